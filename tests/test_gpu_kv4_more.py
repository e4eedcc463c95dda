"""The 4-bit cache where other parts of the library meet it: the two-tier pass, steps that share a context, all layers of the
decode-shaped workload."""
from dataclasses import replace

import numpy as np
import pytest

from workloads import context_kv, get_cascade, get_config, make_batch, model_weights, page_assignment

import kv4_common as K
import parity_common as P

pytestmark = pytest.mark.gpu


def _held(bits):
    return K.values(*K.quantise(P.O.widen_bf16(bits))) if len(bits) else P.O.widen_bf16(bits)


def _contexts(cfg, batch):
    def ctx(i, layer):
        k, v = context_kv(cfg, i, layer, int(batch.ctx_lens[i]))
        return (_held(k), _held(v)) if cfg.kv_format == "int4" else (P.O.widen_bf16(k), P.O.widen_bf16(v))
    return ctx


@pytest.mark.parametrize("formats", [("int4", "int4"), ("int4", "bf16"), ("bf16", "int4")])
def test_the_two_tier_pass(formats):
    """Draft and target over 4-bit caches, and either of them beside a 16-bit one, against the oracle on the values that the codes
    stand for."""
    from paper_2602_18447_b200.runner import CascadeSession
    casc = get_cascade("cascade_tiny")
    cfg_d, cfg_t = (replace(c, ctx_kv="synthetic", kv_format=f) for c, f in zip((casc.draft, casc.target), formats))
    wd, wt = P.planted_weights(cfg_d), P.planted_weights(cfg_t)
    batch = make_batch(cfg_d)
    toks, ctx_lens = P.steps_of(batch), [int(c) for c in batch.ctx_lens]
    of_d, of_t = _contexts(cfg_d, batch), _contexts(cfg_t, batch)
    conf = np.sort(P.O.verify_steps(wd, toks, ctx_lens, of_d, cfg_d.verdict_ids, 0.5)["conf"])
    at = 1 + int(np.argmax(np.diff(conf)[1:-1]))                         # the widest gap that leaves steps on both sides
    tau, gap = float(conf[at:at + 2].mean()), float(conf[at + 1] - conf[at])
    ref = P.O.verify_cascade(wd, wt, toks, ctx_lens, of_d, of_t, cfg_d.verdict_ids, tau)
    assert 0 < ref["escalated"].size < batch.n_steps
    sd = P.build_session(cfg_d, wd, batch)
    try:
        st = P.build_session(cfg_t, wt, batch)
    except BaseException:
        sd.close()
        raise
    cs = CascadeSession(sd, st)
    try:
        cs.verify(tau=tau)
        g = cs.results()
        assert np.max(np.abs(g["conf_d"] - ref["draft"]["conf"])) < 0.45 * gap
        esc = np.nonzero(g["trusted"] == 0)[0]
        assert np.array_equal(esc, ref["escalated"]) and g["n_escalated"] == esc.size
        assert np.max(np.abs(g["conf_t"][esc] - ref["target"]["conf"])) <= P.planted_tols(cfg_t)[1]
        P.check_verdict({"verdict": g["verdict_d"]}, ref["draft"], cfg_d.verdict_ids)
        P.check_verdict({"verdict": g["verdict_t"][esc]}, ref["target"], cfg_d.verdict_ids)
        tr = g["trusted"] != 0
        assert np.array_equal(g["conf"], np.where(tr, g["conf_d"], g["conf_t"]))
        assert np.array_equal(g["verdict"], np.where(tr, g["verdict_d"], g["verdict_t"]))
    finally:
        cs.close()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_the_same_context_for_several_long_steps(dtype):
    """Steps of more than 96 query rows on one sequence (given keys), beside one on another sequence that shares its pages: the context
    is expanded for each as for the step on its own."""
    import torch
    rng = np.random.default_rng(12)
    rows = lambda n, h: torch.from_numpy(rng.standard_normal((n, h, 64))).to(getattr(torch, dtype)).cuda()  # noqa: E731
    with K.Cache(8, 2, 64, n_seqs=3) as c:
        c.B.cs_plan_set(c.plan, [1], [77])
        c.B.cs_kv_append(c.plan, 0, rows(77, 2), rows(77, 2))
        c.B.cs_kv_commit(c.plan)
        c.B.cs_kv_set_seq(c.kv, 2, c.pages[1][:3], 40)                   # the first 40 of the same tokens
        steps = [(1, 30), (1, 26), (2, 33), (1, 100)]
        n = sum(m for _, m in steps)
        q, k, v = rows(n, 8), rows(n, 2), rows(n, 2)
        out, one = torch.empty_like(q), torch.empty_like(q)
        c.B.cs_plan_set(c.plan, [s for s, _ in steps], [m for _, m in steps], given=True)
        c.B.cs_attention_4bit(c.plan, 0, q, out, k, v)
        a = 0
        for s, m in steps:
            c.B.cs_plan_set(c.plan, [s], [m], given=True)
            c.B.cs_attention_4bit(c.plan, 0, q[a:a + m], one[a:a + m], k[a:a + m], v[a:a + m])
            a += m
        torch.cuda.synchronize()
        # a context may be cut into pieces on its own and not in the batch: both are within the roundings of P (2^-11 each way) and
        # of the output of one another; |out| <= max |v|
        eps = 2.0 ** -11 if dtype == "float16" else 2.0 ** -8
        most = float(v.abs().max().clamp(min=5.0))
        assert float((out.double() - one.double()).abs().max()) <= (2 * 2.0 ** -11 + 2 * eps) * most
        assert bool(torch.isfinite(out).all())


def test_cfg11_short_steps_on_long_contexts_full_depth():
    """The decode-shaped workload over the 4-bit cache, all 28 layers and all 64 contexts of 2 K to 8 K tokens. The oracle recomputes
    three steps, whose contexts are the workload's; the others' rows are drawn on the device."""
    import torch
    from paper_2602_18447_b200 import VerifySession, binding as B
    cfg = get_config("cfg11_q3_short_int4")
    weights, batch, sample = model_weights(cfg.model, cfg.seed), make_batch(cfg), [0, 33, 63]
    lens = [int(c) for c in batch.ctx_lens]
    ses = VerifySession(cfg, weights, batch)
    try:
        B.cs_set_keep_logits(ses.model, True)
        total, pages = page_assignment(cfg, batch.ctx_lens)
        ses.alloc_cache(pages, total, batch.ctx_lens, room_for_prefill=True)
        others = [i for i in range(batch.n_steps) if i not in sample]
        plan = B.cs_plan_create(ses.kv)
        B.cs_plan_set(plan, others, [lens[i] for i in others])
        gen = torch.Generator(device="cuda").manual_seed(cfg.seed)
        shape = (sum(lens[i] for i in others), cfg.model.n_kv_heads, cfg.model.head_dim)
        for layer in range(cfg.model.n_layers):
            k, v = (torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) * cfg.kv_std for _ in range(2))
            B.cs_kv_append(plan, layer, k, v, rotate=False)
        B.cs_kv_commit(plan)
        torch.cuda.synchronize()
        B.cs_plan_free(plan)
        held = {}
        for i in sample:
            B.cs_kv_set_seq(ses.kv, i, pages[i], lens[i])
            for layer in range(cfg.model.n_layers):
                k, v = context_kv(cfg, i, layer, lens[i])
                B.cs_kv_fill(ses.kv, i, layer, k, v)
                held[i, layer] = _held(k).astype(np.float32), _held(v).astype(np.float32)
        ses.verify()
        gpu = ses.results()
        assert np.all(np.isfinite(gpu["conf"])) and np.all(gpu["conf"] > 0) and np.all(gpu["conf"] <= 1)
        toks = P.steps_of(batch)
        ref = P.O.verify_steps(weights, [toks[i] for i in sample], [lens[i] for i in sample],
                               lambda j, layer: held[sample[j], layer], cfg.verdict_ids, cfg.tau)
        stats = P.compare(gpu, ses.last_logits(), ref, cfg.tau, steps=sample, gpu_lse=ses.last_lse())
        P.check_verdict(gpu, ref, cfg.verdict_ids, steps=sample)
        assert stats["logit_err"] <= P.LOGIT_TOL and stats["conf_err"] <= P.CONF_TOL
        B.cs_check_workspace(ses.model)
    finally:
        ses.close()
