"""Passes over a model whose projections are 8-bit integers (cs_model_quantize_i8): bit for bit against the public calls where the
attention is the identity, and whole workloads against the oracle with quantised rows and weights."""
from dataclasses import replace

import numpy as np
import pytest

import i8_common as I
import parity_common as P
from workloads import context_kv, get_config, make_batch, model_weights, page_assignment, scaled_config

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2602_18447_b200 import binding
    return binding


def _f16(a):
    """bf16 patterns as the library's fp16 matrix."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).half().cuda()


def _session(B, cfg, weights, batch):
    """As P.build_session, over 8-bit projections from the first prefill on."""
    from paper_2602_18447_b200 import VerifySession
    ses = VerifySession(cfg, weights, batch, i8=True)
    B.cs_set_keep_logits(ses.model, True)
    total, pages = page_assignment(cfg, batch.ctx_lens)
    ses.alloc_cache(pages, total, batch.ctx_lens, room_for_prefill=cfg.ctx_kv == "prefill")
    if cfg.ctx_kv == "prefill":
        ses.prefill_context(batch.ctx_tokens)
    else:
        ses.fill_synthetic_context(lambda i, l: context_kv(cfg, i, l, int(batch.ctx_lens[i])))
    return ses


@pytest.mark.parametrize("name,batch", [("cfg1_tiny", 1), ("cfg1_tiny", 7), ("cfg1_tiny", 40), ("cfg8_tiny_qknorm", 11), ("cfg2", 5), ("cfg2", 150)])
def test_single_tokens_without_context_are_the_public_calls(B, name, batch):
    """One key to attend to: attention leaves the token's own values, and position 0 turns nothing."""
    import torch
    base = scaled_config("cfg2_1p5b_b16", n_layers=3, batch=batch, vocab=2056) if name == "cfg2" else get_config(name)
    cfg = replace(base, batch=batch, ctx_dist=("fixed", 0), step_dist=("fixed", 1), suffix_len=0, ctx_kv="synthetic")
    w, data = model_weights(cfg.model, cfg.seed), make_batch(cfg)
    g = np.random.default_rng(batch)
    for layer in w["layers"]:                      # gains that are not all 1
        for n in ("norm1", "norm2"):
            layer[n] = np.exp(0.3 * g.standard_normal(cfg.model.d_model)).astype(np.float32)
    m = cfg.model
    ses = _session(B, cfg, w, data)
    try:
        ses.verify()
        got = ses.last_logits()
        ses.results()
    finally:
        ses.close()
    x = _f16(w["embed"])[torch.from_numpy(np.asarray(data.step_tokens, np.int64)).cuda()].float()
    T = x.shape[0]
    codes = lambda d: torch.empty(T, d, dtype=torch.int8, device="cuda")  # noqa: E731
    half = lambda n: torch.empty(T, n, dtype=torch.float16, device="cuda")  # noqa: E731
    s, delta = torch.empty(T, device="cuda"), None
    dev = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731

    def coded(mat):
        c, sc = torch.empty(mat.shape, dtype=torch.int8, device="cuda"), torch.empty(mat.shape[0], device="cuda")
        B.cs_quantize_i8(mat, c, sc)
        return c, sc

    for li, l in enumerate(w["layers"]):
        c = codes(m.d_model)
        B.cs_rmsnorm_i8(x, dev(l["norm1"]), c, s, m.rms_eps, delta=delta)
        v = half(m.kv_dim)
        B.cs_gemm_i8(c, s, *coded(_f16(l["wv"])), v)
        o = v.view(T, m.n_kv_heads, 1, m.head_dim).expand(T, m.n_kv_heads, m.group, m.head_dim).reshape(T, m.q_dim).contiguous()
        c = codes(m.q_dim)
        B.cs_quantize_i8(o, c, s)
        last = li == m.n_layers - 1
        delta = None if last else half(m.d_model)
        B.cs_gemm_i8(c, s, *coded(_f16(l["wo"])), x if last else delta, add=x if last else None)
        c = codes(m.d_model)
        B.cs_rmsnorm_i8(x, dev(l["norm2"]), c, s, m.rms_eps, delta=delta)
        h = half(m.d_ffn)
        wu = coded(_f16(l["wu"]))
        B.cs_gemm_i8(c, s, *coded(_f16(l["wg"])), h, w2=wu[0], w2_scales=wu[1])
        c = codes(m.d_ffn)
        B.cs_quantize_i8(h, c, s)
        delta = None if last else half(m.d_model)
        B.cs_gemm_i8(c, s, *coded(_f16(l["wd"])), x if last else delta, add=x if last else None)
    hid = half(m.d_model)
    B.cs_rmsnorm(x, dev(w["final_norm"]), hid, T, m.d_model, m.rms_eps)
    hid, head = hid.double(), _f16(w["lm_head"]).double()
    want = (hid @ head.T).cpu().numpy()
    # the final norm's own rounding to fp16 may fall the other way by its last fp32 bits: one step (2^-10) of a hidden value
    bound = 2.0 ** -10 * (hid.abs() @ head.abs().T).cpu().numpy() * 0.25 + 1e-6
    I.check(got, want, bound)


def _oracle(cfg, weights, batch, noise, monkeypatch):
    monkeypatch.setattr(P.O, "LayerWeights", I.layer_weights(_ORACLE))
    monkeypatch.setattr(P.O, "decoder_layer_extend", I.decoder_layer(_ORACLE, noise))
    try:
        return P.oracle_outputs(cfg, weights, batch)
    finally:
        monkeypatch.undo()


class _Plain:
    """The oracle's own functions, whatever is patched."""
    def __init__(self, O):
        self.__dict__.update({k: getattr(O, k) for k in ("LayerWeights", "rmsnorm", "rope", "silu", "attention_extend")})


_ORACLE = _Plain(P.O)

CASES = [
    ("tiny", replace(get_config("cfg1_tiny"), batch=12)),
    ("tiny, second family", get_config("cfg8_tiny_qknorm")),
    ("1.5B-shaped, 2 layers", scaled_config("cfg2_1p5b_b16", n_layers=2, batch=5, vocab=4104)),
    ("1.7B-shaped, short steps", scaled_config("cfg7_q3_short", n_layers=1, batch=9, vocab=4104)),
    ("1.7B-shaped, short steps, 8-bit cache", scaled_config("cfg9_q3_short_fp8", n_layers=1, batch=9, vocab=4104)),
    ("tiny, five heads to turn", replace(get_config("cfg1_tiny"), batch=5, model=replace(get_config("cfg1_tiny").model, n_kv_heads=1))),
    ("tiny, second family, nine heads to turn",
     replace(get_config("cfg8_tiny_qknorm"), model=replace(get_config("cfg8_tiny_qknorm").model, n_q_heads=6, n_kv_heads=3))),
]


@pytest.mark.parametrize("name,cfg", CASES, ids=[c[0] for c in CASES])
def test_workloads_against_the_oracle_on_codes(B, name, cfg, monkeypatch):
    """A value that fp16 has rounded may fall on the other side of a code's border, and that is most of what the library and the
    oracle differ by. How far that may take the logits is what the oracle itself says: three runs whose fp16 values are off by up to
    half a step at random. The library's largest difference, over as many values, is held to three times theirs."""
    w, batch = P.planted_weights(cfg), make_batch(cfg)
    ref = _oracle(cfg, w, batch, None, monkeypatch)
    runs = [_oracle(cfg, w, batch, np.random.default_rng(k), monkeypatch) for k in range(3)]
    spread = lambda pick: max(float(np.abs(pick(r) - pick(ref)).max()) for r in runs)  # noqa: E731
    vids = list(cfg.verdict_ids)
    rest = lambda r: np.delete(r["logits"], vids, axis=1)  # noqa: E731
    planted = lambda r: r["logits"][:, vids]  # noqa: E731
    conf = lambda r: r["conf"]  # noqa: E731
    ses = _session(B, cfg, w, batch)
    try:
        ses.verify()
        gpu, logits = ses.results(), ses.last_logits().astype(np.float64)
        B.cs_check_workspace(ses.model)
        got = dict(gpu, logits=logits)
        for what, pick in (("logits", rest), ("planted rows", planted), ("confidence", conf)):
            off, bound = float(np.abs(pick(got) - pick(ref)).max()), 3 * spread(pick) + 1e-4
            print(name, what, off, "bound", bound)
            assert off <= bound, (what, off, bound)
        far = np.abs(ref["conf"] - cfg.tau) > 3 * spread(conf) + 1e-4
        assert np.array_equal(gpu["accept"][far], ref["accept"][far])
        ses.verify(host_tokens=True)                                       # the same bits again
        assert np.array_equal(ses.results()["conf"].view(np.uint32), gpu["conf"].view(np.uint32))
        assert np.array_equal(ses.last_logits(), logits.astype(np.float32))
    finally:
        ses.close()


def test_two_tiers_one_of_them_quantised(B):
    """The draft on codes, the target as loaded: the two-tier pass gives what the two passes give."""
    import torch
    from paper_2602_18447_b200.runner import CascadeSession
    from workloads import get_cascade
    c = get_cascade("cascade_tiny")
    batch = make_batch(c.draft)
    draft = _session(B, c.draft, P.planted_weights(c.draft), batch)
    target = P.build_session(c.target, P.planted_weights(c.target), batch)
    two = CascadeSession(draft, target)
    try:
        draft.verify()
        alone = draft.results()
        n = two.verify()
        got = two.results()
        assert n == int((alone["accept"] == 0).sum())
        assert np.array_equal(got["conf_d"].view(np.uint32), alone["conf"].view(np.uint32))
        trusted = got["trusted"] == 1
        assert np.array_equal(got["verdict"][trusted], alone["verdict"][trusted])
        assert np.array_equal(got["conf"][~trusted], got["conf_t"][~trusted])
        torch.cuda.synchronize()
    finally:
        two.close()


def test_4bit_cache_appends_and_grows(B):
    """Prefill of a 4-bit cache and a pass over it, on codes, twice the same."""
    cfg = replace(get_config("cfg1_tiny"), batch=6, ctx_dist=("uniform", 20, 150), kv_format="int4")
    w, batch = P.planted_weights(cfg), make_batch(cfg)
    confs = []
    for _ in range(2):
        ses = _session(B, cfg, w, batch)
        try:
            ses.verify()
            confs.append(ses.results()["conf"])
            B.cs_check_workspace(ses.model)
        finally:
            ses.close()
    assert np.isfinite(confs[0]).all() and np.array_equal(confs[0].view(np.uint32), confs[1].view(np.uint32))


def test_what_is_refused_and_what_is_freed(B):
    import torch
    cfg = scaled_config("cfg2_1p5b_b16", n_layers=4, batch=2, vocab=2056)
    w = model_weights(cfg.model, cfg.seed)
    m = B.cs_model_load(cfg.model, w)
    try:
        before = torch.cuda.mem_get_info()[0]
        B.cs_model_quantize_i8(m)
        gained = torch.cuda.mem_get_info()[0] - before
        assert gained > 0.4 * 2 * cfg.model.params_per_layer() * 4
        with pytest.raises(B.ConfSpecError) as e:
            B.cs_model_quantize_i8(m)
        assert e.value.status == B.CS_ESTATE
    finally:
        B.cs_model_free(m)
    odd = replace(cfg.model, d_ffn=200, n_layers=1)
    m = B.cs_model_load(odd, model_weights(odd, 3))
    try:
        with pytest.raises(B.ConfSpecError) as e:
            B.cs_model_quantize_i8(m)
        assert e.value.status == B.CS_EINVAL
    finally:
        B.cs_model_free(m)
