"""The verification pass over a 4-bit cache: steps that read the codes and steps whose contexts are expanded, against the oracle on
the values that the codes stand for; prefill and the append of accepted steps; a decode step of the program's own next to a pass."""
from dataclasses import replace

import numpy as np
import pytest

from workloads import context_kv, get_cascade, get_config, make_batch, model_weights, scaled_config

import kv4_common as K
import parity_common as P

pytestmark = pytest.mark.gpu


def _held(bits):
    """What the 4-bit cache holds for bf16 rows."""
    return K.values(*K.quantise(P.O.widen_bf16(bits)))


def _oracle(cfg, weights, batch):
    def ctx(i, layer):
        k, v = context_kv(cfg, i, layer, int(batch.ctx_lens[i]))
        if not len(k):
            return P.O.widen_bf16(k), P.O.widen_bf16(v)
        return _held(k), _held(v)
    return P.O.verify_steps(weights, P.steps_of(batch), [int(c) for c in batch.ctx_lens], ctx, cfg.verdict_ids, cfg.tau)


def _run(cfg, weights, batch, planted):
    from paper_2602_18447_b200 import binding as B
    ses = P.build_session(cfg, weights, batch)
    try:
        ses.verify()
        gpu = ses.results()
        logits, lse = ses.last_logits(), ses.last_lse()
        ref = _oracle(cfg, weights, batch)
        if planted:
            P.compare_planted(gpu, logits, ref, cfg.tau, cfg, weights)
        else:
            P.compare(gpu, logits, ref, cfg.tau, gpu_lse=lse)
            P.check_verdict(gpu, ref, cfg.verdict_ids)
        B.cs_check_workspace(ses.model)
        ses.verify(host_tokens=True)
        again = ses.results()
        assert np.array_equal(again["conf"].view(np.uint32), gpu["conf"].view(np.uint32))
    finally:
        ses.close()


def _cfg(name, **kw):
    base = dict(ctx_kv="synthetic", kv_format="int4", suffix_len=0)
    base.update(kw)
    return replace(get_config(name), **base)


# one and two query heads per kv head: up to 96 query rows read the codes, longer steps the expanded pages
@pytest.mark.parametrize("name,steps", [("cfg1_tiny", ("uniform", 1, 32)), ("cfg1_tiny", ("uniform", 90, 140)),
                                        ("cfg8_tiny_qknorm", ("uniform", 1, 40)), ("cfg8_tiny_qknorm", ("uniform", 1, 80))])
def test_small_models_every_step(name, steps):
    cfg = _cfg(name, batch=7, ctx_dist=("uniform", 1, 300), step_dist=steps)
    _run(cfg, P.planted_weights(cfg), make_batch(cfg), True)
    _run(cfg, model_weights(cfg.model, cfg.seed), make_batch(cfg), False)


@pytest.mark.parametrize("ctx,step", [(0, 1), (0, 130), (1, 1), (15, 3), (16, 16), (17, 130), (257, 2)])
def test_context_and_step_length_edges(ctx, step):
    cfg = _cfg("cfg1_tiny", batch=3, ctx_dist=("fixed", ctx), step_dist=("fixed", step))
    _run(cfg, P.planted_weights(cfg), make_batch(cfg), True)


@pytest.mark.parametrize("name", ["cfg9_q3_short_fp8", "cfg2_1p5b_b16"])
def test_large_shapes_reduced_depth(name):
    cfg = replace(scaled_config(name, n_layers=2, batch=5, vocab=20480 + 8), kv_format="int4")
    _run(cfg, P.planted_weights(cfg), make_batch(cfg), True)


def _read_all(B, kv, shape, layer, lens):
    import torch
    seq = np.repeat(np.arange(len(lens)), lens)
    pos = np.concatenate([np.arange(n) for n in lens])
    k = torch.empty(len(seq), shape.n_kv_heads, shape.head_dim, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    B.cs_kv_read(kv, layer, torch.tensor(seq, dtype=torch.int32, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda"),
                 k, v)
    torch.cuda.synchronize()
    cut = np.cumsum(lens)[:-1]
    return list(zip(np.split(k.double().cpu().numpy(), cut), np.split(v.double().cpu().numpy(), cut)))


def test_prefill_quantises_what_the_16_bit_cache_would_hold_and_verifies_on_it():
    """From empty contexts of more than 96 query rows both caches see the same activations, so a 4-bit value is off from the 16-bit
    one by half a code step, the ends' roundings (15 s 2^-11, 2^-11 |min|), the fp16 rounding of the read (2^-11) and the bf16
    rounding of the 16-bit cell (2^-8). Verification on the prefilled cache is then held to the oracle on the values read back."""
    from paper_2602_18447_b200 import VerifySession, binding as B
    cfg = replace(get_config("cfg8_tiny_qknorm"), batch=4, ctx_dist=("uniform", 60, 150), step_dist=("uniform", 1, 30))
    w, batch = P.planted_weights(cfg), make_batch(cfg)
    lens = [int(c) for c in batch.ctx_lens]
    ses = {}
    try:
        for fmt in ("bf16", "int4"):
            ses[fmt] = VerifySession(replace(cfg, kv_format=fmt), w, batch)
            B.cs_set_keep_logits(ses[fmt].model, True)
            total, pages = P.page_assignment(cfg, batch.ctx_lens)
            ses[fmt].alloc_cache(pages, total, batch.ctx_lens, room_for_prefill=True)
            ses[fmt].prefill_context(batch.ctx_tokens)
        held = [_read_all(B, ses["int4"].kv, cfg.model, layer, lens) for layer in range(cfg.model.n_layers)]
        for layer in range(cfg.model.n_layers):
            for (k4, v4), (k16, v16) in zip(held[layer], _read_all(B, ses["bf16"].kv, cfg.model, layer, lens)):
                for x4, x16 in ((k4, k16), (v4, v16)):
                    g = x16.reshape(*x16.shape[:-1], -1, K.GROUP)
                    most = np.abs(g).max(-1, keepdims=True)
                    s = (np.ptp(g, axis=-1, keepdims=True) + 2 * 2.0 ** -8 * most) / 15 * (1 + 2.0 ** -11)
                    bound = s * (0.5 + 15 * 2.0 ** -11) + (2 * 2.0 ** -11 + 2.0 ** -8) * (most + s) * (1 + 2.0 ** -7)
                    assert np.all(np.abs(x4 - x16) <= np.broadcast_to(bound, g.shape).reshape(x16.shape))
        ses["int4"].verify()
        gpu = ses["int4"].results()
        ref = P.O.verify_steps(w, P.steps_of(batch), lens, lambda i, layer: held[layer][i], cfg.verdict_ids, cfg.tau)
        P.compare_planted(gpu, ses["int4"].last_logits(), ref, cfg.tau, cfg, w)
    finally:
        for s in ses.values():
            s.close()


def test_accepted_steps_are_appended_to_a_4_bit_cache():
    """cs_append_accepted writes the accepted steps' rows behind the context (in front of it nothing changes), the context grows by
    them, and the next pass is held to the oracle on the values read back."""
    import torch
    from paper_2602_18447_b200 import binding as B
    cfg = get_cascade("cascade_tiny").draft
    w = P.planted_weights(cfg)
    g = np.random.default_rng(5)
    lens, steps, drafts = [40, 7], np.array([9, 12, 10, 11], np.int32), np.array([5, 12, 0, 3], np.int32)
    model = B.cs_model_load(cfg.model, w)
    kv = B.cs_kv_alloc_4bit(model, 20, 16, 2, 10)
    try:
        B.cs_set_keep_logits(model, True)
        order = g.permutation(20).astype(np.int32)
        for r in range(2):
            B.cs_kv_set_seq(kv, r, order[10 * r:10 * r + 10], 0)
        ctx = [g.integers(3, cfg.model.vocab, n).astype(np.int32) for n in lens]
        B.cs_prefill(model, kv, [0, 1], np.concatenate(ctx), lens)
        before = [_read_all(B, kv, cfg.model, layer, lens) for layer in range(cfg.model.n_layers)]
        toks = g.integers(3, cfg.model.vocab, int(steps.sum())).astype(np.int32)
        prefix = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
        got = B.cs_append_accepted(model, kv, [0, 1], [0, 2, 4], prefix, toks, steps, drafts)
        assert got.tolist() == [2, 1]
        after_lens = [40 + 17, 7]                              # the second request's accepted step drafted nothing
        after = [_read_all(B, kv, cfg.model, layer, after_lens) for layer in range(cfg.model.n_layers)]
        for layer in range(cfg.model.n_layers):
            for r in range(2):
                for x, y in zip(before[layer][r], after[layer][r]):
                    assert np.array_equal(x, y[:lens[r]])
            assert np.abs(after[layer][0][0][40:]).min(axis=(1, 2)).max() > 0
        span = [g.integers(3, cfg.model.vocab, n).astype(np.int32) for n in (4, 6)]
        conf, acc = torch.empty(2, device="cuda"), torch.empty(2, dtype=torch.uint8, device="cuda")
        ver = torch.empty(2, dtype=torch.int32, device="cuda")
        B.cs_verify_steps(model, kv, [0, 1], np.concatenate(span), [4, 6], cfg.verdict_ids, cfg.tau, conf, acc, ver)
        logits = torch.empty(2, cfg.model.vocab, device="cuda")
        B.cs_get_last_logits(model, logits, 2)
        torch.cuda.synchronize()
        B.cs_last_status(model)
        ref = P.O.verify_steps(w, span, after_lens, lambda i, layer: after[layer][i], cfg.verdict_ids, cfg.tau)
        P.compare_planted({"conf": conf.cpu().numpy(), "accept": acc.cpu().numpy(), "verdict": ver.cpu().numpy()},
                          logits.cpu().numpy(), ref, cfg.tau, cfg, w)
    finally:
        B.cs_kv_free(kv)
        B.cs_model_free(model)
