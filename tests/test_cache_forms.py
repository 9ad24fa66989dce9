"""Engines with a 4-bit K/V cache, per-head norms of queries and keys, and token scores, against the oracle.

Tolerance of a 4-bit engine's logits. Its k and v are the oracle's to about 2^-17 (split-bf16 GEMMs), so an element falls
on the other side of a code border with probability 2 * 2^-17 / (1/3) (a step is a third of a row's standard deviation)
= 5e-5: a few of the 30k elements of a batch, and then by a whole step. What one of them does: where w_q and w_k are eight
times their draw, q and k have a deviation of 8 * 0.02 * sqrt(256) = 2.6, a step of k is 0.9, and one element moves a score by
2.6 * 0.9 / sqrt(64) = 0.3; scores spread over 2.6^2 = 6.8, so few keys share the weight, which moves by up to 0.3 / 4 of it:
8% of an attention output that is a part of the residual, some 1e-2 of logits with a deviation of 0.3. So the bf16 bound of
the parity tests, 2e-2, is kept; 4 bits themselves move these logits by 0.2 to 0.6, which is asserted. Batches without a
code on the other side are at 1e-5. Other engines keep the parity tests' bounds (2e-2 for bf16, 1e-4 for f32).
"""
import math

import numpy as np
import pytest

from moa_inputs import ModelShape, f32_to_bf16_bits, generate_weights, pack_blob
from moa_inputs.configs import EngineConsts
from moa_inputs.weights import bf16_bits_to_f32
from oracle import transformer as T
from paper_2606_03014_amd import Engine
from paper_2606_03014_amd import moa as M
from tests.gpu_helpers import check_tokens, say

gpu = pytest.mark.gpu
INT4_TOL = 2e-2


def shape(n_h=8, n_kv=2, hd=64, layers=2, vocab=1024, d=256):
    return ModelShape(n_layers=layers, d_model=d, n_heads=n_h, n_kv_heads=n_kv, head_dim=hd, ffn_dim=512, vocab=vocab)


def weights(sh, dtype, seed, qk_norm=False):
    w = generate_weights(sh, dtype, seed, 98, 0, qk_norm=qk_norm)
    rng = np.random.default_rng(seed)
    for n in w:
        if n.endswith("norm"):
            g = rng.uniform(0.5, 1.5, w[n].shape).astype(np.float32)
            w[n] = f32_to_bf16_bits(g) if dtype == "bf16" else g
    return w


def serve(eng, reqs, noalloc=False, scores=None, history=()):
    """Run (tokens, model, G) requests to the end. Returns tokens, captured logits and score arrays by request."""
    rids, caps, sc = [], [], []
    for toks, m, G in reqs:
        rids.append(eng.submit(np.asarray(toks, np.int32), m, G))
    for (m, tok, L, kv, G) in history:
        rids.append(eng.submit_with_history(m, tok, L, G, kv))
    V = eng.shape.vocab
    for i, rid in enumerate(rids):
        G = eng.request(rid).max_new_tokens
        caps.append(np.full(G * V, np.nan, np.float32))
        eng.capture_logits(rid, caps[-1])
        k = scores[i] if scores else None
        sc.append(None if k is None else eng.request_scores(rid, k))
    while (eng.step_noalloc() if noalloc else eng.step()).step >= 0:
        pass
    got = {r[0]: r[3] for r in eng.collect()}
    eng.sync()
    return [got[r] for r in rids], [c.reshape(-1, V) for c in caps], sc


# ------------------------------------------------------------------ host side (CPU)

def test_flags_are_checked_and_sized():
    sh, c = shape(), EngineConsts(64, 4, 64, 256)
    with pytest.raises(M.MoaError) as err:
        Engine(sh, "f32", c, 1, plan_only=True, kv_int4=True)
    assert err.value.code == M.MOA_EINVAL
    sizes = {}
    for name, kw in dict(plain={}, int4=dict(kv_int4=True), qk=dict(qk_norm=True), scores=dict(scores=True)).items():
        eng = Engine(sh, "bf16", c, 1, plan_only=True, **kw)
        sizes[name] = eng.arena_bytes
        eng.close()
    saved = 64 * sh.n_layers * sh.n_kv_heads * (2 * 16 * 64 * 2 - (16 * 64 + 128))
    assert sizes["int4"] <= sizes["plain"] - saved + 4096
    assert sizes["qk"] > sizes["plain"] - 4096 and sizes["scores"] > sizes["plain"]


def test_weight_blobs_hold_the_head_norms_only_with_the_flag():
    sh, c = shape(), EngineConsts(64, 4, 64, 256)
    plain, qk = (np.zeros((sh.n_params() + extra) * 2, np.uint8) for extra in (0, 2 * sh.n_layers * sh.head_dim))
    for kw, ok, bad in (({}, plain, qk), (dict(qk_norm=True), qk, plain)):
        eng = Engine(sh, "bf16", c, 1, plan_only=True, **kw)
        with pytest.raises(M.MoaError):
            eng.load(bad)
        assert eng.load(ok) == 0
        eng.close()
    w = weights(sh, "bf16", 1, qk_norm=True)
    assert pack_blob(w, sh).nbytes == qk.nbytes


def test_score_and_read_requests_are_refused_on_a_dry_run():
    sh = shape()
    eng = Engine(sh, "bf16", EngineConsts(64, 4, 64, 256), 1, plan_only=True, scores=True)
    eng.load(np.zeros(sh.n_params() * 2, np.uint8))
    rid = eng.submit(np.arange(5, dtype=np.int32), 0, 3)
    for call in (lambda: eng.request_scores(rid, 2), lambda: eng.kv(rid, 0, 1)):
        with pytest.raises(M.MoaError) as err:
            call()
        assert err.value.code == M.MOA_ESTATE
    a, b = np.zeros(3, np.float32), np.zeros(3, np.float32)
    for args in ((rid + 1, a, b), (rid, None, b), (rid, a, None), (rid, a, b, np.zeros((3, 33), np.int32), np.zeros((3, 33), np.float32)),
                 (rid, a, b, np.zeros((3, 2), np.int32), None)):
        with pytest.raises(M.MoaError) as err:
            M.moa_request_scores(eng.h, *args)
        assert err.value.code == M.MOA_EINVAL
    for args in ((rid, 2, 1), (rid, -1, 1), (rid, 0, 17), (rid, 0, -1), (99, 0, 1)):
        with pytest.raises((M.MoaError, ValueError)) as err:
            eng.kv(*args)
    with pytest.raises(ValueError):
        M.moa_request_scores(eng.h, rid, a.astype(np.float64), b)
    eng.close()


def test_dry_run_of_a_4_bit_engine_keeps_the_step_rule():
    """The cache's form changes no admission, chunk or retirement."""
    sh, c = shape(), EngineConsts(200, 6, 64, 3000)
    rng = np.random.default_rng(3)
    reqs = [(int(rng.integers(1, 300)), int(rng.integers(1, 60))) for _ in range(25)]
    traces = []
    for kw in ({}, dict(kv_int4=True)):
        eng = Engine(sh, "bf16", c, 1, plan_only=True, **kw)
        eng.load(np.zeros(sh.n_params() * 2, np.uint8))
        for n, G in reqs:
            eng.submit(np.zeros(n, np.int32), 0, G)
        while eng.step().step >= 0:
            pass
        traces.append(eng.steps().tolist())
        eng.close()
    assert traces[0] == traces[1]


def test_oracle_4_bit_rows():
    """16 levels reproduce themselves; the error is at most half a step plus the minimum's and step's rounding."""
    rng = np.random.default_rng(1)
    levels = 0.25 * rng.integers(0, 16, (50, 64)) - 2.0
    levels[:, 0], levels[:, 1] = -2.0, 1.75
    assert np.array_equal(T.int4_round(levels), levels)
    x = rng.standard_normal((200, 128))
    step = (x.max(-1) - x.min(-1))[:, None] / 15
    assert (np.abs(T.int4_round(x) - x) <= step * (0.5 + 15 * 2.0 ** -9) + 2.0 ** -9 * np.abs(x.min(-1))[:, None] + 1e-6).all()
    assert np.array_equal(T.int4_round(np.full((2, 8), 3.0)), np.full((2, 8), 3.0))


def test_oracle_head_norms():
    """Unit vectors in, gains out: a normalised head scaled by any factor gives the same logits."""
    sh = shape(layers=1)
    w = weights(sh, "f32", 3, qk_norm=True)
    big = dict(w)
    big["layers.0.wq"], big["layers.0.wk"] = w["layers.0.wq"] * 64, w["layers.0.wk"] * 64
    toks = np.arange(12)
    sh0 = ModelShape(**{**sh.__dict__, "rms_eps": 1e-30})
    a, b = (T.forward_full(T.OracleModel(sh0, x), toks) for x in (w, big))
    assert np.abs(a - b).max() < 1e-9
    plain = {k: v for k, v in w.items() if "q_norm" not in k and "k_norm" not in k}
    assert np.abs(T.forward_full(T.OracleModel(sh0, plain), toks) - a).max() > 1e-3


# ------------------------------------------------------------------ engines (GPU)

@pytest.fixture(scope="module")
def on_gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need the MI355X"


def check(sh, w, reqs, toks, logits, tol, what, telling=False, **kw):
    for i, (p, _, G) in enumerate(reqs):
        om = T.OracleModel(sh, w, cache=True)
        ref = T.teacher_forced_logits(om, p, toks[i], **kw)
        err = float(np.abs(logits[i] - ref).max())
        seen = float(np.abs(ref - T.teacher_forced_logits(om, p, toks[i], bf16_kv=kw.get("bf16_kv", False))).max()) if kw.get("int4_kv") else None
        say(f"{what} {i}: |engine - oracle| {err:.2e}" + (f" (4 bits alone: {seen:.2e})" if seen else ""))
        assert err <= tol
        if telling:
            assert seen > 5 * tol, "the batch does not tell 4 bits from more"
        if kw.get("int4_kv"):             # logits within tol of the oracle's: the token is the engine's own largest
            assert np.array_equal(toks[i], logits[i].argmax(1))
        else:
            check_tokens(ref, toks[i], what)


@gpu
@pytest.mark.parametrize("n_h,n_kv,hd", [(8, 2, 64), (4, 2, 128), (8, 1, 64), (2, 2, 128), (4, 4, 64)])
def test_4_bit_engine(on_gpu, n_h, n_kv, hd):
    """Prompts in chunks of any cut, beside decode rows; steps of a few rows and of many."""
    sh = shape(n_h, n_kv, hd)
    w = weights(sh, "bf16", 11)
    w["layers.0.wq"], w["layers.0.wk"] = (_times(w[f"layers.0.{n}"], 8) for n in ("wq", "wk"))      # scores that matter
    rng = np.random.default_rng(5)
    reqs = [(rng.integers(0, sh.vocab, n), 0, G) for n, G in ((1, 7), (150, 5), (33, 9), (64, 3), (17, 6), (260, 4), (5, 12))]
    eng = Engine(sh, "bf16", EngineConsts(128, 5, 100, 512), 1, kv_int4=True)
    eng.load(pack_blob(w, sh))
    toks, logits, _ = serve(eng, reqs)
    eng.close()
    check(sh, w, reqs, toks, logits, INT4_TOL, f"int4 {n_h}/{n_kv}/{hd}", telling=True, int4_kv=True)


def _times(bits, f):
    return f32_to_bf16_bits(bf16_bits_to_f32(bits) * np.float32(f))


@gpu
@pytest.mark.parametrize("dtype,int4", [("f32", False), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("hd", [64, 128])
def test_engine_with_head_norms(on_gpu, dtype, int4, hd):
    sh = shape(4, 2, hd)
    w = weights(sh, dtype, 12, qk_norm=True)
    rng = np.random.default_rng(6)
    reqs = [(rng.integers(0, sh.vocab, n), 0, G) for n, G in ((1, 6), (90, 5), (40, 7), (130, 3))]
    eng = Engine(sh, dtype, EngineConsts(128, 3, 64, 512), 1, kv_int4=int4, qk_norm=True)
    eng.load(pack_blob(w, sh))
    toks, logits, _ = serve(eng, reqs)
    eng.close()
    tol = INT4_TOL if int4 else (1e-4 if dtype == "f32" else 2e-2)
    check(sh, w, reqs, toks, logits, tol, f"head norms {dtype} int4 {int4} {hd}", bf16_kv=dtype == "bf16" and not int4, int4_kv=int4)


@gpu
def test_two_models_on_two_streams_allocation_free(on_gpu):
    """Two models' gains and caches side by side, all flags, through both step calls: the same bits."""
    sh = shape(8, 2, 64)
    ws = [weights(sh, "bf16", s, qk_norm=True) for s in (13, 14)]
    rng = np.random.default_rng(7)
    reqs = [(rng.integers(0, sh.vocab, n), m, G) for n, m, G in ((70, 0, 6), (30, 1, 8), (1, 1, 5), (129, 0, 4))]
    runs = []
    for noalloc in (False, True):
        eng = Engine(sh, "bf16", EngineConsts(128, 4, 96, 512), 2, kv_int4=True, qk_norm=True, scores=True)
        for w in ws:
            eng.load(pack_blob(w, sh))
        runs.append(serve(eng, reqs, noalloc, scores=[3, 0, 5, 1]))
        eng.close()
    for a, b in zip(runs[0][0] + runs[0][1], runs[1][0] + runs[1][1]):
        assert np.array_equal(a, b)
    for a, b in zip(runs[0][2], runs[1][2]):
        assert all(np.array_equal(x, y) for x, y in zip(a, b))
    toks, logits, _ = runs[0]
    for m in range(2):
        mine = [i for i, r in enumerate(reqs) if r[1] == m]
        check(sh, ws[m], [reqs[i] for i in mine], [toks[i] for i in mine], [logits[i] for i in mine], INT4_TOL, f"model {m}", int4_kv=True)


@gpu
@pytest.mark.parametrize("hd", [64, 128])
def test_histories_in_4_bits(on_gpu, hd):
    """Injected rows are stored as the definition says (read back bit for bit), and attention over 1 to 2,500 of them,
    split and not, is the oracle's."""
    sh = shape(4, 2, hd, layers=2)
    w = weights(sh, "bf16", 15)
    w["layers.0.wq"] = _times(w["layers.0.wq"], 16)
    rng = np.random.default_rng(8)
    eng = Engine(sh, "bf16", EngineConsts(500, 8, 64, 3000), 1, kv_int4=True)
    eng.load(pack_blob(w, sh))
    lens = (1, 16, 100, 1023, 1024, 2500)
    hist = []
    for L in lens:
        kv = f32_to_bf16_bits(rng.standard_normal((sh.n_layers, 2, L, sh.n_kv_heads, hd)).astype(np.float32))
        hist.append((0, int(rng.integers(0, sh.vocab)), L, kv, 3))
    rids = [eng.submit_with_history(m, tok, L, G, kv) for m, tok, L, kv, G in hist]
    fill = eng.submit_with_history(0, 5, 37, 3)
    caps = [np.full(3 * sh.vocab, np.nan, np.float32) for _ in rids]
    for rid, c in zip(rids, caps):
        eng.capture_logits(rid, c)
    eng.step()
    for rid, (_, _, L, kv, _) in zip(rids, hist):
        for layer in range(sh.n_layers):
            got = eng.kv(rid, layer, L)
            for i in range(2):
                want = f32_to_bf16_bits(T.int4_round(bf16_bits_to_f32(kv[layer, i])).astype(np.float32))
                assert np.array_equal(got[i], want), (L, layer, i)
    fk, fv = (bf16_bits_to_f32(x) for x in eng.kv(fill, 1, 37))
    assert np.isfinite(fk).all() and 0.9 < np.abs(fk).max() <= 1.05 and 0.5 < fv.std() < 0.65
    while eng.step().step >= 0:
        pass
    toks = {r[0]: r[3] for r in eng.collect()}
    eng.sync()
    eng.close()
    om = T.OracleModel(sh, w)
    for rid, cap, (_, tok, L, kv, _) in zip(rids, caps, hist):
        kvf = T.int4_round(bf16_bits_to_f32(kv))
        ref = T.decode_from_history(om, kvf[:, 0], kvf[:, 1], tok, L, int4_kv=True)
        err = float(np.abs(cap.reshape(3, -1)[0] - ref).max())
        say(f"history {L} hd {hd}: {err:.2e}")
        assert err <= INT4_TOL
        assert toks[rid][0] == cap.reshape(3, -1)[0].argmax()


def check_scores(logits, toks, arrays, k):
    lp, H, ids, tops = arrays
    x = logits.astype(np.float64)
    d = x - x.max(1, keepdims=True)
    ref = d - np.log(np.exp(d).sum(1, keepdims=True))
    r = np.arange(len(toks))
    assert np.abs(lp - ref[r, toks]).max() <= 2e-5
    assert np.abs(H + (np.exp(ref) * ref).sum(1)).max() <= 2e-5 * (1 + math.log(x.shape[1]))
    assert ids.shape == tops.shape == (len(toks), k)
    order = np.argsort(-x, axis=1, kind="stable")[:, :k]
    assert np.array_equal(ids, order)
    if k:
        assert np.abs(tops - np.take_along_axis(ref, order, 1)).max() <= 2e-5
        assert np.array_equal(ids[:, 0], toks) and np.array_equal(tops[:, 0], lp)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_scores_of_requests(on_gpu, dtype):
    """Some requests of a batch ask, with different numbers of alternatives; more gaps between them than launches; the
    others' steps and tokens are as without."""
    sh = shape(4, 2, 64, layers=1, vocab=2048)
    ws = [weights(sh, dtype, s) for s in (16, 17)]
    rng = np.random.default_rng(9)
    reqs = [(rng.integers(0, sh.vocab, 1 + i % 5), i % 2, 2 + i % 7) for i in range(40)]
    ask = [(None, 4, None, 0, 32)[i % 5] for i in range(40)]
    out = []
    for flag, scores in ((True, ask), (False, None)):
        eng = Engine(sh, dtype, EngineConsts(128, 40, 256, 64), 2, scores=flag)
        for w in ws:
            eng.load(pack_blob(w, sh))
        out.append(serve(eng, reqs, scores=scores))
        if not flag:
            rid = eng.submit(np.arange(3, dtype=np.int32), 0, 2)
            with pytest.raises(M.MoaError) as err:
                eng.request_scores(rid, 1)
            assert err.value.code == M.MOA_ESTATE
        else:
            rid = eng.submit(np.arange(3, dtype=np.int32), 0, 4)
            eng.step()
            with pytest.raises(M.MoaError) as err:
                eng.request_scores(rid, 1)                # its prompt has been processed
            assert err.value.code == M.MOA_ESTATE
            with pytest.raises(M.MoaError):
                eng.request_scores(rid, 33)
        eng.close()
    for i, k in enumerate(ask):
        assert np.array_equal(out[0][0][i], out[1][0][i]) and np.array_equal(out[0][1][i], out[1][1][i])
        if k is not None:
            check_scores(out[0][1][i], out[0][0][i], out[0][2][i], k)


@gpu
def test_scores_of_a_feeder_run(on_gpu):
    """Scores asked for as calls are submitted, collected step by step over more steps than staging slots."""
    from types import SimpleNamespace

    from paper_2606_03014_amd import run_feeder
    sh = shape(4, 2, 64, layers=1, vocab=1024)
    eng = Engine(sh, "bf16", EngineConsts(256, 6, 64, 128), 3, kv_int4=True, scores=True)
    for s in (18, 19, 20):
        eng.load(pack_blob(weights(sh, "bf16", s), sh))
    rng = np.random.default_rng(2)
    wl = SimpleNamespace(prompts=[rng.integers(0, sh.vocab, n).astype(np.int32) for n in (5, 40, 17, 9, 22)], experts=[(0, 1)] * 5,
                         n_queries=5, n_experts=2, agg_max_new=12, expert_requests=lambda: [(q, e, 4 + 3 * q) for q in range(5) for e in range(2)])
    got, caps = {}, {}

    def on_submit(rid, q, model, G):
        got[q, model] = eng.request_scores(rid, 2)
        caps[q, model] = np.full(G * sh.vocab, np.nan, np.float32)
        eng.capture_logits(rid, caps[q, model])

    res = run_feeder(eng, wl, [0, 1], agg_model=2, on_submit=on_submit)
    eng.sync()
    assert len(got) == 15 and len(res.outputs) == 15
    for key, toks in res.outputs.items():
        check_scores(caps[key].reshape(len(toks), -1), toks, got[key], 2)
    eng.close()
