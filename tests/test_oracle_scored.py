"""CPU checks of the definitions of scores of the caller's and shared beginnings, and of what the binding does by itself."""
import ctypes
import gc
import math
import weakref

import numpy as np
import pytest

import oracle
from helpers import load_binding
from oracle import drafts, scored


def _cache(rng, bt, hkv, n, scale=1.0):
    oc = oracle.OracleLayerCache(bt, hkv)
    if n:
        oc.append((rng.standard_normal((bt, hkv, n, 128)) * scale).astype(np.float16), rng.standard_normal((bt, hkv, n, 128)).astype(np.float16))
    return oc


def _drafts(rng, bt, hkv, n):
    return tuple(rng.standard_normal((bt, hkv, n, 128)).astype(np.float16) for _ in range(2))


@pytest.mark.parametrize("n_tokens", [0, 7, 53])
def test_the_plain_scores_are_those_of_drafted_tokens(n_tokens):
    rng = np.random.default_rng(n_tokens)
    oc, n = _cache(rng, 2, 1, n_tokens), 5
    q = rng.standard_normal((2, n, 2, 128)).astype(np.float16)
    kd, vd = _drafts(rng, 2, 1, n)
    seen = np.stack([drafts.ancestors([-1, 0, 0, 1, 1])] * 2)
    a = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    b = scored.decode(None, oc, q, kd, vd, seen, oracle.Tolerances())
    for x, y in zip((r for s in a for m in s for r in m), (r for s in b for m in s for r in m)):
        for f in x:
            assert np.allclose(x[f], y[f], rtol=1e-12, atol=1e-15), f


def _originals(shared, oc, kd, vd, b, h):
    each = oc.bt // shared.bt if shared is not None else 1
    k, v = [oc.k16[b, h], kd[b, h]], [oc.v16[b, h], vd[b, h]]
    if shared is not None:
        k.insert(0, shared.k16[b // each, h])
        v.insert(0, shared.v16[b // each, h])
    return np.concatenate(k).astype(np.float64), np.concatenate(v).astype(np.float64)


@pytest.mark.parametrize("beginning,n_tokens,cap,biased,scale,keys", [
    (0, 48, 5.0, False, 0.0, 1.0), (0, 53, 0.5, True, 0.3, 3.0), (35, 20, 2.0, True, 0.0, 1.0), (64, 0, 0.0, True, 0.0, 1.0), (17, 33, 30.0, False, 1.0, 2.0)])
def test_the_certificate_bounds_the_distance_to_attention_on_the_originals(beginning, n_tokens, cap, biased, scale, keys):
    """Sequences of two beginnings, spans that begin and end inside blocks."""
    rng = np.random.default_rng(beginning + n_tokens)
    shared = _cache(rng, 2, 1, beginning, keys) if beginning else None
    oc, n = _cache(rng, 4, 1, n_tokens, keys), 3
    q = rng.standard_normal((4, n, 2, 128)).astype(np.float16)
    kd, vd = _drafts(rng, 4, 1, n)
    seen = np.tile(np.tril(np.ones((n, n), bool)), (4, 1, 1))
    total = beginning + n_tokens
    spans = np.sort(rng.integers(0, total + 1, (4, n, 4)), axis=-1)
    slopes = np.array([0.3, -0.02], np.float32) if biased else None
    res = scored.decode(shared, oc, q, kd, vd, seen, oracle.Tolerances(), scale, cap, slopes, None, spans)
    for b in range(4):
        k, v = _originals(shared, oc, kd, vd, b, 0)
        for i in range(n):
            j = np.arange(total + n)
            s = spans[b, i]
            at = np.where(j < total, ((j >= s[0]) & (j < s[1])) | ((j >= s[2]) & (j < s[3])), j - total <= i)
            for h in range(2):
                x = (k @ q[b, i, h].astype(np.float64)) * (scale or 128 ** -0.5)
                x = cap * np.tanh(x / cap) if cap else x
                if biased:
                    x = x - float(slopes[h]) * np.abs(total + i - j)
                w = np.exp(x[at] - x[at].max())
                r = res[b][i][h]
                assert np.linalg.norm(r["O"] - (w / w.sum()) @ v[at]) <= r["E_key"] + r["E_val"] + 1e-9


def test_a_cap_narrows_differences_of_scores_by_the_bound():
    rng = np.random.default_rng(5)
    a, b = rng.standard_normal(100000) * 20, rng.standard_normal(100000) * 20
    for cap in (0.1, 3.0, 50.0):
        far = np.abs(cap * np.tanh(a / cap) - cap * np.tanh(b / cap))
        assert (far <= 2 * cap * np.tanh(np.abs(a - b) / (2 * cap)) * (1 + 1e-12)).all()
        assert np.isclose(2 * cap * np.tanh(1.0 / (2 * cap)), cap * np.tanh(0.5 / cap) - cap * np.tanh(-0.5 / cap))


def test_rows_that_attend_nothing():
    rng = np.random.default_rng(9)
    oc = _cache(rng, 1, 1, 20)
    q = rng.standard_normal((1, 2, 1, 128)).astype(np.float16)
    spans = np.array([[[5, 5, 9, 3], [0, 0, 4, 5]]])
    r = scored.decode(None, oc, q, None, None, None, oracle.Tolerances(), spans=spans)[0]
    assert r[0][0]["lse"] == -math.inf and (r[0][0]["O"] == 0).all() and r[0][0]["flags"] == 0
    v = drafts.to_fp16(drafts.read_back(oc, 0, 20)[1])[0, 0, 4]
    assert np.allclose(r[1][0]["O"], v.astype(np.float64))


def test_calls_without_handles_are_refused():
    """On the host, before anything is read: the addresses are not."""
    cqa = load_binding()
    n = ctypes.c_int64(0)
    tol, s = cqa.Tolerances(), cqa.Scoring()
    lib = cqa._lib
    assert lib.cqa_scored_workspace_bytes(None, 1, ctypes.byref(n)) == cqa.ERR_INVALID_ARG
    assert lib.cqa_prefix_workspace_bytes(None, None, 1, ctypes.byref(n)) == cqa.ERR_INVALID_ARG
    args = (4096, 4096, 4096, 1, None, ctypes.byref(s), ctypes.byref(tol), 4096, 4096, 4096, 4096, None)
    assert lib.cqa_scored_decode(None, 0, *args) == cqa.ERR_INVALID_ARG
    assert lib.cqa_prefix_decode(None, None, 0, *args) == cqa.ERR_INVALID_ARG
    assert ctypes.sizeof(cqa.Scoring) == 32


def test_a_scoring_keeps_its_tensors():
    import torch
    cqa = load_binding()
    spans = torch.zeros((1, 1, 4), dtype=torch.int64)
    ref, at = weakref.ref(spans), spans.data_ptr()
    s = cqa.Scoring(spans_dev=spans)
    del spans
    gc.collect()
    assert ref() is not None and s.spans_dev == at and s.slopes_dev is None
    del s
    gc.collect()
    assert ref() is None
