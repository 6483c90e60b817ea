"""Drafted tokens over the cache where attention and its certificate are most easily wrong: against oracle/drafts.py, with the tolerances of
test_gpu_drafts.py."""
import functools
import math

import numpy as np
import pytest

import oracle
import workloads
from helpers import GpuLayerCache
from oracle import drafts, quantizer
from test_gpu_drafts import assert_nodes, random_tree, tree_call

pytestmark = pytest.mark.gpu


def sequences(x, bt):
    """Up to four sequences over and over."""
    return np.tile(x, ((bt + len(x) - 1) // len(x),) + (1,) * (x.ndim - 1))[:bt]


# 33 .. 64, 65 .. 128 and up to 256 rows; a workgroup has a sequence, more than 64 blocks of it and not a multiple of 32
@pytest.mark.parametrize("n,n_tokens", [(13, 1157), (13, 1293), (27, 1093), (27, 1347), (64, 1093), (64, 1285)])
def test_widths_of_two_blocks_do_not_meet(n, n_tokens):
    """The first blocks are wide in one half of the channels, all others in the other half: a Delta over channels of two blocks is up to
    twice that of any block."""
    print("tree widths", n, n_tokens, flush=True)
    rng = np.random.default_rng(60 + n_tokens)
    bt = 256 if n * 4 <= 64 else 160
    k = rng.standard_normal((4, 1, n_tokens, 128)) * 0.05
    k[:, :, :64, :64] *= 20.0
    k[:, :, 64:, 64:] *= 20.0
    k, kd = k.astype(np.float16), workloads.normal_f16(rng, (4, 1, n, 128))
    v, vd = workloads.normal_f16(rng, (4, 1, n_tokens, 128)), workloads.normal_f16(rng, (4, 1, n, 128))
    q = workloads.normal_f16(rng, (4, n, 4, 128))
    seen = random_tree(rng, 4, n)
    nodes = np.unique([0, 1, n // 2, n - 1])
    oc = oracle.OracleLayerCache(4, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q[:, nodes], kd, vd, seen[:, nodes], oracle.Tolerances())
    with GpuLayerCache(bt, 4, 1, n_tokens, tier2=False) as gc:
        gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)))
    for at in range(4):
        for y in (O, flags, *cert.values()):
            assert all(np.array_equal(z, y[at]) for z in y[at::4])
        assert_nodes(ref[at:at + 1], O[at:at + 1, nodes], {f: y[at:at + 1, nodes] for f, y in cert.items()}, flags[at:at + 1, nodes], at)


SCORE = 1.0 / math.sqrt(128.0)


def determined(oc, q, kd, seen, scale):
    """bool [Bt, n, Hq]: rows whose result FP32 sums of products determine.  A score of 128 products is off by at most 128 * 2^-23 sum |q k|;
    the largest one has to be beyond twice that, and 30 (e^-30 = 1e-13) on top, of the next -- or to be the same number by its keys."""
    k_all, _ = drafts.read_back(oc, 0, oc.length)
    bt, n, hq, _ = q.shape
    g = hq // oc.hkv
    out = np.ones((bt, n, hq), bool)
    for b, i, h in np.ndindex(bt, n, hq):
        k = np.concatenate([drafts.to_fp16(k_all[b, h // g]), kd[b, h // g][seen[b, i]]]).astype(np.float64)
        x = q[b, i, h].astype(np.float64)
        s = (k @ x) * SCORE
        if len(s) < 2 or np.abs(s).max() < 1000.0:
            continue
        off = 128 * 2.0 ** -23 * (np.abs(k) @ np.abs(x)).max() * SCORE
        near = s >= s.max() - 2 * off - 30.0
        out[b, i, h] = (k[near] == k[near][0]).all()
    return out


# few rows; 64, 128 and 256 rows by a workgroup; several tokens' turns; nothing sealed
LARGE = [(1, 1, 6, 0), (2, 1, 6, 37), (1, 2, 27, 700), (1, 1, 4, 3001), (256, 1, 13, 1157), (160, 1, 27, 613), (160, 1, 64, 203)]


@pytest.mark.parametrize("scale", [400.0, 2000.0, 8000.0, 50000.0, -2000.0, -50000.0])
@pytest.mark.parametrize("bt,hkv,n,n_tokens", LARGE)
def test_large_keys_meet_large_queries(bt, hkv, n, n_tokens, scale):
    """Scores up to 2^35 of either sign: of FP32's spacing there, the largest weight must not be more than FP16 holds, nor nothing.  Every other
    head has ordinary scores over the same keys."""
    print("tree large scores", bt, hkv, n, n_tokens, scale, flush=True)
    rng = np.random.default_rng(70 + n_tokens)
    few, size = min(bt, 4), abs(scale)
    u = rng.choice([-1.0, 1.0], 128)
    around = lambda shape: 1.0 + 0.1 * rng.standard_normal(shape)  # noqa: E731
    k, kd = (np.clip(u * size * around((few, hkv, m, 128)), -65504.0, 65504.0).astype(np.float16) for m in (n_tokens, n))
    v, vd = (workloads.normal_f16(rng, (few, hkv, m, 128)) for m in (n_tokens, n))
    q = np.clip(u * scale * around((few, n, hkv * 4, 128)), -65504.0, 65504.0)
    q[:, :, 1::2] *= 20.0 / (128.0 * size * size) / SCORE
    q = q.astype(np.float16)
    seen = random_tree(rng, few, n)
    nodes = np.unique([0, 1, n // 2, n - 1])
    oc = oracle.OracleLayerCache(few, hkv)
    oc.append(k, v)
    tol = oracle.Tolerances(key_bound_mode=2)
    ref = drafts.tree_decode(oc, q[:, nodes], kd, vd, seen[:, nodes], tol)
    clear = determined(oc, q[:, nodes], kd, seen[:, nodes], scale)
    assert clear.mean() > 0.9
    with GpuLayerCache(bt, hkv * 4, hkv, max(n_tokens, 16), tier2=False) as gc:
        if n_tokens:
            gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)),
                                   gc.cqa.Tolerances(key_bound_mode=2))
    assert np.isfinite(O).all() and all(np.isfinite(x).all() for x in cert.values()) and not (flags & oracle.FLAG_PRECOND).any()
    for b, i, h in np.ndindex(few, len(nodes), hkv * 4):
        if clear[b, i, h]:
            at = (slice(b, b + 1), slice(nodes[i], nodes[i] + 1), slice(h, h + 1))
            assert_nodes([[[ref[b][i][h]]]], O[at], {f: y[at] for f, y in cert.items()}, flags[at], (b, nodes[i], h))


# nothing sealed; one workgroup, some, more than 16 and more than 32 of few rows; 64, 128 and 256 rows, by one workgroup and by some
@pytest.mark.parametrize("bt,hkv,n,n_tokens", [(2, 1, 6, 0), (1, 2, 70, 0), (1, 1, 6, 5), (1, 1, 6, 200), (1, 1, 7, 2003), (1, 2, 30, 6000), (1, 1, 6, 12000),
                                               (256, 1, 13, 1030), (96, 1, 27, 1001), (160, 1, 64, 203), (4, 1, 64, 10029)])
def test_queries_that_are_not_finite(bt, hkv, n, n_tokens):
    """All scores of such a row can be -inf, which leaves its weights nothing as an empty mask does: only the latter is an answer."""
    print("tree queries not finite", bt, hkv, n, n_tokens, flush=True)
    rng = np.random.default_rng(80 + n_tokens)
    few = min(bt, 2)
    k, kd = (workloads.normal_f16(rng, (few, hkv, m, 128)) for m in (n_tokens, n))
    v, vd = (workloads.normal_f16(rng, (few, hkv, m, 128)) for m in (n_tokens, n))
    k[..., 7], kd[..., 7] = np.float16(0.5), np.float16(0.5)
    q = workloads.normal_f16(rng, (few, n, hkv * 4, 128))
    seen = random_tree(rng, few, n)
    seen[:, n // 2] = False
    hit = np.zeros((few, n, hkv * 4), bool)
    for i, x in ((0, -np.inf), (1, np.inf), (2, np.nan), (n - 1, -np.inf), (n // 2, -np.inf)):
        q[:, i, 1, 7] = x
        hit[:, i, 1] = True
    if n_tokens == 0:   # this node attends nothing, whatever its query
        hit[:, n // 2] = False
    nodes = np.unique([0, 1, 2, n // 2, n - 1])
    oc = oracle.OracleLayerCache(few, hkv)
    oc.append(k, v)
    plain = np.where(np.isfinite(q), q, np.float16(0.0))
    ref = drafts.tree_decode(oc, plain[:, nodes], kd, vd, seen[:, nodes], oracle.Tolerances())
    with GpuLayerCache(bt, hkv * 4, hkv, max(n_tokens, 16), tier2=False) as gc:
        if n_tokens:
            gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)))
    for b, i, h in np.ndindex(few, len(nodes), hkv * 4):
        at = (slice(b, b + 1), slice(nodes[i], nodes[i] + 1), slice(h, h + 1))
        if hit[b, nodes[i], h]:
            assert np.isnan(O[at]).all() and (flags[at] & oracle.FLAG_PRECOND).all(), at
            assert np.isnan(cert["lse"][at]).all(), at
        else:
            assert_nodes([[[ref[b][i][h]]]], O[at], {f: y[at] for f, y in cert.items()}, flags[at], (b, nodes[i], h))
    if n_tokens == 0:
        assert (O[:, n // 2] == 0).all() and (cert["lse"][:, n // 2] == -math.inf).all() and (flags[:, n // 2] == 0).all()


@pytest.mark.parametrize("bt,hkv,n,n_tokens", [(1, 4, 26, 2053), (256, 1, 13, 1157), (96, 1, 27, 1001), (160, 1, 64, 427)])
def test_outlier_channels_and_peaked_queries(bt, hkv, n, n_tokens):
    """Keys of 20 to 80 and queries of 3 to 9: one step of FP16 of one key is up to 4 % of its weight."""
    print("tree outliers", bt, hkv, n, n_tokens, flush=True)
    rng = np.random.default_rng(90 + n_tokens)
    few = min(bt, 4)
    k, kd = (rng.standard_normal((few, hkv, m, 128)) for m in (n_tokens, n))
    k[..., 11::32] *= 20.0
    kd[..., 11::32] *= 20.0
    k, kd = k.astype(np.float16), kd.astype(np.float16)
    v, vd = (workloads.normal_f16(rng, (few, hkv, m, 128)) for m in (n_tokens, n))
    q = rng.standard_normal((few, n, hkv * 4, 128))
    q[:, :, ::2] *= 3.0
    q = q.astype(np.float16)
    seen = random_tree(rng, few, n)
    nodes = np.arange(n) if bt == 1 else np.unique([0, 1, n // 3, n // 2, n - 2, n - 1])
    oc = oracle.OracleLayerCache(few, hkv)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q[:, nodes], kd, vd, seen[:, nodes], oracle.Tolerances())
    with GpuLayerCache(bt, hkv * 4, hkv, n_tokens, tier2=False) as gc:
        gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)))
    assert_nodes(ref, O[:few, nodes], {f: y[:few, nodes] for f, y in cert.items()}, flags[:few, nodes])


@functools.lru_cache
def columns_at_a_border(count):
    """[16, count] FP16 keys of one channel and block, one of them, near the largest, reconstructed to another FP16 number where the product
    code sigma is rounded before z is added: the definition rounds the sum once."""
    found, rng = [], np.random.default_rng(101)
    for _ in range(40):
        k = (rng.standard_normal((100000, 16, 1)) * 20.0).astype(np.float16)
        codes, sigma, z = quantizer.quantize_key_blocks(k)
        once = quantizer.dequantize_keys(codes, sigma, z).astype(np.float32)[:, :, 0]
        twice = (codes.astype(np.float32) * sigma[:, None] + z[:, None])[:, :, 0]
        told = (once.astype(np.float16) != twice.astype(np.float16)) & (once >= 16.0) & (once >= once.max(1, keepdims=True) - 12.0)
        found.append(k[told.any(1), :, 0].T)
    found = np.concatenate(found, 1)
    assert found.shape[1] >= count, found.shape
    return found[:, :count]


@pytest.mark.parametrize("bt,n_tokens", [(1, 16), (1, 100), (256, 1157)])
def test_keys_are_rounded_once(bt, n_tokens):
    """A key at a border of FP16 in each of 32 channels, rows that ask for one channel, and values that show every weight of the first block."""
    print("tree rounding", bt, n_tokens, flush=True)
    rng = np.random.default_rng(100)
    n = 13
    k, kd = (workloads.normal_f16(rng, (1, 1, m, 128)) for m in (n_tokens, n))
    k[0, 0, :16, :32] = columns_at_a_border(32)
    v, vd = np.zeros((1, 1, n_tokens, 128), np.float16), np.zeros((1, 1, n, 128), np.float16)
    v[0, 0, np.arange(128) // 8, np.arange(128)] = 1.0
    q = np.zeros((1, n, 4, 128), np.float16)
    q.reshape(4 * n, 128)[np.arange(4 * n), np.arange(4 * n) % 32] = 3.0
    seen = np.eye(n, dtype=bool)[None]
    oc = oracle.OracleLayerCache(1, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    # with the other rounding, a step of FP16 from 2^-6 on, every row is further off than it may be
    with pytest.MonkeyPatch.context() as m:
        m.setattr(quantizer, "dequantize_keys", lambda codes, sigma, z: codes.astype(np.float32) * sigma[..., None, :] + z[..., None, :])
        wrong = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    for r, w in zip(sum(ref[0], []), sum(wrong[0], [])):
        assert (np.abs(w["O"] - r["O"]) > 2.0 ** -11 * np.abs(r["O"]) + (2.0 ** -11 + 1e-4) * r["spread"] + 2.0 ** -25 * r["floor"]).any()
    with GpuLayerCache(bt, 4, 1, n_tokens, tier2=False) as gc:
        gc.append(sequences(k, bt), sequences(v, bt))
        O, cert, flags = tree_call(gc, sequences(q, bt), sequences(kd, bt), sequences(vd, bt), drafts.mask_words(sequences(seen, bt)))
    assert_nodes(ref, O[:1], {f: y[:1] for f, y in cert.items()}, flags[:1])
    for y in (O, flags, *cert.values()):
        assert all(np.array_equal(z, y[0]) for z in y)


@pytest.mark.parametrize("n_tokens", [48, 704, 5008])
def test_sealed_tokens_too_light_for_fp32_still_have_a_key_error(n_tokens):
    """Each node's draft is 150 above all sealed scores, which are themselves off by up to Delta = 50 and more: their mass, e^-150, is nothing in
    FP32, but e^(4 Delta) times that is not."""
    print("tree light sealed tokens", n_tokens, flush=True)
    rng = np.random.default_rng(110 + n_tokens)
    n = 5
    k, v = ((rng.standard_normal((1, 1, n_tokens, 128)) * s).astype(np.float16) for s in (32.0, 1.0))
    q = (rng.standard_normal((1, n, 1, 128)) * 32.0).astype(np.float16)
    oc = oracle.OracleLayerCache(1, 1)
    oc.append(k, v)
    sealed = drafts.read_back(oc, 0, n_tokens)[0][0, 0].astype(np.float64)
    x = q[0, :, 0].astype(np.float64)
    top = (x @ sealed.T).max(1) * SCORE
    kd = (x * ((top + 150.0) / SCORE / (x * x).sum(1))[:, None]).astype(np.float16)[None, None]
    vd = workloads.normal_f16(rng, (1, 1, n, 128))
    seen = np.eye(n, dtype=bool)[None]
    tol = oracle.Tolerances(eps_key=0.01)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, tol)
    for r in ref[0]:
        assert r[0]["delta_h"] > 45.0 and 1e-80 < r[0]["alpha_tail_hat"] < 1e-45 and r[0]["E_key"] == 2 * r[0]["v_max"] and r[0]["flags"] & oracle.FLAG_KEY
    with GpuLayerCache(1, 1, 1, n_tokens, tier2=False) as gc:
        gc.append(k, v)
        assert_nodes(ref, *tree_call(gc, q, kd, vd, drafts.mask_words(seen), gc.cqa.Tolerances(eps_key=0.01)))
