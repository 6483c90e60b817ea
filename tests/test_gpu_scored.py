"""Nodes with scores of the caller's and sequences behind a shared beginning, against the 64-bit definition of oracle/scored.py.

Tolerances as in test_gpu_drafts.py: O its own rounding 2^-11 |O|, the weights' 2^-11 sum a |v| and 2^-25 count max |v| / sum exp(s - max), and the
library's bar for the certificate, 1e-4, for the scores' FP32 arithmetic: 1e-4 sum a |v|.  A cap's tanh is off by 2^-24 of 2 cap with a cap up to 256
(3e-5) and relatively by 2^-22 beyond; a bias counts from the row's nearest token.  Certificate: 1e-4 relative (lse: 1e-4 max(1, |lse|))."""
import math

import numpy as np
import pytest

import oracle
import workloads
from helpers import GpuLayerCache, load_binding
from oracle import drafts, scored
from test_gpu_drafts import NODE_FIELDS, _off, assert_nodes, random_tree

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


class Call:
    """Outputs with guard rows behind them, a workspace whose every byte is set, and the inputs of one call."""

    def __init__(self, shared, gc, q, kd=None, vd=None, mask=None, scale=0.0, cap=0.0, slopes=None, places=None, spans=None, tol=None, layer=0, by=0,
                 plain=False):
        t, cqa = gc.torch, gc.cqa
        bt, n, hq, _ = q.shape
        self.cqa, self.gc, self.shared, self.shape, self.layer = cqa, gc, shared, (bt, n, hq), layer
        rows = bt * n * hq
        self.O = t.full((rows + 4, 128), 7.0, dtype=t.float16, device="cuda")
        self.cert = t.full((rows + 4, 8), 7.0, device="cuda")
        self.flags = t.full((rows + 4,), 77, dtype=t.int32, device="cuda")
        size = cqa.cqa_prefix_workspace_bytes(shared.h, gc.h, n) if shared is not None else cqa.cqa_scored_workspace_bytes(gc.h, n)
        self.ws_bytes = size
        self.ws = t.full((size + 256,), 0xFF, dtype=t.uint8, device="cuda")
        self.inputs = [None if x is None else _off(x, by) for x in (q, kd, vd)]
        self.mask = None if mask is None else t.from_numpy(np.ascontiguousarray(mask).view(np.int64)).cuda()
        dev = lambda x, d: None if x is None else t.from_numpy(np.ascontiguousarray(x, dtype=d)).cuda()  # noqa: E731
        self.slopes, self.places, self.spans = dev(slopes, np.float32), dev(places, np.int64), dev(spans, np.int64)
        self.scoring = None if plain else cqa.Scoring(scale, cap, self.slopes, self.places, self.spans)
        self.tol = tol or cqa.Tolerances()
        t.cuda.synchronize()

    def enqueue(self, stream=None):
        rest = (self.layer, *self.inputs, self.shape[1], self.mask, self.scoring, self.tol, self.O, self.cert, self.flags, self.ws, stream)
        if self.shared is not None:
            self.cqa.cqa_prefix_decode(self.shared.h, self.gc.h, *rest)
        else:
            self.cqa.cqa_scored_decode(self.gc.h, *rest)

    def results(self):
        t = _torch()
        t.cuda.synchronize()
        rows = int(np.prod(self.shape))
        assert (self.O[rows:] == 7.0).all() and (self.cert[rows:] == 7.0).all() and (self.flags[rows:] == 77).all()
        assert (self.ws[self.ws_bytes:] == 0xFF).all()
        cert = self.cert[:rows].cpu().numpy().reshape(self.shape + (8,))
        return (self.O[:rows].cpu().numpy().astype(np.float64).reshape(self.shape + (128,)),
                {n: cert[..., i].astype(np.float64) for i, n in enumerate(NODE_FIELDS)},
                self.flags[:rows].cpu().numpy().view(np.uint32).reshape(self.shape))


def call(shared, gc, q, *args, **kw):
    c = Call(shared, gc, q, *args, **kw)
    c.enqueue()
    return c.results()


def same(x, y):
    return all(np.array_equal(a, b, equal_nan=True) if not isinstance(a, dict) else all(np.array_equal(a[f], b[f], equal_nan=True) for f in a) for a, b in zip(x, y))


def make_spans(rng, kind, bt, n, total, places):
    """None, or int64 [bt][n][4]."""
    s = np.zeros((bt, n, 4), np.int64)
    if kind == "all":
        return None
    if kind == "window":
        s[..., 1] = min(3, total)
        s[..., 2], s[..., 3] = np.maximum(places - max(1, total // 3), 0), total
    elif kind == "padded":
        s[..., 2], s[..., 3] = rng.integers(0, total + 1, (bt, 1)), total
        s[-1] = 0
    elif kind == "sorted":     # two pieces that begin and end anywhere
        s = np.sort(rng.integers(0, total + 1, (bt, n, 4)), axis=-1)
    elif kind == "any":        # overlapping, empty, turned round, beyond the cached tokens
        s = rng.integers(-20, total + 40, (bt, n, 4))
        s[0, 0] = [0, 1, total - 1, total]
        if n > 1:
            s[0, 1] = [-5, 10 ** 12, 4, 2]
        if n > 2:
            s[0, 2] = [7, 3, -9 * 10 ** 15, 0]
    return s.astype(np.int64)


def make(rng, bt, hkv, g, tokens, n, drafted, keys="normal", peak=1.0, shared=0, beginning=0):
    draw = workloads.student_t3_f16 if keys == "student" else workloads.normal_f16
    x = dict(k=draw(rng, (bt, hkv, tokens, 128)), v=workloads.normal_f16(rng, (bt, hkv, tokens, 128)),
             q=workloads.normal_f16(rng, (bt, n, hkv * g, 128)), kd=None, vd=None)
    x["q"][:, :, ::2] *= np.float16(peak)
    if drafted:
        x["kd"], x["vd"] = draw(rng, (bt, hkv, n, 128)), workloads.normal_f16(rng, (bt, hkv, n, 128))
    if shared:
        x["sk"], x["sv"] = draw(rng, (shared, hkv, beginning, 128)), workloads.normal_f16(rng, (shared, hkv, beginning, 128))
    return x


class Caches:
    """The device's and the oracle's caches of one layer, the shared beginning's among them."""

    def __init__(self, x, g, room=16):
        bt, hkv, tokens = x["k"].shape[:3]
        self.gc = GpuLayerCache(bt, hkv * g, hkv, tokens + room, tier2=False)
        self.oc = oracle.OracleLayerCache(bt, hkv)
        self.shared = self.shared_oc = None
        if "sk" in x:
            count, _, beginning = x["sk"].shape[:3]
            self.shared = GpuLayerCache(count, hkv * g, hkv, max(beginning, 1), tier2=False)
            self.shared_oc = oracle.OracleLayerCache(count, hkv)
        for gc, oc, k, v in ((self.gc, self.oc, x["k"], x["v"]), (self.shared, self.shared_oc, x.get("sk"), x.get("sv"))):
            if gc is not None and k.shape[2]:
                gc.append(k, v)
                oc.append(k, v)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.gc.close()
        if self.shared is not None:
            self.shared.close()


def compare(x, g, seen, where, by=False, nodes=None, **score):
    """The call against the definition; `nodes`: those the definition is asked for."""
    with Caches(x, g) as c:
        mask = None if seen is None else drafts.mask_words(seen)
        gpu = dict(score)
        got = call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, **gpu)
        ref_seen = seen
        n = x["q"].shape[1]
        if x["kd"] is not None and seen is None:
            ref_seen = np.tile(np.tril(np.ones((n, n), bool)), (x["q"].shape[0], 1, 1))
        ref = scored.decode(c.shared_oc, c.oc, x["q"], x["kd"], x["vd"], ref_seen, oracle.Tolerances(), **score)
        assert_nodes(ref, *got, where)
        if by:   # at any address an FP16 number may have: the same bits
            assert same(got, call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, by=1, **gpu))
    return got


def slopes_of(hq, kind):
    s = 2.0 ** (-8.0 * (np.arange(hq) + 1.0) / hq)
    return None if kind == 0 else (s * (np.where(np.arange(hq) % 2, -0.05, 1.0) if kind < 0 else 1.0)).astype(np.float32)


# few rows; 33 .. 64, 65 .. 128, up to 256 rows and several tiles of 256; no block, ragged ends; every kind of score
CASES = [
    (1, 1, 1, 0, 1, "tree", 0.0, 0, "all"), (1, 1, 4, 1, 1, None, 5.0, 1, "all"), (1, 1, 4, 1029, 1, None, 50.0, 0, "all"),
    (2, 2, 2, 777, 1, None, 3.0, 1, "window"), (3, 1, 4, 333, 5, "tree", 0.0, 1, "padded"), (1, 2, 4, 16, 3, "chunk", 30.0, -1, "any"),
    (1, 2, 1, 700, 26, "tree", 2.0, 1, "sorted"), (1, 1, 4, 333, 13, "tree", 20.0, 1, "any"), (1, 1, 4, 700, 27, "tree", 10.0, 0, "window"),
    (1, 1, 4, 2101, 16, "chunk", 30.0, -1, "sorted"), (2, 1, 2, 257, 100, "tree", 50.0, 1, "any"), (1, 1, 1, 100, 256, "chunk", 1e5, 1, "all"),
    (1, 1, 4, 81, 256, "chunk", 1.0, 0, "padded"), (1, 1, 4, 1500, 64, "tree", 300.0, 1, "sorted"), (1, 1, 2, 4099, 1, None, 0.5, -1, "any"),
    (8, 2, 1, 143, 2, "tree", 0.0, 1, "padded"), (5, 3, 1, 31, 7, "tree", 7.0, 0, "any"), (1, 2, 2, 160, 63, "chunk", 0.0, 1, "window"),
]


@pytest.mark.parametrize("bt,hkv,g,tokens,n,kind,cap,bias,spans", CASES)
def test_scores_match_the_definition(bt, hkv, g, tokens, n, kind, cap, bias, spans):
    print("scored", bt, hkv, g, tokens, n, kind, cap, bias, spans, flush=True)
    rng = np.random.default_rng(1000 * tokens + n)
    x = make(rng, bt, hkv, g, tokens, n, kind is not None, "student" if n % 2 else "normal", 4.0 if n % 3 == 0 else 1.0)
    seen = random_tree(rng, bt, n) if kind == "tree" else None
    places = scored.default_places(bt, n, tokens, kind is not None)
    sp = make_spans(rng, spans, bt, n, tokens, places)
    if kind == "tree":
        places = tokens + seen.sum(-1) - 1
    compare(x, g, seen, (tokens, n), by=n < 8, scale=0.05 if n % 2 else 0.0, cap=cap, slopes=slopes_of(hkv * g, bias), places=places if bias and kind == "tree" else None,
            spans=sp)


# (batch, beginnings, kv heads, group, their tokens, own tokens, nodes, kind, cap, bias, spans)
SHARED = [
    (1, 1, 1, 1, 1, 0, 1, None, 0.0, 0, "all"), (2, 1, 1, 4, 1029, 37, 1, None, 0.0, 0, "all"), (2, 2, 2, 4, 0, 100, 1, None, 0.0, 0, "all"),
    (4, 2, 1, 4, 500, 0, 1, None, 5.0, 1, "all"), (4, 2, 2, 2, 700, 90, 3, "tree", 0.0, 0, "all"), (9, 3, 1, 4, 333, 48, 5, "tree", 30.0, 1, "padded"),
    (16, 1, 1, 4, 1000, 17, 1, None, 0.0, 0, "all"), (40, 1, 1, 4, 2000, 33, 1, None, 50.0, 0, "padded"), (70, 1, 1, 4, 1100, 20, 1, None, 0.0, 0, "all"),
    (6, 2, 1, 2, 1200, 65, 30, "chunk", 3.0, -1, "sorted"), (3, 1, 2, 1, 100, 31, 40, "tree", 0.0, 1, "any"), (2, 1, 1, 4, 77, 900, 70, "chunk", 20.0, 0, "window"),
    (3, 3, 1, 4, 260, 5, 2, "chunk", 0.0, 0, "any"), (5, 1, 1, 1, 16, 16, 1, None, 4.0, 1, "any"), (2, 1, 1, 4, 300, 0, 4, "tree", 0.0, 0, "all"),
]


@pytest.mark.parametrize("bt,count,hkv,g,beginning,tokens,n,kind,cap,bias,spans", SHARED)
def test_sequences_behind_a_beginning_match_the_definition(bt, count, hkv, g, beginning, tokens, n, kind, cap, bias, spans):
    print("prefix", bt, count, hkv, g, beginning, tokens, n, kind, cap, bias, spans, flush=True)
    rng = np.random.default_rng(1000 * tokens + beginning)
    x = make(rng, bt, hkv, g, tokens, n, kind is not None, "student" if n % 2 else "normal", 3.0 if bt % 2 == 0 else 1.0, count, beginning)
    seen = random_tree(rng, bt, n) if kind == "tree" else None
    total = beginning + tokens
    places = scored.default_places(bt, n, total, kind is not None)
    sp = make_spans(rng, spans, bt, n, total, places)
    if seen is not None and spans == "padded":
        seen[-1] = False   # the last sequence is idle
    compare(x, g, seen, (beginning, tokens, n), by=bt < 4, cap=cap, slopes=slopes_of(hkv * g, bias), spans=sp)


@pytest.mark.parametrize("n,tokens", [(1, 400), (20, 400), (64, 1200)])
@pytest.mark.parametrize("cap,scale", [(2.0 ** -20, 0.0), (256.0, 2.0), (257.0, 2.0), (1e6, 0.0), (2.0 ** 60, 1.0), (0.0, 2.0 ** -40), (0.0, 20.0), (5.0, 2.0 ** 40)])
def test_the_ends_of_caps_and_scales(n, tokens, cap, scale):
    """A cap of 2^-20 makes all weights alike, one of 2^60 none; a scale of 2^40 saturates every score but those of q . k = 0."""
    print("caps", n, tokens, cap, scale, flush=True)
    rng = np.random.default_rng(7)
    x = make(rng, 1, 1, 4, tokens, n, True)
    if scale == 20.0:   # FP32 sums are off by some 2^-24 sum |q k|: 20 times that is below the bar for such queries
        x["q"] *= np.float16(0.25)
    compare(x, 4, None, (cap, scale), cap=cap, scale=scale)


# up to 16, 32, 64, 128 and 256 rows a workgroup; the last with the tokens as a beginning's
@pytest.mark.parametrize("n,bt,tokens,beginning", [(1, 1, 1300, 0), (8, 1, 1300, 0), (13, 256, 1300, 0), (27, 160, 1300, 0), (64, 160, 1300, 0), (64, 160, 40, 1300), (13, 160, 40, 1300)])
@pytest.mark.parametrize("cap", [30.0, 64.0, 250.0])
def test_a_cap_keeps_the_bits_of_small_scores(n, bt, tokens, beginning, cap):
    """Rows that attend two tokens each, whose q . k are whole numbers, so that the cap is what rounds.  A score is off by cap (2^-25 + |tanh| 2^-21), caps
    beyond 128 by the second alone (include/cqa.h): scale / cap, its product with q . k, 1 - E, 1 + E and the quotient by some 8 2^-24 of the tanh, E by half of 2^-24.  Two weights beside each other are off by twice that; their exponents of 2, of 14 at most, by half a step, 2^-21 ln 2, each, the exponentials by 2^-23 each; sum, quotient, the
    block's error and the product by 2^-24 each: 1.2e-6.  lse, besides its score's part, by a step of ln(2^15) = 10.4, 2^-20, and of the numbers taken off it, as large: 2e-6."""
    print("bits of caps", n, bt, tokens, beginning, cap, flush=True)
    rng = np.random.default_rng(n + beginning)
    g, scale = 4, 2.0 ** -4
    x = make(rng, 1, 1, g, tokens, n, False, shared=1 if beginning else 0, beginning=beginning)
    for name in ("k", "sk"):
        if name in x:
            x[name] = np.where(rng.random(x[name].shape) < 0.5, -1.0, 1.0).astype(np.float16)
    x["q"] = rng.integers(-2, 3, x["q"].shape).astype(np.float16)
    total = beginning + tokens
    keys = np.concatenate([x[name][0, 0] for name in ("sk", "k") if name in x]).astype(np.float64)
    with Caches(x, g) as c, Caches({k: again(v, bt) for k, v in x.items()}, g) as w:
        for turn in range(4):
            spans = np.zeros((1, n, 4), np.int64)
            spans[..., 0] = rng.integers(0, total // 2 - 16, (1, n))
            spans[..., 2] = rng.integers(total // 2, total // 16 * 16 if not beginning else total - 16, (1, n))
            spans[..., 1], spans[..., 3] = spans[..., 0] + 1, spans[..., 2] + 1
            ref = scored.decode(c.shared_oc, c.oc, x["q"], None, None, None, oracle.Tolerances(), scale=scale, cap=cap, spans=spans)[0]
            O, cert, flags = call(w.shared, w.gc, again(x["q"], bt), scale=scale, cap=cap, spans=again(spans, bt))
            for i in range(n):
                pair = keys[[spans[0, i, 0], spans[0, i, 2]]]
                for h in range(g):
                    r = ref[i][h]
                    most = float(np.tanh(np.abs(pair @ x["q"][0, i, h].astype(np.float64)) * scale / cap).max())
                    off = cap * ((2.0 ** -25 if cap <= 128 else 0.0) + most * 2.0 ** -21)
                    for field in ("alpha_tail_hat", "max_block_contrib", "E_val"):
                        tol = 2 * off + 1.2e-6
                        assert abs(cert[field][0, i, h] - r[field]) <= tol * r[field], (field, turn, i, h, cert[field][0, i, h] / r[field] - 1, tol)
                    assert abs(cert["lse"][0, i, h] - r["lse"]) <= off + 2e-6, (turn, i, h, cert["lse"][0, i, h] - r["lse"], off)
            assert (flags == 0).all() and all(np.array_equal(O[i], O[0]) for i in range(bt))


@pytest.mark.parametrize("n", [1, 20, 64])
@pytest.mark.parametrize("far", [0, 1000, 10 ** 6, 2 ** 29, 2 ** 33, -(2 ** 29), -(2 ** 40)])
def test_rows_that_attend_only_far_tokens_keep_their_weights(n, far):
    """Places far from every token attended, ahead of them and behind them, with slopes of either sign."""
    print("far", n, far, flush=True)
    rng = np.random.default_rng(abs(far) % 1000 + n)
    tokens = 700
    x = make(rng, 2, 1, 4, tokens, n, False)
    places = np.full((2, n), tokens + far, np.int64) + rng.integers(0, 5, (2, n))
    spans = make_spans(rng, "sorted", 2, n, tokens, places)
    slopes = np.array([0.5, 0.01, -0.02, 0.0], np.float32)
    limit = 2 ** 29
    held = np.clip(places, -limit, tokens + limit)
    with Caches(x, 4) as c:
        got = call(None, c.gc, x["q"], slopes=slopes, places=places, spans=spans)
        ref = scored.decode(None, c.oc, x["q"], None, None, None, oracle.Tolerances(), slopes=slopes, places=held, spans=spans)
        assert_nodes(ref, *got, far)


def test_places_among_the_cached_tokens_and_of_drafted_ones_anywhere():
    print("places", flush=True)
    rng = np.random.default_rng(12)
    for n, tokens in ((3, 200), (40, 333), (64, 900)):
        x = make(rng, 1, 1, 4, tokens, n, True)
        places = rng.integers(-30, tokens + 60, (1, n))
        seen = rng.random((1, n, n)) < 0.5
        compare(x, 4, seen, n, slopes=np.array([0.25, 0.03, -0.01, 1.0], np.float32), places=places, cap=4.0, spans=make_spans(rng, "any", 1, n, tokens, places))


@pytest.mark.parametrize("n", [2, 20, 64])
def test_drafted_tokens_at_both_ends_of_the_places(n):
    """Distances of almost 2^31, which the slopes make heavy or light."""
    print("ends of places", n, flush=True)
    rng = np.random.default_rng(n)
    x = make(rng, 1, 1, 4, 300, n, True)
    places = np.where(np.arange(n) % 2, -2 ** 40, 2 ** 40)[None]
    held = np.clip(places, -2 ** 29, 300 + 2 ** 29)
    seen = rng.random((1, n, n)) < 0.6
    slopes = np.array([1e-9, -1e-9, 3.0, 0.0], np.float32)
    with Caches(x, 4) as c:
        got = call(None, c.gc, x["q"], x["kd"], x["vd"], drafts.mask_words(seen), slopes=slopes, places=places)
        assert_nodes(scored.decode(None, c.oc, x["q"], x["kd"], x["vd"], seen, oracle.Tolerances(), slopes=slopes, places=held), *got, n)


@pytest.mark.parametrize("beginning", [0, 210])
@pytest.mark.parametrize("n", [3, 40])
def test_numbers_that_are_not_finite(n, beginning):
    """A query makes its own row NaN, with a cap too; a drafted token the rows that attend it; a slope its head's rows; rows that attend nothing are
    none of these."""
    print("not finite", n, beginning, flush=True)
    rng = np.random.default_rng(n)
    bt, tokens = 2, 130
    x = make(rng, bt, 1, 4, tokens, n, True, shared=1 if beginning else 0, beginning=beginning)
    seen = random_tree(rng, bt, n)
    x["q"][0, 1, 2, 77] = np.inf
    x["q"][1, n - 1, 0, 0] = np.nan
    x["kd"][0, 0, n - 1, 5] = np.nan       # only the last node attends itself
    x["vd"][1, 0, n - 2, 9] = -np.inf
    spans = np.tile(np.array([0, beginning + tokens, 0, 0]), (bt, n, 1))
    spans[1, 0] = 0
    seen[1, 0] = False
    x["q"][1, 0, 1, 3] = np.nan            # of a node that attends nothing
    clean = {k: (None if v is None else np.where(np.isfinite(v), v, 0).astype(np.float16)) for k, v in x.items()}
    slopes = np.array([0.1, 0.0, 0.01, 0.2], np.float32)
    with Caches(clean, 4) as c:
        mask = drafts.mask_words(seen)
        score = dict(cap=6.0, slopes=slopes, spans=spans)
        O, cert, flags = call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, **score)
        rO, rc, rf = call(c.shared, c.gc, clean["q"], clean["kd"], clean["vd"], mask, **score)
        bad = np.zeros((bt, n, 4), bool)
        bad[0, 1, 2] = bad[1, n - 1, 0] = True
        bad[0, n - 1, :] = True
        bad[1, :, :] |= seen[1, :, n - 2][:, None]
        assert np.isnan(O[bad]).all() and (flags[bad] & 8 != 0).all()
        assert np.array_equal(O[~bad], rO[~bad]) and (flags[~bad] == 0).all()
        assert (O[1, 0] == 0).all() and (cert["lse"][1, 0] == -np.inf).all()
        for s in (np.nan, np.inf, -np.inf):
            slopes[1] = s
            O, cert, flags = call(c.shared, c.gc, clean["q"], clean["kd"], clean["vd"], mask, cap=6.0, slopes=slopes, spans=spans)
            assert np.isnan(O[0, :, 1]).all() and (flags[0, :, 1] & 8 != 0).all()
            assert np.array_equal(O[:, :, 2:], rO[:, :, 2:]) and (flags[:, :, 2:] == 0).all()
            assert (O[1, 0] == 0).all() and (flags[1, 0] == 0).all() and (cert["lse"][1, 0] == -np.inf).all()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n,hkv", [(1, 1), (1, 70), (6, 1), (16, 1), (30, 1), (64, 1), (90, 2)])
def test_padding_that_is_not_finite(n, hkv, shared):
    """Cached padding of NaN and infinities, sealed and trailing, before and between what is attended: to the rows that leave it out it is as any
    other padding, bit for bit, and the rows that attend it are NaN with PRECOND.  (In a block with attended tokens it is NaN, and in its stead the
    other padding repeats one of them, which leaves the block's steps and errors.)"""
    print("padding", n, hkv, shared, flush=True)
    rng = np.random.default_rng(n)
    bt, tokens, pads = 2, 714, (37, 64)
    x = make(rng, bt, hkv, 4, tokens, n, False, shared=1 if shared else 0, beginning=150)
    clean = {k: None if v is None else v.copy() for k, v in x.items()}
    for name in ("k", "v"):
        clean[name][0, :, :37] = clean[name][0, :, 37:38]
        x[name][0, :, :37] = np.nan
        x[name][0, :, 704:] = np.nan                                              # trailing ones
    x["k"][1, :, :48, 7::16] = np.inf
    x["k"][1, :, 20:30] = -np.inf
    x["v"][1, :, 30:64] = np.where(np.arange(128) % 3 == 0, np.inf, -np.inf)
    x["v"][1, :, 336:352, 5] = np.inf                                             # a block between the spans
    lead = 150 if shared else 0
    spans = np.zeros((bt, n, 4), np.int64)
    spans[0, :] = [lead + 37, lead + 300, lead + 300, lead + 704]
    spans[1, :] = [lead + 64, lead + 336, lead + 352, lead + tokens]
    score = dict(cap=6.0, slopes=slopes_of(4 * hkv, 1))
    with Caches(clean, 4) as c:
        good = call(c.shared, c.gc, x["q"], spans=spans, **score)
        gc = GpuLayerCache(bt, 4 * hkv, hkv, tokens + 16, tier2=False)
        gc.append(x["k"], x["v"])
        got = call(c.shared, gc, x["q"], spans=spans, **score)
        assert same(good, got) and np.isfinite(got[0]).all() and (got[2] == 0).all()
        some = np.arange(0, n, 3)
        rest = np.setdiff1d(np.arange(n), some)
        for first, second in (([lead + 37, lead + 705, 0, 0], [lead + 300, lead + 337, 0, 0]), ([lead, lead + 17, 0, 0], [0, 0, lead + 47, lead + 49])):
            wide = spans.copy()
            wide[0, some], wide[1, some] = first, second
            O, _, flags = call(c.shared, gc, x["q"], spans=wide, **score)
            assert np.isnan(O[:, some]).all() and (flags[:, some] & 8 != 0).all()
            # (the other rows' sums are in the order that this call's spans give them)
            assert np.array_equal(O[:, rest], call(c.shared, c.gc, x["q"], spans=wide, **score)[0][:, rest]) and (flags[:, rest] == 0).all()
        gc.close()


@pytest.mark.parametrize("steep", [30.0, 1e5, 1e20, -1e5])
@pytest.mark.parametrize("n,cap,beginning", [(1, 5.0, 0), (20, 30.0, 0), (64, 30.0, 0), (64, 1e4, 0), (32, 30.0, 700), (64, 30.0, 700)])
def test_steep_biases(n, cap, beginning, steep):
    """Tokens whose weights are nothing beside the nearest ones', in workgroups that see no others: their scores are far beyond what a rounding of
    the largest leaves."""
    print("steep", n, cap, beginning, steep, flush=True)
    rng = np.random.default_rng(n)
    x = make(rng, 1, 1, 4, 1500, n, n > 1, shared=1 if beginning else 0, beginning=beginning)
    seen = random_tree(rng, 1, n) if n > 1 else None
    compare(x, 4, seen, (n, steep), cap=cap, slopes=np.array([steep, steep / 3, 0.01, 0.0], np.float32))


@pytest.mark.parametrize("steep", [30.0, 1e5, 1e20, -1e5])
@pytest.mark.parametrize("n,cap,tokens", [(64, 30.0, 1290), (32, 200.0, 2500)])
def test_steep_biases_of_many_rows(n, cap, tokens, steep):
    """The same in the workgroups that reconstruct for 128 and 256 rows."""
    print("steep, many rows", n, cap, steep, flush=True)
    rng = np.random.default_rng(n)
    bt, g = 130, 4
    x = make(rng, 1, 2, g, tokens, n, True)
    seen = random_tree(rng, 1, n)
    score = dict(cap=cap, slopes=np.array([steep, steep / 3, 0.01, 0.0, -0.01, steep / 7, 0.5, steep], np.float32))
    with Caches(x, g) as c:
        ref = scored.decode(None, c.oc, x["q"], x["kd"], x["vd"], seen, oracle.Tolerances(), **score)
        gc = GpuLayerCache(bt, 2 * g, 2, tokens, tier2=False)
        many = [np.tile(x[i], (bt, 1, 1, 1)) for i in ("k", "v", "q", "kd", "vd")]
        gc.append(*many[:2])
        O, cert, flags = call(None, gc, *many[2:], drafts.mask_words(np.tile(seen, (bt, 1, 1))), **score)
        assert_nodes(ref, O[:1], {f: y[:1] for f, y in cert.items()}, flags[:1], (n, steep))
        assert all(np.array_equal(O[i], O[0]) for i in range(bt))
        gc.close()


# up to 16, 32, 64, 128 and 256 rows a workgroup; the last with the tokens as a beginning's
@pytest.mark.parametrize("n,bt,tokens,beginning", [(1, 2, 300, 0), (3, 2, 300, 700), (8, 2, 300, 0), (13, 160, 1290, 0), (32, 130, 1300, 0), (64, 130, 1290, 0), (64, 130, 40, 1290)])
@pytest.mark.parametrize("cap,scale", [(30.0, 0.0), (200.0, 0.0), (1e4, 0.0), (0.0, 0.0), (0.0, 4.0)])
def test_a_bias_is_too_steep_from_the_same_slope_on(n, bt, tokens, beginning, cap, scale):
    """10^28 cap, or 10^28 scale without one, whichever kernel a row's number and the cache's length choose."""
    print("too steep", n, bt, tokens, beginning, cap, scale, flush=True)
    rng = np.random.default_rng(n + tokens)
    g, hkv = 4, 2
    x = make(rng, 1, hkv, g, tokens, n, True, shared=1 if beginning else 0, beginning=beginning)
    seen = random_tree(rng, 1, n)
    unit = cap or scale or 1.0 / math.sqrt(128.0)
    slopes = (np.array([0.9e28, 1.1e28, -1.1e28, 1.9e28, 0.01, -1.9e28, 2.1e28, -0.9e28]) * unit).astype(np.float32)
    undefined = np.abs(slopes) > 1e28 * unit
    score = dict(cap=cap, scale=scale, slopes=slopes)
    with Caches(x, g) as c:
        ref = scored.decode(c.shared_oc, c.oc, x["q"], x["kd"], x["vd"], seen, oracle.Tolerances(), **score)
        wide = {k: again(v, bt) for k, v in x.items()}
        with Caches(wide, g) as w:
            O, cert, flags = call(w.shared, w.gc, wide["q"], wide["kd"], wide["vd"], drafts.mask_words(again(seen, bt)), **score)
    for y in (O, flags, *cert.values()):
        assert all(np.array_equal(y[i], y[0], equal_nan=True) for i in range(bt))
    assert np.isnan(O[0][:, undefined]).all() and (flags[0][:, undefined] & 8 != 0).all()
    fine = np.flatnonzero(~undefined)
    assert_nodes([[[heads[h] for h in fine] for heads in ref[0]]], O[:1][:, :, fine], {f: y[:1][:, :, fine] for f, y in cert.items()}, flags[:1][:, :, fine], (n, cap))


@pytest.mark.parametrize("n,bt,hkv", [(1, 1, 1), (13, 1, 1), (27, 1, 1), (64, 1, 1), (64, 130, 2)])
def test_spans_at_the_ends_of_blocks_tiles_and_turns(n, bt, hkv):
    """Spans of one token, of a tile, one short of and one beyond it, alike for all nodes and not."""
    print("span ends", n, bt, flush=True)
    rng = np.random.default_rng(n)
    tokens = 1300 if bt == 1 else 330
    x = make(rng, min(bt, 2), hkv, 4, tokens, n, False)
    some = np.unique([0, n // 2, n - 1])
    with Caches(dict(x), 4) as c:
        gc = c.gc
        if bt > 2:
            gc = GpuLayerCache(bt, 4 * hkv, hkv, tokens, tier2=False)
            gc.append(np.tile(x["k"], (bt // 2, 1, 1, 1)), np.tile(x["v"], (bt // 2, 1, 1, 1)))
        for a, b in ((0, 1), (15, 16), (16, 32), (31, 33), (63, 64), (64, 128), (127, 257), (tokens - 21, tokens), (tokens - 1, tokens), (tokens // 16 * 16 - 1, tokens // 16 * 16 + 1)):
            spans = np.zeros((min(bt, 2), n, 4), np.int64)
            spans[..., 0], spans[..., 1] = a, b
            spans[0, n // 2] = [a, b, 300, 310]
            q = x["q"]
            ref = scored.decode(None, c.oc, q[:, some], None, None, None, oracle.Tolerances(), spans=spans[:, some])
            if bt > 2:
                q, spans = np.tile(q, (bt // 2, 1, 1, 1)), np.tile(spans, (bt // 2, 1, 1))
            O, cert, flags = call(None, gc, q, spans=spans)
            assert_nodes(ref, O[:2, some], {f: y[:2, some] for f, y in cert.items()}, flags[:2, some], (a, b))
            if bt > 2:
                assert all(np.array_equal(O[i], O[i % 2]) for i in range(bt))
        if bt > 2:
            gc.close()


def again(x, bt):
    """Up to four sequences over and over."""
    return None if x is None else np.tile(x, ((bt + len(x) - 1) // len(x),) + (1,) * (x.ndim - 1))[:bt]


# caches that are long for the device: up to 16 rows by twelve waves; 33 .. 64, 65 .. 128, up to 256 rows by a workgroup that reconstructs once for all
@pytest.mark.parametrize("n,tokens,cap,bias,spans", [
    (1, 1157, 30.0, 0, "all"), (1, 2053, 0.0, 1, "window"), (4, 1293, 5.0, 1, "sorted"), (4, 1029, 0.0, 0, "any"), (2, 1290, 500.0, -1, "padded"), (13, 1157, 5.0, 1, "sorted"), (13, 1293, 0.0, -1, "window"), (13, 1290, 50.0, 0, "any"), (27, 1093, 3.0, 1, "padded"), (27, 1347, 1e3, 1, "sorted"),
    (27, 1100, 0.0, 0, "window"), (64, 1093, 30.0, 0, "sorted"), (64, 1285, 2.0, 1, "window"), (64, 1029, 0.0, 1, "any"), (64, 1290, 9.0, 0, "all")])
@pytest.mark.parametrize("beginnings", [False, True])
def test_many_rows_of_many_sequences(n, tokens, cap, bias, spans, beginnings):
    """The tokens as the sequences' own, with drafted ones, or as their beginnings', one a sequence, with a few of their own behind."""
    print("scored many rows", n, tokens, cap, bias, spans, beginnings, flush=True)
    rng = np.random.default_rng(tokens + n)
    bt = 256 if n * 4 <= 64 else 160
    own = 21 if beginnings else tokens
    total = own + (tokens if beginnings else 0)
    x = make(rng, 4, 1, 4, own, n, True, "student", 2.0, 4 if beginnings else 0, tokens)
    seen = random_tree(rng, 4, n)
    places = total + seen.sum(-1) - 1
    sp, slopes = make_spans(rng, spans, 4, n, total, places), slopes_of(4, bias)
    some = np.unique([0, min(1, n - 1), n // 2, n - 1])
    with Caches(x, 4) as c:
        # (the definition's rows are some of the nodes: drafted tokens are all there, with the masks and places of all)
        keep = dict(cap=cap, slopes=slopes, spans=None if sp is None else sp[:, some])
        wide = {k: again(v, bt) for k, v in x.items()}
        with Caches(wide, 4) as w:
            O, cert, flags = call(w.shared, w.gc, wide["q"], wide["kd"], wide["vd"], drafts.mask_words(again(seen, bt)), cap=cap, slopes=slopes,
                                  places=again(places, bt), spans=again(sp, bt))
        ref = some_nodes(c, x, seen, places, some, **keep)
    for at in range(4):
        for y in (O, flags, *cert.values()):
            assert all(np.array_equal(z, y[at]) for z in y[at::4])
        assert_nodes(ref[at:at + 1], O[at:at + 1, some], {f: y[at:at + 1, some] for f, y in cert.items()}, flags[at:at + 1, some], at)


def some_nodes(c, x, seen, places, some, **score):
    """The definition for some of the nodes: the others' queries are left out, their drafted tokens not."""
    n = x["q"].shape[1]
    full = []
    for i in some:
        one = np.zeros_like(x["q"][:, :1]) + x["q"][:, i:i + 1]
        s = dict(score)
        if s.get("spans") is not None:
            s["spans"] = s["spans"][:, list(some).index(i)][:, None]
        full.append(scored.decode(c.shared_oc, c.oc, one, x["kd"], x["vd"], seen[:, i:i + 1], oracle.Tolerances(), places=places[:, i:i + 1], where_drafted=places, **s))
    return [[full[j][b][0] for j in range(len(some))] for b in range(x["q"].shape[0])]


@pytest.mark.parametrize("n,blocks", [(13, 68), (13, 76), (13, 67), (13, 69), (13, 72), (27, 69), (27, 71), (64, 68), (64, 70)])
@pytest.mark.parametrize("beginnings", [False, True])
def test_a_bound_is_over_blocks_that_are_there(n, blocks, beginnings):
    """A tile of 64 and more rows ends behind the last sealed block: what it holds there is no block of the row's, also where the row attends the trailing
    tokens, whose places these would be.  The first block's keys, far wider than all others, are left out by most rows."""
    print("blocks that are there", n, blocks, beginnings, flush=True)
    rng = np.random.default_rng(100 * blocks + n)
    bt = 256 if n * 4 <= 64 else 160
    tokens, own = 16 * blocks + 5, 21
    x = make(rng, 4, 1, 4, own if beginnings else tokens, n, False, shared=4 if beginnings else 0, beginning=tokens)
    x["sk" if beginnings else "k"][:, :, :16] *= np.float16(256.0)
    spans = np.zeros((4, n, 4), np.int64)
    spans[0] = [40, tokens, 0, 0]                                  # padded
    spans[1] = [16 * blocks, tokens, 0, 0]                         # trailing tokens only: no sealed one bounds anything
    spans[2] = [tokens - 150, tokens, 0, 0]                        # a window
    spans[2, n // 2] = [0, 3, 16 * blocks + 2, tokens]             # ... with the first tokens
    spans[3] = [0, 0, 16 * blocks - 1, 16 * blocks + 1]
    spans[3, 0] = 0                                                # nothing
    some = np.unique([0, n // 2, n - 1])
    with Caches(x, 4) as c:
        ref = scored.decode(c.shared_oc, c.oc, x["q"][:, some], None, None, None, oracle.Tolerances(), spans=spans[:, some])
        wide = {k: again(v, bt) for k, v in x.items()}
        with Caches(wide, 4) as w:
            O, cert, flags = call(w.shared, w.gc, wide["q"], spans=again(spans, bt))
    assert (cert["delta_h"][1] == 0).all()
    for y in (O, flags, *cert.values()):
        assert all(np.array_equal(y[i], y[i % 4]) for i in range(bt))
    O, cert, flags = O[:4, some], {f: y[:4, some] for f, y in cert.items()}, flags[:4, some]
    wide_rows(ref[2][1], x["q"][2, n // 2], x["sk" if beginnings else "k"][2, 0, :3], {f: y[2, 1] for f, y in cert.items()}, flags[2, 1])
    for field in cert:
        cert[field][2, 1] = [r.get(field, 0.0) for r in ref[2][1]]
    O[2, 1], flags[2, 1] = [r["O"] for r in ref[2][1]], [r["flags"] for r in ref[2][1]]
    assert_nodes(ref, O, cert, flags, (n, blocks))


def wide_rows(ref, q, k, cert, flags):
    """The certificate of a node's heads that attend keys of some 256 times the ordinary size, whose scores the bar of 1e-4 for FP32's arithmetic does not
    cover.  A score is a sum of 128 products, exact in FP32 each: it is off by 128 2^-24 of the sum of their sizes s at most, so that a weight beside
    another's is off by the factor e^(2 128 2^-24 s), and a mass by as much.  Delta, a sum of 128 numbers of one sign, is relatively off by 128 2^-24, and
    E_key, which has e^(mass_exp Delta) and e^(2 Delta), by that of (mass_exp + 2) Delta."""
    for h, r in enumerate(ref):
        size = float((np.abs(k.astype(np.float64)) @ np.abs(q[h].astype(np.float64))).max()) / math.sqrt(128.0)
        weight = math.expm1(2 * 128 * 2.0 ** -24 * size)
        bound = 128 * 2.0 ** -24 * (oracle.Tolerances().mass_exp + 2) * r["delta_h"]
        for field, tol in (("delta_h", 0.0), ("v_max", 0.0), ("E_val", weight), ("alpha_tail_hat", weight), ("max_block_contrib", weight), ("E_key", weight + math.expm1(bound))):
            assert abs(float(cert[field][h]) - r[field]) <= (1e-4 + tol) * abs(r[field]) + 1e-9, (field, h, float(cert[field][h]), r[field])
        assert abs(float(cert["lse"][h]) - r["lse"]) <= 1e-4 * max(1.0, abs(r["lse"])) + 128 * 2.0 ** -24 * size
        assert int(flags[h]) == r["flags"]


def test_the_plain_scores_are_the_tree_calls():
    """No scoring, a scoring of nothing, and a span of everything."""
    print("plain", flush=True)
    from test_gpu_drafts import tree_call
    rng = np.random.default_rng(3)
    for n, tokens in ((5, 700), (30, 700), (60, 2000)):
        x = make(rng, 2, 1, 4, tokens, n, True)
        seen = random_tree(rng, 2, n)
        mask = drafts.mask_words(seen)
        with Caches(x, 4) as c:
            tree = tree_call(c.gc, x["q"], x["kd"], x["vd"], mask)
            assert same(tree, call(None, c.gc, x["q"], x["kd"], x["vd"], mask, plain=True))
            assert same(tree, call(None, c.gc, x["q"], x["kd"], x["vd"], mask))
            ref = scored.decode(None, c.oc, x["q"], x["kd"], x["vd"], seen, oracle.Tolerances())
            assert_nodes(ref, *call(None, c.gc, x["q"], x["kd"], x["vd"], mask, spans=np.tile([0, tokens, 0, 0], (2, n, 1))), n)


def test_thresholds_and_forced_flags():
    print("scored flags", flush=True)
    rng = np.random.default_rng(4)
    x = make(rng, 2, 2, 2, 200, 6, True, shared=1, beginning=300)
    seen = random_tree(rng, 2, 6)
    with Caches(x, 2) as c:
        mask = drafts.mask_words(seen)
        _, cert, _ = call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, cap=3.0)
        for field, name in (("E_key", "eps_key"), ("E_val", "eps_val"), ("max_block_contrib", "v_tol")):
            at = float(np.median(cert[field]))
            _, _, flags = call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, cap=3.0, tol=c.gc.cqa.Tolerances(**{name: at}))
            assert np.array_equal(flags, np.where(cert[field] > np.float32(at), 1 if name == "eps_key" else 2, 0))
        _, _, flags = call(c.shared, c.gc, x["q"], x["kd"], x["vd"], mask, cap=3.0, tol=c.gc.cqa.Tolerances(force_flags=4))
        assert (flags == 4).all()


def test_layers_are_apart_and_a_single_token_is_a_node():
    """Three layers of different lengths; an appended token attended without drafted ones is the single-token step up to the rounding."""
    print("scored layers", flush=True)
    t, cqa = _torch(), load_binding()
    rng = np.random.default_rng(8)
    gc = GpuLayerCache(1, 4, 1, 400, tier2=False, n_layers=3)
    shared = GpuLayerCache(1, 4, 1, 400, tier2=False, n_layers=3)
    try:
        for layer, (own, beginning) in enumerate(((33, 200), (0, 47), (150, 0))):
            ocs = []
            for g, n in ((shared, beginning), (gc, own)):
                oc = oracle.OracleLayerCache(1, 1)
                if n:
                    k, v = (workloads.normal_f16(rng, (1, 1, n, 128)) for _ in range(2))
                    g.append(k, v, layer)
                    oc.append(k, v)
                ocs.append(oc)
            q = workloads.normal_f16(rng, (1, 1, 4, 128))
            assert_nodes(scored.decode(*ocs, q, None, None, None, oracle.Tolerances(), cap=9.0), *call(shared, gc, q, cap=9.0, layer=layer), layer)
            if own:
                O, _, _ = call(None, gc, q, layer=layer)
                gc.cqa.cqa_certified_decode(gc.h, layer, _off(q[0]), cqa.Tolerances(), gc.O, gc.cert, gc.flags)
                t.cuda.synchronize()
                assert np.abs(O[0, 0] - gc.O[0].cpu().numpy()).max() <= 4e-3
    finally:
        gc.close()
        shared.close()


@pytest.mark.parametrize("n,bt,beginning,tokens", [(1, 4, 600, 70), (20, 2, 300, 40)])
def test_recorded_calls_follow_their_buffers(n, bt, beginning, tokens):
    """Queries, spans and slopes are read by each replay; eager work of the program's goes on between them."""
    print("scored graph", n, flush=True)
    t = _torch()
    rng = np.random.default_rng(21)
    x = make(rng, bt, 1, 4, tokens, n, True, shared=1, beginning=beginning)
    with Caches(x, 4) as c:
        total = beginning + tokens
        args = dict(cap=5.0, slopes=slopes_of(4, 1), spans=make_spans(rng, "sorted", bt, n, total, None))
        a = Call(c.shared, c.gc, x["q"], x["kd"], x["vd"], None, **args)
        b = Call(None, c.gc, x["q"], x["kd"], x["vd"], None, cap=2.0)
        s = t.cuda.Stream()
        with t.cuda.stream(s):
            a.enqueue(s.cuda_stream)
            b.enqueue(s.cuda_stream)
        s.synchronize()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph, stream=s):
            a.enqueue(s.cuda_stream)
            b.enqueue(s.cuda_stream)
        for turn in range(4):
            q = workloads.normal_f16(rng, x["q"].shape)
            spans = make_spans(rng, ("any", "sorted", "padded", "window")[turn], bt, n, total, scored.default_places(bt, n, total, True))
            slopes = np.abs(rng.standard_normal(4)).astype(np.float32)
            for z in (a, b):
                z.inputs[0].copy_(t.from_numpy(q))
            a.spans.copy_(t.from_numpy(spans))
            a.slopes.copy_(t.from_numpy(slopes))
            a.ws.fill_(0xFF)
            b.ws.fill_(0xFF)
            t.cuda.synchronize()
            graph.replay()
            got = a.results(), b.results()
            args.update(slopes=slopes, spans=spans)
            assert same(got[0], call(c.shared, c.gc, q, x["kd"], x["vd"], None, **args))
            assert same(got[1], call(None, c.gc, q, x["kd"], x["vd"], None, cap=2.0))


def test_two_streams_at_a_time():
    print("scored streams", flush=True)
    t = _torch()
    rng = np.random.default_rng(22)
    x = make(rng, 4, 2, 4, 300, 3, True, shared=2, beginning=2000)
    with Caches(x, 4) as c:
        calls = [Call(c.shared, c.gc, workloads.normal_f16(rng, x["q"].shape), x["kd"], x["vd"], None, cap=float(3 + i)) for i in range(2)]
        alone = []
        for z in calls:
            z.enqueue()
            alone.append(z.results())
            z.O[:-4].fill_(0.0)
        streams = [t.cuda.Stream() for _ in calls]
        t.cuda.synchronize()
        for _ in range(3):
            for z, s in zip(calls, streams):
                z.enqueue(s.cuda_stream)
        for z, ref in zip(calls, alone):
            assert same(z.results(), ref)


def test_more_sequences_than_compute_units_and_more_than_256_rows():
    """300 sequences behind one beginning, 1200 rows; each three times the same four."""
    print("scored many sequences", flush=True)
    rng = np.random.default_rng(31)
    x = make(rng, 4, 1, 4, 37, 1, False, shared=1, beginning=900)
    with Caches(x, 4) as c:
        ref = scored.decode(c.shared_oc, c.oc, x["q"], None, None, None, oracle.Tolerances())
        for bt in (300, 64):
            gc = GpuLayerCache(bt, 4, 1, 64, tier2=False)
            gc.append(np.tile(x["k"], (bt // 4, 1, 1, 1)), np.tile(x["v"], (bt // 4, 1, 1, 1)))
            O, cert, flags = call(c.shared, gc, np.tile(x["q"], (bt // 4, 1, 1, 1)))
            assert_nodes(ref, O[:4], {f: y[:4] for f, y in cert.items()}, flags[:4], bt)
            assert all(np.array_equal(O[i], O[i % 4]) and np.array_equal(cert["E_key"][i], cert["E_key"][i % 4]) for i in range(bt))
            gc.close()


@pytest.mark.parametrize("tokens,bt,hkv,g,n,cap,bias,spans", [
    (0, 200, 4, 4, 4, 0.0, 0, "all"), (37, 200, 4, 4, 1, 0.0, 0, "all"), (263, 200, 4, 2, 7, 30.0, 0, "all"), (130, 400, 2, 4, 3, 300.0, 1, "padded"),
    (2053, 100, 8, 4, 1, 5.0, 1, "any"), (519, 400, 4, 1, 16, 0.0, -1, "sorted"), (33, 200, 4, 4, 4, 0.0, 0, "window")])
@pytest.mark.parametrize("beginning", [0, 85])
def test_more_short_sequences_than_the_device_holds(tokens, bt, hkv, g, n, cap, bias, spans, beginning):
    """Workgroups of two waves: every kind of score, trailing and drafted tokens of several turns, groups of one row and of sixteen."""
    print("short sequences", tokens, bt, hkv, g, n, beginning, flush=True)
    rng = np.random.default_rng(tokens + beginning)
    x = make(rng, 4, hkv, g, tokens, n, n > 1, "student", 2.0, 1 if beginning else 0, beginning)
    seen = random_tree(rng, 4, n) if n > 1 else None
    total = beginning + tokens
    places = total - (0 if n > 1 else 1) + rng.integers(0, 9, (4, n))
    at = make_spans(rng, spans, 4, n, total, places)
    score = dict(cap=cap, slopes=slopes_of(hkv * g, bias), places=places if bias else None, spans=at)
    tile = lambda y: None if y is None else np.tile(y, (bt // 4,) + (1,) * (y.ndim - 1))  # noqa: E731
    with Caches(x, g) as c:
        ref = scored.decode(c.shared_oc, c.oc, x["q"], x["kd"], x["vd"], seen, oracle.Tolerances(), **score)
        gc = GpuLayerCache(bt, hkv * g, hkv, max(tokens, 1), tier2=False)
        if tokens:
            gc.append(tile(x["k"]), tile(x["v"]))
        many = dict(score, places=tile(score["places"]), spans=tile(at))
        mask = None if seen is None else drafts.mask_words(tile(seen))
        O, cert, flags = call(c.shared, gc, tile(x["q"]), tile(x["kd"]), tile(x["vd"]), mask, **many)
        assert_nodes(ref, O[:4], {f: y[:4] for f, y in cert.items()}, flags[:4], bt)
        assert all(np.array_equal(O[i], O[i % 4]) and np.array_equal(flags[i], flags[i % 4]) for i in range(bt))
        gc.close()


@pytest.mark.parametrize("hkv,g,beginning,bt,n,cap", [(4, 4, 20016, 32, 1, 0.0), (4, 4, 20005, 16, 1, 40.0), (2, 4, 33003, 12, 6, 0.0), (8, 2, 5001, 160, 1, 20.0)])
def test_many_sequences_behind_a_long_beginning(hkv, g, beginning, bt, n, cap):
    """33 and more rows of several sequences by a workgroup that reconstructs once for all."""
    print("prefix long", hkv, g, beginning, bt, n, flush=True)
    rng = np.random.default_rng(bt)
    x = make(rng, 4, hkv, g, 35, n, n > 1, "student", 2.0, 1, beginning)
    seen = random_tree(rng, 4, n) if n > 1 else None
    some = np.unique([0, n - 1])
    with Caches(x, g) as c:
        gc = GpuLayerCache(bt, hkv * g, hkv, 64, tier2=False)
        gc.append(again(x["k"], bt), again(x["v"], bt))
        O, cert, flags = call(c.shared, gc, again(x["q"], bt), again(x["kd"], bt), again(x["vd"], bt), None if seen is None else drafts.mask_words(again(seen, bt)), cap=cap)
        places = scored.default_places(4, n, beginning + 35, n > 1)
        if n > 1:
            ref = some_nodes(c, x, seen, places, some, cap=cap)
        else:
            ref = scored.decode(c.shared_oc, c.oc, x["q"], None, None, None, oracle.Tolerances(), cap=cap)
        gc.close()
    assert_nodes(ref, O[:4, some], {f: y[:4, some] for f, y in cert.items()}, flags[:4, some], bt)
    for y in (O, flags, *cert.values()):
        assert all(np.array_equal(y[i], y[i % 4]) for i in range(bt))


def test_joining_as_many_sets_as_two_caches_can_leave():
    """One KV head: three workgroups a compute unit in either pass, 1536 sets of a row, whose weights take more of LDS than 64 KB beside what is joined."""
    print("scored most sets", flush=True)
    t = _torch()
    rng = np.random.default_rng(61)
    tokens, beginning = 98437, 98506
    x = make(rng, 1, 1, 4, tokens, 1, False, "student", 2.0, 1, beginning)
    with Caches(x, 4) as c:
        sets = 3 * t.cuda.get_device_properties(0).multi_processor_count
        assert min(tokens, beginning) // 128 >= sets
        for score in (dict(), dict(cap=30.0, slopes=np.array([0.001, 0.0, 1e-5, -1e-6], np.float32))):
            assert_nodes(scored.decode(c.shared_oc, c.oc, x["q"], None, None, None, oracle.Tolerances(), **score), *call(c.shared, c.gc, x["q"], **score), "sets")


def test_nothing_at_all_is_attended():
    """Empty caches and no drafted tokens, and an empty mask."""
    print("scored empty", flush=True)
    rng = np.random.default_rng(2)
    for n in (1, 9, 70):
        x = make(rng, 2, 1, 4, 0, n, True, shared=1, beginning=0)
        with Caches(x, 4) as c:
            for shared in (None, c.shared):
                for got in (call(shared, c.gc, x["q"], cap=3.0), call(shared, c.gc, x["q"], x["kd"], x["vd"], np.zeros((2, n, (n + 63) // 64), np.uint64))):
                    assert (got[0] == 0).all() and (got[2] == 0).all()
                    assert all((y == (-np.inf if f == "lse" else 0)).all() for f, y in got[1].items())


def test_the_calls_refuse_what_they_do_not_do():
    print("scored refusals", flush=True)
    t, cqa = _torch(), load_binding()
    rng = np.random.default_rng(1)
    x = make(rng, 4, 2, 2, 40, 2, True, shared=2, beginning=50)
    with Caches(x, 2) as c:
        z = Call(c.shared, c.gc, x["q"], x["kd"], x["vd"], None)
        base = dict(shared=c.shared.h, h=c.gc.h, layer=0, q=z.inputs[0], kd=z.inputs[1], vd=z.inputs[2], n=2, mask=None, scoring=cqa.Scoring(), tol=z.tol, O=z.O,
                    cert=z.cert, flags=z.flags, ws=z.ws)

        def status(**change):
            a = dict(base, **change)
            try:
                rest = (a["layer"], a["q"], a["kd"], a["vd"], a["n"], a["mask"], a["scoring"], a["tol"], a["O"], a["cert"], a["flags"], a["ws"])
                if a["shared"] == 0:
                    cqa.cqa_scored_decode(a["h"], *rest)
                else:
                    cqa.cqa_prefix_decode(a["shared"], a["h"], *rest)
            except cqa.CqaError as e:
                return e.status
            return cqa.OK

        bad, no = cqa.ERR_INVALID_ARG, cqa.ERR_UNSUPPORTED
        other = [GpuLayerCache(b, hq, hkv, 64, tier2=False) for b, hq, hkv in ((3, 4, 2), (8, 4, 2), (2, 8, 2), (2, 2, 1))]
        for shared in (0, c.shared.h):
            assert status(shared=shared) == cqa.OK
            for name in ("q", "O", "cert", "flags", "ws", "kd", "vd"):
                assert status(shared=shared, **{name: None}) == bad, name
            for name in ("O", "cert", "flags", "ws"):
                assert status(shared=shared, **{name: base[name].data_ptr() + 8}) == bad, name
            assert status(shared=shared, q=z.inputs[0].data_ptr() + 1) == bad and status(shared=shared, kd=z.inputs[1].data_ptr() + 1) == bad
            assert status(shared=shared, kd=None, vd=None) == cqa.OK
            assert status(shared=shared, kd=None, vd=None, mask=z.ws) == bad and status(shared=shared, mask=z.ws.data_ptr() + 4) == bad
            assert status(shared=shared, layer=1) == bad and status(shared=shared, layer=-1) == bad
            assert status(shared=shared, n=0) == bad and status(shared=shared, n=257) == no
            for s in (dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=2.0 ** -41), dict(scale=2.0 ** 41), dict(cap=-1.0), dict(cap=math.nan),
                      dict(cap=math.inf), dict(cap=2.0 ** -21), dict(cap=2.0 ** 61), dict(slopes_dev=z.ws.data_ptr() + 2), dict(places_dev=z.ws.data_ptr() + 4),
                      dict(spans_dev=z.ws.data_ptr() + 4)):
                assert status(shared=shared, scoring=cqa.Scoring(**s)) == bad, s
            assert status(shared=shared, scoring=None) == cqa.OK
            for tol, want in ((cqa.Tolerances(mass_exp=-1), bad), (cqa.Tolerances(rank_depth=1), no), (cqa.Tolerances(int8_query=True), no), (cqa.Tolerances(key_bound_mode=3), bad)):
                assert status(shared=shared, tol=tol) == want
        for o in other:
            assert status(shared=o.h) == bad
            with pytest.raises(cqa.CqaError) as e:
                cqa.cqa_prefix_workspace_bytes(o.h, c.gc.h, 1)
            assert e.value.status == bad
        wide = GpuLayerCache(300, 4, 1, 16, tier2=False)
        one = GpuLayerCache(1, 4, 1, 16, tier2=False)
        with pytest.raises(cqa.CqaError) as e:   # 300 x 256 x 4 rows
            cqa.cqa_prefix_workspace_bytes(one.h, wide.h, 256)
        assert e.value.status == no
        assert cqa.cqa_prefix_workspace_bytes(one.h, wide.h, 218) > 0
        for o in (*other, wide, one):
            o.close()
        z.results()


def test_a_turn_of_a_batch_behind_a_system_prompt():
    """Drafted tokens of four left-padded sequences with capped scores, then one of each is appended and attended as a single token: the two calls as a
    program makes them, over two layers."""
    print("scored turn", flush=True)
    t = _torch()
    rng = np.random.default_rng(40)
    bt, hkv, g, beginning, tokens, n = 4, 2, 2, 83, 30, 3
    shared, gc = GpuLayerCache(1, hkv * g, hkv, 128, tier2=False, n_layers=2), GpuLayerCache(bt, hkv * g, hkv, 64, tier2=False, n_layers=2)
    try:
        begin = beginning + rng.integers(0, tokens, bt)
        spans = np.zeros((bt, n, 4), np.int64)
        spans[..., 1], spans[..., 2], spans[..., 3] = beginning, begin[:, None], 10 ** 6
        for layer in range(2):
            ocs = [oracle.OracleLayerCache(1, hkv), oracle.OracleLayerCache(bt, hkv)]
            for cache, oc, b, m in ((shared, ocs[0], 1, beginning), (gc, ocs[1], bt, tokens)):
                k, v = (workloads.normal_f16(rng, (b, hkv, m, 128)) for _ in range(2))
                cache.append(k, v, layer)
                oc.append(k, v)
            q, kd, vd = (workloads.normal_f16(rng, s) for s in ((bt, n, hkv * g, 128), (bt, hkv, n, 128), (bt, hkv, n, 128)))
            seen = np.tile(np.tril(np.ones((n, n), bool)), (bt, 1, 1))
            assert_nodes(scored.decode(*ocs, q, kd, vd, seen, oracle.Tolerances(), cap=4.0, spans=spans),
                         *call(shared, gc, q, kd, vd, None, cap=4.0, spans=spans, layer=layer), layer)
            gc.append(kd[:, :, :1], vd[:, :, :1], layer)
            ocs[1].append(kd[:, :, :1], vd[:, :, :1])
            assert_nodes(scored.decode(*ocs, q[:, :1], None, None, None, oracle.Tolerances(), cap=4.0, spans=spans[:, :1]),
                         *call(shared, gc, q[:, :1], cap=4.0, spans=spans[:, :1], layer=layer), layer)
    finally:
        gc.close()
        shared.close()
