"""Drafted tokens: rotary rows, reading the cache back and attention of trees and chunks over the cache, against the 64-bit
definitions of oracle/drafts.py.

Tolerances.  A rounding to FP16 is off by at most 2^-11 of the value (BF16 2^-8, FP32 2^-24).
  read    bit-exact in every type (the definition names each rounding; a BF16 or FP32 value by its own definition in float64).
  rotary  two products and a sum in FP32 with sine and cosine within 2^-22, and one rounding to the type.
  tree    O: its own rounding 2^-11 |O|, the weights' 2^-11 sum a |v| and 2^-25 count max |v| / sum exp(s - max) (weights below
          FP16's normal range), and the library's bar for the certificate, 1e-4, for the scores' FP32 sums: 1e-4 sum a |v|.
          Certificate: the library's bar, 1e-4 relative (lse: 1e-4 max(1, |lse|)).
"""
import math

import numpy as np
import pytest

import oracle
import workloads
from helpers import CERT_REL, GpuLayerCache, load_binding
from oracle import drafts

pytestmark = pytest.mark.gpu

NODE_FIELDS = ("E_key", "E_val", "delta_h", "v_max", "alpha_tail_hat", "lse", "max_block_contrib", "reserved")


def _torch():
    import torch
    return torch


def _off(x, by=1):
    """The same FP16 numbers on the device, `by` numbers behind an aligned address."""
    t = _torch()
    buf = t.empty(x.size + 16, dtype=t.float16, device="cuda")
    out = buf[by:by + x.size].view(x.shape)
    out.copy_(t.from_numpy(np.ascontiguousarray(x)))
    return out


class Nodes:
    """Output buffers of a tree call with guard rows behind them."""

    def __init__(self, cqa, h, bt, n, hq, ws_fill=0xFF):
        t = _torch()
        self.cqa, self.shape = cqa, (bt, n, hq)
        rows = bt * n * hq
        self.O = t.full((rows + 4, 128), 7.0, dtype=t.float16, device="cuda")
        self.cert = t.full((rows + 4, 8), 7.0, device="cuda")
        self.flags = t.full((rows + 4,), 77, dtype=t.int32, device="cuda")
        self.ws_bytes = cqa.cqa_tree_workspace_bytes(h, n)
        # every byte set: a NaN pattern where a set is read that was not written
        self.ws = t.full((self.ws_bytes + 256,), ws_fill, dtype=t.uint8, device="cuda")

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


def tree_call(gc, q, kd, vd, mask, tol=None, layer=0, stream=None, by=0):
    cqa, t = gc.cqa, gc.torch
    bt, n, hq, _ = q.shape
    out = Nodes(cqa, gc.h, bt, n, hq)
    md = None if mask is None else t.from_numpy(np.ascontiguousarray(mask).view(np.int64)).cuda()
    args = [_off(x, by) for x in (q, kd, vd)]
    t.cuda.synchronize()
    cqa.cqa_tree_decode(gc.h, layer, *args, n, md, tol or cqa.Tolerances(), out.O, out.cert, out.flags, out.ws, stream)
    return out.results()


def assert_nodes(ref, O, cert, flags, where=""):
    for b, nodes in enumerate(ref):
        for i, heads in enumerate(nodes):
            for h, r in enumerate(heads):
                at = (where, b, i, h)
                tol = 2.0 ** -11 * np.abs(r["O"]) + (2.0 ** -11 + 1e-4) * r["spread"] + 2.0 ** -25 * r["floor"]
                err = np.abs(O[b, i, h] - r["O"])
                assert (err <= tol).all(), (at, float((err - tol).max()), float(np.abs(r["O"]).max()))
                for name in ("E_key", "E_val", "delta_h", "v_max", "alpha_tail_hat", "max_block_contrib"):
                    x, y = float(cert[name][b, i, h]), r[name]
                    assert x == y or abs(x - y) <= CERT_REL * abs(y) + 1e-9, (at, name, x, y)
                x = float(cert["lse"][b, i, h])
                assert x == r["lse"] or abs(x - r["lse"]) <= 1e-4 * max(1.0, abs(r["lse"])), (at, "lse", x, r["lse"])
                assert cert["reserved"][b, i, h] == 0
                assert int(flags[b, i, h]) == r["flags"], (at, "flags", int(flags[b, i, h]), r["flags"])


def random_tree(rng, bt, n):
    return np.stack([drafts.ancestors([-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, n)]) for _ in range(bt)])


def make(rng, bt, hkv, g, n_tokens, n, keys="normal", peaked=False):
    draw = workloads.student_t3_f16 if keys == "student" else workloads.normal_f16
    k, kd = draw(rng, (bt, hkv, n_tokens, 128)), draw(rng, (bt, hkv, n, 128))
    v, vd = workloads.normal_f16(rng, (bt, hkv, n_tokens, 128)), workloads.normal_f16(rng, (bt, hkv, n, 128))
    q = workloads.normal_f16(rng, (bt, n, hkv * g, 128))
    if peaked:
        q[:, :, ::2] *= np.float16(4.0)
    return k, v, q, kd, vd


# few rows, 33 .. 64, 65 .. 128, up to 256 and several tiles of 256; a block short, blocks that do not fill a record, ragged ends
CASES = [
    (1, 1, 1, 0, 1, True), (1, 1, 4, 0, 3, True), (2, 1, 2, 1, 2, False), (1, 2, 4, 15, 3, True), (2, 3, 2, 16, 5, True), (1, 1, 4, 17, 1, False),
    (1, 2, 4, 1029, 8, True), (1, 2, 4, 337, 13, True), (1, 1, 4, 333, 27, True), (1, 2, 4, 700, 64, True), (1, 1, 2, 257, 200, True),
    (1, 1, 1, 100, 256, False), (3, 1, 4, 2053, 31, True), (1, 1, 4, 81, 256, False), (1, 1, 2, 64, 65, True), (1, 1, 1, 4099, 1, True),
    (2, 1, 1, 143, 33, False), (1, 2, 2, 160, 63, True), (5, 3, 1, 31, 7, True),
]


@pytest.mark.parametrize("bt,hkv,g,n_tokens,n,tree", CASES)
def test_nodes_match_the_definition(bt, hkv, g, n_tokens, n, tree):
    print("tree", bt, hkv, g, n_tokens, n, tree, flush=True)
    rng = np.random.default_rng(1000 * n_tokens + n)
    k, v, q, kd, vd = make(rng, bt, hkv, g, n_tokens, n, keys="student" if n % 2 else "normal", peaked=n % 3 == 0)
    seen = random_tree(rng, bt, n) if tree else np.tile(np.tril(np.ones((n, n), bool)), (bt, 1, 1))
    oc = oracle.OracleLayerCache(bt, hkv)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    with GpuLayerCache(bt, hkv * g, hkv, n_tokens + 32, tier2=False) as gc:
        if n_tokens:
            gc.append(k, v)
        mask = drafts.mask_words(seen) if tree else None
        got = tree_call(gc, q, kd, vd, mask)
        assert_nodes(ref, *got)
        # at any address an FP16 number may have: the same bits
        for x, y in zip(got, tree_call(gc, q, kd, vd, mask, by=1)):
            assert all((x[f] == y[f]).all() for f in x) if isinstance(x, dict) else np.array_equal(x, y)


def test_thresholds_and_forced_flags():
    print("tree flags", flush=True)
    rng = np.random.default_rng(4)
    k, v, q, kd, vd = make(rng, 1, 2, 2, 200, 6)
    oc = oracle.OracleLayerCache(1, 2)
    oc.append(k, v)
    seen = random_tree(rng, 1, 6)
    plain = [r for heads in drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())[0] for r in heads]

    def between(name):
        """The middle of the widest gap of a field's values: no row is near it."""
        x = np.sort([r[name] for r in plain])
        i = int(np.argmax(np.diff(x)))
        assert x[i + 1] - x[i] > 4 * CERT_REL * x[i + 1]
        return float(np.float32((x[i] + x[i + 1]) / 2))

    total = np.sort([r["E_key"] + r["E_val"] for r in plain])
    with GpuLayerCache(1, 4, 2, 256, tier2=False) as gc:
        gc.append(k, v)
        for kw in (dict(eps_key=between("E_key")), dict(eps_val=between("E_val")), dict(v_tol=between("max_block_contrib")),
                   dict(eps_total=float(total[0] / 2)), dict(force_flags=0x14), dict(mass_exp=3), dict(key_bound_mode=1), dict(key_bound_mode=2)):
            ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances(**kw))
            assert_nodes(ref, *tree_call(gc, q, kd, vd, drafts.mask_words(seen), gc.cqa.Tolerances(**kw)), where=str(kw))


def test_rows_that_attend_nothing_and_bits_behind_the_last_node():
    print("tree empty rows", flush=True)
    rng = np.random.default_rng(5)
    for n_tokens in (0, 5, 40):
        k, v, q, kd, vd = make(rng, 2, 1, 4, n_tokens, 7)
        seen = random_tree(rng, 2, 7)
        seen[0, 3] = seen[1, 0] = False
        oc = oracle.OracleLayerCache(2, 1)
        oc.append(k, v)
        ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
        mask = drafts.mask_words(seen) | np.uint64(0xFFFFFFFFFFFFFF80)   # nodes that there are not
        with GpuLayerCache(2, 4, 1, 64, tier2=False) as gc:
            if n_tokens:
                gc.append(k, v)
            O, cert, flags = tree_call(gc, q, kd, vd, mask)
            assert_nodes(ref, O, cert, flags)
            if n_tokens == 0:
                assert (O[0, 3] == 0).all() and (cert["lse"][0, 3] == -math.inf).all() and (flags == 0).all()


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_numbers_that_are_not_finite_reach_only_the_nodes_that_attend_them(what):
    print("tree not finite", what, flush=True)
    rng = np.random.default_rng(6)
    for n_tokens, n in ((0, 4), (53, 20), (70, 90)):
        k, v, q, kd, vd = make(rng, 1, 1, 2, n_tokens, n)
        seen = random_tree(rng, 1, n)
        oc = oracle.OracleLayerCache(1, 1)
        oc.append(k, v)
        ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
        kd2, vd2 = kd.copy(), vd.copy()
        kd2[0, 0, 2, 9] = what
        vd2[0, 0, n - 1, 100] = what
        hit = seen[0, :, 2] | seen[0, :, n - 1]
        assert hit.any() and not hit.all()
        with GpuLayerCache(1, 2, 1, 128, tier2=False) as gc:
            if n_tokens:
                gc.append(k, v)
            O, cert, flags = tree_call(gc, q, kd2, vd2, drafts.mask_words(seen))
            keep = np.where(~hit)[0]
            assert_nodes([[ref[0][i] for i in keep]], O[:, keep], {f: x[:, keep] for f, x in cert.items()}, flags[:, keep])
            assert np.isnan(O[:, hit]).all() and (flags[:, hit] == oracle.FLAG_PRECOND).all()


def test_a_query_that_is_not_finite_stays_in_its_row():
    print("tree query not finite", flush=True)
    rng = np.random.default_rng(7)
    k, v, q, kd, vd = make(rng, 1, 2, 4, 100, 5)
    seen = random_tree(rng, 1, 5)
    oc = oracle.OracleLayerCache(1, 2)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    q2 = q.copy()
    q2[0, 2, 5, 17] = np.nan
    with GpuLayerCache(1, 8, 2, 128, tier2=False) as gc:
        gc.append(k, v)
        O, cert, flags = tree_call(gc, q2, kd, vd, drafts.mask_words(seen))
        assert np.isnan(O[0, 2, 5]).all() and flags[0, 2, 5] & oracle.FLAG_PRECOND
        for i in range(5):
            for h in range(8):
                if (i, h) != (2, 5):
                    assert_nodes([[[ref[0][i][h]]]], O[:, i:i + 1, h:h + 1], {f: x[:, i:i + 1, h:h + 1] for f, x in cert.items()}, flags[:, i:i + 1, h:h + 1])


@pytest.mark.parametrize("ks,vs,qs", [(65504.0, 65504.0, 1e-3), (1e-3, 1e-3, 100.0), (4000.0, 1.0, 2e-3), (6e-8, 6e-8, 1.0)])
def test_the_ends_of_the_range(ks, vs, qs):
    """Keys and values up to FP16's largest number (whose reconstruction can lie beyond it) and down to its smallest."""
    print("tree range", ks, vs, qs, flush=True)
    rng = np.random.default_rng(8)
    n_tokens, n = 150, 6
    sign = lambda shape: rng.choice([-1.0, 1.0, 0.5], shape)  # noqa: E731
    k, v = (sign((1, 1, n_tokens, 128)) * ks).astype(np.float16), (sign((1, 1, n_tokens, 128)) * vs).astype(np.float16)
    kd, vd = (sign((1, 1, n, 128)) * ks).astype(np.float16), (sign((1, 1, n, 128)) * vs).astype(np.float16)
    q = (rng.standard_normal((1, n, 4, 128)) * qs).astype(np.float16)
    seen = random_tree(rng, 1, n)
    oc = oracle.OracleLayerCache(1, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    with GpuLayerCache(1, 4, 1, 160, tier2=False) as gc:
        gc.append(k, v)
        O, cert, flags = tree_call(gc, q, kd, vd, drafts.mask_words(seen))
        for b, i, h in np.ndindex(1, n, 4):
            r = ref[b][i][h]
            # results among FP16's subnormals: half their step
            r["floor"] += 1.0 if vs > 1e-6 else 2.0 * vs * 2.0 ** 25
        assert_nodes(ref, O, cert, flags)


@pytest.mark.parametrize("n", [3, 12, 30, 40])
def test_light_tokens_among_some_that_hold_nothing(n):
    """A token of each block has a score 18.4 above the others' and the value 0: what comes out is those others, of weights that FP16 does not
    hold beside 1.  Not off by more than FP16's step of their own."""
    print("tree light tokens", n, flush=True)
    n_tokens = 1000
    k, v = np.zeros((1, 1, n_tokens, 128), np.float16), np.full((1, 1, n_tokens, 128), 30000.0, np.float16)
    k[:, :, 3::16, 5], v[:, :, 3::16] = 16.0, 0.0
    kd, vd = np.zeros((1, 1, n, 128), np.float16), np.zeros((1, 1, n, 128), np.float16)
    q = np.zeros((1, n, 4, 128), np.float16)
    q[..., 5] = 13.0
    seen = np.eye(n, dtype=bool)[None]
    oc = oracle.OracleLayerCache(1, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    assert 0.002 < ref[0][0][0]["O"][0] < 0.01
    for b, i, h in np.ndindex(1, n, 4):
        ref[b][i][h]["floor"] = 0.0
    with GpuLayerCache(1, 4, 1, n_tokens, tier2=False) as gc:
        gc.append(k, v)
        assert_nodes(ref, *tree_call(gc, q, kd, vd, drafts.mask_words(seen)))


@pytest.mark.parametrize("n,n_tokens", [(2, 700), (11, 390), (27, 203), (40, 150), (130, 75)])
def test_more_sequences_than_compute_units(n, n_tokens):
    """A workgroup has all of a sequence's tokens, several turns of them, and finishes its rows."""
    print("tree of many sequences", n, n_tokens, flush=True)
    rng = np.random.default_rng(20 + n)
    bt, hkv, g = (43, 3, 2) if n > 100 else (87, 3, 4)
    k, v, q, kd, vd = make(rng, bt, hkv, g, n_tokens, n)
    seen = random_tree(rng, bt, n)
    oc = oracle.OracleLayerCache(bt, hkv)
    oc.append(k, v)
    some = [0, 1, bt // 2, bt - 1]
    part = oracle.OracleLayerCache(len(some), hkv)
    part.append(k[some], v[some])
    ref = drafts.tree_decode(part, q[some], kd[some], vd[some], seen[some], oracle.Tolerances())
    with GpuLayerCache(bt, hkv * g, hkv, n_tokens, tier2=False) as gc:
        gc.append(k, v)
        O, cert, flags = tree_call(gc, q, kd, vd, drafts.mask_words(seen))
        assert_nodes(ref, O[some], {f: x[some] for f, x in cert.items()}, flags[some])
        assert np.isfinite(O).all() and (flags == 0).all()


# the first and the last lengths of a tile, and of one and two workgroups
@pytest.mark.parametrize("g,n", [(4, 3), (4, 9), (4, 20), (2, 127), (4, 256)])
def test_lengths_at_the_tiles_ends(g, n):
    print("tree lengths", g, n, flush=True)
    rng = np.random.default_rng(30 + n)
    few = [3, n - 1] if n > 100 else range(n)   # nodes that are compared
    for n_tokens in (63, 64, 80, 127, 128, 129, 144, 192, 255, 256, 257, 272, 528, 1040):
        k, v, q, kd, vd = make(rng, 1, 1, g, n_tokens, n)
        seen = random_tree(rng, 1, n)
        oc = oracle.OracleLayerCache(1, 1)
        oc.append(k, v)
        few = list(few)
        ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances()) if n <= 100 else None
        with GpuLayerCache(1, g, 1, 1100, tier2=False) as gc:
            gc.append(k, v)
            O, cert, flags = tree_call(gc, q, kd, vd, drafts.mask_words(seen))
            if ref is None:   # a few rows: of each, the call with that node's mask alone for all of them
                for i in few:
                    one = drafts.tree_decode(oc, q[:, i:i + 1], np.ascontiguousarray(kd[:, :, seen[0, i]]), np.ascontiguousarray(vd[:, :, seen[0, i]]),
                                             np.ones((1, 1, int(seen[0, i].sum())), bool), oracle.Tolerances())
                    assert_nodes(one, O[:, i:i + 1], {f: x[:, i:i + 1] for f, x in cert.items()}, flags[:, i:i + 1], (n_tokens, i))
            else:
                assert_nodes(ref, O, cert, flags, n_tokens)


# caches that are long for the device, by many sequences or tokens: 33 .. 64, 65 .. 128, up to 256 rows and several tiles of 256; a sequence by one workgroup, by
# some, and by more than 32; without sealed tokens
WIDE = [(87, 3, 4, 1029, 16), (96, 1, 4, 2811, 13), (88, 3, 4, 300, 27), (48, 2, 4, 1029, 19), (88, 3, 4, 150, 40), (48, 1, 4, 1029, 50),
        (44, 3, 2, 75, 130), (24, 1, 4, 603, 130), (24, 1, 4, 0, 256), (12, 2, 4, 5, 255), (4, 1, 4, 10029, 64), (4, 1, 1, 20007, 201), (4, 1, 4, 12001, 8),
        (4, 1, 4, 20007, 32)]


@pytest.mark.parametrize("bt,hkv,g,n_tokens,n", WIDE)
def test_caches_that_are_long_for_the_device(bt, hkv, g, n_tokens, n):
    """Four sequences over and over, behind a reset: one as it comes, one with drafts that are no finite numbers, one with nodes that attend no draft,
    a chunk."""
    print("tree of many rows", bt, hkv, g, n_tokens, n, flush=True)
    rng = np.random.default_rng(50 + n)
    k, v, q, kd, vd = make(rng, 4, hkv, g, n_tokens, n, keys="student" if n % 2 else "normal", peaked=n % 3 == 0)
    seen = random_tree(rng, 4, n)
    seen[2, [0, n // 3, n - 1]] = False
    seen[3] = np.tril(np.ones((n, n), bool))
    nodes = np.unique(np.concatenate([[0, n // 3, n - 1], rng.choice(n, 6)]))
    oc = oracle.OracleLayerCache(4, hkv)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q[:, nodes], kd, vd, seen[:, nodes], oracle.Tolerances())
    kd[1, :, 1, 9], vd[1, :, n - 2, 100] = np.nan, np.inf
    hit = np.zeros((4, n), bool)
    hit[1] = seen[1, :, 1] | seen[1, :, n - 2]
    assert hit[1].any() and not hit[1].all()
    times = (bt + 3) // 4
    wide = lambda x: np.tile(x, (times,) + (1,) * (x.ndim - 1))[:bt]  # noqa: E731
    with GpuLayerCache(bt, hkv * g, hkv, n_tokens + 64, tier2=False) as gc:
        old = np.full((1, 1, n_tokens + 64, 128), 50.0, np.float16)
        old[..., ::3] = -700.0
        old[:, :, 1::2] *= -1
        gc.append(*[np.broadcast_to(old, (bt, hkv) + old.shape[2:])] * 2)   # larger widths and values than any that follow
        gc.cqa.cqa_cache_reset(gc.h, 0)
        if n_tokens:
            gc.append(wide(k), wide(v))
        O, cert, flags = tree_call(gc, wide(q), wide(kd), wide(vd), drafts.mask_words(wide(seen)))
    for at in range(4):
        for y in (O, flags, *cert.values()):
            assert all(np.array_equal(z, y[at], equal_nan=True) for z in y[at::4])
        assert np.isnan(O[at, hit[at]]).all() and (flags[at, hit[at]] == oracle.FLAG_PRECOND).all()
        keep = [i for i, node in enumerate(nodes) if not hit[at, node]]
        which = nodes[keep]
        assert_nodes([[ref[at][i] for i in keep]], O[at:at + 1, which], {f: y[at:at + 1, which] for f, y in cert.items()}, flags[at:at + 1, which], at)


def test_a_cache_that_is_filled_again():
    """What an earlier, longer sequence left behind the last block of a record is not the new one's: neither widths nor errors."""
    print("tree after a reset", flush=True)
    rng = np.random.default_rng(40)
    with GpuLayerCache(1, 4, 1, 1100, tier2=False) as gc:
        for n in (5, 30):
            k, v, q, kd, vd = make(rng, 1, 1, 4, 1024, n)
            gc.append((k.astype(np.float32) * 50).astype(np.float16), (v.astype(np.float32) * 50).astype(np.float16))
            tree_call(gc, q, kd, vd, None)
            for n_tokens in (0, 7, 16, 83, 100):
                gc.cqa.cqa_cache_reset(gc.h, 0)
                k, v, q, kd, vd = make(rng, 1, 1, 4, n_tokens, n)
                seen = random_tree(rng, 1, n)
                oc = oracle.OracleLayerCache(1, 1)
                if n_tokens:
                    oc.append(k, v)
                    gc.append(k, v)
                ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
                assert_nodes(ref, *tree_call(gc, q, kd, vd, drafts.mask_words(seen)), where=n_tokens)
            gc.cqa.cqa_cache_reset(gc.h, 0)


def test_one_node_agrees_with_the_appended_token_and_layers_are_apart():
    print("tree of one node against append + decode, three layers", flush=True)
    rng = np.random.default_rng(9)
    with GpuLayerCache(2, 8, 2, 400, n_layers=3) as gc:
        data = []
        for layer in range(3):
            k, v, q, kd, vd = make(rng, 2, 2, 4, 100 + 97 * layer, 1)
            gc.append(k, v, layer)
            data.append((q, kd, vd))
        for layer, (q, kd, vd) in enumerate(data):
            O, cert, flags = tree_call(gc, q, kd, vd, None, layer=layer)
            gc.append(kd, vd, layer)
            O1, c1, f1 = gc.certified_decode(q[:, 0], layer=layer)
            assert (np.linalg.norm(O[:, 0] - O1, axis=-1) <= 2e-3 * np.linalg.norm(O1, axis=-1)).all()
            for name in ("E_key", "E_val", "delta_h"):
                assert (cert[name][:, 0] >= c1[name] * (1 - 2e-3)).all() and (cert[name][:, 0] <= c1[name] * 1.25).all(), name


def test_a_layer_beyond_32_bits_of_offset():
    """The records of the last layer start 4.6 GB behind the first."""
    print("tree and read in a layer far behind", flush=True)
    rng = np.random.default_rng(10)
    layers, cap, n_tokens, n = 63, 262144, 1000, 9
    assert (layers - 1) * cap * 290 > 2 ** 32
    k, v, q, kd, vd = make(rng, 1, 1, 4, n_tokens, n)
    seen = random_tree(rng, 1, n)
    oc = oracle.OracleLayerCache(1, 1)
    oc.append(k, v)
    ref = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    with GpuLayerCache(1, 4, 1, cap, tier2=False, n_layers=layers) as gc:
        gc.append(k, v, layers - 1)
        assert_nodes(ref, *tree_call(gc, q, kd, vd, drafts.mask_words(seen), layer=layers - 1))
        check_read(gc, oc, 3, 995, "fp16", layer=layers - 1)


def test_a_long_cache_against_the_single_token_pass():
    """128K tokens: O and the certificate of a chain's nodes whose drafts are masked out are those of the single-token call, up to
    the rounding of the reconstruction (O 2e-3 of its norm; lse 1e-3)."""
    print("tree over 128K", flush=True)
    t = _torch()
    n_tokens, n = 131072 + 11, 5
    k, v = workloads.torch_device_kv("t128k", 0, t.device("cuda:0"), seed=3, context=n_tokens)
    rng = np.random.default_rng(11)
    q = workloads.normal_f16(rng, (1, n, 32, 128))
    kd, vd = workloads.normal_f16(rng, (1, 8, n, 128)), workloads.normal_f16(rng, (1, 8, n, 128))
    with GpuLayerCache(1, 32, 8, n_tokens + 16, tier2=False) as gc:
        gc.append(k, v)
        O, cert, flags = tree_call(gc, q, kd, vd, np.zeros((1, n, 1), np.uint64))
        for i in range(n):
            O1, c1, _ = gc.certified_decode(q[:, i])
            assert (np.linalg.norm(O[:, i] - O1, axis=-1) <= 2e-3 * np.linalg.norm(O1, axis=-1)).all()
            assert np.abs(cert["lse"][:, i] - c1["lse"]).max() <= 1e-3
            assert (cert["delta_h"][:, i] >= c1["delta_h"]).all() and (cert["delta_h"][:, i] <= 1.25 * c1["delta_h"]).all()
            assert (cert["v_max"][:, i] == c1["v_max"]).all()


def test_recorded_calls_follow_their_buffers():
    """Two calls with workspaces of their own in one graph, replayed with other queries, masks and eager work in between."""
    print("tree in a graph", flush=True)
    rng = np.random.default_rng(12)
    bt, hkv, g, n_tokens, n = 1, 2, 4, 900, 12
    with GpuLayerCache(bt, hkv * g, hkv, 1024, tier2=False) as gc:
        t, cqa = gc.torch, gc.cqa
        k, v, q, kd, vd = make(rng, bt, hkv, g, n_tokens, n)
        gc.append(k, v)
        qd, kdd, vdd = (gc.to_dev(x).clone() for x in (q, kd, vd))
        mask = t.from_numpy(drafts.mask_words(random_tree(rng, bt, n)).view(np.int64)).cuda()
        a, b = Nodes(cqa, gc.h, bt, n, hkv * g), Nodes(cqa, gc.h, bt, n, hkv * g)
        s, graph = t.cuda.Stream(), t.cuda.CUDAGraph()
        t.cuda.synchronize()
        with t.cuda.graph(graph, stream=s):
            cqa.cqa_tree_decode(gc.h, 0, qd, kdd, vdd, n, mask, cqa.Tolerances(), a.O, a.cert, a.flags, a.ws, s.cuda_stream)
            cqa.cqa_tree_decode(gc.h, 0, qd, kdd, vdd, n, None, cqa.Tolerances(), b.O, b.cert, b.flags, b.ws, s.cuda_stream)
        for rep in range(4):
            _, _, q, kd, vd = make(rng, bt, hkv, g, 1, n)
            seen = random_tree(rng, bt, n)
            for x, y in ((qd, q), (kdd, kd), (vdd, vd)):
                x.copy_(gc.to_dev(y))
            mask.copy_(t.from_numpy(drafts.mask_words(seen).view(np.int64)))
            want = [tree_call(gc, q, kd, vd, drafts.mask_words(seen)), tree_call(gc, q, kd, vd, None)]
            for out in (a, b):
                out.ws.fill_(0xFF)
                out.O.fill_(7.0)
            t.cuda.synchronize()
            graph.replay()
            for out, w in zip((a, b), want):
                got = out.results()
                assert np.array_equal(got[0], w[0]) and np.array_equal(got[2], w[2]), rep
                assert all(np.array_equal(got[1][f], w[1][f]) for f in w[1]), rep


def test_two_streams_at_a_time():
    print("tree on two streams", flush=True)
    rng = np.random.default_rng(13)
    k, v, q, kd, vd = make(rng, 1, 4, 4, 6000, 30)
    mask = drafts.mask_words(random_tree(rng, 1, 30))
    with GpuLayerCache(1, 16, 4, 6100, tier2=False) as gc:
        t, cqa = gc.torch, gc.cqa
        gc.append(k, v)
        want = [tree_call(gc, q, kd, vd, mask), tree_call(gc, q, kd, vd, None)]
        qd, kdd, vdd, md = *(gc.to_dev(x) for x in (q, kd, vd)), t.from_numpy(mask.view(np.int64)).cuda()
        outs = [Nodes(cqa, gc.h, 1, 30, 16) for _ in range(2)]
        streams = [t.cuda.Stream() for _ in range(2)]
        t.cuda.synchronize()
        for _ in range(8):
            for out, s, m in zip(outs, streams, (md, None)):
                cqa.cqa_tree_decode(gc.h, 0, qd, kdd, vdd, 30, m, cqa.Tolerances(), out.O, out.cert, out.flags, out.ws, s.cuda_stream)
        for out, w in zip(outs, want):
            got = out.results()
            assert np.array_equal(got[0], w[0]) and all(np.array_equal(got[1][f], w[1][f]) for f in w[1])


def test_the_tree_call_refuses_what_it_does_not_do():
    print("tree refusals", flush=True)
    cqa = load_binding()
    with GpuLayerCache(1, 8, 2, 64, tier2=False) as gc:
        tol = cqa.Tolerances()

        def refused(status, layer=0, q=4096, k=4096, v=4096, n=4, mask=None, tol=tol, O=4096, cert=4096, flags=4096, ws=4096):
            with pytest.raises(cqa.CqaError) as e:
                cqa.cqa_tree_decode(gc.h, layer, q, k, v, n, mask, tol, O, cert, flags, ws)
            assert e.value.status == status

        bad, no = cqa.ERR_INVALID_ARG, cqa.ERR_UNSUPPORTED
        for kw in (dict(layer=-1), dict(layer=1), dict(q=None), dict(k=None), dict(v=None), dict(O=None), dict(cert=None), dict(flags=None),
                   dict(ws=None), dict(n=0), dict(n=-1), dict(q=4097), dict(k=4097), dict(v=4097), dict(mask=4100), dict(O=4104), dict(cert=4100),
                   dict(flags=4100), dict(ws=4104), dict(tol=cqa.Tolerances(mass_exp=-1)), dict(tol=cqa.Tolerances(key_bound_mode=3))):
            refused(bad, **kw)
        for kw in (dict(n=257), dict(tol=cqa.Tolerances(rank_depth=1)), dict(tol=cqa.Tolerances(int8_query=True))):
            refused(no, **kw)
        for n, status in ((0, bad), (257, no)):
            with pytest.raises(cqa.CqaError) as e:
                cqa.cqa_tree_workspace_bytes(gc.h, n)
            assert e.value.status == status
        assert cqa._lib.cqa_tree_workspace_bytes(gc.h, 1, None) == bad


# ---- reading back ----------------------------------------------------------------------------------------------------------

def rounded(x, name):
    """float64 or binary32 numbers rounded to the type, as float64."""
    t = _torch()
    if name == "fp16":
        return drafts.to_fp16(x).astype(np.float64)
    y = np.asarray(x, np.float64).astype(np.float32)
    return (t.from_numpy(y).to(t.bfloat16).double().numpy() if name == "bf16" else y.astype(np.float64))


def check_read(gc, oc, first, n, name, strides=None, layer=0, only=None):
    cqa, t = gc.cqa, gc.torch
    dt = {"fp16": t.float16, "bf16": t.bfloat16, "fp32": t.float32}[name]
    bt, hkv = oc.bt, oc.hkv
    if strides is None:
        size, view = bt * hkv * n * 128, lambda x: x.view(bt, hkv, n, 128)
    else:
        size, view = strides[3], lambda x: x.as_strided((bt, hkv, n, 128), (*strides[:3], 1))
    bufs = [t.full((size + 32,), 7.0, dtype=dt, device="cuda") for _ in range(2)]
    outs = [None if only is not None and only != i else x for i, x in enumerate(bufs)]
    cqa.cqa_cache_read(gc.h, layer, first, n, {"fp16": cqa.FP16, "bf16": cqa.BF16, "fp32": cqa.FP32}[name], outs[0], outs[1],
                       None if strides is None else strides[:3])
    t.cuda.synchronize()
    for i, (x, want) in enumerate(zip(bufs, drafts.read_back(oc, first, n))):
        got = view(x[:size]).double().cpu().numpy()
        if outs[i] is None:
            assert (x == 7.0).all()
            continue
        ok = got == rounded(want, name)
        assert ok.all(), (name, i, first, n, np.argwhere(~ok)[:3], got[~ok][:3], rounded(want, name)[~ok][:3])
        keep = t.zeros_like(x, dtype=t.bool)
        view(keep[:size])[:] = True
        assert (x[~keep] == 7.0).all()          # between and behind the rows nothing is written


@pytest.mark.parametrize("bt,hkv,n_tokens,keys", [(1, 1, 1, "normal"), (1, 2, 15, "normal"), (2, 3, 16, "student"), (1, 2, 333, "student"), (3, 1, 1029, "normal")])
def test_reading_back_gives_the_definition(bt, hkv, n_tokens, keys):
    print("read", bt, hkv, n_tokens, flush=True)
    rng = np.random.default_rng(n_tokens)
    k, v, *_ = make(rng, bt, hkv, 1, n_tokens, 1, keys)
    k[..., 5] += np.float16(30.0)                # a channel far from zero
    v[..., 16:32] = v[..., 16:17]                # groups of one value
    oc = oracle.OracleLayerCache(bt, hkv)
    oc.append(k, v)
    with GpuLayerCache(bt, hkv, hkv, n_tokens + 5, tier2=False) as gc:
        gc.append(k, v)
        spans = {(0, n_tokens), (0, 1), (n_tokens - 1, 1), (n_tokens // 2, (n_tokens + 2) // 3), (max(0, n_tokens - 20), min(n_tokens, 20))}
        for first, n in sorted(spans):
            n = min(n, n_tokens - first)
            for name in ("fp16", "bf16", "fp32"):
                check_read(gc, oc, first, n, name)
                # token-major rows with gaps between them
                check_read(gc, oc, first, n, name, (n * hkv * 136 + 8, 136, hkv * 136, bt * (n * hkv * 136 + 8)))
        check_read(gc, oc, 0, n_tokens, "fp16", only=0)
        check_read(gc, oc, 0, n_tokens, "fp16", only=1)


def test_reading_back_at_the_ends_of_the_range_and_refusals():
    print("read range", flush=True)
    cqa = load_binding()
    rng = np.random.default_rng(1)
    for scale in (65504.0, 6e-8):
        k, v = ((rng.choice([-1.0, 1.0, 0.3], (1, 1, 40, 128)) * scale).astype(np.float16) for _ in range(2))
        oc = oracle.OracleLayerCache(1, 1)
        oc.append(k, v)
        with GpuLayerCache(1, 1, 1, 64, tier2=False) as gc:
            gc.append(k, v)
            for name in ("fp16", "bf16", "fp32"):
                check_read(gc, oc, 0, 40, name)
            for args, status in (((0, -1, 1), 1), ((0, 0, -1), 1), ((0, 0, 41), 1), ((0, 40, 1), 1), ((0, 41, 0), 1), ((1, 0, 1), 1), ((-1, 0, 1), 1)):
                with pytest.raises(cqa.CqaError) as e:
                    cqa.cqa_cache_read(gc.h, *args, cqa.FP16, 4096, 4096)
                assert e.value.status == cqa.ERR_INVALID_ARG
            for typ, kk, vv in ((cqa.FP16, None, None), (3, 4096, 4096), (-1, 4096, 4096), (cqa.FP16, 4097, None), (cqa.FP32, None, 4098)):
                with pytest.raises(cqa.CqaError) as e:
                    cqa.cqa_cache_read(gc.h, 0, 0, 1, typ, kk, vv)
                assert e.value.status == cqa.ERR_INVALID_ARG
            cqa.cqa_cache_read(gc.h, 0, 40, 0, cqa.FP16, 4096, 4096)    # nothing to read
            gc.torch.cuda.synchronize()


# ---- rotary ----------------------------------------------------------------------------------------------------------------

SCALINGS = {"plain": {}, "linear": dict(factor=4.0), "parts": dict(factor=8.0, low_rotations=1.0, high_rotations=4.0, trained_tokens=8192)}
STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


@pytest.mark.parametrize("rot,interleaved,scaling,src,dst,bt,n", [
    (128, False, "plain", "bf16", "fp16", 1, 1), (128, True, "parts", "fp32", "fp16", 2, 27), (64, False, "linear", "fp16", "fp16", 3, 33),
    (64, True, "plain", "fp16", "bf16", 1, 100), (16, False, "parts", "fp32", "fp32", 1, 5), (2, True, "plain", "fp32", "fp32", 2, 9),
    (2, False, "plain", "bf16", "bf16", 1, 64), (102, False, "parts", "fp32", "fp32", 1, 31), (126, True, "linear", "bf16", "fp32", 2, 3),
    (96, False, "plain", "fp32", "bf16", 1, 1000), (48, True, "parts", "fp16", "fp32", 5, 65)])
def test_rotary_matches_the_definition(rot, interleaved, scaling, src, dst, bt, n):
    print("rotary", rot, interleaved, scaling, src, dst, bt, n, flush=True)
    t = _torch()
    cqa = load_binding()
    types = {"fp16": (t.float16, cqa.FP16), "bf16": (t.bfloat16, cqa.BF16), "fp32": (t.float32, cqa.FP32)}
    rng = np.random.default_rng(rot + n)
    hq, hk, magnitude = 5, 2, 1.0 if scaling == "plain" else 1.25
    kw = SCALINGS[scaling]
    f = drafts.rotary_frequencies(rot, 500000.0, scaling, kw.get("factor", 1.0), kw.get("low_rotations", 0), kw.get("high_rotations", 0), kw.get("trained_tokens", 0))
    x = t.from_numpy(rng.standard_normal((bt, n, hq + 2 * hk, 128)).astype(np.float32)).to(types[src][0])
    xd = x.cuda()
    # near, far, beyond 32 bits, and turning back
    pos = np.stack([rng.choice([0, 1, 131071, 2 ** 31 + 7, 2 ** 40 + 3, -5, -131000], n) + np.arange(n) for _ in range(bt)]).astype(np.int64)
    pd = t.from_numpy(pos).cuda()
    q_out = t.full((bt, n, hq, 128), 9.0, dtype=types[dst][0], device="cuda")
    k_out = t.full((bt, hk, n + 1, 128), 9.0, dtype=types[dst][0], device="cuda")
    r = cqa.cqa_rotary_create(rot_dim=rot, layout=cqa.ROTARY_INTERLEAVED if interleaved else cqa.ROTARY_HALF, base=500000.0,
                              scaling={"plain": cqa.ROTARY_PLAIN, "linear": cqa.ROTARY_LINEAR, "parts": cqa.ROTARY_PARTS}[scaling], magnitude=magnitude, **kw)
    row = (hq + 2 * hk) * 128
    rows = [cqa.RotaryRows(xd, q_out, hq, (n * row, 128, row), (n * hq * 128, 128, hq * 128)),
            cqa.RotaryRows(xd[:, :, hq:], k_out, hk, (n * row, 128, row), (hk * (n + 1) * 128, (n + 1) * 128, 128))]
    cqa.cqa_rotary_apply(r, pd, n, bt, n, rows, types[src][1], types[dst][1])
    t.cuda.synchronize()
    x64 = x.double().numpy()
    for b in range(bt):
        want = drafts.rotary(x64[b, :, :hq + hk].transpose(1, 0, 2), pos[b], f, interleaved, magnitude)
        a = np.abs(x64[b, :, :hq + hk].transpose(1, 0, 2))
        pair = a.copy()          # |a| + |b| of the pair a channel belongs to
        half = rot // 2
        at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
        pair[..., at[0]] = pair[..., at[1]] = a[..., at[0]] + a[..., at[1]]
        # sine and cosine within 2^-22 (2^-24 of a turn: 2 pi 2^-25 of the angle, and their own rounding), two roundings of FP32
        tol = STEP[dst] * np.abs(want) + 2.0 ** -21 * magnitude * pair + 2.0 ** -25
        tol[..., rot:] = STEP[dst] * np.abs(want[..., rot:])
        got = np.concatenate([q_out[b].transpose(0, 1).double().cpu().numpy(), k_out[b, :, :n].double().cpu().numpy()])
        assert (np.abs(got - want) <= tol).all(), (b, float((np.abs(got - want) - tol).max()))
    assert (k_out[:, :, n] == 9.0).all()
    if src == dst:      # in place: the same bits
        cqa.cqa_rotary_apply(r, pd, n, bt, n, [cqa.RotaryRows(xd, xd, hq, (n * row, 128, row), (n * row, 128, row))], types[src][1], types[dst][1])
        t.cuda.synchronize()
        assert (xd[:, :, :hq] == q_out).all() and (xd[:, :, hq:].cpu() == x[:, :, hq:]).all()
    # one set of positions for all sequences, at an odd address, on a stream of its own
    s = t.cuda.Stream()
    if bt > 1:
        buf = t.empty(bt * n * hq * 128 + 1, dtype=types[dst][0], device="cuda")
        out = buf[1:].view(bt, n, hq, 128)
        fresh = x.cuda()
        t.cuda.synchronize()
        cqa.cqa_rotary_apply(r, pd, 0, bt, n, [cqa.RotaryRows(fresh, out, hq, (n * row, 128, row), (n * hq * 128, 128, hq * 128))],
                             types[src][1], types[dst][1], s.cuda_stream)
        t.cuda.synchronize()
        assert (out[0] == q_out[0]).all()
        same = t.empty_like(out)
        cqa.cqa_rotary_apply(r, pd[:1].expand(bt, n).contiguous(), n, bt, n,
                             [cqa.RotaryRows(fresh, same, hq, (n * row, 128, row), (n * hq * 128, 128, hq * 128))], types[src][1], types[dst][1])
        t.cuda.synchronize()
        assert (out == same).all()
    cqa.cqa_rotary_destroy(r)


def test_many_tokens_and_heads_and_the_gradient():
    """Every thread walks over several heads here; turning back by the same positions is the gradient, checked against differences."""
    print("rotary large", flush=True)
    t = _torch()
    cqa = load_binding()
    n, h = 9001, 40
    r = cqa.cqa_rotary_create(rot_dim=128, base=500000.0)
    g = t.Generator(device="cuda")
    g.manual_seed(1)
    x, dx, dy = (t.randn((1, n, h, 128), generator=g, device="cuda") for _ in range(3))
    pos = t.arange(n, device="cuda") + 100000
    st = (n * h * 128, 128, h * 128)

    def turn(x, pos):
        y = t.empty_like(x)
        cqa.cqa_rotary_apply(r, pos, 0, 1, n, [cqa.RotaryRows(x, y, h, st, st)], cqa.FP32, cqa.FP32)
        return y

    back = turn(turn(x, pos), -pos)
    # two turns: twice the forward error 2^-21 (|a| + |b|) of numbers within 6 sigma
    assert (back - x).abs().max() <= 2 * 2.0 ** -21 * 2 * x.abs().max() * 1.5
    diff = (turn(x + dx, pos) - turn(x - dx, pos)) / 2
    lhs, rhs = (dy.double() * diff.double()).sum(), (turn(dy, -pos).double() * dx.double()).sum()
    # sums of 46 M products of magnitude 1 with errors of 2^-20 each, added up at random: 7000 * 2^-20 and a margin of 10
    assert abs(lhs - rhs) <= 0.1
    cqa.cqa_rotary_destroy(r)


# ---- together --------------------------------------------------------------------------------------------------------------

def test_a_speculative_turn_from_the_projection_to_the_appended_path():
    """Prompt rows are turned and appended; drafted rows are turned, attend the cache as a tree, the accepted path is appended, and
    the next step decodes; a second cache gets the reconstruction moved towards the front.  Each stage against the oracle on the
    numbers that the stage before gave."""
    print("speculative turn", flush=True)
    t = _torch()
    cqa = load_binding()
    rng = np.random.default_rng(21)
    hkv, g, n_tokens, n = 2, 4, 150, 11
    hq = hkv * g
    row = (hq + 2 * hkv) * 128
    r = cqa.cqa_rotary_create(rot_dim=128, base=500000.0, scaling=cqa.ROTARY_PARTS, **SCALINGS["parts"])
    f = drafts.rotary_frequencies(128, 500000.0, "parts", 8.0, 1.0, 4.0, 8192)

    def project(m, pos):
        fused = t.from_numpy(rng.standard_normal((1, m, hq + 2 * hkv, 128)).astype(np.float32)).to(t.bfloat16).cuda()
        q, k = t.empty((1, m, hq, 128), dtype=t.float16, device="cuda"), t.empty((1, hkv, m, 128), dtype=t.float16, device="cuda")
        cqa.cqa_rotary_apply(r, t.from_numpy(np.asarray(pos, np.int64)).cuda(), 0, 1, m,
                             [cqa.RotaryRows(fused, q, hq, (m * row, 128, row), (m * hq * 128, 128, hq * 128)),
                              cqa.RotaryRows(fused[:, :, hq:], k, hkv, (m * row, 128, row), (hkv * m * 128, m * 128, 128))], cqa.BF16, cqa.FP16)
        v = fused[:, :, hq + hkv:].transpose(1, 2).to(t.float16).contiguous()
        want = drafts.rotary(fused[0, :, hq:hq + hkv].double().cpu().numpy().transpose(1, 0, 2), pos, f, False)
        assert np.abs(k[0].double().cpu().numpy() - want).max() <= 2.0 ** -11 * np.abs(want).max() + 1e-5
        return q, k, v

    with GpuLayerCache(1, hq, hkv, 256) as gc, GpuLayerCache(1, hq, hkv, 256, tier2=False) as moved:
        _, k, v = project(n_tokens, np.arange(n_tokens))
        cqa.cqa_cache_append(gc.h, 0, k, v, n_tokens)
        oc = oracle.OracleLayerCache(1, hkv)
        oc.append(k.cpu().numpy(), v.cpu().numpy())
        parents = [-1, 0, 0, 1, 1, 2, 3, 3, 6, 6, 8]
        seen = drafts.ancestors(parents)[None]
        depth = seen[0].sum(1) - 1
        q, kd, vd = project(n, n_tokens + depth)
        got = tree_call(gc, q.cpu().numpy(), kd.cpu().numpy(), vd.cpu().numpy(), drafts.mask_words(seen))
        assert_nodes(drafts.tree_decode(oc, q.cpu().numpy(), kd.cpu().numpy(), vd.cpu().numpy(), seen, oracle.Tolerances()), *got)
        path = [0, 1, 3, 6, 8]
        assert [parents[i] for i in path[1:]] == path[:-1]
        ka, va = kd[:, :, path].contiguous(), vd[:, :, path].contiguous()
        cqa.cqa_cache_append(gc.h, 0, ka, va, len(path))
        oc.append(ka.cpu().numpy(), va.cpu().numpy())
        q, k1, v1 = project(1, [n_tokens + len(path)])
        cqa.cqa_append_decode_step(gc.h, 0, k1, v1, q, cqa.Tolerances(), gc.O, gc.cert, gc.flags)
        oc.append(k1.cpu().numpy(), v1.cpu().numpy())
        O, _, _ = gc.results()
        for h, ref in enumerate(oc.decode_step(q[0].cpu().numpy(), oracle.Tolerances())):
            assert np.linalg.norm(O[0, h] - ref["O"]) <= 1e-3 * np.linalg.norm(ref["O"])
        # the last 100 tokens into another cache, 56 positions further to the front
        total, keep = oc.length, 100
        check_read(gc, oc, total - keep, keep, "fp16")
        kr, vr = (t.empty((1, hkv, keep, 128), dtype=t.float16, device="cuda") for _ in range(2))
        cqa.cqa_cache_read(gc.h, 0, total - keep, keep, cqa.FP16, kr, vr)
        before = kr.clone()
        st = (hkv * keep * 128, keep * 128, 128)
        shift = t.full((keep,), keep - total, dtype=t.int64, device="cuda")
        cqa.cqa_rotary_apply(r, shift, 0, 1, keep, [cqa.RotaryRows(kr, kr, hkv, st, st)])
        cqa.cqa_cache_append(moved.h, 0, kr, vr, keep)
        assert moved.length() == keep
        want = drafts.rotary(before[0].double().cpu().numpy(), np.full(keep, keep - total), f, False)
        assert np.abs(kr[0].double().cpu().numpy() - want).max() <= 2.0 ** -11 * np.abs(want).max() + 1e-5
    cqa.cqa_rotary_destroy(r)
