"""CPU checks of the drafted tokens' definitions and of the calls' refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest

import oracle
from helpers import load_binding
from oracle import drafts


def _cache(rng, bt, hkv, n, scale=1.0):
    oc = oracle.OracleLayerCache(bt, hkv)
    oc.append((rng.standard_normal((bt, hkv, n, 128)) * scale).astype(np.float16), rng.standard_normal((bt, hkv, n, 128)).astype(np.float16))
    return oc


@pytest.mark.parametrize("shift,scale", [(0.0, 1.0), (30.0, 1.0), (0.0, 1e-4), (0.0, 2000.0)])
def test_widths_and_value_errors_cover_the_rounding_to_fp16(shift, scale):
    """|FP16(k^) - k| <= w / 2 and max_t ||FP16(v^) - v|| <= eta', also where rounding dominates (a channel far from zero)."""
    rng = np.random.default_rng(3)
    oc = oracle.OracleLayerCache(1, 2)
    k = ((rng.standard_normal((1, 2, 64, 128)) + shift) * scale).astype(np.float16)
    v = ((rng.standard_normal((1, 2, 64, 128)) + shift) * scale).astype(np.float16)
    oc.append(k, v)
    kr, vr = drafts.read_back(oc, 0, 64)
    dk = np.abs(drafts.to_fp16(kr).astype(np.float64) - k.astype(np.float64)).reshape(1, 2, 4, 16, 128).max(3)
    w = drafts.key_widths(oc.sigma, oc.z)
    # sigma, z and the reconstruction itself are binary32: 2^-22 of the largest key
    assert (dk <= w / 2 + np.abs(k.astype(np.float64)).max() * 2.0 ** -22).all()
    assert (w <= oc.sigma.astype(np.float64) * 2.002 + 1e-7).all()
    dv = np.sqrt(((drafts.to_fp16(vr).astype(np.float64) - v.astype(np.float64)) ** 2).sum(-1)).reshape(1, 2, 4, 16).max(-1)
    assert (dv <= drafts.value_errors(oc.eta, oc.nu) * (1 + 1e-6)).all()


@pytest.mark.parametrize("n_tokens,n,scale", [(48, 5, 1.0), (53, 9, 0.3), (7, 4, 1.0), (0, 3, 1.0)])
def test_the_certificate_bounds_the_distance_to_attention_on_the_originals(n_tokens, n, scale):
    rng = np.random.default_rng(n_tokens)
    oc = _cache(rng, 1, 1, n_tokens, scale)
    q = rng.standard_normal((1, n, 2, 128)).astype(np.float16)
    kd, vd = (rng.standard_normal((1, 1, n, 128)).astype(np.float16) for _ in range(2))
    seen = drafts.ancestors([-1] + [int(rng.integers(0, i)) for i in range(1, n)])[None]
    res = drafts.tree_decode(oc, q, kd, vd, seen, oracle.Tolerances())
    for i in range(n):
        k = np.concatenate([oc.k16[0, 0], kd[0, 0][seen[0, i]]])
        v = np.concatenate([oc.v16[0, 0], vd[0, 0][seen[0, i]]])
        for h in range(2):
            r = res[0][i][h]
            ref = oracle.softmax_attention(q[0, i, h], k, v)
            assert np.linalg.norm(r["O"] - ref) <= r["E_key"] + r["E_val"] + 1e-9
            assert r["flags"] == 0
            if n_tokens < 16:
                assert r["E_key"] == 0 and r["E_val"] == 0 and np.allclose(r["O"], ref, atol=1e-12)


def test_one_node_is_an_appended_token_up_to_the_rounding():
    rng = np.random.default_rng(11)
    oc = _cache(rng, 1, 1, 70)
    q = rng.standard_normal((1, 1, 4, 128)).astype(np.float16)
    kd, vd = (rng.standard_normal((1, 1, 1, 128)).astype(np.float16) for _ in range(2))
    res = drafts.tree_decode(oc, q, kd, vd, np.ones((1, 1, 1), bool), oracle.Tolerances())
    oc.append(kd, vd)
    for a, b in zip(res[0][0], oc.certified_decode(q[0], oracle.Tolerances())):
        assert np.linalg.norm(a["O"] - b["O"]) <= 2e-3 * np.linalg.norm(b["O"])
        for name in ("E_key", "E_val", "delta_h", "max_block_contrib"):
            assert b[name] * (1 - 2e-3) <= a[name] <= b[name] * 1.25, name
        assert a["v_max"] == b["v_max"]


def test_masks_are_packed_by_node():
    seen = drafts.ancestors([-1, 0, 0, 1] + [3] * 66)[None]
    w = drafts.mask_words(seen)
    assert w.shape == (1, 70, 2) and w[0, 0, 0] == 1 and w[0, 3, 0] == 0b1011 and w[0, 69, 0] == 0b1011 and w[0, 69, 1] == 1 << 5


def test_turning_back_undoes_turning_and_is_its_gradient():
    rng = np.random.default_rng(2)
    for interleaved in (False, True):
        f = drafts.rotary_frequencies(96, 500000.0, "parts", 8.0, 1.0, 4.0, 8192)
        pos = np.array([0, 3, 131071, 2 ** 33])
        x = rng.standard_normal((2, 4, 128))
        y = drafts.rotary(x, pos, f, interleaved)
        assert np.allclose(drafts.rotary(y, -pos, f, interleaved), x, atol=1e-12)
        # <dy, J dx> = <J^T dy, dx>, J^T = the turn back; and J dx by differences (the map is linear)
        dx, dy = rng.standard_normal(x.shape), rng.standard_normal(x.shape)
        diff = (drafts.rotary(x + dx, pos, f, interleaved) - drafts.rotary(x - dx, pos, f, interleaved)) / 2
        assert math.isclose((dy * diff).sum(), (drafts.rotary(dy, -pos, f, interleaved) * dx).sum(), rel_tol=1e-10)


def _refused(cqa, status, call, *args, **kw):
    with pytest.raises(cqa.CqaError) as e:
        call(*args, **kw)
    assert e.value.status == status, (e.value.status, status, args, kw)


def test_rotary_tables_refuse_what_has_no_meaning():
    cqa = load_binding()
    good = dict(rot_dim=128, base=10000.0, scaling=cqa.ROTARY_PARTS, factor=8.0, low_rotations=1.0, high_rotations=4.0, trained_tokens=8192)
    cqa.cqa_rotary_destroy(cqa.cqa_rotary_create(**good))
    for bad in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=130), dict(rot_dim=-2), dict(layout=2), dict(layout=-1), dict(scaling=3),
                dict(scaling=-1), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan), dict(factor=0.0),
                dict(factor=math.nan), dict(factor=math.inf), dict(low_rotations=-1.0), dict(low_rotations=4.0), dict(high_rotations=math.inf),
                dict(high_rotations=math.nan), dict(trained_tokens=0), dict(magnitude=0.0), dict(magnitude=math.nan), dict(magnitude=math.inf),
                dict(base=0.99), dict(factor=0.99)):
        _refused(cqa, cqa.ERR_INVALID_ARG, cqa.cqa_rotary_create, **{**good, **bad})
    cqa.cqa_rotary_destroy(cqa.cqa_rotary_create(rot_dim=2, factor=0.0))        # PLAIN reads no factor
    assert cqa._lib.cqa_rotary_create(None, ctypes.byref(ctypes.c_void_p())) == cqa.ERR_INVALID_ARG
    assert cqa._lib.cqa_rotary_create(ctypes.byref(cqa.RotaryDesc(128, 0, 0, 1.0, 1e4, 1.0, 0, 0, 0)), None) == cqa.ERR_INVALID_ARG
    _refused(cqa, cqa.ERR_INVALID_ARG, cqa.cqa_rotary_destroy, None)


def test_rotary_refuses_bad_rows_before_anything_is_read():
    """The addresses are not memory: nothing may be launched."""
    cqa = load_binding()
    r = cqa.cqa_rotary_create()
    st = (128, 128, 128)
    row = lambda i=4096, o=8192, h=1: cqa.RotaryRows(i, o, h, st, st)  # noqa: E731
    call = cqa.cqa_rotary_apply
    bad = cqa.ERR_INVALID_ARG
    _refused(cqa, bad, call, None, 4096, 1, 1, 1, [row()])
    _refused(cqa, bad, call, r, None, 1, 1, 1, [row()])
    _refused(cqa, bad, call, r, 4100, 1, 1, 1, [row()])
    for batch in (0, -1, 65536):
        _refused(cqa, bad, call, r, 4096, 1, batch, 1, [row()])
    _refused(cqa, bad, call, r, 4096, 1, 1, -1, [row()])
    _refused(cqa, bad, call, r, 4096, 1, 1, 1, [])
    _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row(), row(), row()])
    for x in (row(i=None), row(o=None), row(h=0), row(h=-3), row(h=65536), row(i=4097), row(o=8193)):
        _refused(cqa, bad, call, r, 4096, 1, 1, 1, [x])
        _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row(), x])
    _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row(i=4098)], cqa.FP32, cqa.FP16)
    _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row(o=8194)], cqa.FP16, cqa.FP32)
    for t in (3, -1):
        _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row()], t, cqa.FP16)
        _refused(cqa, bad, call, r, 4096, 1, 1, 1, [row()], cqa.FP16, t)
    x = row()
    x.reserved = 1
    _refused(cqa, bad, call, r, 4096, 1, 1, 1, [x])
    _refused(cqa, cqa.ERR_UNSUPPORTED, call, r, 4096, 1, 1, 1 << 40, [row()])
    call(r, None, 1, 1, 0, [row()])                                             # no tokens: nothing to do
    cqa.cqa_rotary_destroy(r)


def test_struct_layouts_of_the_drafted_calls():
    cqa = load_binding()
    assert ctypes.sizeof(cqa.NodeCert) == 32
    assert ctypes.sizeof(cqa.Strides) == 24
    assert ctypes.sizeof(cqa.RotaryDesc) == 56
    assert ctypes.sizeof(cqa.RotaryRows) == 72


def test_no_handle_no_call():
    cqa = load_binding()
    _refused(cqa, cqa.ERR_INVALID_ARG, cqa.cqa_cache_read, None, 0, 0, 1, cqa.FP16, 4096, 4096)
    _refused(cqa, cqa.ERR_INVALID_ARG, cqa.cqa_tree_workspace_bytes, None, 1)
    _refused(cqa, cqa.ERR_INVALID_ARG, cqa.cqa_tree_decode, None, 0, 4096, 4096, 4096, 1, None, cqa.Tolerances(), 4096, 4096, 4096, 4096)
