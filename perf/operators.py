"""The operators that a program puts around the certified cache when it decodes several drafted tokens at once, and how
they are measured: rotary positions of the projections' rows, attention of a tree of drafted tokens over the quantized
cache, and the reading back of the cache's reconstruction.

`run` computes each in its plain form (elementary torch operations, `own` false) or by the calls a user makes of the
library (`own` true); both take the same state.  Sizes are those of this repository's caches: head_dim 128, 1, 2 or 4
query heads per KV head, keys N(0, 1), N(0, 1) with outlier channels x 20 or Student-t(3).

kinds
  rotary  queries and keys of a fused projection [batch][token][heads of q, k, v][128] turned by their positions and
          written as the cache takes them: keys [batch][head][token][128], queries [batch][token][head][128].
  read    tokens first .. first + count of every sequence as the cache reconstructs them.
  tree    drafted tokens, each attending the cache, its ancestors and itself, with the certificate of every (node, head).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 128
BLK = 16
NG = 8
T1_BYTES = 288.5         # quantized bytes per token and KV head: codes, metadata, block annotations
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"fp16": 2, "bf16": 2, "fp32": 4}
F16_MAX = 65504.0
HALF_STEP = 2.0 ** -11   # half a unit in the last place of FP16, relative


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one generated token of one sequence: the latency of a launch
        dict(name="rotary-token", kind="rotary", batch=1, kv=8, group=4, count=1, start=8191, rot=128, layout="half", scaling="plain",
             source="bf16", target="fp16", back=False),
        # the drafted tokens of three sequences at far positions, part of the head, interleaved pairs, scaled by parts
        dict(name="rotary-draft", kind="rotary", batch=3, kv=4, group=4, count=27, start=130009, rot=64, layout="interleaved",
             scaling="parts", source="fp32", target="fp16", back=False),
        # a prompt
        dict(name="rotary-prompt-8k", kind="rotary", batch=1, kv=8, group=4, count=8192, start=0, rot=128, layout="half", scaling="parts",
             source="bf16", target="fp16", back=False),
        # the gradient of a rotated batch: turned back, in 32 bits, ragged length
        dict(name="rotary-back-4k", kind="rotary", batch=2, kv=8, group=2, count=4099, start=17, rot=128, layout="half", scaling="linear",
             source="fp32", target="fp32", back=True),
        # a few tokens out of the middle of a short cache, across block borders
        dict(name="read-37", kind="read", batch=1, kv=8, group=4, tokens=1029, first=501, count=37, keys="normal", target="fp16",
             token_major=False),
        # one whole layer at 128K, for a program that goes on in FP16
        dict(name="read-128k", kind="read", batch=1, kv=8, group=4, tokens=131085, first=0, count=131085, keys="student", target="fp16",
             token_major=False),
        # the end of four sequences in 32 bits, token-major, from an odd token on
        dict(name="read-9k-fp32", kind="read", batch=4, kv=8, group=4, tokens=16399, first=7001, count=9398, keys="outlier", target="fp32",
             token_major=True),
        # one KV group of a small model or of one tensor-parallel rank: eight drafts, latency
        dict(name="tree-1k-8", kind="tree", batch=1, kv=1, group=4, tokens=1029, count=8, keys="normal", tree=True, peaked=False),
        # the ordinary turn: a tree of 26 drafts over 8K
        dict(name="tree-8k-26", kind="tree", batch=1, kv=8, group=4, tokens=8229, count=26, keys="outlier", tree=True, peaked=True),
        # few drafts for several long sequences: the cache's bytes bound it
        dict(name="tree-32k-5", kind="tree", batch=4, kv=8, group=4, tokens=32775, count=5, keys="student", tree=True, peaked=False),
        # a wide tree over 128K: the products bound it
        dict(name="tree-128k-64", kind="tree", batch=1, kv=8, group=4, tokens=131085, count=64, keys="student", tree=True, peaked=False),
        # a chunk of a prompt over its cached beginning: every token attends the ones before it
        dict(name="chunk-20k-256", kind="tree", batch=1, kv=8, group=2, tokens=20011, count=256, keys="normal", tree=False, peaked=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rotary", "read", "tree", "tree"])
    batch, kv, group = rng.choice([1, 1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4])
    if kind == "rotary":
        target = rng.choice(["fp16", "fp16", "bf16", "fp32"])
        return dict(kind=kind, batch=batch, kv=kv, group=group, count=_log_int(rng, 1, min(8192, (1 << 18) // (batch * kv * (group + 2)))),
                    start=rng.randint(0, 131072), rot=2 * rng.randint(1, 64) if rng.random() < 0.3 else rng.choice([32, 64, 96, 128]),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["plain", "linear", "parts"]),
                    source=rng.choice(["fp16", "bf16", "fp32"]), target=target, back=rng.random() < 0.3)
    # KV heads x tokens bounds what a case reads, query rows x tokens what it computes: the largest listed cases are the limit
    tokens = _log_int(rng, 1, min(131072, (1 << 20) // (batch * kv)))
    keys = rng.choice(["normal", "outlier", "student"])
    if kind == "read":
        target = rng.choice(["fp16", "bf16", "fp32"])
        tokens = min(tokens, (1 << 20) // (batch * kv * (SIZE[target] // 2)))
        first = rng.randint(0, tokens - 1)
        return dict(kind=kind, batch=batch, kv=kv, group=group, tokens=tokens, first=first, count=_log_int(rng, 1, tokens - first),
                    keys=keys, target=target, token_major=rng.random() < 0.4)
    count = _log_int(rng, 1, min(256, max(1, (32 * 64 * 131072) // (batch * kv * group * (tokens + 256)))))
    return dict(kind=kind, batch=batch, kv=kv, group=group, tokens=tokens, count=count, keys=keys, tree=rng.random() < 0.7,
                peaked=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs

def _gen(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + case["count"] * 7919 + case["batch"] * 31 + case["kv"]) & 0x7FFFFFFF)
    return g


def _randn(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _keys(case, g, shape):
    z = _randn(g, shape)
    if case["keys"] == "student":
        z = z / torch.sqrt((_randn(g, shape).square() + _randn(g, shape).square() + _randn(g, shape).square()) / 3.0)
    elif case["keys"] == "outlier":
        z[..., 11::32] *= 20.0
    return z.clamp(-2e4, 2e4).to(torch.float16)


def _quantized(k, v):
    """The cache's contents for FP16 keys and values of whole blocks: per block and channel INT8 keys with FP32 step and zero
    point, per token and 16 channels INT4 values with FP16 step and offset, and the block annotations eta and nu."""
    b, h, n, _ = k.shape
    c255, c15 = torch.full((), 255.0, device="cuda"), torch.full((), 15.0, device="cuda")
    kb = k.float().view(b, h, n // BLK, BLK, D)
    lo = kb.amin(3, keepdim=True)
    sigma = (kb.amax(3, keepdim=True) - lo) / c255
    zero = lo + 128.0 * sigma
    kc = torch.round((kb - zero) / torch.where(sigma == 0, torch.ones_like(sigma), sigma)).clamp(-128, 127)
    kc = torch.where(sigma == 0, torch.zeros_like(kc), kc).to(torch.int8)
    vg = v.float().view(b, h, n // BLK, BLK, NG, D // NG)
    off = vg.amin(5, keepdim=True)
    step = ((vg.amax(5, keepdim=True) - off) / c15).to(torch.float16)
    s = step.float()
    vc = torch.round((vg - off) / torch.where(s == 0, torch.ones_like(s), s)).clamp(0, 15)
    vc = torch.where(s == 0, torch.zeros_like(vc), vc).to(torch.uint8)
    err = (vc.double() * s.double() + off.double() - vg.double()).square().sum((4, 5)).sqrt().amax(3)
    norm = vg.double().square().sum((4, 5)).sqrt().amax(3)
    return dict(kc=kc, sigma=sigma, zero=zero, vc=vc, step=step, off=off.to(torch.float16), eta=err.float(), nu=norm.float())


class _Cache:
    """A cache that holds the tokens of one layer, freed with the state."""

    def __init__(self, case, k, v):
        from paper_2605_20868_amd import binding as cqa
        self.cqa = cqa
        self.h = cqa.cqa_cache_create(1, case["batch"], case["kv"] * case["group"], case["kv"], case["tokens"] + 256,
                                      tier2_mode=cqa.TIER2_NONE)
        cqa.cqa_cache_append(self.h, 0, k, v, case["tokens"])
        torch.cuda.synchronize()

    def __del__(self):
        torch.cuda.synchronize()
        self.cqa.cqa_cache_destroy(self.h)


class _Rotary:
    """The table of one kind of rotary positions, freed with the state."""

    def __init__(self, case):
        from paper_2605_20868_amd import binding as cqa
        self.cqa = cqa
        self.h = cqa.cqa_rotary_create(rot_dim=case["rot"], layout={"half": cqa.ROTARY_HALF, "interleaved": cqa.ROTARY_INTERLEAVED}[case["layout"]],
                                       base=500000.0, **_scaling(case, {"plain": cqa.ROTARY_PLAIN, "linear": cqa.ROTARY_LINEAR, "parts": cqa.ROTARY_PARTS}))

    def __del__(self):
        self.cqa.cqa_rotary_destroy(self.h)


def _scaling(case, names):
    more = {"plain": {}, "linear": dict(factor=4.0), "parts": dict(factor=8.0, low_rotations=1.0, high_rotations=4.0, trained_tokens=8192, magnitude=1.25)}
    return dict(scaling=names[case["scaling"]], **more[case["scaling"]])


def _prepare_rotary(case, seed):
    g = _gen(case, seed)
    b, n, kv, hq = case["batch"], case["count"], case["kv"], case["kv"] * case["group"]
    fused = _randn(g, (b, n, hq + 2 * kv, D)).to(TYPES[case["source"]])
    # each sequence at a place of its own; a batch that is turned back has negated positions
    pos = (case["start"] + torch.randint(0, 64, (b, 1), generator=g, device="cuda") + torch.arange(n, device="cuda")).to(torch.int64)
    t = TYPES[case["target"]]
    return dict(case=case, fused=fused, pos=-pos if case["back"] else pos, q_out=torch.empty((b, n, hq, D), dtype=t, device="cuda"),
                k_out=torch.empty((b, kv, n, D), dtype=t, device="cuda"), rotary=_Rotary(case) if own else None)


def _prepare_cache(case, g):
    b, kv, n = case["batch"], case["kv"], case["tokens"]
    k, v = _keys(case, g, (b, kv, n, D)), _randn(g, (b, kv, n, D)).to(torch.float16)
    whole = n // BLK * BLK
    state = _quantized(k[:, :, :whole].contiguous(), v[:, :, :whole].contiguous())
    state.update(case=case, trail_k=k[:, :, whole:].clone(), trail_v=v[:, :, whole:].clone(), cache=_Cache(case, k, v) if own else None)
    return state


def _prepare_read(case, seed):
    state = _prepare_cache(case, _gen(case, seed))
    b, kv, n, t = case["batch"], case["kv"], case["count"], TYPES[case["target"]]
    shape = (b, n, kv, D) if case["token_major"] else (b, kv, n, D)
    state.update(k_out=torch.empty(shape, dtype=t, device="cuda"), v_out=torch.empty(shape, dtype=t, device="cuda"))
    return state


def _parents(case, seed):
    """Per sequence the parent of every drafted node, -1 for the first: a chain, or a tree grown at random."""
    n, rng = case["count"], np.random.default_rng(seed)
    if not case["tree"]:
        return np.tile(np.arange(n) - 1, (case["batch"], 1))
    i = np.arange(n)
    return np.where(i == 0, -1, (rng.random((case["batch"], n)) * np.minimum(i, 12)).astype(np.int64) + np.maximum(i - 12, 0))


def _ancestors(parents):
    """True where the second node is the first one or an ancestor of it."""
    b, n = parents.shape
    m = np.zeros((b, n, n), bool)
    for i in range(n):
        m[:, i, i] = True
        if i:
            m[np.arange(b), i] |= m[np.arange(b), parents[:, i]]
    return m


def _prepare_tree(case, seed):
    g = _gen(case, seed)
    state = _prepare_cache(case, g)
    b, n, kv, hq = case["batch"], case["count"], case["kv"], case["kv"] * case["group"]
    scale = torch.where(torch.arange(hq, device="cuda") % 2 == 0, 3.0 if case["peaked"] else 1.0, 1.0).view(hq, 1)
    q = (_randn(g, (b, n, hq, D)) * scale).to(torch.float16)
    mask = None
    if case["tree"]:   # bit j of a node's words: it attends node j
        words = (n + 63) // 64
        bits = np.zeros((b, n, words * 64), bool)
        bits[:, :, :n] = _ancestors(_parents(case, seed))
        packed = np.packbits(bits, axis=-1, bitorder="little").view("<i8")
        mask = torch.from_numpy(packed.reshape(b, n, words)).cuda()
    state.update(q=q, k_draft=_keys(case, g, (b, kv, n, D)), v_draft=_randn(g, (b, kv, n, D)).to(torch.float16), mask=mask,
                 O=torch.empty((b, n, hq, D), dtype=torch.float16, device="cuda"), cert=torch.empty((b, n, hq, 8), device="cuda"),
                 flags=torch.empty((b, n, hq), dtype=torch.int32, device="cuda"))
    if own:
        cqa = state["cache"].cqa
        state.update(tol=cqa.Tolerances(), ws=torch.empty(cqa.cqa_tree_workspace_bytes(state["cache"].h, n), dtype=torch.uint8, device="cuda"))
    return state


def prepare(case, seed):
    return {"rotary": _prepare_rotary, "read": _prepare_read, "tree": _prepare_tree}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rotary": _own_rotary, "read": _own_read, "tree": _own_tree}[kind](state)
    return {"rotary": _plain_rotary, "read": _plain_read, "tree": _plain_tree}[kind](state)


def _own_rotary(s):
    case, cqa = s["case"], s["rotary"].cqa
    b, n, kv, hq = case["batch"], case["count"], case["kv"], case["kv"] * case["group"]
    row = (hq + 2 * kv) * D
    types = {"fp16": cqa.FP16, "bf16": cqa.BF16, "fp32": cqa.FP32}
    cqa.cqa_rotary_apply(s["rotary"].h, s["pos"], n, b, n,
                         [cqa.RotaryRows(s["fused"], s["q_out"], hq, (n * row, D, row), (n * hq * D, D, hq * D)),
                          cqa.RotaryRows(s["fused"][:, :, hq:], s["k_out"], kv, (n * row, D, row), (kv * n * D, n * D, D))],
                         types[case["source"]], types[case["target"]])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_read(s):
    case, cqa = s["case"], s["cache"].cqa
    kv, n = case["kv"], case["count"]
    strides = (n * kv * D, D, kv * D) if case["token_major"] else None
    cqa.cqa_cache_read(s["cache"].h, 0, case["first"], n, {"fp16": cqa.FP16, "bf16": cqa.BF16, "fp32": cqa.FP32}[case["target"]],
                       s["k_out"], s["v_out"], strides)
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_tree(s):
    cqa = s["cache"].cqa
    cqa.cqa_tree_decode(s["cache"].h, 0, s["q"], s["k_draft"], s["v_draft"], s["case"]["count"], s["mask"], s["tol"], s["O"], s["cert"],
                        s["flags"], s["ws"])
    return _outputs(s["O"], s["cert"].unbind(-1), s["flags"])


def _outputs(O, cert, flags):
    return dict(O=O, E_key=cert[0], E_val=cert[1], delta_h=cert[2], v_max=cert[3], alpha_tail_hat=cert[4], lse=cert[5], max_block_contrib=cert[6],
                flags=flags)


def _frequencies(case):
    """Radians per position of every pair, in 64 bits."""
    f = 500000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
    if case["scaling"] == "linear":
        return f / 4.0, 1.0
    if case["scaling"] == "parts":   # pairs that turn less than once in the trained length are stretched, those that turn often are not
        keep = ((8192.0 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / 8.0), 1.25
    return f, 1.0


def _turned(x, cos, sin, rot, layout):
    """x [..., 128], 32 bits; cos, sin [..., rot / 2]."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if layout == "interleaved" else (x[..., : rot // 2], x[..., rot // 2: rot])
    pair = a * cos - b * sin, a * sin + b * cos
    head = torch.stack(pair, -1).flatten(-2) if layout == "interleaved" else torch.cat(pair, -1)
    return torch.cat((head, x[..., rot:]), -1)


def _plain_rotary(s):
    case = s["case"]
    hq, kv = case["kv"] * case["group"], case["kv"]
    f, magnitude = _frequencies(case)
    angle = s["pos"].double()[..., None] * f                                   # far positions lose their angle in 32 bits
    cos, sin = (angle.cos() * magnitude).float()[:, :, None], (angle.sin() * magnitude).float()[:, :, None]
    x = _turned(s["fused"][:, :, : hq + kv].float(), cos, sin, case["rot"], case["layout"])
    t = TYPES[case["target"]]
    return {"q": x[:, :, :hq].to(t).contiguous(), "k": x[:, :, hq:].transpose(1, 2).to(t).contiguous()}


def _dequantized(s, lo, hi):
    """Keys and values of blocks lo .. hi, in 32 bits."""
    k = torch.addcmul(s["zero"][:, :, lo:hi], s["kc"][:, :, lo:hi].float(), s["sigma"][:, :, lo:hi])
    v = torch.addcmul(s["off"][:, :, lo:hi].float(), s["vc"][:, :, lo:hi].float(), s["step"][:, :, lo:hi].float())
    b, h = k.shape[:2]
    return k.view(b, h, -1, D), v.view(b, h, -1, D)


def _plain_read(s):
    case = s["case"]
    first, end = case["first"], case["first"] + case["count"]
    nb = case["tokens"] // BLK
    lo, hi = min(first // BLK, nb), min((end + BLK - 1) // BLK, nb)
    k, v = _dequantized(s, lo, hi)
    t = TYPES[case["target"]]
    cut = slice(first - lo * BLK, end - lo * BLK)
    k = torch.cat((k, s["trail_k"].float()), 2)[:, :, cut].to(t)
    v = torch.cat((v, s["trail_v"].float()), 2)[:, :, cut].to(t)
    return {"k": k.transpose(1, 2).contiguous(), "v": v.transpose(1, 2).contiguous()} if case["token_major"] else {"k": k.contiguous(), "v": v.contiguous()}


def _fp16(x):
    return x.clamp(-F16_MAX, F16_MAX).to(torch.float16)


def _rounded_up(x):
    """The smallest FP16 numbers that are not below x >= 0, 32 bits."""
    h = x.to(torch.float16)
    return torch.where(h.float() < x, (h.view(torch.int16) + 1).view(torch.float16), h).float()


def _widths(s):
    """Per block and channel: the key's quantization step with what rounding the reconstruction to FP16 adds to it, rounded up to FP16."""
    sigma, zero = s["sigma"][:, :, :, 0], s["zero"][:, :, :, 0]
    most = torch.maximum((zero - 128.0 * sigma).abs(), (zero + 127.0 * sigma).abs())
    return _rounded_up(sigma + 2.0 * torch.minimum(0.5 * sigma, HALF_STEP * most + 2.0 ** -25))


def _etas(s):
    """Per block: the value error with what rounding the reconstruction to FP16 adds to it."""
    return s["eta"] + torch.minimum(s["eta"], HALF_STEP * (s["nu"] + s["eta"]) + 2.0 ** -21)


def _plain_tree(s):
    case = s["case"]
    b, n, kv, g = case["batch"], case["count"], case["kv"], case["group"]
    nb = case["tokens"] // BLK
    sealed, trail = nb * BLK, case["tokens"] % BLK
    q = s["q"].float().view(b, n, kv, g, D).transpose(1, 2).reshape(b, kv, n * g, D)
    k, v = _dequantized(s, 0, nb)
    k = torch.cat((_fp16(k), s["trail_k"], s["k_draft"]), 2).float()
    v = torch.cat((_fp16(v), s["trail_v"], s["v_draft"]), 2).float()
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    if s["mask"] is None:
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril().expand(b, n, n)
    else:
        j = torch.arange(n, device="cuda")
        seen = (s["mask"][:, :, j // 64] >> (j % 64)) & 1 != 0
    rows = seen[:, None, :, None, :].expand(b, kv, n, g, n).reshape(b, kv, n * g, n)
    scores[..., sealed + trail:] = scores[..., sealed + trail:].masked_fill(~rows, -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - m)
    total = p.sum(-1)
    O = torch.matmul(p, v) / total[..., None]
    rho = p[..., :sealed].view(b, kv, n * g, nb, BLK).sum(-1) / total[..., None]
    contrib = rho * _etas(s)[:, :, None]
    alpha = rho.sum(-1)
    none = torch.zeros((b, kv, n * g, 1), device="cuda")
    delta = torch.cat((torch.matmul(q.abs(), _widths(s).transpose(2, 3).contiguous()) * (0.5 / math.sqrt(D)), none), -1).amax(-1)
    drafts = s["v_draft"].float().norm(dim=-1)[:, :, None].expand(b, kv, n * g, n) * rows
    norms = torch.cat((s["nu"], s["trail_v"].float().norm(dim=-1)), -1)[:, :, None].expand(b, kv, n * g, nb + trail)
    v_max = torch.cat((drafts, norms), -1).amax(-1)
    tail = torch.minimum(torch.ones_like(alpha), torch.exp(2.0 * delta) * alpha) * torch.expm1(2.0 * delta)
    e_key = 2.0 * v_max * torch.minimum(torch.tanh(delta), torch.where(alpha > 0, tail, torch.zeros_like(tail)))
    cert = torch.stack((e_key, contrib.sum(-1), delta, v_max, alpha, m[..., 0] + torch.log(total), torch.cat((contrib, none), -1).amax(-1)))
    back = lambda x: x.view(b, kv, n, g, -1).transpose(1, 2).reshape(b, n, kv * g, -1)  # noqa: E731
    finite = torch.isfinite(O).all(-1) & torch.isfinite(cert).all(0)
    return _outputs(back(O).to(torch.float16), [back(c)[..., 0] for c in cert], torch.where(back(finite)[..., 0], 0, 8).to(torch.int32))


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "read": _exact_read, "tree": _exact_tree}[case["kind"]](s, case, seed)


def _exact_rotary(s, case, seed):
    hq, kv, half = case["kv"] * case["group"], case["kv"], case["rot"] // 2
    factor = {"plain": 1.0, "linear": 4.0, "parts": 8.0}[case["scaling"]]
    turn = []
    for i in range(half):
        f = math.exp(-2.0 * i / case["rot"] * math.log(500000.0))
        share = 0.0 if case["scaling"] == "linear" else 1.0
        if case["scaling"] == "parts":
            share = min(1.0, max(0.0, (8192.0 / (2.0 * math.pi / f) - 1.0) / 3.0))
        turn.append(share * f + (1.0 - share) * f / factor)
    phase = s["pos"].double()[..., None] * torch.tensor(turn, dtype=torch.float64, device="cuda")
    unit = torch.polar(torch.full_like(phase, 1.25 if case["scaling"] == "parts" else 1.0), phase)[:, :, None]
    x = s["fused"][:, :, : hq + kv].double().clone()
    index = torch.arange(half, device="cuda")
    re, im = (2 * index, 2 * index + 1) if case["layout"] == "interleaved" else (index, index + half)
    z = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * unit
    x[..., re], x[..., im] = z.real, z.imag
    return {"q": x[:, :, :hq].contiguous(), "k": x[:, :, hq:].transpose(1, 2).contiguous()}


def _exact_read(s, case, seed):
    t = torch.arange(case["first"], case["first"] + case["count"], device="cuda")
    nb = case["tokens"] // BLK
    k = torch.empty((case["batch"], case["kv"], case["count"], D), dtype=torch.float64, device="cuda")
    v = torch.empty_like(k)
    old, new = t < nb * BLK, t >= nb * BLK
    blk, tok = t[old] // BLK, t[old] % BLK
    k[:, :, old] = s["kc"][:, :, blk, tok].double() * s["sigma"][:, :, blk, 0].double() + s["zero"][:, :, blk, 0].double()
    v[:, :, old] = (s["vc"][:, :, blk, tok].double() * s["step"][:, :, blk, tok].double() + s["off"][:, :, blk, tok].double()).flatten(3)
    k[:, :, new], v[:, :, new] = s["trail_k"][:, :, t[new] - nb * BLK].double(), s["trail_v"][:, :, t[new] - nb * BLK].double()
    return {"k": k.transpose(1, 2).contiguous(), "v": v.transpose(1, 2).contiguous()} if case["token_major"] else {"k": k, "v": v}


def _exact_tree(s, case, seed):
    b, n, kv, g, nb = case["batch"], case["count"], case["kv"], case["group"], case["tokens"] // BLK
    seen = torch.from_numpy(_ancestors(_parents(case, seed))).cuda()
    out = {k: torch.zeros((b, n, kv * g), dtype=torch.float64, device="cuda") for k in
           ("E_key", "E_val", "delta_h", "v_max", "alpha_tail_hat", "lse", "max_block_contrib")}
    O = torch.zeros((b, n, kv * g, D), dtype=torch.float64, device="cuda")
    for i in range(b):
        for h in range(kv):
            sg, z = s["sigma"][i, h, :, 0].double(), s["zero"][i, h, :, 0].double()
            kk = s["kc"][i, h].double() * sg[:, None] + z[:, None]
            vv = (s["vc"][i, h].double() * s["step"][i, h].double() + s["off"][i, h].double()).reshape(-1, D)
            to16 = lambda x: x.clamp(-65504, 65504).half().double()  # noqa: E731
            kk = torch.cat((to16(kk.reshape(-1, D)), s["trail_k"][i, h].double(), s["k_draft"][i, h].double()))
            vv = torch.cat((to16(vv), s["trail_v"][i, h].double(), s["v_draft"][i, h].double()))
            allowed = torch.ones((n, kk.shape[0]), dtype=torch.bool, device="cuda")
            allowed[:, case["tokens"]:] = seen[i]
            half_step = torch.minimum(sg / 2, torch.maximum((z - 128 * sg).abs(), (z + 127 * sg).abs()) / 2048 + 2.0 ** -25)
            wide = (sg + 2 * half_step).cpu().numpy()
            up = wide.astype(np.float16)
            up = torch.from_numpy(np.where(up.astype(np.float64) < wide, np.nextafter(up, np.float16(np.inf)), up).astype(np.float64)).cuda()
            eta, nu = s["eta"][i, h].double(), s["nu"][i, h].double()
            eta = eta + torch.minimum(eta, (nu + eta) / 2048 + 2.0 ** -21)
            norms = torch.cat((nu, vv[nb * BLK:].square().sum(1).sqrt()))
            open_ = torch.ones((n, norms.shape[0]), dtype=torch.bool, device="cuda")
            open_[:, nb + case["tokens"] % BLK:] = seen[i]
            v_max = torch.where(open_, norms, torch.zeros_like(norms)).amax(1)
            for j in range(g):
                qh = s["q"][i, :, h * g + j].double()
                w = (qh @ kk.T / math.sqrt(128.0)).masked_fill(~allowed, -math.inf)
                lse = torch.logsumexp(w, 1)
                w = torch.exp(w - lse[:, None])
                col = h * g + j
                O[i, :, col], out["lse"][i, :, col], out["v_max"][i, :, col] = w @ vv, lse, v_max
                if nb:
                    rho = w[:, : nb * BLK].reshape(n, nb, BLK).sum(2)
                    dl = ((qh.abs() @ up.T) / (2 * math.sqrt(128.0))).amax(1)
                    al = rho.sum(1)
                    tv = torch.minimum(torch.tanh(dl), torch.clamp(torch.exp(2 * dl) * al, max=1.0) * torch.expm1(2 * dl))
                    out["E_val"][i, :, col], out["max_block_contrib"][i, :, col] = rho @ eta, (rho * eta).amax(1)
                    out["delta_h"][i, :, col], out["alpha_tail_hat"][i, :, col], out["E_key"][i, :, col] = dl, al, 2 * v_max * tv
    return dict(out, O=O, flags=None)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    b, kv, hq, n = case["batch"], case["kv"], case["kv"] * case["group"], case["count"]
    if case["kind"] == "rotary":
        values = b * n * (hq + kv) * D
        return dict(bytes=values * (SIZE[case["source"]] + SIZE[case["target"]]) + 8 * b * n, flops=3 * b * n * (hq + kv) * case["rot"])
    if case["kind"] == "read":
        whole = case["tokens"] // BLK * BLK
        sealed = max(0, min(case["first"] + n, whole) - case["first"])
        return dict(bytes=b * kv * (sealed * (T1_BYTES - 0.5) + (n - sealed) * 4 * D + n * 2 * D * SIZE[case["target"]]), flops=4 * b * kv * n * D)
    nb = case["tokens"] // BLK
    trail = case["tokens"] % BLK
    pairs = b * hq * n * (nb * BLK + trail + n)
    return dict(bytes=b * kv * (nb * BLK * T1_BYTES + (trail + n) * 4 * D) + b * n * hq * (4 * D + 36) + (8 * b * n * ((n + 63) // 64) if case["tree"] else 0),
                flops=4 * D * pairs + 2 * D * b * hq * n * nb)
