"""Attention over the certified cache for models whose scores are not the plain ones, and for batches that share a long
beginning, and how they are measured.

`run` computes each in its plain form (elementary torch operations, `own` false) or by the calls a user makes of the
library (`own` true); both take the same state.  Sizes are those of this repository's caches: head_dim 128, 1, 2 or 4
query heads per KV head, keys N(0, 1), N(0, 1) with outlier channels x 20 or Student-t(3).

kinds
  scored  nodes (single tokens, drafted trees, chunks of a prompt) over the cache, with any of: scores capped by a tanh, a
          bias by distance and head, spans of cached tokens (sliding windows, left-padded batches, packed documents).
  prefix  the same nodes of many sequences over the cached tokens of a beginning that they share, held once, and their own.
Either returns the attention's result and the certificate of every (node, query head).

For node i at place p_i and token j at place p_j (cached tokens: their index, those of the shared beginning first)
  x = scale q . k,  y = cap tanh(x / cap),  score = y - slope |p_i - p_j|  over the tokens attended:
cached ones of the node's two spans, drafted ones by its mask.  Sealed tokens enter as the cache reads back in FP16.
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
F16_MAX = 65504.0
HALF_STEP = 2.0 ** -11   # half a unit in the last place of FP16, relative
SINKS = 4                # first tokens that a window keeps


# ---------------------------------------------------------------------------------------------- cases

_BASE = dict(kind="scored", batch=1, shared=0, kv=8, group=4, prefix=0, tokens=0, count=1, drafts="none", cap=0.0, scale=0.0, slopes=False,
             spans="all", window=0, keys="normal", peaked=False)


def listed():
    return [dict(_BASE, **c) for c in (
        # one token over one KV group of a small model or of one tensor-parallel rank: latency
        dict(name="scored-token-1k", kv=1, tokens=1029, cap=50.0),
        # a layer with a sliding window in a model of capped scores, four long sequences
        dict(name="scored-window-32k", batch=4, tokens=32775, cap=50.0, spans="window", window=4096, keys="student", peaked=True),
        # one token over 128K with a scale of the model's own: the cache's bytes bound it
        dict(name="scored-token-128k", tokens=131085, cap=30.0, scale=0.0625, keys="student"),
        # drafted tokens of a left-padded batch of eight, one place of it idle, biased by distance
        dict(name="scored-padded-9k-5", batch=8, kv=4, group=2, tokens=9001, count=5, drafts="tree", slopes=True, spans="padded"),
        # the ordinary turn of a biased model with as many KV heads as query heads
        dict(name="scored-tree-8k-26", group=1, tokens=8229, count=26, drafts="tree", slopes=True, keys="outlier"),
        # a chunk of packed documents: the last cached one goes on, then a new one, both behind a common beginning
        dict(name="scored-documents-20k-256", group=2, tokens=20011, count=256, drafts="chunk", cap=50.0, spans="documents", window=9000),
        # a wide tree over 128K with capped scores: products and weights bound it
        dict(name="scored-tree-128k-64", tokens=131085, count=64, drafts="tree", cap=50.0, keys="student", peaked=True),
        # two requests behind one short instruction: latency
        dict(name="prefix-2-1k", kind="prefix", batch=2, shared=1, kv=1, prefix=1029, tokens=37),
        # a small batch behind a long document
        dict(name="prefix-16-32k", kind="prefix", batch=16, shared=1, prefix=32775, tokens=517, keys="student"),
        # a full batch behind a very long one
        dict(name="prefix-64-128k", kind="prefix", batch=64, shared=1, prefix=131085, tokens=1029, keys="outlier", peaked=True),
        # drafted tokens, two beginnings with four sequences each, unequal lengths, capped scores, one place idle
        dict(name="prefix-8-16k-5", kind="prefix", batch=8, shared=2, prefix=16399, tokens=2053, count=5, drafts="tree", cap=50.0, spans="padded"),
        # many short requests behind a system prompt: their own tokens bound it
        dict(name="prefix-200-2k", kind="prefix", batch=200, shared=1, kv=4, prefix=2053, tokens=263),
    )]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["scored", "prefix"])
    kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4])
    shared = prefix = 0
    # KV heads x cached tokens bounds what a case reads, query rows x tokens what it computes: the largest listed cases are the limit
    if kind == "prefix":
        shared = rng.choice([1, 1, 1, 2, 3])
        batch = shared * _log_int(rng, 1, 200 // shared)
        prefix = _log_int(rng, 1, min(131072, (1 << 20) // (shared * kv)))
        tokens = _log_int(rng, 1, min(8192, (1 << 19) // (batch * kv)))
    else:
        batch = rng.choice([1, 1, 2, 3, 4, 8, 16])
        tokens = _log_int(rng, 1, min(131072, (1 << 20) // (batch * kv)))
    drafts = rng.choice(["none", "tree", "chunk"])
    most = min(256, max(1, (1 << 28) // (batch * kv * group * (prefix + tokens + 256))))
    count = 1 if drafts == "none" else _log_int(rng, 1, most)
    spans = rng.choice(["all", "all", "window", "padded", "documents"])
    return dict(_BASE, kind=kind, batch=batch, shared=shared, kv=kv, group=group, prefix=prefix, tokens=tokens, count=count, drafts=drafts,
                cap=rng.choice([0.0, 30.0, 50.0]), scale=rng.choice([0.0, 0.0, 0.0625]), slopes=rng.random() < 0.3, spans=spans,
                window=_log_int(rng, 1, prefix + tokens) if spans in ("window", "documents") else 0,
                keys=rng.choice(["normal", "outlier", "student"]), peaked=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs

def _gen(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + case["count"] * 7919 + case["batch"] * 31 + case["kv"] + case["tokens"] * 131) & 0x7FFFFFFF)
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
    """A cache's contents for FP16 keys and values: of the whole blocks, per block and channel INT8 keys with FP32 step and zero
    point, per token and 16 channels INT4 values with FP16 step and offset, and the block annotations eta and nu; and the rest."""
    b, h, n, _ = k.shape
    whole = n // BLK * BLK
    trail = dict(trail_k=k[:, :, whole:].clone(), trail_v=v[:, :, whole:].clone())
    k, v = k[:, :, :whole].contiguous(), v[:, :, :whole].contiguous()
    c255, c15 = torch.full((), 255.0, device="cuda"), torch.full((), 15.0, device="cuda")
    kb = k.float().view(b, h, whole // BLK, BLK, D)
    lo = kb.amin(3, keepdim=True)
    sigma = (kb.amax(3, keepdim=True) - lo) / c255
    zero = lo + 128.0 * sigma
    kc = torch.round((kb - zero) / torch.where(sigma == 0, torch.ones_like(sigma), sigma)).clamp(-128, 127)
    kc = torch.where(sigma == 0, torch.zeros_like(kc), kc).to(torch.int8)
    vg = v.float().view(b, h, whole // BLK, BLK, NG, D // NG)
    off = vg.amin(5, keepdim=True)
    step = ((vg.amax(5, keepdim=True) - off) / c15).to(torch.float16)
    s = step.float()
    vc = torch.round((vg - off) / torch.where(s == 0, torch.ones_like(s), s)).clamp(0, 15)
    vc = torch.where(s == 0, torch.zeros_like(vc), vc).to(torch.uint8)
    err = (vc.double() * s.double() + off.double() - vg.double()).square().sum((4, 5)).sqrt().amax(3)
    norm = vg.double().square().sum((4, 5)).sqrt().amax(3)
    return dict(kc=kc, sigma=sigma, zero=zero, vc=vc, step=step, off=off.to(torch.float16), eta=err.float(), nu=norm.float(), **trail)


class _Cache:
    """A cache that holds the tokens of one layer, freed with the state."""

    def __init__(self, case, k, v):
        from paper_2605_20868_amd import binding as cqa
        self.cqa = cqa
        self.h = cqa.cqa_cache_create(1, k.shape[0], case["kv"] * case["group"], case["kv"], k.shape[2] + 256, tier2_mode=cqa.TIER2_NONE)
        cqa.cqa_cache_append(self.h, 0, k, v, k.shape[2])
        torch.cuda.synchronize()

    def __del__(self):
        torch.cuda.synchronize()
        self.cqa.cqa_cache_destroy(self.h)


def _parents(case, seed):
    """Per sequence the parent of every drafted node, -1 for the first: a chain, or a tree grown at random."""
    n, rng = case["count"], np.random.default_rng(seed)
    if case["drafts"] != "tree":
        return np.tile(np.arange(n) - 1, (case["batch"], 1))
    i = np.arange(n)
    return np.where(i == 0, -1, (rng.random((case["batch"], n)) * np.minimum(i, 12)).astype(np.int64) + np.maximum(i - 12, 0))


def _layout(case, seed):
    """(seen, places, spans): which drafted nodes a node attends [batch][n][n], its place [batch][n], its spans of cached tokens
    [batch][n][4] (two of them, from and to).  Cached tokens count from the shared beginning's first."""
    b, n, prefix, length = case["batch"], case["count"], case["prefix"], case["prefix"] + case["tokens"]
    rng = np.random.default_rng(seed + 77)
    seen = np.zeros((b, n, n), bool)
    places = np.full((b, n), length - 1, np.int64)   # a single token that is the cache's last
    if case["drafts"] != "none":
        parents = _parents(case, seed)
        for i in range(n):
            seen[:, i, i] = True
            places[:, i] = length
            if i:
                seen[np.arange(b), i] |= seen[np.arange(b), parents[:, i]]
                places[:, i] = places[np.arange(b), parents[:, i]] + 1
    spans = np.zeros((b, n, 4), np.int64)
    spans[..., 1] = length
    if case["spans"] == "window":       # the first tokens and the last ones up to the node
        spans[..., 1] = min(SINKS, length)
        spans[..., 2] = np.maximum(places - case["window"] + 1, 0)
        spans[..., 3] = length
    elif case["spans"] == "padded":     # a sequence's own tokens begin late; in a larger batch the last place is idle
        begin = prefix + (rng.random(b) * case["tokens"]).astype(np.int64)
        spans[..., 1], spans[..., 2], spans[..., 3] = prefix, begin[:, None], length
        if b > 3:
            spans[-1], seen[-1] = 0, False
    elif case["spans"] == "documents":  # a common beginning; the last cached document goes on up to some node, where a new one begins
        border = (rng.random(b) * (n + 1)).astype(np.int64)[:, None] if case["drafts"] == "chunk" else np.full((b, 1), n)
        old = np.arange(n)[None] < border
        spans[..., 1] = min(64, length)
        spans[..., 2] = max(length - case["window"], 0)
        spans[..., 3] = np.where(old, length, spans[..., 2])
        if case["drafts"] == "chunk":
            seen &= old[:, :, None] == old[:, None, :]
    return seen, places, spans


def _slopes(case):
    hq = case["kv"] * case["group"]
    return 2.0 ** (-8.0 * (torch.arange(hq, device="cuda", dtype=torch.float32) + 1.0) / hq)


def prepare(case, seed):
    g = _gen(case, seed)
    b, n, kv, hq = case["batch"], case["count"], case["kv"], case["kv"] * case["group"]
    state = dict(case=case)
    for name, batch, tokens in (("shared", case["shared"], case["prefix"]), ("mine", b, case["tokens"])):
        if batch:
            k, v = _keys(case, g, (batch, kv, tokens, D)), _randn(g, (batch, kv, tokens, D)).to(torch.float16)
            state[name] = dict(_quantized(k, v), cache=_Cache(case, k, v) if own else None)
    scale = torch.where(torch.arange(hq, device="cuda") % 2 == 0, 3.0 if case["peaked"] else 1.0, 1.0).view(hq, 1)
    q = (_randn(g, (b, n, hq, D)) * scale).to(torch.float16)
    seen, places, spans = _layout(case, seed)
    mask = kd = vd = None
    if case["drafts"] != "none":
        kd, vd = _keys(case, g, (b, kv, n, D)), _randn(g, (b, kv, n, D)).to(torch.float16)
        if case["drafts"] == "tree" or case["spans"] != "all":   # bit j of a node's words: it attends node j
            words = (n + 63) // 64
            bits = np.zeros((b, n, words * 64), bool)
            bits[:, :, :n] = seen
            mask = torch.from_numpy(np.packbits(bits, axis=-1, bitorder="little").view("<i8").reshape(b, n, words)).cuda()
    state.update(q=q, k_draft=kd, v_draft=vd, mask=mask, slopes=_slopes(case) if case["slopes"] else None,
                 places=torch.from_numpy(places).cuda() if case["slopes"] and case["drafts"] == "tree" else None,
                 spans=torch.from_numpy(spans).cuda() if case["spans"] != "all" else None,
                 O=torch.empty((b, n, hq, D), dtype=torch.float16, device="cuda"), cert=torch.empty((b, n, hq, 8), device="cuda"),
                 flags=torch.empty((b, n, hq), dtype=torch.int32, device="cuda"))
    if own:
        cqa, mine = state["mine"]["cache"].cqa, state["mine"]["cache"].h
        size = (cqa.cqa_prefix_workspace_bytes(state["shared"]["cache"].h, mine, n) if case["kind"] == "prefix"
                else cqa.cqa_scored_workspace_bytes(mine, n))
        state.update(tol=cqa.Tolerances(), ws=torch.empty(size, dtype=torch.uint8, device="cuda"),
                     scoring=cqa.Scoring(scale=case["scale"], cap=case["cap"], slopes_dev=state["slopes"], places_dev=state["places"],
                                         spans_dev=state["spans"]))
    return state


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    return _own_run(state) if own else _plain_run(state)


def _own_run(s):
    cqa, mine = s["mine"]["cache"].cqa, s["mine"]["cache"].h
    rest = (0, s["q"], s["k_draft"], s["v_draft"], s["case"]["count"], s["mask"], s["scoring"], s["tol"], s["O"], s["cert"], s["flags"], s["ws"])
    if s["case"]["kind"] == "prefix":
        cqa.cqa_prefix_decode(s["shared"]["cache"].h, mine, *rest)
    else:
        cqa.cqa_scored_decode(mine, *rest)
    return _outputs(s["O"], s["cert"].unbind(-1), s["flags"])


def _outputs(O, cert, flags):
    return dict(O=O, E_key=cert[0], E_val=cert[1], delta_h=cert[2], v_max=cert[3], alpha_tail_hat=cert[4], lse=cert[5], max_block_contrib=cert[6],
                flags=flags)


def _fp16(x):
    return x.clamp(-F16_MAX, F16_MAX).to(torch.float16)


def _rounded_up(x):
    """The smallest FP16 numbers that are not below x >= 0, 32 bits."""
    h = x.to(torch.float16)
    return torch.where(h.float() < x, (h.view(torch.int16) + 1).view(torch.float16), h).float()


def _attended(c):
    """Keys and values of a cache's tokens as attention takes them, 32 bits, [batch][heads][tokens][128]."""
    k = _fp16(torch.addcmul(c["zero"], c["kc"].float(), c["sigma"])).float()
    v = _fp16(torch.addcmul(c["off"].float(), c["vc"].float(), c["step"].float())).float()
    b, h = k.shape[:2]
    return torch.cat((k.view(b, h, -1, D), c["trail_k"].float()), 2), torch.cat((v.view(b, h, -1, D), c["trail_v"].float()), 2)


def _widths(c):
    """Per block and channel: the key's quantization step with what rounding the reconstruction to FP16 adds to it, rounded up to FP16."""
    sigma, zero = c["sigma"][:, :, :, 0], c["zero"][:, :, :, 0]
    most = torch.maximum((zero - 128.0 * sigma).abs(), (zero + 127.0 * sigma).abs())
    return _rounded_up(sigma + 2.0 * torch.minimum(0.5 * sigma, HALF_STEP * most + 2.0 ** -25))


def _etas(c):
    """Per block: the value error with what rounding the reconstruction to FP16 adds to it."""
    return c["eta"] + torch.minimum(c["eta"], HALF_STEP * (c["nu"] + c["eta"]) + 2.0 ** -21)


def _plain_run(s):
    case = s["case"]
    b, n, kv, g, cap = case["batch"], case["count"], case["kv"], case["group"], case["cap"]
    scale = case["scale"] or 1.0 / math.sqrt(D)
    length = case["prefix"] + case["tokens"]
    drafted = case["drafts"] != "none"
    q = s["q"].float().view(b, n, kv, g, D).transpose(1, 2).reshape(b, kv, n * g, D)
    q_abs = q.abs()

    def with_rows(x, rows, parts):
        """Products of every row with its sequence's x [parts][kv][m][128], -> [batch][kv][n g][m]; a part is several sequences'."""
        each = b // parts
        y = rows.view(parts, each, kv, n * g, D).transpose(1, 2).reshape(parts, kv, each * n * g, D)
        y = torch.matmul(y, x.transpose(2, 3).contiguous())
        return y.view(parts, kv, each, n * g, -1).transpose(1, 2).reshape(b, kv, n * g, -1)

    def by_rows(w, x, parts):
        """Sums of x [parts][kv][m][128] under the rows' weights, -> [batch][kv][n g][128]."""
        each = b // parts
        w = w.reshape(parts, each, kv, n * g, -1).transpose(1, 2).reshape(parts, kv, each * n * g, -1)
        return torch.matmul(w, x).view(parts, kv, each, n * g, D).transpose(1, 2).reshape(b, kv, n * g, D)

    def of_nodes(x):
        """[batch][n][m] of the nodes for the rows, [batch][1][n g][m]."""
        return x[:, None, :, None].expand(b, 1, n, g, x.shape[-1]).reshape(b, 1, n * g, -1)

    # tokens attended, in the order of their places: the shared beginning, the sequence's own, the drafted ones
    j = torch.arange(length, device="cuda")
    if s["spans"] is None:
        open_ = torch.ones((b, n, length), dtype=torch.bool, device="cuda")
    else:
        f = s["spans"][..., None]
        open_ = ((j >= f[:, :, 0]) & (j < f[:, :, 1])) | ((j >= f[:, :, 2]) & (j < f[:, :, 3]))
    if drafted:
        if s["mask"] is None:
            seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril().expand(b, n, n)
        else:
            i = torch.arange(n, device="cuda")
            seen = (s["mask"][:, :, i // 64] >> (i % 64)) & 1 != 0
        open_ = torch.cat((open_, seen), -1)
    first = length if drafted else length - n
    places = s["places"] if s["places"] is not None else (first + torch.arange(n, device="cuda")).expand(b, n)

    parts = [(s["mine"], b, case["prefix"], case["tokens"])]
    if case["shared"]:
        parts.insert(0, (s["shared"], case["shared"], 0, case["prefix"]))
    kv_of = [_attended(c) for c, _, _, _ in parts]
    scores = [with_rows(k, q, p) for (_, p, _, _), (k, _) in zip(parts, kv_of)]
    if drafted:
        scores.append(with_rows(s["k_draft"].float(), q, b))
    x = torch.cat(scores, -1) * scale
    if cap:
        x = cap * torch.tanh(x / cap)
    if s["slopes"] is not None:
        at = torch.cat((j.expand(b, length), places), -1) if drafted else j.expand(b, length)
        far = (places[:, :, None] - at[:, None]).abs().float()
        x = x - (s["slopes"].view(1, kv, 1, g, 1) * far[:, None, :, None]).reshape(b, kv, n * g, -1)
    rows_open = of_nodes(open_)
    x = x.masked_fill(~rows_open, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1)
    inv = torch.where(total == 0, torch.zeros_like(total), 1.0 / total)
    zero = torch.zeros((b, kv, n * g), device="cuda")
    O, e_val, contrib, alpha, delta, v_max = 0.0, zero, zero, zero, zero, zero
    for (c, count, at, tokens), (_, v) in zip(parts, kv_of):
        nb, sealed = tokens // BLK, tokens // BLK * BLK
        w = p[..., at:at + tokens] * inv[..., None]
        O = O + by_rows(w, v, count)
        each = b // count
        per_seq = lambda y: y[:, None].expand(count, each, *y.shape[1:]).reshape(b, *y.shape[1:])  # noqa: E731
        if nb:
            rho = w[..., :sealed].reshape(b, kv, n * g, nb, BLK).sum(-1)
            some = of_nodes(open_[..., at:at + sealed].reshape(b, n, nb, BLK).any(-1))
            e = rho * per_seq(_etas(c))[:, :, None]
            e_val, contrib, alpha = e_val + e.sum(-1), torch.maximum(contrib, e.amax(-1)), alpha + rho.sum(-1)
            d = with_rows(_widths(c), q_abs, count) * (0.5 * scale)
            delta = torch.maximum(delta, d.masked_fill(~some, 0.0).amax(-1))
            v_max = torch.maximum(v_max, (per_seq(c["nu"])[:, :, None] * some).amax(-1))
        if tokens > sealed:
            norms = per_seq(c["trail_v"].float().norm(dim=-1))[:, :, None]
            v_max = torch.maximum(v_max, (norms * of_nodes(open_[..., at + sealed:at + tokens])).amax(-1))
    if drafted:
        O = O + by_rows(p[..., length:] * inv[..., None], s["v_draft"].float(), b)
        v_max = torch.maximum(v_max, (s["v_draft"].float().norm(dim=-1)[:, :, None] * of_nodes(open_[..., length:])).amax(-1))
    if cap:
        delta = 2.0 * cap * torch.tanh(delta / (2.0 * cap))
    tail = torch.minimum(torch.ones_like(alpha), torch.exp(2.0 * delta) * alpha) * torch.expm1(2.0 * delta)
    e_key = 2.0 * v_max * torch.minimum(torch.tanh(delta), torch.where(alpha > 0, tail, zero))
    lse = m[..., 0] + torch.log(total)
    cert = torch.stack((e_key, e_val, delta, v_max, alpha, lse, contrib))
    back = lambda y: y.view(b, kv, n, g, -1).transpose(1, 2).reshape(b, n, kv * g, -1)  # noqa: E731
    finite = torch.isfinite(O).all(-1) & (torch.isfinite(cert).all(0) | (total == 0))
    return _outputs(back(O).to(torch.float16), [back(c)[..., 0] for c in cert], torch.where(back(finite)[..., 0], 0, 8).to(torch.int32))


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    b, n, kv, g = case["batch"], case["count"], case["kv"], case["group"]
    scale, cap = case["scale"] or 128.0 ** -0.5, case["cap"]
    seen, places, spans = _layout(case, seed)
    length = case["prefix"] + case["tokens"]
    names = ("E_key", "E_val", "delta_h", "v_max", "alpha_tail_hat", "lse", "max_block_contrib")
    out = {k: torch.zeros((b, n, kv * g), dtype=torch.float64, device="cuda") for k in names}
    O = torch.zeros((b, n, kv * g, D), dtype=torch.float64, device="cuda")
    to16 = lambda x: x.clamp(-65504, 65504).half().double()  # noqa: E731

    def contents(c, i, h):
        """(keys, values, widths, value errors, norm bounds of the blocks, of the rest) of one head."""
        sg, z = c["sigma"][i, h, :, 0].double(), c["zero"][i, h, :, 0].double()
        kk = to16(c["kc"][i, h].double() * sg[:, None] + z[:, None]).reshape(-1, D)
        vv = to16((c["vc"][i, h].double() * c["step"][i, h].double() + c["off"][i, h].double()).reshape(-1, D))
        half_step = torch.minimum(sg / 2, torch.maximum((z - 128 * sg).abs(), (z + 127 * sg).abs()) / 2048 + 2.0 ** -25)
        wide = (sg + 2 * half_step).cpu().numpy()
        up = wide.astype(np.float16)
        up = torch.from_numpy(np.where(up.astype(np.float64) < wide, np.nextafter(up, np.float16(np.inf)), up).astype(np.float64)).cuda()
        eta, nu = c["eta"][i, h].double(), c["nu"][i, h].double()
        tk, tv = c["trail_k"][i, h].double(), c["trail_v"][i, h].double()
        return torch.cat((kk, tk)), torch.cat((vv, tv)), up, eta + torch.minimum(eta, (nu + eta) / 2048 + 2.0 ** -21), nu, tv.square().sum(1).sqrt()

    slopes = s["slopes"].double().cpu().numpy() if case["slopes"] else None
    for h in range(kv):
        for i in range(b):
            if case["shared"] and i % (b // case["shared"]) == 0:
                common = contents(s["shared"], i // (b // case["shared"]), h)
            pieces = ([common] if case["shared"] else []) + [contents(s["mine"], i, h)]
            keys, values = [p[0] for p in pieces], [p[1] for p in pieces]
            if case["drafts"] != "none":
                keys.append(s["k_draft"][i, h].double())
                values.append(s["v_draft"][i, h].double())
            keys, values = torch.cat(keys), torch.cat(values)
            where = torch.arange(keys.shape[0], device="cuda")
            node_at = torch.from_numpy(places[i]).cuda()
            if case["drafts"] != "none":
                where[length:] = node_at
            allowed = torch.zeros((n, keys.shape[0]), dtype=torch.bool, device="cuda")
            for r in range(n):
                lo0, hi0, lo1, hi1 = (int(v) for v in spans[i, r])
                allowed[r, lo0:hi0] = True
                if hi1 > lo1:
                    allowed[r, lo1:hi1] = True
            if case["drafts"] != "none":
                allowed[:, length:] = torch.from_numpy(seen[i]).cuda()
            any_ = allowed.any(1)
            for j in range(g):
                col = h * g + j
                qh = s["q"][i, :, col].double()
                w = qh @ keys.T * scale
                if cap:
                    w = cap * torch.tanh(w / cap)
                if slopes is not None:
                    w = w - slopes[col] * (node_at[:, None] - where[None]).abs().double()
                lse = torch.logsumexp(w.masked_fill(~allowed, -math.inf), 1)
                w = torch.where(allowed, torch.exp(w - torch.where(any_, lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(w))
                O[i, :, col], out["lse"][i, :, col] = w @ values, lse
                dl, al, vm = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(3))
                at = 0
                for kk, _, up, eta, nu, norms in pieces:
                    nb = up.shape[0]
                    if nb:
                        hit = allowed[:, at:at + nb * BLK].reshape(n, nb, BLK).any(2)
                        rho = w[:, at:at + nb * BLK].reshape(n, nb, BLK).sum(2)
                        out["E_val"][i, :, col] += rho @ eta
                        out["max_block_contrib"][i, :, col] = torch.maximum(out["max_block_contrib"][i, :, col], (rho * eta).amax(1))
                        al = al + rho.sum(1)
                        dl = torch.maximum(dl, torch.where(hit, (qh.abs() @ up.T) * (scale / 2), torch.zeros_like(rho)).amax(1))
                        vm = torch.maximum(vm, torch.where(hit, nu.expand(n, nb), torch.zeros_like(rho)).amax(1))
                    rest = allowed[:, at + nb * BLK:at + kk.shape[0]]
                    if rest.shape[1]:
                        vm = torch.maximum(vm, torch.where(rest, norms.expand(n, -1), torch.zeros_like(rest, dtype=torch.float64)).amax(1))
                    at += kk.shape[0]
                if case["drafts"] != "none":
                    norms = values[length:].square().sum(1).sqrt().expand(n, n)
                    vm = torch.maximum(vm, torch.where(allowed[:, length:], norms, torch.zeros_like(norms)).amax(1))
                if cap:
                    dl = 2 * cap * torch.tanh(dl / (2 * cap))
                tv = torch.minimum(torch.tanh(dl), torch.clamp(torch.exp(2 * dl) * al, max=1.0) * torch.expm1(2 * dl))
                out["delta_h"][i, :, col], out["alpha_tail_hat"][i, :, col], out["v_max"][i, :, col], out["E_key"][i, :, col] = dl, al, vm, 2 * vm * tv
    return dict(out, O=O, flags=None)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without

def _read_tokens(case):
    """Cached tokens of a sequence that some node of it attends: (of the shared beginning, its own, of all sequences on the average)."""
    prefix, tokens = case["prefix"], case["tokens"]
    length = prefix + tokens
    if case["spans"] == "padded":
        live = (case["batch"] - 1) / case["batch"] if case["batch"] > 3 else 1.0
        return prefix, live * tokens / 2
    if case["spans"] == "all":
        return prefix, tokens
    first, last = min(SINKS if case["spans"] == "window" else 64, length), min(case["window"], length)
    from_ = max(length - last, first)
    in_prefix = min(first, prefix) + max(prefix - from_, 0)
    return in_prefix, first + (length - from_) - in_prefix


def work(case):
    b, kv, hq, n = case["batch"], case["kv"], case["kv"] * case["group"], case["count"]
    shared, mine = _read_tokens(case)
    drafted = n if case["drafts"] != "none" else 0
    live = (b - 1) / b if case["spans"] == "padded" and b > 3 else 1.0
    late = 0.5 if case["spans"] == "documents" and case["drafts"] == "chunk" else 1.0   # nodes of the new document, half of them, attend no old one
    pairs = b * hq * n * (late * (live * shared + mine) + live * drafted)
    nodes = b * n * (8 * ((n + 63) // 64 if drafted else 0) + (32 if case["spans"] != "all" else 0))
    return dict(bytes=kv * T1_BYTES * (case["shared"] * shared + b * mine) + b * kv * drafted * 4 * D + b * n * hq * (4 * D + 36) + nodes,
                flops=4 * D * pairs + 2 * D * pairs / BLK)
