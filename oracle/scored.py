"""CPU oracle, part 5: nodes with scores of the caller's, and sequences behind a beginning that is cached once (test
infrastructure only; see quantizer.py's header).  float64 apart from the roundings that drafts.py states.

* Node i at place p_i attends cached tokens of two spans and drafted ones of its mask:
      x = scale q . k,  y = cap tanh(x / cap) (cap 0: x),  score = y - slope |p_i - p_j|
  A cached token's place is its index, the beginning's first; a drafted token's is its node's.
* The certificate of drafts.py, over the blocks of which the node attends a token, with
      Delta_b = scale / 2 sum_c |q_c| w_c,  Delta = 2 cap tanh(max Delta_b / (2 cap)) where there is a cap.
  tanh a - tanh b <= 2 tanh((a - b) / 2) for a >= b: the difference is largest where a = -b.
"""
from __future__ import annotations

import math

import numpy as np

from . import attention as att
from . import quantizer as qz
from .drafts import key_widths, read_back, to_fp16, value_errors


def default_places(bt, n, cached, drafted):
    return np.tile(np.arange(n) + cached - (0 if drafted else n), (bt, 1))


class _Contents:
    """By [b, h]: (keys, values, widths, value errors, norms of the blocks, norms of the trailing tokens) of a head, as attended."""

    def __init__(self, oc):
        self.oc, self.kv = oc, read_back(oc, 0, oc.length)

    def __getitem__(self, bh):
        oc, nb = self.oc, self.oc.n_blocks
        k, v = (to_fp16(x[bh]).astype(np.float64) for x in self.kv)
        return (k, v, key_widths(oc.sigma[bh], oc.z[bh]), value_errors(oc.eta[bh], oc.nu[bh]), oc.nu[bh].astype(np.float64),
                np.sqrt((v[nb * qz.B:] ** 2).sum(1)))


def decode(shared, oc, q16, k_draft, v_draft, seen, tol, scale=0.0, cap=0.0, slopes=None, places=None, spans=None, where_drafted=None):
    """shared: OracleLayerCache or None; q16 [Bt, n, Hq, d]; k_draft, v_draft [Bt, Hkv, n, d] or None; seen bool [Bt, n, n] or None.
    where_drafted [Bt, drafted tokens]: their places, where they are not the nodes'.  Dicts [Bt][n][Hq] as drafts.tree_decode returns them."""
    bt, n, hq, d = q16.shape
    g = hq // oc.hkv
    ahead = shared.length if shared is not None else 0
    cached = ahead + oc.length
    drafted = k_draft is not None
    if places is None:
        places = default_places(bt, n, cached, drafted)
    if spans is None:
        spans = np.tile(np.array([0, cached, 0, 0]), (bt, n, 1))
    if where_drafted is None:
        where_drafted = places
    scale = scale or 1.0 / math.sqrt(d)
    out = [[[None] * hq for _ in range(n)] for _ in range(bt)]
    mine, common = _Contents(oc), _Contents(shared) if shared is not None else None
    for b in range(bt):
        for h in range(oc.hkv):
            parts = ([common[b // (bt // shared.bt), h]] if shared is not None else []) + [mine[b, h]]
            k, v = np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts])
            where = np.arange(cached, dtype=np.float64)
            if drafted:
                k = np.concatenate([k, k_draft[b, h].astype(np.float64)])
                v = np.concatenate([v, v_draft[b, h].astype(np.float64)])
                where = np.concatenate([where, where_drafted[b].astype(np.float64)])
            for i in range(n):
                j = np.arange(cached)
                s = spans[b, i]
                at = ((j >= s[0]) & (j < s[1])) | ((j >= s[2]) & (j < s[3]))
                if drafted:
                    at = np.concatenate([at, seen[b, i]])
                for e in range(g):
                    col = h * g + e
                    bias = None if slopes is None else -float(slopes[col]) * np.abs(float(places[b, i]) - where)
                    out[b][i][col] = _row(q16[b, i, col].astype(np.float64), k, v, at, bias, parts, scale, cap, tol)
    return out


def _row(q, k, v, at, bias, parts, scale, cap, tol):
    d = q.shape[0]
    if not at.any():
        return dict(O=np.zeros(d), E_key=0.0, E_val=0.0, delta_h=0.0, v_max=0.0, alpha_tail_hat=0.0, lse=-math.inf, max_block_contrib=0.0,
                    flags=tol.force_flags, spread=np.zeros(d), floor=0.0)
    s = scale * (k @ q)
    if cap:
        s = cap * np.tanh(s / cap)
    if bias is not None:
        s = s + bias
    s = np.where(at, s, -math.inf)
    m = s.max()
    e = np.exp(s - m)
    a = e / e.sum()
    lse = m + math.log(e.sum())
    delta = alpha = e_val = contrib = v_max = 0.0
    first = 0
    for keys, _, widths, eta, nu, norms in parts:
        nb, n = len(eta), len(keys)
        if nb:
            some = at[first:first + nb * qz.B].reshape(nb, qz.B).any(1)
            rho = a[first:first + nb * qz.B].reshape(nb, qz.B).sum(1)
            alpha += float(rho.sum())
            e_val += float(rho @ eta)
            contrib = max(contrib, float((rho * eta).max()))
            if some.any():
                delta = max(delta, float((widths[some] @ np.abs(q)).max()) * scale / 2)
                v_max = max(v_max, float(nu[some].max()))
        tail = norms[at[first + nb * qz.B:first + n]]
        v_max = max(v_max, float(tail.max()) if tail.size else 0.0)
        first += n
    drafted = np.sqrt((v[first:][at[first:]] ** 2).sum(1))
    v_max = max(v_max, float(drafted.max()) if drafted.size else 0.0)
    if cap:
        delta = 2 * cap * math.tanh(delta / (2 * cap))
    e_key = att.key_term(delta, max(alpha, 2.0 ** -110) if delta else alpha, v_max, tol.mass_exp, tol.key_bound_mode)
    O = a @ np.where(at[:, None], v, 0.0)
    flags = tol.force_flags
    if e_key > tol.eps_key:
        flags |= att.FLAG_KEY
    if e_val > tol.eps_val or contrib > tol.v_tol:
        flags |= att.FLAG_VAL
    if e_key + e_val > tol.eps_total:
        flags |= att.FLAG_TOTAL
    if not all(math.isfinite(x) for x in (e_key, e_val, delta, v_max, lse)) or not np.isfinite(O).all():
        flags |= att.FLAG_PRECOND
    return dict(O=O, E_key=e_key, E_val=e_val, delta_h=delta, v_max=v_max, alpha_tail_hat=alpha, lse=lse, max_block_contrib=contrib, flags=flags,
                spread=a[at] @ np.abs(v[at]), floor=float(np.abs(v[at]).max()) * int(at.sum()) / float(e.sum()))
