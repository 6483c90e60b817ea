"""CPU oracle, part 4: drafted tokens over the cache, rotary positions, reading the cache back (test infrastructure
only; see quantizer.py's header).  float64 apart from the roundings that the definitions state.

* Reading back: k = code * sigma + z as one fused binary32 operation, v = code * scale + offset exactly, each rounded
  once to the asked type (values to BF16 by way of binary32); what overflows FP16 becomes its largest number.
* A node attends the sealed tokens as read back in FP16, the trailing tokens and the drafted tokens of its mask, which are
  exact.  The certificate is that of attention.py with the widths and value errors that cover the rounding to FP16:
      w_c   = FP16 upwards(sigma_c + 2 min(sigma_c / 2, 2^-11 max(|z_c - 128 sigma_c|, |z_c + 127 sigma_c|) + 2^-25))
      eta'_b = eta_b + min(eta_b, 2^-11 (nu_b + eta_b) + 2^-21)
  The originals are FP16 numbers, so the nearest FP16 number to k^ is no further from k^ than k is; and it is within half a
  step of FP16 (2^-11 relative, 2^-25 among the subnormals).
* Rotary: the pair (a, b) turns by p f_i.
"""
from __future__ import annotations

import math

import numpy as np

from . import attention as att
from . import quantizer as qz

F16_MAX = 65504.0


def to_fp16(x):
    """Rounded to FP16, saturating; infinite and undefined numbers stay."""
    x = np.asarray(x, np.float64)
    return np.where(np.isfinite(x), np.clip(x, -F16_MAX, F16_MAX), x).astype(np.float16)


def read_back(oc, first, n):
    """(k binary32, v float64) [Bt, Hkv, n, d] of an OracleLayerCache's tokens, not yet rounded to a type."""
    nb, d = oc.n_blocks, oc.d
    k = qz.dequantize_keys(oc.k_codes, oc.sigma, oc.z).astype(np.float32).reshape(oc.bt, oc.hkv, nb * qz.B, d)
    v = qz.dequantize_values(oc.v_codes, oc.v_scale, oc.v_offset).reshape(oc.bt, oc.hkv, nb * qz.B, d)
    k = np.concatenate([k, oc.k16[:, :, nb * qz.B:].astype(np.float32)], axis=2)
    v = np.concatenate([v, oc.v16[:, :, nb * qz.B:].astype(np.float64)], axis=2)
    return k[:, :, first:first + n], v[:, :, first:first + n]


def key_widths(sigma, z):
    sg, zz = sigma.astype(np.float64), z.astype(np.float64)
    most = np.maximum(np.abs(zz - 128 * sg), np.abs(zz + 127 * sg))
    w = sg + 2 * np.minimum(sg / 2, most / 2048 + 2.0 ** -25)
    h = w.astype(np.float16)
    return np.where(h.astype(np.float64) < w, np.nextafter(h, np.float16(np.inf)), h).astype(np.float64)


def value_errors(eta, nu):
    e, n = eta.astype(np.float64), nu.astype(np.float64)
    return e + np.minimum(e, (n + e) / 2048 + 2.0 ** -21)


def ancestors(parents):
    """bool [n, n] of a list of parents (-1: none): the node itself and its ancestors."""
    n = len(parents)
    seen = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while j >= 0:
            seen[i, j] = True
            j = parents[j]
    return seen


def mask_words(seen):
    """bool [Bt, n, n] -> uint64 [Bt, n, ceil(n / 64)]."""
    bt, n, _ = seen.shape
    words = (n + 63) // 64
    bits = np.zeros((bt, n, words * 64), bool)
    bits[:, :, :n] = seen
    return np.packbits(bits, axis=-1, bitorder="little").view("<u8").reshape(bt, n, words)


def tree_decode(oc, q16, k_draft, v_draft, seen, tol):
    """q16 [Bt, n, Hq, d]; k_draft, v_draft [Bt, Hkv, n, d]; seen bool [Bt, n, n].  Dicts [Bt][n][Hq], each with what errors
    of the weights amount to: `spread` = sum_t a_t |v_t| per channel (relative ones) and `floor` = count max |v| / sum_t
    exp(s_t - max s) (absolute ones)."""
    bt, n, hq, d = q16.shape
    g, nb = hq // oc.hkv, oc.n_blocks
    k_all, v_all = read_back(oc, 0, oc.length)
    out = []
    for b in range(bt):
        rows = [[None] * hq for _ in range(n)]
        for h in range(oc.hkv):
            k = np.concatenate([to_fp16(k_all[b, h]).astype(np.float64), k_draft[b, h].astype(np.float64)])
            v = np.concatenate([to_fp16(v_all[b, h]).astype(np.float64), v_draft[b, h].astype(np.float64)])
            norms = np.sqrt((v[nb * qz.B:] ** 2).sum(1))
            widths, eta = key_widths(oc.sigma[b, h], oc.z[b, h]), value_errors(oc.eta[b, h], oc.nu[b, h])
            for i in range(n):
                at = np.concatenate([np.ones(oc.length, bool), seen[b, i]])
                for j in range(g):
                    q = q16[b, i, h * g + j].astype(np.float64)
                    rows[i][h * g + j] = _node(q, k, v, at, norms, widths, eta, oc.nu[b, h], nb, tol)
        out.append(rows)
    return out


def _node(q, k, v, at, norms, widths, eta, nu, nb, tol):
    d = q.shape[0]
    if not at.any():
        zero = dict(O=np.zeros(d), E_key=0.0, E_val=0.0, delta_h=0.0, v_max=0.0, alpha_tail_hat=0.0, lse=-math.inf,
                    max_block_contrib=0.0, flags=tol.force_flags, spread=np.zeros(d), floor=0.0)
        return zero
    s = (k[at] @ q) / math.sqrt(d)
    m = s.max()
    e = np.exp(s - m)
    a = e / e.sum()
    lse = m + math.log(e.sum())
    O = a @ v[at]
    rho = a[:nb * qz.B].reshape(nb, qz.B).sum(1)
    delta = float((widths @ np.abs(q)).max() / (2 * math.sqrt(d))) if nb else 0.0
    alpha, e_val = float(rho.sum()), float(rho @ eta)
    contrib = float((rho * eta).max()) if nb else 0.0
    tail = norms[at[nb * qz.B:]]
    v_max = max(float(nu.max()) if nb else 0.0, float(tail.max()) if tail.size else 0.0)
    e_key = att.key_term(delta, alpha, v_max, tol.mass_exp, tol.key_bound_mode)
    flags = tol.force_flags
    if e_key > tol.eps_key:
        flags |= att.FLAG_KEY
    if e_val > tol.eps_val or contrib > tol.v_tol:
        flags |= att.FLAG_VAL
    if e_key + e_val > tol.eps_total:
        flags |= att.FLAG_TOTAL
    if not all(math.isfinite(x) for x in (e_key, e_val, delta, v_max, lse)) or not np.isfinite(O).all():
        flags |= att.FLAG_PRECOND
    return dict(O=O, E_key=e_key, E_val=e_val, delta_h=delta, v_max=v_max, alpha_tail_hat=alpha, lse=lse,
                max_block_contrib=contrib, flags=flags, spread=a @ np.abs(v[at]),
                floor=float(np.abs(v[at]).max()) * int(at.sum()) / float(e.sum()))


def rotary_frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, low=0.0, high=0.0, trained=0):
    i = np.arange(0, rot_dim, 2, dtype=np.longdouble)
    f = np.power(np.longdouble(base), -i / rot_dim)
    if scaling == "linear":
        f = f / np.longdouble(factor)
    elif scaling == "parts":
        keep = np.clip((np.longdouble(trained) * f / (2 * np.longdouble(math.pi)) - low) / (np.longdouble(high) - low), 0, 1)
        f = f * (keep + (1 - keep) / np.longdouble(factor))
    return f


def rotary(x, positions, f, interleaved, magnitude=1.0):
    """x [..., n, 128] rows of tokens n, positions [n]; float64."""
    x = np.asarray(x, np.float64).copy()
    half = len(f)
    w = np.asarray(positions, np.longdouble)[:, None] * f
    c, s = (magnitude * np.cos(w)).astype(np.float64), (magnitude * np.sin(w)).astype(np.float64)
    at = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., at[0]].copy(), x[..., at[1]].copy()
    x[..., at[0]], x[..., at[1]] = a * c - b * s, a * s + b * c
    return x
