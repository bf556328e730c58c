"""Plain 64-bit reference of the cache in 4 bits: quantiser by exact fractions, decoder, and attention with derived bounds."""
import math
from fractions import Fraction

import numpy as np
import torch

HALF_BF16 = 2.0 ** -8            # a rounding to bf16 is off by at most this, relative to the value
ORDER = [0, 2, 4, 6, 1, 3, 5, 7]  # nibble n of a word holds value ORDER[n] of its eight


def bits_of(x):
    """bf16 tensor -> uint16 bit patterns."""
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def from_bits(b):
    return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _nearest(f):
    """Nearest whole number of a fraction, from the middle away from zero."""
    n = math.floor(abs(f) + Fraction(1, 2))
    return n if f >= 0 else -n


def quantise_row(bits):
    """One head's row (uint16 bf16 patterns) -> (codes uint8 [d], scale pattern, zero point): the definition, by fractions."""
    if ((bits & 0x7F80) == 0x7F80).any():
        return np.zeros(len(bits), np.uint8), 0x7FFF, 0
    x = [Fraction(float(v)) for v in from_bits(bits)]
    lo, hi = min(min(x), 0), max(max(x), 0)
    low, high = 0x0380, 0x7F7F                       # 2^-120 .. the largest bf16: the patterns of positive numbers are in order
    while low < high:
        mid = (low + high) // 2
        if Fraction(float(from_bits(np.array([mid], np.uint16))[0])) * 15 >= hi - lo:
            high = mid
        else:
            low = mid + 1
    s = Fraction(float(from_bits(np.array([low], np.uint16))[0]))
    z = _nearest(-lo / s)
    return np.array([min(15, max(0, _nearest(v / s) + z)) for v in x], np.uint8), low, z


def pack_row(codes):
    n = codes.reshape(-1, 8)[:, ORDER]
    return (n[:, 0::2] | (n[:, 1::2] << 4)).astype(np.uint8).reshape(-1)


def unpack(codes, params):
    """Bytes uint8 [..., d / 2] and words int32 [...] -> values in 64 bits."""
    n = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1, 8)
    c = np.empty_like(n)
    c[..., ORDER] = n
    p = params.astype(np.int64) & 0xFFFFFFFF
    s = from_bits((p & 0xFFFF).astype(np.uint16))
    z = (p >> 16) & 15
    assert (p >> 20 == 0).all()
    return s[..., None] * (c.reshape(*codes.shape[:-1], -1).astype(np.float64) - z[..., None])


def cache_values(cache, layer, device="cpu"):
    """What a layer of the cache stands for: K and V in 64 bits, [slots][H][d]."""
    kc, kp, vc, vp = (t[layer].cpu().numpy() for t in cache.tensors)
    return (torch.from_numpy(unpack(kc, kp)).to(device), torch.from_numpy(unpack(vc, vp)).to(device))


def ancestors(parent):
    T = len(parent)
    see = np.zeros((T, T), bool)
    for t in range(T):
        a = t
        while a >= 0:
            see[t, a] = True
            a = parent[a]
    return see


def value_scales(cache, layer, device="cpu"):
    """Scales of a layer's values, [slots][H], 0 where they are not finite."""
    s = torch.from_numpy(from_bits((cache.tensors[3][layer].cpu().numpy() & 0xFFFF).astype(np.uint16))).to(device)
    return torch.nan_to_num(s, nan=0.0, posinf=0.0)


def attention(parent, gamma, scale, q_main, q_spec, k_held, v_held, k_tree, v_tree, k_spec, v_spec, v_scale=None):
    """One sequence in 64 bits.  Rows are the nodes, then the nodes' streams; returns o, lse and the bounds of both.  v_scale: scales of
    the held values, [L][H].

    Bound of o: the weights meet V rounded to 8 bits (2^-8 of sum p |v| / l), the output is rounded once (2^-8 of itself), and a
    score is off by what fp32 sums of its d products, the scales and the exponential lose: delta, which moves weights and their sum.
    Sums over cached keys: sum p s c and sum p s z are taken apart, in fp32, 16 keys at a time; both are at most 15 sum p s, a step rounds
    by at most 2^-23 of that, and there are L / 16 steps and what joins partial sums: (L / 16 + 64) 2^-22 15 sum p s in all.  A weight
    p s is off by at most 2^-31 of the largest scale where it is too small for fp16's 11 bits: 15 L 2^-31 max s."""
    T, H, d = q_main.shape
    rows = [q_main.double()] + ([q_spec.double().flatten(0, 1)] if gamma else [])
    keys = [k_held, k_tree.double()] + ([k_spec.double().flatten(0, 1)] if gamma else [])
    vals = [v_held, v_tree.double()] + ([v_spec.double().flatten(0, 1)] if gamma else [])
    q, k, v = torch.cat(rows), torch.cat(keys), torch.cat(vals)
    L = k_held.shape[0]
    anc = ancestors(parent)
    see = np.zeros((T * (1 + gamma), L + T * (1 + gamma)), bool)
    see[:, :L] = True
    see[:T, L:L + T] = anc
    for t in range(T):
        for j in range(gamma):
            see[T + t * gamma + j, L:L + T] = anc[t]
            see[T + t * gamma + j, L + T + t * gamma:L + T + t * gamma + j + 1] = True
    see = torch.from_numpy(see).to(q.device)
    # (keys that a row does not see may hold anything)
    s = torch.einsum("rhd,khd->hrk", q, k) * scale
    s = torch.where(see, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None])
    o = torch.einsum("hrk,khd->rhd", p, v)
    mass = torch.einsum("hrk,khd->rhd", p, v.abs())
    size = torch.where(see, torch.einsum("rhd,khd->hrk", q.abs(), k.abs()) * abs(scale), torch.zeros_like(s)).amax(-1)
    delta = ((d + 16) * 2.0 ** -23 * size + 2.0 ** -20 + (L / 32 + 64) * 2.0 ** -24).T                      # [rows][H]
    o_tol = HALF_BF16 * (mass + o.abs()) * (1 + 2.0 ** -6) + 2 * delta[..., None] * mass + 2.0 ** -126
    lse_tol = delta + 2.0 ** -22 * lse.T.abs() + 2.0 ** -20
    if v_scale is not None and L:
        sums = torch.einsum("hrk,kh->rh", p[..., :L], v_scale)
        o_tol = o_tol + (15 * (L / 16 + 64) * 2.0 ** -22 * sums + 15 * L * 2.0 ** -31 * v_scale.amax(0))[..., None]
    return o, lse.T, o_tol, lse_tol
