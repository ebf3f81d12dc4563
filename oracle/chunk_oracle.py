"""CPU oracle for chunks of new tokens: rotary positions, the append of rotated keys to the pages, and causal attention of
packed chunks over the pages.  TEST INFRASTRUCTURE, as ``attention_oracle``; it shares no code with the library.

Rotary positions.  Pair i of a head's channels is a point of the plane and is turned by pos * theta_i; theta_i =
base^(-2 i / R), scaled for long contexts in one of four ways.  Angles are worked out in 60-digit decimal arithmetic and kept
in turns as 128-bit fixed-point integers, so that pos * theta modulo one turn is exact far beyond float64 for any position.

Append.  bf16 rounding to nearest even by bit arithmetic; E4M3 by search in the sorted list of the 254 finite codes
(nearest, ties to the even code, beyond the largest to the largest).

Attention.  Row i of a chunk of n new tokens of a sequence of L sees cached tokens 0 .. L - n + i; float64 softmax.
"""
from __future__ import annotations

import math
from decimal import Decimal, getcontext

import numpy as np

from oracle import attention_oracle as O

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899863")
HALF, INTERLEAVED = "half", "interleaved"


def rope_turns(rotary_dim: int, base: float, scaling: str = "none", factor: float = 1.0, low: float = 0.0, high: float = 0.0,
               original_len: int = 0):
    """Turns per position of each pair, as integers in units of 2^-128 turn."""
    getcontext().prec = 60
    R, f, b = rotary_dim, Decimal(factor), Decimal(base)
    if scaling == "base":
        b = b * f ** (Decimal(R) / Decimal(R - 2))
    out = []
    for i in range(R // 2):
        theta = b ** (Decimal(-2 * i) / Decimal(R))
        if scaling == "linear":
            theta = theta / f
        elif scaling == "bands":
            n = Decimal(original_len) * theta / (2 * PI)
            keep = min(max((n - Decimal(low)) / (Decimal(high) - Decimal(low)), Decimal(0)), Decimal(1))
            theta = theta * keep + theta / f * (1 - keep)
        elif scaling == "ramp":
            pair = [Decimal(R) * (Decimal(original_len) / (2 * PI * Decimal(n))).ln() / (2 * Decimal(base).ln()) for n in (high, low)]
            lo, hi = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), R - 1)
            gone = min(max(Decimal(i - lo) / max(Decimal(hi - lo), Decimal("0.001")), Decimal(0)), Decimal(1))
            theta = theta * (1 - gone) + theta / f * gone
        elif scaling not in ("none", "base"):
            raise ValueError(scaling)
        out.append(int((theta / (2 * PI) * (1 << 128)).to_integral_value()))
    return out


def rope_angles(positions, turns) -> np.ndarray:
    """float64 [positions, pairs]: the angle in (-pi, pi], from exact integer arithmetic."""
    one = 1 << 128
    a = np.empty((len(positions), len(turns)), dtype=np.float64)
    for t, pos in enumerate(positions):
        for i, w in enumerate(turns):
            phase = (int(pos) * w) % one
            if phase > one // 2:
                phase -= one
            a[t, i] = (phase / one) * 2 * math.pi
    return a


def rotate(x, angles, layout: str, magnitude: float = 1.0) -> np.ndarray:
    """x: float64 [tokens, heads, channels]; angles [tokens, pairs]."""
    y = np.array(x, dtype=np.float64)
    n = angles.shape[1]
    for i in range(n):
        a, b = (i, i + n) if layout == HALF else (2 * i, 2 * i + 1)
        c, s = np.cos(angles[:, i])[:, None], np.sin(angles[:, i])[:, None]
        u, v = x[:, :, a], x[:, :, b]
        y[:, :, a] = magnitude * (u * c - v * s)
        y[:, :, b] = magnitude * (u * s + v * c)
    return y


def e4m3_values() -> np.ndarray:
    """Value of every code 0 .. 255 (NaN codes: NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    mag = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e.astype(float) - 7))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c & 128, -mag, mag)


def e4m3_encode(x) -> np.ndarray:
    """Nearest code, ties to the even mantissa, saturating; NaN -> 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    vals = e4m3_values()[:127]                                      # ascending magnitudes of codes 0 .. 126
    a = np.minimum(np.abs(x), vals[-1])
    hi = np.clip(np.searchsorted(vals, np.nan_to_num(a)), 1, 126)
    lo = hi - 1
    dl, dh = a - vals[lo], vals[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def row_positions(q_lens, seq_lens) -> np.ndarray:
    """Position of every packed row."""
    return np.array([L - n + i for n, L in zip(q_lens, seq_lens) for i in range(n)], dtype=np.int64)


def packed_chunk_attention(q, k_tokens, v_tokens, q_lens, seq_lens, sm_scale: float | None = None):
    """q: float64 [rows, Hq, d]; k_tokens[b], v_tokens[b]: float64 [Hkv, L_b, d].
    Returns out [rows, Hq, d], lse [rows, Hq] and spread [rows, Hq, d] = sum_t p_t |v_t|, the scale that the rounding of the
    probabilities acts on."""
    rows, Hq, d = q.shape
    scale = 1.0 / math.sqrt(d) if sm_scale is None else float(sm_scale)
    out, spread = np.zeros((rows, Hq, d)), np.zeros((rows, Hq, d))
    lse = np.full((rows, Hq), -np.inf)
    r = 0
    for b, (n, L) in enumerate(zip(q_lens, seq_lens)):
        for i in range(n):
            seen = L - n + i + 1
            if seen > 0:
                K, V = k_tokens[b][:, :seen], v_tokens[b][:, :seen]
                G = Hq // K.shape[0]
                s = np.einsum("hgd,htd->hgt", q[r].reshape(-1, G, d), K) * scale
                m = s.max(axis=-1, keepdims=True)
                p = np.exp(s - m)
                z = p.sum(axis=-1, keepdims=True)
                out[r] = np.einsum("hgt,htd->hgd", p / z, V).reshape(Hq, d)
                spread[r] = np.einsum("hgt,htd->hgd", p / z, np.abs(V)).reshape(Hq, d)
                lse[r] = (m + np.log(z))[..., 0].reshape(Hq)
            r += 1
    return out, lse, spread


def sequence_tokens(pages, block_table, seq_lens, layout: str = "HND", scale: float | None = None):
    """Per sequence float64 [Hkv, L, d]; pages are bf16 bits (uint16) or, with a scale, E4M3 codes (uint8)."""
    out = []
    for b, L in enumerate(seq_lens):
        P = pages.shape[2] if layout == "HND" else pages.shape[1]
        ids = np.asarray(block_table[b, :-(-int(L) // P)], dtype=np.int64)
        got = pages[ids] if layout == "HND" else pages[ids].transpose(0, 2, 1, 3)
        x = got.transpose(1, 0, 2, 3).reshape(got.shape[1], -1, got.shape[3])[:, :int(L)]
        out.append(O.bf16_bits_to_f64(x) if scale is None else e4m3_values()[x] * scale)
    return out
