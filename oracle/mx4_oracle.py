"""The latent cache in 4 bits in fp64 numpy: encoding, decoding and decode attention from their definitions.

E2M1 elements (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with one E8M0 scale per 32 channels.
Encoding looks for the nearest representable value by comparing distances; it shares no code and no method with the kernels,
which scale and round.
"""
import math

import numpy as np

GROUP = 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_exponent(top):
    """Exponent of a group's power of two from its largest magnitude (finite): that of the magnitude rounded to one mantissa
    bit, less two, kept where every value is a normal bf16 number or zero."""
    if top == 0.0:
        return -125
    m, e = math.frexp(top)                       # top = 2 m 2^(e - 1), 1 <= 2 m < 2
    return min(max(e - 1 + (1 if 2 * m >= 1.75 else 0) - 2, -125), 125)


def encode_group(x):
    """32 values -> (codes 0..15, scale byte)."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(GROUP, dtype=np.uint8), 255
    e = scale_exponent(float(np.abs(x).max()))
    y = np.abs(x) / 2.0 ** e
    codes = np.zeros(GROUP, dtype=np.uint8)
    for i, v in enumerate(y):
        d = np.abs(VALUES - v)
        near = np.flatnonzero(d == d.min())      # two of them: a tie, whose even code has the even mantissa
        codes[i] = near[0] if len(near) == 1 else near[near % 2 == 0][0]
    return codes | (np.signbit(x).astype(np.uint8) << 3), e + 127


def encode(rows):
    """rows [..., channels] -> packed codes [..., channels / 2], scale bytes [..., channels / 32]."""
    rows = np.asarray(rows, dtype=np.float64)
    flat = rows.reshape(-1, GROUP)
    codes, scales = np.zeros(flat.shape, dtype=np.uint8), np.zeros(len(flat), dtype=np.uint8)
    for i, g in enumerate(flat):
        codes[i], scales[i] = encode_group(g)
    codes = codes.reshape(rows.shape)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales.reshape(rows.shape[:-1] + (rows.shape[-1] // GROUP,))


def decode(packed, scales):
    """Packed codes and scale bytes -> the fp64 values that they stand for."""
    codes = np.stack((packed & 15, packed >> 4), axis=-1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))
    v = np.where(codes >= 8, -1.0, 1.0) * VALUES[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    with np.errstate(invalid="ignore"):
        return v * np.repeat(s, GROUP, axis=-1)


def attend(latent, rope, lens, q_abs, q_rope, w_uv, tau, out_scale=1.0, groups=1, gate=None):
    """latent: list of [n][blocks][d_cb] per sequence, rope: list of [n][d_r]; q_abs [batch][q_len][blocks][hb][d_cb],
    q_rope [batch][q_len][h][d_r], w_uv [blocks][d_cb][hb * d_h] -> out [batch][q_len][h][d_h], lse [batch][q_len][blocks][hb].
    Query j of a sequence of n tokens sees the first n - (q_len - 1 - j) of them."""
    batch, q_len, blocks, hb, d_cb = q_abs.shape
    d_h = w_uv.shape[2] // hb
    w = w_uv.reshape(blocks, d_cb, hb, d_h)
    out = np.zeros((batch, q_len, groups * hb, d_h))
    lse = np.full((batch, q_len, blocks, hb), -np.inf)
    for s in range(batch):
        for j in range(q_len):
            n = int(lens[s]) - (q_len - 1 - j)
            if n <= 0:
                continue
            for b in range(blocks):
                g = b // (blocks // groups)
                c = latent[s][:n, b]
                score = tau * (q_abs[s, j, b] @ c.T + q_rope[s, j, g * hb:(g + 1) * hb] @ rope[s][:n].T)
                top = score.max(axis=1, keepdims=True)
                p = np.exp(score - top)
                lse[s, j, b] = top[:, 0] + np.log(p.sum(axis=1))
                z = (p / p.sum(axis=1, keepdims=True)) @ c
                out[s, j, g * hb:(g + 1) * hb] += out_scale * np.einsum("ic,cid->id", z, w[b])
    return (out if gate is None else out * gate), lse
