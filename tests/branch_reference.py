"""The branching operators in 64 bits (positions in the host's long double),
from their definitions, and the bounds on what a kernel may differ by."""
import numpy as np
import torch

EPS_OF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative


# Sequences (tokens before, new tokens) whose workgroups are a few more than full rounds of 256, so that the keys of the
# last rows are cut: float32 or bf16, head_dim, key heads, query heads per key head, sequences.
LAST_ROUND = [(torch.bfloat16, 128, 24, 1, [(900, 1500), (1100, 1321)]), (torch.bfloat16, 64, 40, 2, [(3000, 800)]),
              (torch.bfloat16, 64, 7, 1, [(2000, 5000), (0, 1), (600, 4900)]), (torch.float32, 64, 33, 1, [(700, 290)]),
              (torch.float32, 32, 5, 4, [(900, 210), (1000, 230)])]


def gather(buf, block, table):
    """[tokens, kv_heads, d] of a sequence, float64 on the CPU."""
    first, tokens, pages = table
    page = buf.shape[3]
    at = np.arange(first, first + tokens)
    p = torch.from_numpy(pages[at // page].astype(np.int64)).to(buf.device)
    r = torch.from_numpy(at % page).to(buf.device)
    return buf[block][p, :, r].double().cpu()


def attention(q, k, v, scale):
    """q [rows, heads, d], k / v [keys, kv_heads, d] (float64): the result and its bound for a
    kernel whose scores and sums are float32 and whose probabilities have half a step p_eps.

    Score: a sum of d float32 products, relative error d 2^-24 of sum |q||k|, as an exponent twice (the
    score and the maximum it is taken against) plus the rounding of the exponent itself.  Sum over keys:
    at most (keys + 64) 2^-24, numerator and denominator."""
    heads, kv, d = q.shape[1], k.shape[1], q.shape[2]
    out, size, spread = torch.empty_like(q), torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64)
    for h in range(heads):
        kh, vh = k[:, h * kv // heads], v[:, h * kv // heads]
        s = q[:, h] @ kh.T * scale
        p = torch.softmax(s, -1)
        out[:, h] = p @ vh
        size[:, h] = p @ vh.abs()
        spread[:, h] = (q[:, h].abs() @ kh.abs().T * scale).amax(-1)
    return out, size, spread


def attention_bound(out, size, spread, d, keys, dtype, p_eps):
    f32 = 2.0 ** -24
    arith = 2 * (d + 4) * f32 * spread[..., None] + 2 * (keys + 64) * f32
    return EPS_OF[dtype] * out.abs() + (p_eps + arith * (1 + p_eps)) * size * (1 + EPS_OF[dtype]) + 1e-30


def axis_dims(d, axes):
    return [d] if axes == 1 else [d - 4 * (d // 6), 2 * (d // 6), 2 * (d // 6)]


def turns(positions, d, theta):
    """cos, sin [rows, d / 2] of the rotation angles, in long double."""
    pos = positions.numpy().astype(np.longdouble)
    parts = []
    for a, n in enumerate(axis_dims(d, pos.shape[1])):
        f = np.longdouble(theta) ** (-np.arange(0, n, 2).astype(np.longdouble) / n)
        parts.append(pos[:, a:a + 1] * f)
    ang = np.concatenate(parts, 1)
    return (torch.from_numpy(np.cos(ang).astype(np.float64)), torch.from_numpy(np.sin(ang).astype(np.float64)),
            torch.from_numpy(np.abs(ang).astype(np.float64)))


def norm_rope(x, gain, positions, theta, dtype):
    """x [rows, heads, d] float64 -> the result and its bound.

    Float32 arithmetic up to the one rounding: sum of squares, root, division and the gain's products within
    16 float32 half steps; sine and cosine of a float32 fraction of a turn (absolute 2^-25 turns, 2 pi of that as an
    angle) with two units in the last place; two products and a sum: 32 half steps of |a| + |b| in all.  The
    angle itself is a double product of three rounded factors: 4 half steps of a double, relative."""
    d = x.shape[-1]
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain
    if positions is None:
        out, pair, ang = y, y.abs(), torch.zeros(x.shape[0], d, dtype=torch.float64)
    else:
        c, s, ang = turns(positions, d, theta)
        c, s = c[:, None], s[:, None]
        a, b = y[..., 0::2], y[..., 1::2]
        out = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
        pair = (a.abs() + b.abs()).repeat_interleave(2, -1)
        ang = ang.repeat_interleave(2, -1)
    return out, EPS_OF[dtype] * out.abs() + pair * (2.0 ** -19 + ang[:, None] * 2.0 ** -51) + 1e-30
