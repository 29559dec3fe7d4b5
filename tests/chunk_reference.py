"""The operators of chunks under a mask in 64 bits, from their definitions, and the bounds on what a kernel may differ
by."""
import torch

from branch_reference import EPS_OF, attention_bound

F32 = 2.0 ** -24


def sees(tokens, new, group, window, sinks):
    """[new, tokens] truth values: what each of the last `new` rows sees."""
    out = torch.zeros(new, tokens, dtype=torch.bool)
    for r in range(new):
        end = tokens - new + min(new, (r // group + 1) * group) if group else tokens
        begin = max(0, end - window) if window else 0
        out[r, begin:end] = True
        out[r, :min(sinks, end)] |= bool(window)
    return out


def scores(q, k, scale, visible):
    """[heads, rows, keys] in 64 bits, -infinity where a row does not see, and the largest |q||k| of each row."""
    heads, kv = q.shape[1], k.shape[1]
    s = torch.stack([q[:, h] @ k[:, h * kv // heads].T * scale for h in range(heads)])
    size = torch.stack([q[:, h].abs() @ k[:, h * kv // heads].abs().T * scale for h in range(heads)])
    size = torch.where(visible, size, torch.zeros_like(size)).amax(-1)
    return torch.where(visible, s, torch.full_like(s, -torch.inf)), size


def attention(q, k, v, scale, visible, dtype, p_eps):
    """Outputs [rows, heads, d] and log-sum-exps [rows, heads] with their bounds.

    The output's bound is that of attention without a mask (branch_reference).  The log-sum-exp: a score is off by
    (d + 4) 2^-24 of sum |q||k| at most, their sum by (keys + 64) 2^-24 of itself; a maximum, the logarithm of a sum
    (two units in the last place) and their sum are rounded, none larger than the scores and the logarithm of the keys."""
    heads, kv, d = q.shape[1], k.shape[1], q.shape[2]
    s, spread = scores(q, k, scale, visible)
    p = torch.softmax(s, -1)
    vh = torch.stack([v[:, h * kv // heads] for h in range(heads)])
    keep = visible.any(0)
    vh = torch.where(keep[None, :, None], vh, torch.zeros_like(vh))
    out, size = (p @ vh).transpose(0, 1), (p @ vh.abs()).transpose(0, 1)
    lse = torch.logsumexp(s, -1).T
    n = visible.sum(-1).max().item()
    spread = spread.T
    tol = attention_bound(out, size, spread, d, n, dtype, p_eps)
    lse_tol = (d + 4) * F32 * spread + (n + 64) * F32 + 8 * F32 * (spread + torch.log(torch.tensor(n + 1.0)))
    return out, tol, lse, lse_tol


def weights(q, k, scale, visible, lse):
    """[keys]: the sum over rows and heads of exp(scale q k - lse), lse as given [rows, heads], and its bound.

    A term's exponent is off by (d + 4) 2^-24 of sum |q||k| and by four half steps of the score and of the
    log-sum-exp, its exponential by four half steps more; the sum of n terms by n + 64 half steps of each."""
    d = q.shape[2]
    s, spread = scores(q, k, scale, visible)
    lse = lse.T[..., None]
    p = torch.exp(s - lse)
    off = (d + 8) * F32 * spread[..., None] + 4 * F32 * lse.abs() + (p.shape[0] * p.shape[1] + 72) * F32
    return p.sum((0, 1)), (p * off).sum((0, 1)) * 1.01


def kept(w, keep, sinks, recent):
    """Numbers of the tokens that a sequence keeps, by their weights (float32)."""
    tokens = len(w)
    if keep >= tokens:
        return list(range(tokens))
    mid = range(sinks, tokens - recent)
    key = [(0, 0.0) if w[t] != w[t] else (1, float(w[t])) for t in range(tokens)]
    best = sorted(mid, key=lambda t: (-key[t][0], -key[t][1], t))[:keep - sinks - recent]
    return list(range(sinks)) + sorted(best) + list(range(tokens - recent, tokens))
