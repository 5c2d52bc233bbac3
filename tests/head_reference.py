"""Plain references of the classifier-head operators, from their definitions: NumPy and torch in 64 bits, on the CPU."""
import math

import numpy as np
import torch

GOLDEN = 0x9E3779B97F4A7C15
M64 = (1 << 64) - 1

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


def draw(key, j):
    """Draw j of the generator, in Python integers."""
    z = (key + (j + 1) * GOLDEN) & M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def kept(rows, cols, rate, key, first_row=0):
    """Which elements dropout keeps, [rows][cols]."""
    pairs = (cols + 1) // 2
    threshold = np.uint32(int(float(np.float32(rate)) * 2.0 ** 32))
    with np.errstate(over="ignore"):
        row = np.uint64(first_row) + np.arange(rows, dtype=np.uint64)[:, None]
        j = row * np.uint64(pairs) + np.arange(pairs, dtype=np.uint64)[None, :]
        z = np.uint64(key) + (j + np.uint64(1)) * np.uint64(GOLDEN)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return np.ascontiguousarray(z).view(np.uint32).reshape(rows, 2 * pairs)[:, :cols] >= threshold


def dropout(x, rate, key, first_row=0):
    """x: a float32 or bfloat16 CPU tensor; the float32 product rounded once, as the operator defines it."""
    scale = np.float32(1.0 / (1.0 - float(np.float32(rate))))
    y = x.float() * torch.tensor(scale)
    return torch.where(torch.from_numpy(kept(*x.shape, rate, key, first_row)), y, torch.zeros_like(y)).to(x.dtype)


def log_probs(z, targets, top=0):
    """(log_prob, entropy, lse, top_log_prob, top_class) of rows of float64 logits, as include/edl.h defines them."""
    rows, classes = z.shape
    bad = (torch.isnan(z) | (z == math.inf)).any(1)
    empty = (z == -math.inf).all(1)
    safe = torch.where((bad | empty)[:, None], torch.zeros_like(z), z)
    lse = torch.logsumexp(safe, 1)
    lp = safe - lse[:, None]
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    nan, inf = torch.full_like(lse, math.nan), torch.full_like(lse, -math.inf)
    lse = torch.where(bad, nan, torch.where(empty, inf, lse))
    entropy = torch.where(bad, nan, torch.where(empty, torch.zeros_like(entropy), entropy))
    lp = torch.where(bad[:, None], nan[:, None], torch.where(empty[:, None], inf[:, None], lp))
    log_prob = None
    if targets is not None:
        has = (targets >= 0) & (targets < classes)
        at = torch.where(has, targets, torch.zeros_like(targets)).long()
        log_prob = torch.where(has, lp.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    rank = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :top]
    return log_prob, entropy, lse, lp.gather(1, order), order.to(torch.int32)


def log_probs_backward(z, targets, dlog_prob, dentropy):
    """Gradient of rows of float64 logits, from the formula."""
    rows, classes = z.shape
    _, entropy, lse, _, _ = log_probs(z, None)
    has = torch.zeros(rows, dtype=torch.bool) if targets is None else (targets >= 0) & (targets < classes)
    g = torch.where(has, dlog_prob.double() if dlog_prob is not None else torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64))
    h = dentropy.double() if dentropy is not None else torch.zeros(rows, dtype=torch.float64)
    lp = z - lse[:, None]
    p = torch.where(z == -math.inf, torch.zeros_like(z), lp.exp())
    d = -g[:, None] * p - h[:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), p)
    for r in torch.nonzero(has)[:, 0].tolist():
        d[r, int(targets[r])] += g[r]
    return torch.where(((g == 0) & (h == 0))[:, None], torch.zeros_like(d), d)
