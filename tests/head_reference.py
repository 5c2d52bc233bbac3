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
