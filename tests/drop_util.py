"""The masks of dropout from their definition, in numpy."""
import numpy as np
import torch

STEP_STRIDE = 0xD1342543DE82EF95


def kept(rows, hidden, p, seed, step=0):
    """[rows, hidden] truth values."""
    u = np.uint64
    z = u((seed + step * STEP_STRIDE) % (1 << 64)) + np.arange(1, rows + 1, dtype=u) * u(0x9E3779B97F4A7C15)
    z = (z ^ z >> u(30)) * u(0xBF58476D1CE4E5B9)
    z = (z ^ z >> u(27)) * u(0x94D049BB133111EB)
    z ^= z >> u(31)
    k0, k1 = z.astype(np.uint32)[:, None], (z >> u(32)).astype(np.uint32)[:, None]
    x = (k0 + np.arange(hidden, dtype=np.uint32)) * np.uint32(0x9E3779B1)
    x = (x ^ x >> np.uint32(15) ^ k1) * np.uint32(0x85EBCA6B)
    x ^= x >> np.uint32(16)
    return x >> np.uint32(8) >= int(np.floor(p * 2.0 ** 24 + 0.5))


def factors(rows, hidden, p, seed, step=0, device="cuda:0"):
    """The mask as fp64 factors: 0, or what is kept is multiplied with."""
    top = int(np.floor(p * 2.0 ** 24 + 0.5))
    scale = 2.0 ** 24 / (2 ** 24 - top) if top < 1 << 24 else 0.0
    return torch.from_numpy(kept(rows, hidden, p, seed, step) * scale).to(device)
