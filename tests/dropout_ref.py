"""The generator of the dropout operators in numpy, and plain results in 64 bits."""
import numpy as np
import torch


def philox(c, k, rounds=10):
    """Philox4x32 of uint32 counters c [4, n] and key k [2]."""
    c = [v.astype(np.uint64) for v in c]
    k = [int(v) for v in k]
    low = np.uint64(0xffffffff)
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [q >> np.uint64(32) ^ c[1] ^ np.uint64(k[0]), q & low, p >> np.uint64(32) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c).astype(np.uint32)


def bits(count, rng, site, first=0):
    """The 16 random bits of values first .. first + count - 1 (multiples of 8)."""
    seed, step = (int(v) % 2 ** 64 for v in rng.tolist())
    g = np.arange(first // 8, (first + count) // 8, dtype=np.uint64)
    low = np.uint64(0xffffffff)
    words = philox([g & low, g >> np.uint64(32), np.full_like(g, step % 2 ** 32), np.full_like(g, site)],
                   [seed % 2 ** 32, seed >> 32])
    return np.stack([words & 0xffff, words >> 16], 2).transpose(1, 0, 2).reshape(-1)


def cut_of(p):
    return int(np.rint(p * 65536))


def factor(shape, p, rng, site, device="cuda"):
    """0 or 1 / (1 - q) of each value, in 64 bits."""
    cut = cut_of(p)
    keep = torch.from_numpy(bits(int(np.prod(shape)), rng, site) >= cut).to(device).view(shape)
    return keep.double() * (65536 / (65536 - cut) if cut < 65536 else 0.0)
