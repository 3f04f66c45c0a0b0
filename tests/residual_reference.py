"""The operators of the residual stream in plain torch and numpy, written from their formulas, for the tests."""
import numpy as np
import torch

PHILOX = (0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85)


def philox(counter, key):
    """Philox 4x32 with ten rounds: four arrays of 32-bit words, two words -> four arrays (uint64 holds the products)."""
    low = np.uint64(0xffffffff)
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        u, v = c[0] * np.uint64(PHILOX[0]), c[2] * np.uint64(PHILOX[1])
        c = [(v >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), v & low, (u >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), u & low]
        k = [(k[0] + PHILOX[2]) & 0xffffffff, (k[1] + PHILOX[3]) & 0xffffffff]
    return c


def threshold(p):
    return min(65535, int(p * 65536 + 0.5))


def factors(seed, offset, rows, cols, p):
    """What a dropout multiplies by, fp64 [rows, cols]; seed and offset: whole numbers, modulo 2^64."""
    t = threshold(p)
    if t == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    octs = -(-cols // 8)
    zero = np.zeros((rows, octs), dtype=np.uint64)
    words = philox((zero + np.arange(octs, dtype=np.uint64), zero + np.arange(rows, dtype=np.uint64)[:, None], zero + np.uint64(offset & 0xffffffff),
                    zero + np.uint64(offset >> 32)), (seed & 0xffffffff, seed >> 32))
    bits = np.stack([w >> np.uint64(s) & np.uint64(0xffff) for w in words for s in (0, 16)], axis=-1).reshape(rows, octs * 8)[:, :cols]
    return torch.from_numpy(np.where(bits >= t, 65536.0 / (65536 - t), 0.0))


def dropped(x, factor):
    """x in fp32 times the factors, which are fp32 numbers in the library; what is dropped is zero whatever it was."""
    f = factor.to(x.device).float()
    return torch.where(f == 0, torch.zeros((), device=x.device), x.float() * f)


def stream(x, residual, factor):
    """h as it is stored: each operation in fp32, rounded once to the stream's type."""
    h = x.float() if factor is None else dropped(x, factor)
    if residual is not None:
        h = residual.float() + h
    return h.to((x if residual is None else residual).dtype)


def normed(h, w, eps):
    """(y, 1 / sqrt) in 64 bits."""
    h = h.double()
    r = 1 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    return h * r * (1.0 if w is None else w.double()), r


def int8_of(v):
    """Values and max |v| of rows in fp32, as the library defines them: each operation rounded once."""
    top = v.abs().amax(dim=1)
    m = top.clamp(min=2.0 ** -100)
    fine = torch.isfinite(v).all(dim=1)
    q = torch.round(torch.where(fine.unsqueeze(1), v, torch.zeros_like(v)) * torch.div(torch.full_like(m, 127.0), m).nan_to_num(0, 0, 0).unsqueeze(1))
    return q.to(torch.int8), m, fine


def gradients(h, dy, dh, w, eps):
    """(gradient of h, of the weight, and for each element what its rounding errors are in proportion to), 64 bits."""
    h, dy = h.double(), dy.double()
    w = torch.ones(h.shape[1], dtype=torch.float64, device=h.device) if w is None else w.double()
    r = 1 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)
    hat, g = h * r, dy * w
    d = r * (g - hat * (g * hat).mean(dim=1, keepdim=True))
    size = r * (g.abs() + hat.abs() * (g * hat).abs().mean(dim=1, keepdim=True))
    if dh is not None:
        d, size = d + dh.double(), size + dh.double().abs()
    return d, (dy * hat).sum(dim=0), size, (dy * hat).abs().sum(dim=0)
