"""The policy's operators in float64 on the CPU, from their definitions (include/wdp.h), element by element where that is plainest."""
import numpy as np
import torch

BLOCK, TINY = 128, 2.0 ** -100
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11,
             torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}  # relative
LEAST_HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float8_e4m3fn: 2.0 ** -10, torch.float8_e5m2: 2.0 ** -17}
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def f64(t):
    return t.detach().cpu().double()


def rounding(values, dtype):
    """How far rounding to dtype may move the values."""
    return (values.abs() * HALF_STEP[dtype]).clamp(min=LEAST_HALF_STEP[dtype])


def blocks_of(v):
    """[rows, width] -> list of the row's blocks of up to 128 columns."""
    return list(v.split(BLOCK, 1))


def norm(x, weight, residual, eps):
    """(h as it is stored, y, rstd) in float64."""
    h = x.cpu() if residual is None else (f64(x) + f64(residual)).to(x.dtype)
    # (float64 to bfloat16 rounds twice at most by way of float32; the sum of two values of 16 bits is exact in float32
    # unless their exponents are far apart, where both ways round to the larger one)
    if residual is not None:
        h = (x.cpu().float() + residual.cpu().float()).to(x.dtype)
    v = f64(h)
    rstd = 1 / torch.sqrt((v * v).mean(1) + eps)
    w = torch.ones(v.shape[1], dtype=torch.float64) if weight is None else f64(weight)
    return h, v * rstd[:, None] * w, rstd


def norm_backward(dy, h, weight, rstd, dh):
    dy, h, r = f64(dy), f64(h), f64(rstd)[:, None]
    w = torch.ones(h.shape[1], dtype=torch.float64) if weight is None else f64(weight)
    xhat, g = h * r, dy * w
    dx = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
    size = r * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))  # of what is added up
    if dh is not None:
        dx, size = dx + f64(dh), size + f64(dh).abs()
    return dx, (dy * xhat).sum(0), size, (dy * xhat).abs().sum(0)


def product(a, a_scale, b, b_scale, by_row):
    """(c, sum of the terms' sizes, sum over the blocks of 128 * (largest a) * (largest b)) in float64."""
    def spread(scale, rows, n, k):
        s = f64(scale).repeat_interleave(BLOCK, 1)[:, :k]
        return s if rows == 1 else s.repeat_interleave(rows, 0)[:n]

    def largest(v):
        return torch.stack([x.abs().amax(1) for x in v.split(BLOCK, 1)], 1)

    (m, k), n = a.shape, b.shape[0]
    av, bv = a.cpu().float().double() * spread(a_scale, 1, m, k), b.cpu().float().double() * spread(b_scale, 1 if by_row else BLOCK, n, k)
    return av @ bv.t(), av.abs() @ bv.abs().t(), BLOCK * largest(av) @ largest(bv).t()


def verify(target, draft, drafts, u, lengths=None):
    """One sequence after the other, one token after the other."""
    p, q, x, u = f64(target).numpy(), f64(draft).numpy(), drafts.cpu().numpy(), f64(u).numpy()
    batch, rows, vocab = p.shape
    n_max = x.shape[1]
    accepted, tokens = np.zeros(batch, np.int32), np.full((batch, rows), -1, np.int32)
    for s in range(batch):
        n = n_max if lengths is None else min(max(int(lengths[s]), 0), n_max)
        a = 0
        while a < n and 0 <= x[s, a] < vocab and u[s, a] * q[s, a, x[s, a]] < p[s, a, x[s, a]]:
            tokens[s, a] = x[s, a]
            a += 1
        accepted[s] = a
        if a == n and rows == n_max:
            continue
        plain = np.where(p[s, a] > 0, p[s, a], 0.0)
        with np.errstate(invalid="ignore"):
            left = p[s, a] - q[s, a] if a < n else p[s, a]
        r = np.where(left > 0, left, 0.0)
        if not r.sum() > 0:
            r = plain
        run = np.cumsum(r)
        with np.errstate(invalid="ignore"):
            past = np.flatnonzero((r > 0) & (run > u[s, n_max] * run[-1]))
        some = np.flatnonzero(r > 0)
        tokens[s, a] = past[0] if len(past) else some[-1] if len(some) else vocab - 1
    return accepted, tokens


def philox_words(seed, four, step):
    """Words of the blocks (seed; four, step, stream 4); four: uint64 array -> [len, 4]."""
    m32 = np.uint64(0xFFFFFFFF)
    four = np.asarray(four, np.uint64)
    c = [four & m32, four >> np.uint64(32), np.full_like(four, step & 0xFFFFFFFF), np.full_like(four, 4 | (step >> 32 << 8))]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1)


def adamw(p, g, m, v, step, lr, betas, eps, decay):
    """(p, m, v) after a step, float64."""
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / (torch.sqrt(v / (1 - b2 ** step)) + eps), m, v


def code_units(z):
    """(z in units of E4M3's step there, that step): the step is 2^-9 below 2^-6 and 2^(e-3) at 2^e."""
    e = torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return z.abs() / step, step
