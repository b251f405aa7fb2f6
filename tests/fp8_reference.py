"""The 8-bit floating-point linear and the norm with codes, stated plainly on the CPU: every binary32 step of the definition as one
torch operation, sums of squares and products in 64 bits."""
from __future__ import annotations

import torch

BLOCK, E4M3_MAX, TINY = 128, torch.tensor(448.0), 2.0 ** -100


def rows(seed, T, K, dtype, outliers=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, K, generator=g)
    if outliers:
        x[:, torch.randperm(K, generator=g)[: max(1, K // 200)]] *= 50.0
    return x.to(dtype)


def padded_rows(T):
    return -(-T // 16) * 16 + 256


def _blocks(v):
    T, K = v.shape
    kb = -(-K // BLOCK)
    return torch.nn.functional.pad(v, (0, kb * BLOCK - K)).view(T, kb, BLOCK)


def _codes(v, a):
    """Codes and scale of blocks whose largest magnitude is `a` (NaN apart)."""
    r = torch.where(a < TINY, torch.zeros_like(a), E4M3_MAX / a)
    return (v * r).to(torch.float8_e4m3fn), torch.where(a < TINY, torch.zeros_like(a), a / E4M3_MAX)


def act_codes(v):
    """fp32 [T, K] -> (e4m3 [T, K], scale [T, ceil(K/128)])."""
    T, K = v.shape
    b = _blocks(v)
    q, s = _codes(b, b.nan_to_num(nan=0.0, posinf=float("inf"), neginf=-float("inf")).abs().amax(dim=2, keepdim=True))
    return q.view(torch.uint8).reshape(T, -1)[:, :K].contiguous().view(torch.float8_e4m3fn), s[:, :, 0]


def weight_codes(w):
    """fp32 [K, N] -> (e4m3 [K, N], scale [ceil(K/128), ceil(N/128)])."""
    K, N = w.shape
    kb, nb = -(-K // BLOCK), -(-N // BLOCK)
    b = torch.nn.functional.pad(w, (0, nb * BLOCK - N, 0, kb * BLOCK - K)).view(kb, BLOCK, nb, BLOCK)
    q, s = _codes(b, b.nan_to_num(nan=0.0, posinf=float("inf"), neginf=-float("inf")).abs().amax(dim=(1, 3), keepdim=True))
    return q.view(torch.uint8).reshape(kb * BLOCK, -1)[:K, :N].contiguous().view(torch.float8_e4m3fn), s[:, 0, :, 0]


def pack_weight(wq):
    """[K, N] codes as haq_pack_weight lays them out."""
    K, N = wq.shape
    kp, npad = -(-K // 64) * 64, -(-N // 256) * 256
    b = torch.nn.functional.pad(wq.view(torch.uint8), (0, npad - N, 0, kp - K))
    return b.view(kp // 16, 16, npad).transpose(1, 2).contiguous().view(-1)


def unpack_act(q_packed, T, K):
    """Packed codes -> [T, K] bytes."""
    return q_packed.view(torch.uint8)[: -(-K // 64) * 64 * padded_rows(T)].view(-1, padded_rows(T), 16)[: K // 16, :T].permute(1, 0, 2).reshape(T, K)


def unpack_scale(scale, T, K):
    return scale.view(-1, padded_rows(T))[: -(-K // BLOCK), :T].t()


def linear(xq, sx, wq, sw, relu=False):
    """(y, bound of the sum's error) in 64 bits.  The bound: a matrix instruction sums products in groups of eight, in whole steps of
    2^-13 of the largest one's power of two: the other seven lose less than a step each, together 7 2^-13 of the magnitudes; the 16
    groups of a block are added in binary32, 16 2^-24 at most.  The scales' product and the sum over the blocks round once each for
    a block, 2^-24 of a partial sum that the magnitudes bound, so kb 2^-23 of their whole sum."""
    K, N = wq.shape
    kb = -(-K // BLOCK)
    a, w = xq.double(), wq.double()
    y, mag = torch.zeros(xq.shape[0], N, dtype=torch.float64), torch.zeros(xq.shape[0], N, dtype=torch.float64)
    for b in range(kb):
        k = slice(b * BLOCK, (b + 1) * BLOCK)
        s = sx[:, b:b + 1].double() * sw[b].double().repeat_interleave(BLOCK)[:N]
        y += s * (a[:, k] @ w[k])
        mag += s.abs() * (a[:, k].abs() @ w[k].abs())
    return (y.clamp(min=0) if relu else y), mag * (7 * 2.0 ** -13 + 2.0 ** -20 + kb * 2.0 ** -23)


def assert_linear(y, ref, bound):
    """y (16 bits) is `ref`, off by `bound` before the one rounding, of half a step (of the smallest normal below it)."""
    info = torch.finfo(y.dtype)
    over = ref.abs() + bound >= info.max  # may round to infinity
    half = (ref.abs() + bound).clamp(min=info.tiny) * info.eps / 2
    far = (y.double() - ref).abs() - bound - half
    ok = (far <= 0) | (over & ((y.double() == ref.sign() * float("inf")) | (far <= 0)))
    assert bool(ok.all()), (int((~ok).sum()), float(far[~ok].max()), ok.logical_not().nonzero()[:4].tolist())


def norm(x, weight, eps, residual=None):
    """(h in 16 bits, v in binary32)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    m = h.double().square().sum(dim=1, keepdim=True) / h.shape[1]
    return h, h.float() * (1.0 / (m + eps).sqrt()).float() * weight


def i8_codes(v):
    """fp32 [T, K] -> (int8 [T, K], scale [T])."""
    a = v.abs().amax(dim=1, keepdim=True)
    s = torch.where(a < TINY, torch.zeros_like(a), a / torch.tensor(127.0))
    fine = (a >= TINY) & a.isfinite()
    q = torch.where(fine, (v / s).round().clamp(-127, 127), torch.zeros_like(v))
    return q.to(torch.int8), s[:, 0]
