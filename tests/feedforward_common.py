"""Plain 64-bit forms of the feed-forward block's operators, and the bounds their tests use.

u(t): the largest relative error of one rounding to type t, eps / 2.  E = 2^-24 is that of FP32.
"""
import math

import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E = 2.0 ** -24


def u(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """Half the spacing of t's denormals: the absolute error of a rounding near zero."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def rand(shape, t, seed, scale=1.0, shift=0.0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    wide = torch.randn(shape[0], shape[1] + pad, generator=g, device="cuda", dtype=torch.float64).mul_(scale).add_(shift).to(t)
    return wide[:, : shape[1]]


def vec(n, t, seed, scale=1.0, shift=0.0):
    return rand((1, n), t, seed, scale, shift)[0].contiguous()


def within(got, ref, bound, what):
    """Every element of got within bound (a tensor) of ref."""
    off = (got.double() - ref).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = int((off / bound.clamp(min=1e-300)).nan_to_num(nan=float("inf")).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} elements off; worst at {i}: got {got.double().flatten()[i]:.9g}, "
                             f"expected {ref.flatten()[i]:.9g}, bound {bound.expand_as(ref).flatten()[i]:.3g}")


def act64(name, v):
    z = torch.special.expit(v)
    if name == "relu":
        return torch.where(v > 0, v, 0.0), (v > 0).double()
    if name == "sigmoid":
        return z, z * torch.special.expit(-v)
    if name == "silu":
        return v * z, z + v * z * torch.special.expit(-v)
    if name == "gelu":
        cdf = torch.special.ndtr(v)
        return v * cdf, cdf + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    th = torch.tanh(k * (v + 0.044715 * v ** 3))
    return 0.5 * v * (1 + th), 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * k * (1 + 3 * 0.044715 * v * v)


def product(A, B, a_err, b_err):
    """(A B^T, bound on what an FP32-accumulated product may be off) of 64-bit A [m][k], B [n][k], whose elements the device holds with
    independent errors of up to a_err, b_err (matrices, or 0).

    S = sqrt(sum a^2 b^2) is the spread of sum a b.  Independent zero-mean errors of at most c_k sum to less than 7 sqrt(sum c_k^2) (Hoeffding:
    but for 2 exp(-7^2 / 2) = 5e-11 of the elements).  Partial sums are at most |ab| + 7 S in the same sense; each of K FP32 additions is off by at
    most 2 E of one (the tensor core cuts off what does not fit), in one direction where the core truncates: 16 terms are one
    addition there, so K / 16 + 8 of them add up, or 7 sqrt(K) E where they round."""
    K = A.shape[1]
    ref = A @ B.T
    S = torch.sqrt((A * A) @ (B * B).T)
    bound = E * (2 * (K / 16 + 8) + 7 * math.sqrt(K)) * (ref.abs() + 7 * S)
    for X, Y, err in ((A, B, a_err), (B, A, b_err)):
        if torch.is_tensor(err):
            q = (err * err) @ (B * B).T if X is A else (A * A) @ (err * err).T
            bound = bound + 7 * torch.sqrt(q)
    return ref, bound


def philox_words(n, key, step):
    """The first n words of Philox4x32-10 with counter (block, step): Salmon et al. 2011, in numpy's 64-bit integers."""
    i = np.arange((n + 3) // 4, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    c = [i & m, i >> np.uint64(32), np.full_like(i, step & 0xFFFFFFFF), np.full_like(i, step >> 32 & 0xFFFFFFFF)]
    k = [key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).reshape(-1)[:n]


def mask_of(shape, p, key, step):
    words = philox_words(shape[0] * shape[1], key, step).reshape(shape)
    return torch.from_numpy(words >= np.uint64(round(p * 2 ** 32))).cuda()
