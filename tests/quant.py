"""Rotary positions, and a small paged cache held in 8 bits, on the host and in 64 bits, from their definition."""
import numpy as np
import torch

import paged
from paper_2609_32663_gb300 import dkv

HEAD = 128
PAIRS = {False: lambda rot: (np.arange(rot // 2), np.arange(rot // 2) + rot // 2),
         True: lambda rot: (2 * np.arange(rot // 2), 2 * np.arange(rot // 2) + 1)}


def turned(x, positions, freq, interleaved, magnitude=1.0):
    """(rows x [T, heads, 128] turned, |a| + |b| of each element's pair times the magnitude) in 64 bits."""
    x = x.double()
    a, b = PAIRS[interleaved](2 * len(freq))
    # Exact for the frequency as it is held: turns modulo 1 in 64-bit integers.
    turns = np.array([int(np.floor(f / (2 * np.pi) % 1 * 2.0 ** 64)) % 2 ** 64 for f in freq], dtype=object)
    frac = np.array([[(int(p) * t % 2 ** 64) / 2.0 ** 64 for t in turns] for p in positions], dtype=np.float64).reshape(len(positions), -1)
    cos, sin = (torch.from_numpy(f(2 * np.pi * frac) * magnitude)[:, None] for f in (np.cos, np.sin))
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    return y, size


def assert_turned(got, want, size, dtype, what=""):
    """An element is rounded once. Before that, in fp32: the angle within a quarter turn is off by 2^-26 of half a turn
    (two roundings of a value below 1/4), 2^-24.4; cos and sin by two last places, 2^-23; the magnitude, the two
    products and their sum by 2^-24 each: below 2^-21 (|a| + |b|) together. fp16 rounds to a step of 2^-24 at least."""
    u = torch.finfo(dtype).eps / 2
    got = got.double().cpu()
    bound = u * (want.abs() + 2.0 ** -21 * size) + 2.0 ** -21 * size + (2.0 ** -25 if dtype == torch.float16 else 1e-38)
    err = ((got - want).abs() / bound)
    assert err.numel() == 0 or float(err.max()) <= 1, f"{what}: {float(err.max()):.3g} times the bound"


def scale_bytes(x):
    """Scale bytes of rows (the last axis): the least e >= -126 with max |x| <= 448 2^e over what is finite, plus 127."""
    x = np.abs(np.asarray(x, np.float64))
    most = np.where(np.isfinite(x), x, 0).max(-1)
    e = np.full(most.shape, -126)
    for i in range(-126, 121):
        e = np.where(most > 448 * 2.0 ** i, i + 1, e)
    return (e + 127).astype(np.uint8)


def codes_of(y):
    """e4m3 bytes of values of at most 448 (0x7f, NaN, for what is not finite): nearest, ties to the even code."""
    y = np.asarray(y, np.float64)
    a = np.where(np.isfinite(y), np.abs(y), 0)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-30))), -6) - 3)
    v = np.round(a / step) * step  # (np.round: ties to even)
    e = np.maximum(np.floor(np.log2(np.maximum(v, 1e-30))), -6)
    code = np.where(v < 2.0 ** -6, v / 2.0 ** -9, (e + 7) * 8 + (v / np.exp2(e) - 1) * 8).astype(np.uint8)
    return np.where(np.isfinite(y), code | np.where(np.signbit(y), 0x80, 0).astype(np.uint8), 0x7f).astype(np.uint8)


def held(x):
    """(codes, scale bytes) of rows as numpy arrays."""
    x = x.double().numpy() if isinstance(x, torch.Tensor) else np.asarray(x, np.float64)
    u = scale_bytes(x)
    return codes_of(x / np.exp2(u.astype(np.float64) - 127)[..., None]), u


def values(codes, scales):
    """What rows stand for, in 64 bits."""
    c = torch.as_tensor(np.asarray(codes)).view(torch.float8_e4m3fn).double()
    return c * torch.exp2(torch.as_tensor(np.asarray(scales)).double() - 127)[..., None]


class Cache8:
    """paged.Cache in 8 bits: K8, V8 uint8 [rows, 128], Ks, Vs uint8 [rows]; rows that no slab holds are NaN."""

    def __init__(self, lens, page, spare=3, wider=2, dtype=torch.bfloat16, seed=0, H=None):
        c = self.cache = paged.Cache(lens, page, spare=spare, wider=wider, dtype=dtype, seed=seed, H=H)
        self.pages, self.dtype = c.pages, dtype
        (self.K8, self.Ks), (self.V8, self.Vs) = ([torch.from_numpy(x) for x in held(p)] for p in (c.Kp, c.Vp))
        unused = torch.isnan(c.Kp[:, 0])
        for codes, scales in ((self.K8, self.Ks), (self.V8, self.Vs)):
            codes[unused], scales[unused] = 0x7f, 255
        self.sync()

    def sync(self):
        """The 64-bit values follow the bytes."""
        self.cache.Kp, self.cache.Vp = values(self.K8, self.Ks), values(self.V8, self.Vs)


def attention(c8, layer, q, cu, causal=True, scale=None):
    out, size, _, _ = paged.attention(c8.cache, layer, q, None, None, cu, causal, scale)
    return out, size


def weight_rounding(tokens, G, dtype, rows, most=0):
    """Half a step of a softmax weight, relative, for each of `rows` tokens: 2^-11 (fp16) where a sequence's tokens x G are at most
    8, or at most 16 if no sequence of the call may have more, else that of the call's type."""
    few = 16 if (most if 0 < most < rows else rows) * G <= 16 else 8
    few = np.repeat([n * G <= few for n in tokens], tokens)
    u = np.full(rows, torch.finfo(dtype).eps / 2)
    u[:few.size][few] = 2.0 ** -11
    return torch.from_numpy(u)[:, None, None]


def assert_attention(got, want, size, dtype, what="", weights=None):
    """Each output is rounded once, u |o|, and so is each weight (`weights`, relative; a sequence of few tokens has them
    times their rows' V scales, in fp16): weights sum w|v|, or half of fp16's least step, 2^-32 of the largest weight times the
    largest scale (below 1e-6 of sum w|v| for the inputs here). Scores are 32-bit sums of 128 products, |error| <= 128 2^-24 sum|q k| scale < 2e-4 for
    the standard normal inputs here (sum |q k| scale < 25), which moves a weight by twice that."""
    u = torch.finfo(dtype).eps / 2
    got = got.double().cpu()
    bound = u * want.abs() * (1 + 1e-3) + ((u if weights is None else weights) + 4e-4) * size + 1e-30
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), what
    err = ((got - want).abs() / bound)[finite]
    assert err.numel() == 0 or float(err.max()) <= 1, f"{what}: {float(err.max()):.3g} times the bound"
