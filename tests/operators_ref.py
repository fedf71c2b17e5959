"""Plain 64-bit forms of the norm, linear, packing and feed-forward operators for the tests (torch, any device), and buffers whose
surroundings show a stray read or write."""
import math

import torch

ACTS = ("none", "gelu", "gelu_tanh", "silu")


def act(v, name):
    if name == "gelu":
        return 0.5 * v * (1 + torch.special.erf(v / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    return v


def stride(K):
    return 4 * ((K + 127) // 128)


def codes(x):
    """Scale codes (int64) of the rows of x [rows, K]: the smallest power of two by which the largest finite magnitude of 32
    channels fits 448."""
    b = x.double().reshape(x.shape[0], -1, 32)
    top = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax(-1)
    m, e = torch.frexp(top / 448)          # top / 448 in (2^(e-1), 2^e) or exactly 2^(e-1); the division by 448 = 7 * 64 rounds,
    e = torch.where(top <= 448 * torch.exp2((e - 1).double()), e - 1, e)   # so the border is decided by an exact product
    e = torch.where(top > 448 * torch.exp2(e.double()), e + 1, e)
    return torch.where(top == 0, torch.zeros_like(e), (e + 127).clamp(min=0)).long()


def pack(x):
    """(elements, scale codes) of x [rows, K] as the library lays them out."""
    rows, K = x.shape
    c = codes(x)
    q = x.double().reshape(rows, K // 32, 32) * torch.exp2(127.0 - c.double())[..., None]
    q = q.float().to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, K)   # (q has at most 24 significant bits: exact in float)
    s = torch.zeros(rows, stride(K), dtype=torch.uint8, device=x.device)
    s[:, :K // 32] = c.to(torch.uint8)
    return q, s


def unpack(q, s):
    rows, K = q.shape
    sc = torch.exp2(s[:, :K // 32].double() - 127)
    return (q.view(torch.float8_e4m3fn).double().reshape(rows, K // 32, 32) * sc[..., None]).reshape(rows, K)


def norm(x, r, g, eps):
    h = x.double() + (r.double() if r is not None else 0.0)
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, y * g.double() if g is not None else y


def guarded(t, fill):
    """A copy of t inside a larger buffer whose ends hold `fill`; returns (view, check): check() fails if the ends changed."""
    n, pad = t.numel(), 4096
    buf = torch.full((n + 2 * pad,), fill, dtype=t.dtype, device="cuda")
    buf[pad:pad + n] = t.reshape(-1).to("cuda")
    ends = torch.cat([buf[:pad], buf[pad + n:]]).clone()
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]

    def check():
        now = torch.cat([buf[:pad], buf[pad + n:]])
        assert torch.equal(now.view(bits), ends.view(bits)), "written outside"

    return buf[pad:pad + n].reshape(t.shape), check
