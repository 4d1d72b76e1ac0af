"""Plain 64-bit forms of the row operators and of the 4-bit cache, for the tests: no code of the
library, and numpy / torch on the CPU throughout."""
import math

import torch

FP4 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def step(dtype):
    """A rounding is off by at most this, relative to the value."""
    return torch.finfo(dtype).eps / 2


def rotated(x, norm, eps, table, at, interleaved):
    """x [n][H][d] (16-bit), at [n][rot / 2]: the table's row of each pair.  Returns the exact rows and a
    bound on what fp32 arithmetic may add to their magnitudes before the last rounding: a factor of the
    norm has three roundings (of the root, and two products), a turn a product and a sum of each part."""
    y = x.double()
    if norm is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * norm.double()
    size = y.abs()
    half = 0 if table is None else table.shape[1] // 2
    if half:
        pair = torch.arange(half)
        c, s = table[at, pair].double()[:, None], table[at, pair + half].double()[:, None]
        a, b = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + half)
        ya, yb = y[..., a].clone(), y[..., b].clone()
        y, size = y.clone(), size.clone()
        y[..., a], y[..., b] = ya * c - yb * s, yb * c + ya * s
        size[..., a] = (ya * c).abs() + (yb * s).abs()
        size[..., b] = (yb * c).abs() + (ya * s).abs()
    # (the exact squares' sum and its root in fp64 add nothing that shows)
    return y, 5 * 2.0 ** -24 * size


def row_bound(y, slack, dtype):
    """|out - y| for a row rounded once to dtype: half a step of what the fp32 value may be (at least half
    of the smallest subnormal), and the fp32 arithmetic's own error."""
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    return slack + torch.clamp(step(dtype) * (y.abs() + slack), min=tiny)


def fp4_quantised(x):
    """bf16 rows [..., d] -> codes (int64) and the scales (fp64), by the definition."""
    x32 = x.float()
    most = x32.abs().amax(-1)
    b = (most / 6.0).view(torch.int32)
    scale = torch.where(most > 0, ((b + 0xffff) & ~0xffff).view(torch.float32), torch.ones_like(most))
    r = (x32.double() / scale.double()[..., None]).float().double()      # (fp64 division, then fp32: rounds once in all)
    grid = FP4
    m = r.abs().clamp(max=6.0)
    hi = torch.searchsorted(grid, m.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - m, m - grid[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return code + 8 * ((r < 0) & (code > 0)), scale.double()


def int8_quantised(x):
    x32 = x.float()
    most = x32.abs().amax(-1)
    scale = torch.where(most > 0, (most.double() / 127.0).float(), torch.ones_like(most))
    r = (x32.double() / scale.double()[..., None]).float()
    return torch.round(r).clamp(-127, 127).long(), scale.double()


def fp4_values(code):
    return FP4[code & 7] * (1 - 2 * (code >> 3)).double()


def fp4_places(S, d):
    """Byte and shift of every (token, channel) of a block: of keys, of values."""
    t, c = torch.meshgrid(torch.arange(S), torch.arange(d), indexing="ij")
    k = t * (d // 2) + c // 2
    v = S * d // 2 + (((t // 8 * (d // 64) + c // 64) * 16 + c % 16) * 4 + c // 16 % 4) * 4 + t % 8 // 2
    return (k, 4 * (c % 2)), (v, 4 * (t % 2))


def fp4_unpacked(blocks, S, d):
    """Blocks uint8 [..., bytes] -> key codes, key scales, value codes, value scales ([..., S, d], [..., S])."""
    blocks = blocks[..., :S * (d + 4)].contiguous()
    (ka, ks), (va, vs) = fp4_places(S, d)
    b = blocks.long()
    sc = blocks[..., S * d:].contiguous().view(torch.bfloat16).double()
    return b[..., ka] >> ks & 15, sc[..., :S], b[..., va] >> vs & 15, sc[..., S:]


def fp4_packed(kc, ks, vc, vs, stride):
    """The other way round, into blocks of `stride` bytes."""
    S, d = kc.shape[-2:]
    (ka, kb), (va, vb) = fp4_places(S, d)
    out = torch.zeros(kc.shape[:-2] + (stride,), dtype=torch.int64)
    lead = kc.shape[:-2]
    for code, at, sh in ((kc, ka, kb), (vc, va, vb)):
        out.scatter_add_(-1, at.reshape(-1).expand(lead + (-1,)), (code << sh).reshape(lead + (-1,)))
    out = out.to(torch.uint8)
    out[..., S * d:S * (d + 4)] = torch.cat([ks, vs], -1).to(torch.bfloat16).contiguous().view(torch.uint8)
    return out


def outwards(x, up):
    """fp64 -> the bf16 number at or next to it on one side, by bisecting the bf16 numbers' order."""
    back = lambda k: torch.where(k < 0, -k - 0x8000, k).to(torch.int16).view(torch.bfloat16).double()  # noqa: E731
    lo = torch.full(x.shape, -0x7f80, dtype=torch.int32)
    hi = torch.full(x.shape, 0x7f80, dtype=torch.int32)
    for _ in range(17):             # the largest number <= x
        mid = (lo + hi + 1) >> 1
        ok = back(mid) <= x
        lo, hi = torch.where(ok, mid, lo), torch.where(ok, hi, mid - 1)
    below = lo
    exact = back(below) == x
    return back(torch.where(exact | torch.tensor(not up), below, below + 1))


def attention(q, k, v, scale):
    """q [H][d] on k, v [Hkv][n][d] (fp64): the output, the log denominators, and a bound of the output's
    error for fp32 sums of exact products and weights of 16 bits and more (relative 2^-18 each)."""
    Hkv, n, d = k.shape
    G = q.shape[0] // Hkv
    q = q.double().view(Hkv, G, d)
    if n == 0:
        z = torch.zeros(Hkv * G, d, dtype=torch.float64)
        return z, torch.full((Hkv * G,), -math.inf, dtype=torch.float64), z
    w = torch.matmul(q, k.transpose(1, 2)) * scale
    # a logit: d products summed in fp32, two factors and log2(e) on top; then the exponent's own rounding
    off = (d + 8) * 2.0 ** -24 * torch.matmul(q.abs(), k.abs().transpose(1, 2)).amax(-1) * abs(scale) + 2.0 ** -22
    lse = torch.logsumexp(w, -1)
    p = torch.exp(w - lse[..., None])
    out = torch.matmul(p, v)
    # weights off by exp(2 off), their roundings, and fp32 sums over n tokens of |p v| (and of p)
    rel = 2 * off + 2.0 ** -17 + (n + 64) * 2.0 ** -23
    bound = rel[..., None] * (torch.matmul(p, v.abs()) + out.abs())
    return out.reshape(Hkv * G, d), lse.reshape(-1), bound.reshape(Hkv * G, d)
