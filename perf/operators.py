"""The operators between the projections of a layer and its decode attention, as cases that can be
timed and compared: norm and rotation of queries and keys, the rotated append to the paged cache, and
attention over a cache held in 4 bits.

Operations ("op"):

  rotate   per-head norms of queries and keys and their position rotation (rotate_rows)
  append   keys and values of one token (decode) or of ragged prompts into the 16-bit paged cache,
           rotated on the way, page boxes kept, the queries rotated in the same call (append_rows)
  step     the same into the 4-bit cache, and the attention of each sequence's last token over all
           its cached tokens (append_rows, dense_decode_attention)
  dense    attention over every cached token of a 4-bit cache (dense_decode_attention)
  aware    scores, page selection and attention over the selected pages of a 4-bit cache
           (query_aware_decode)

The plain forms below compute the same from elementary torch operations.  Where a value is rounded to
a code, to 16 bits for the cache, or outwards for a box, the plain form takes the same roundings in
the same order; sums of squares and page scores are taken in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = float(torch.tensor(1e-6, dtype=torch.float32))
FP4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]      # magnitudes of the codes 0 to 7; bit 3 is the sign
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp4": torch.bfloat16}     # of the rows beside the cache

BASE = dict(B=1, Hq=32, Hkv=4, d=64, S=16, L=0, L_min=0, new=1, kv="bf16", rot=64, interleaved=False, axes=1,
            norm=False, fused=False, topk=0, frac=0.0, out="f32")


def _case(name, op, **kw):
    c = dict(BASE, name=name, op=op, kv="bf16" if op in ("rotate", "append") else "fp4")
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token in a TinyLLaMA-shaped model: 36 rows, all of it is latency
        _case("rotate_token", "rotate", norm=True),
        # one user's prompt of odd length, queries and keys sliced out of one projection's rows
        _case("rotate_prompt", "rotate", new=8191, norm=True, fused=True),
        # a video prompt: three position axes, adjacent channels paired, a part of the head rotated
        _case("rotate_video", "rotate", new=5003, Hkv=8, d=128, kv="fp16", rot=96, interleaved=True, axes=3,
              norm=True),
        # the decode step of the ragged serving batch, many heads: one token for each sequence
        _case("append_step", "append", B=64, Hkv=32, d=128, rot=128, L=2000, L_min=200, fused=True),
        # prompts of several users, of very different lengths, behind what some have cached already
        _case("append_prompts", "append", B=7, Hkv=8, d=128, rot=128, L=900, L_min=1, new=4001, norm=True, fused=True),
        # one user chatting: a short odd context in 4 bits, one token appended and attended
        _case("chat_step", "step", L=2999, norm=True, fused=True, out="bf16"),
        # the first token after the prompts of a batch: they go into the 4-bit cache and are attended
        _case("prompt_step", "step", B=5, Hkv=8, d=128, S=32, rot=128, L=40, L_min=1, new=2500, norm=True, fused=True,
              out="bf16"),
        # the smallest cache: one sequence, one head
        _case("tiny_dense", "dense", Hq=1, Hkv=1, L=4096),
        # the TinyLLaMA-shaped batch
        _case("tinyllama_dense", "dense", B=16, L=16384),
        # the large ragged serving batch, grouped heads, 128 channels: the most work of all
        _case("ragged_dense", "dense", B=64, Hkv=8, d=128, L=32768, L_min=1024, out="bf16"),
        # long documents: few sequences, 128K tokens each, large pages, a fixed number of pages kept
        _case("longctx_aware", "aware", B=4, S=32, L=131072, topk=128),
        # a mid-size ragged batch that keeps a quarter of each sequence's pages
        _case("gqa_aware", "aware", B=24, Hkv=8, d=128, L=8192, L_min=512, frac=0.25, out="bf16"),
    ]


HEADS = [(1, 1), (8, 8), (12, 12), (16, 16), (32, 32), (8, 1), (12, 4), (16, 2), (32, 4), (32, 8), (40, 8), (64, 8)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = work(next(c for c in listed() if c["name"] == "ragged_dense"))["bytes"]
    while True:
        op = rng.choice(["rotate", "append", "step", "dense", "aware"])
        Hq, Hkv = rng.choice(HEADS)
        d = rng.choice([64, 128])
        c = dict(BASE, op=op, Hq=Hq, Hkv=Hkv, d=d, rot=rng.choice([d, d, d // 2, 3 * d // 4]),
                 interleaved=rng.random() < 0.3, axes=rng.choice([1, 1, 3]) if op == "rotate" else 1,
                 norm=rng.random() < 0.6, fused=rng.random() < 0.5, out=rng.choice(["f32", "bf16"]),
                 kv=rng.choice(["bf16", "fp16"]) if op in ("rotate", "append") else "fp4")
        if op == "rotate":
            c["new"] = _log_int(rng, 1, 32768)
        else:
            c["B"] = _log_int(rng, 1, 64)
            c["S"] = rng.choices([4, 8, 16, 32, 64] if op == "append" else [8, 16, 32, 64],
                                 [1, 1, 6, 3, 1] if op == "append" else [1, 6, 3, 1])[0]
            c["L"] = _log_int(rng, 1, 4097) - 1 if op in ("append", "step") else _log_int(rng, 1, 65536)
            c["new"] = rng.choice([1, _log_int(rng, 2, 8192)])
            if c["L"] and rng.random() < 0.5:
                c["L_min"] = max(1, int(c["L"] * rng.uniform(0.03, 0.9)))
        if op == "aware":
            pages = -(-c["L"] // c["S"])
            if c["L_min"]:
                c["frac"] = round(rng.uniform(0.05, 0.5), 3)
            else:
                c["topk"] = max(1, int(pages * math.exp(rng.uniform(math.log(0.03), math.log(0.5)))))
        if op == "step":        # (its output follows from rotated rows rounded to bf16)
            c["out"] = "bf16"
        if op != "rotate" and _capacity(c) // c["S"] > 16384:
            continue
        if work(c)["bytes"] <= most and _padded_bytes(c) <= 10 << 30:
            return c


# ---------------------------------------------------------------------------------- sizes of a case
def _spread(lo, hi, n, i):
    return lo + (hi - lo) * (2 * i + 1) // (2 * n)


def _mean_lens(c):
    """Cached tokens of each sequence, each draw at the middle of its share of the range."""
    if not c["L_min"]:
        return [c["L"]] * c["B"]
    return [_spread(c["L_min"], c["L"], c["B"], i) for i in range(c["B"])]


def _mean_new(c):
    return [1] * c["B"] if c["new"] == 1 else [_spread(1, c["new"], c["B"], i) for i in range(c["B"])]


def _capacity(c):
    """Tokens a row of the block table has room for."""
    most = c["L"] + (c["new"] if c["op"] in ("append", "step") else 0)
    return -(-most // c["S"]) * c["S"]


def _padded_bytes(c):
    """All sequences as long as the longest, in fp32: what the plain forms lay out."""
    return 0 if c["op"] == "rotate" else 4 * c["B"] * c["Hkv"] * c["d"] * _capacity(c)


def work(case):
    c = case
    d, Hq, Hkv = c["d"], c["Hq"], c["Hkv"]
    if c["op"] == "rotate":
        n = c["new"]
        return {"bytes": 4 * n * (Hq + Hkv) * d + 4 * n * c["rot"], "flops": 8 * n * (Hq + Hkv) * d}
    lens, new = _mean_lens(c), _mean_new(c)
    token = 2 * (d + 4) // 2 if c["op"] != "append" else 4 * d          # K and V of one token and head
    out = c["B"] * Hq * d * (2 + (2 if c["out"] == "bf16" else 4))      # queries in, attention out
    if c["op"] in ("append", "step"):
        n = sum(new)
        pages = sum(-(-(a + b) // c["S"]) - a // c["S"] for a, b in zip(lens, new))
        size = 2 * n * (2 * Hq + 2 * Hkv) * d + n * Hkv * token + 4 * n * c["rot"] + pages * Hkv * 4 * d
        flops = 8 * n * (Hq + 2 * Hkv) * d
        if c["op"] == "step":
            cached = sum(lens) + n
            size += cached * Hkv * token + out
            flops += 4 * cached * Hq * d
        return {"bytes": size, "flops": flops}
    if c["op"] == "dense":
        return {"bytes": sum(lens) * Hkv * token + out, "flops": 4 * sum(lens) * Hq * d}
    pages = [-(-n // c["S"]) for n in lens]
    kept = [_kept(c, p) for p in pages]
    return {"bytes": sum(pages) * Hkv * 4 * d + sum(kept) * c["S"] * Hkv * token + out + sum(pages) * Hkv * 4,
            "flops": 4 * sum(kept) * c["S"] * Hq * d + 4 * sum(pages) * Hq * d}


def _kept(c, pages):
    return min(pages, c["topk"] if c["topk"] else max(1, math.ceil(c["frac"] * pages)))


# ------------------------------------------------------------------------------------------- inputs
def _table(rows, rot):
    """Cosines and sines of every position, worked out in 64 bits."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEVICE)
    at = torch.arange(rows, dtype=torch.float64, device=DEVICE)[:, None] * 10000.0 ** (-2.0 * i / rot)
    return torch.cat([at.cos(), at.sin()], dim=1).float().contiguous()


def _axis_of_pair(c):
    """Which axis a pair of channels turns by: sections in turn of time, height and width."""
    return [0] * (c["rot"] // 2) if c["axes"] == 1 else [i % 3 for i in range(c["rot"] // 2)]


def _rows(c, n, g):
    """The projections' rows of n tokens: slices of one matrix, or three of their own."""
    Hq, Hkv, d, t = c["Hq"], c["Hkv"], c["d"], TYPES[c["kv"]]
    heads = [Hq, Hkv, Hkv]
    if c["fused"]:
        x = torch.randn((n, sum(heads), d), generator=g, device=DEVICE).to(t)
        return list(x.split(heads, dim=1))
    return [torch.randn((n, h, d), generator=g, device=DEVICE).to(t) for h in heads]


def _fp4_codes(x):
    """fp32 rows [..., d] -> codes (uint8) and one bf16 scale a row, the scale rounded up."""
    most = x.abs().amax(-1)
    up = ((most / 6.0).view(torch.int32) + 0xffff) & ~0xffff
    scale = torch.where(most > 0, up.view(torch.float32), torch.ones_like(most))
    r = (x.double() / scale[..., None].double()).float()
    m = r.abs()
    code = torch.zeros_like(m, dtype=torch.uint8)
    code += m > 0.25
    code += m >= 0.75
    code += m > 1.25
    code += m >= 1.75
    code += m > 2.5
    code += m >= 3.5
    code += m > 5.0
    code += ((code > 0) & (r < 0)).to(torch.uint8) * 8
    return code, scale.to(torch.bfloat16)


def _block_bytes(S, d):
    return S * (d + 4)


def _pack_pages(kc, ks, vc, vs):
    """Codes [n][Hkv][S][d] and scales [n][Hkv][S] of whole pages -> blocks [n][Hkv][S * (d + 4)]."""
    n, H, S, d = kc.shape
    k = kc[..., 0::2] | kc[..., 1::2] << 4                                            # [n][H][S][d/2]
    v = vc.view(n, H, S // 8, 4, 2, d // 64, 4, 16)             # octet, pair, token of the pair, channels
    v = (v[:, :, :, :, 0] | v[:, :, :, :, 1] << 4).permute(0, 1, 2, 4, 6, 5, 3)       # [o][d/64][16][4][pair]
    parts = [k.reshape(n, H, -1), v.reshape(n, H, -1), ks.contiguous().view(torch.uint8).view(n, H, -1),
             vs.contiguous().view(torch.uint8).view(n, H, -1)]
    return torch.cat(parts, dim=2)


def _unpack_pages(blocks, S, d):
    """The values [n][Hkv][S][d] (fp32) of keys and values of blocks [n][Hkv][S * (d + 4)]."""
    n, H = blocks.shape[:2]
    half = S * d // 2
    table = torch.tensor(FP4 + [-x for x in FP4], device=blocks.device)

    def values(codes):
        return table.index_select(0, codes.reshape(-1).int()).view(codes.shape)

    def scales(at):
        return blocks[:, :, at:at + 2 * S].contiguous().view(torch.bfloat16).float()[..., None]

    k = blocks[:, :, :half].reshape(n, H, S, d // 2)
    k = torch.stack([k & 15, k >> 4], dim=-1).view(n, H, S, d)
    v = blocks[:, :, half:2 * half].reshape(n, H, S // 8, d // 64, 16, 4, 4)          # [o][d/64][16][4][pair]
    v = torch.stack([v & 15, v >> 4], dim=-1).permute(0, 1, 2, 6, 7, 3, 5, 4).reshape(n, H, S, d)
    return values(k) * scales(2 * half), values(v) * scales(2 * half + 2 * S)


def _outwards(v, up):
    """Values (fp32 or fp64) to the bf16 number next to them on one side."""
    n = v.to(torch.bfloat16)
    off = (n.double() < v.double()) if up else (n.double() > v.double())
    b = n.view(torch.int16).int()
    key = torch.where(b < 0, -(b & 0x7fff), b) + off.int() * (1 if up else -1)
    return torch.where(key < 0, -key - 0x8000, key).to(torch.int16).view(torch.bfloat16)


def _shuffled(x, g):
    return [x[i] for i in torch.randperm(len(x), generator=g).tolist()]


def _pool_pages(c):
    """Pages enough for however the lengths and the new tokens fall together."""
    S, grows = c["S"], c["op"] in ("append", "step")
    return sum(-(-n // S) for n in _mean_lens(c)) + (sum(-(-n // S) for n in _mean_new(c)) if grows else 0)


def _paged(c, lens, gc):
    """A shuffled block table whose rows have pages for all their tokens, -1 behind them."""
    S = c["S"]
    wide, n_phys = _capacity(c) // S, _pool_pages(c)
    need = [-(-n // S) for n in lens]
    perm = torch.randperm(n_phys, generator=gc)
    table = torch.full((c["B"], wide), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n].int()
        at += n
    return table.to(DEVICE), n_phys


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    gc = torch.Generator()
    gc.manual_seed(seed)
    B, Hq, Hkv, d, S, rot = c["B"], c["Hq"], c["Hkv"], c["d"], c["S"], c["rot"]
    s = dict(case=c, scale=1.0 / math.sqrt(d), axis=_axis_of_pair(c))
    if c["norm"]:
        s["q_norm"], s["k_norm"] = (1.0 + 0.2 * torch.randn((2, d), generator=g, device=DEVICE)).unbind(0)
    else:
        s["q_norm"] = s["k_norm"] = None
    if c["op"] == "rotate":
        n = c["new"]
        start = int(torch.randint(0, 32768, (1,), generator=gc))
        at = torch.arange(start, start + n, dtype=torch.int32)
        if c["axes"] == 3:                      # frames of 24 by 36 patches
            at = torch.arange(n, dtype=torch.int32)
            at = torch.stack([start + at // 864, start + at // 36 % 24, start + at % 36])
        s["positions"] = at.view(c["axes"], n).to(DEVICE)
        s["table"] = _table(start + n, rot)
        s["q"], s["k"], _ = _rows(c, n, g)
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=x.dtype, device=DEVICE) for x in (s["q"], s["k"]))
        if own:
            from paper_2509_12211_amd import tinyserve as ts
            s["rotary"] = ts.make_rotary(s["table"], positions=s["positions"], interleaved=c["interleaved"],
                                         axis_of_pair=s["axis"], q_norm=s["q_norm"], k_norm=s["k_norm"], norm_eps=EPS)
        return s

    # the batch's lengths are the same whatever the seed; which sequence has which is not
    grows = c["op"] in ("append", "step")
    lens = _shuffled(_mean_lens(c), gc)
    new = _shuffled(_mean_new(c), gc) if grows else [0] * B
    full = [a + b for a, b in zip(lens, new)]
    table, n_phys = _paged(c, full, gc)
    wide = table.shape[1]
    s.update(block_table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEVICE), n_phys=n_phys)
    page_type = TYPES[c["kv"]]
    # what the sequences hold already: every page of the pool is filled, what lies behind a length counts as absent
    if c["op"] == "append":
        kv = torch.randn((n_phys, Hkv, 2, S * d), generator=g, device=DEVICE).to(page_type)
        s["k_pool"], s["v_pool"] = kv[:, :, 0].view(n_phys, Hkv, S, d), kv[:, :, 1].view(n_phys, Hkv, d, S)
    else:
        s["pool"] = torch.empty((n_phys, Hkv, _block_bytes(S, d)), dtype=torch.uint8, device=DEVICE)
        offset = torch.randn((Hkv, 1, d), generator=g, device=DEVICE)
        step = max(1, (64 << 20) // (Hkv * S * d))
        for at in range(0, n_phys, step):
            n = min(step, n_phys - at)
            k = torch.randn((n, Hkv, S, d), generator=g, device=DEVICE) + offset
            v = torch.randn((n, Hkv, S, d), generator=g, device=DEVICE)
            s["pool"][at:at + n] = _pack_pages(*_fp4_codes(k.bfloat16().float()), *_fp4_codes(v.bfloat16().float()))
    s["page_min"] = torch.zeros((B, Hkv, wide, d), dtype=page_type, device=DEVICE)
    s["page_max"] = torch.zeros_like(s["page_min"])
    for b, n in enumerate(lens if c["op"] != "dense" else []):
        pages = -(-n // S)
        if pages:
            at = table[b, :pages].long()
            k = s["k_pool"][at].float() if c["op"] == "append" else _unpack_pages(s["pool"][at], S, d)[0]
            behind = (torch.arange(pages * S, device=DEVICE) >= n).view(pages, 1, S, 1)
            s["page_min"][b, :, :pages] = _outwards_as(k.masked_fill(behind, math.inf).amin(2), page_type, False).transpose(0, 1)
            s["page_max"][b, :, :pages] = _outwards_as(k.masked_fill(behind, -math.inf).amax(2), page_type, True).transpose(0, 1)
    out_type = torch.bfloat16 if c["out"] == "bf16" else torch.float32
    if c["op"] != "append":
        s["out"] = torch.empty((B, Hq, d), dtype=out_type, device=DEVICE)
    if grows:
        n = sum(new)
        s["table"] = _table(_capacity(c), rot)
        s["q"], s["k"], s["v"] = _rows(c, n, g)
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        cu = [0]
        for x in new:
            cu.append(cu[-1] + x)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEVICE)
        s["lens_after"] = torch.tensor(full, dtype=torch.int32, device=DEVICE)
        s["last"] = s["cu"][1:].long() - 1
    else:
        s["query"] = torch.randn((B, Hq, d), generator=g, device=DEVICE).bfloat16()
    if c["op"] == "aware":
        pages = [-(-n // S) for n in lens]
        s["kept"] = torch.tensor([_kept(c, p) for p in pages], dtype=torch.int32, device=DEVICE)
        s["most"] = max(_kept(c, p) for p in pages)
        s["scores"] = torch.empty((B, Hkv, wide), dtype=torch.float32, device=DEVICE)
        s["sel"] = torch.empty((B, Hkv, s["most"]), dtype=torch.int32, device=DEVICE)
        s["count"] = torch.empty((B,), dtype=torch.int32, device=DEVICE)
    if own:
        from paper_2509_12211_amd import tinyserve as ts
        fmt = ts.TS_OUT_BF16 if c["out"] == "bf16" else ts.TS_OUT_F32

        def layout(lens_of):
            return ts.make_layout(B, Hq, Hkv, d, S, wide, s["k_pool"] if c["op"] == "append" else s["pool"],
                                  s.get("v_pool"), table, lens_of, s["page_min"], s["page_max"], out_format=fmt)

        s["layout"] = layout(s["lens"])
        if grows:
            s["layout_after"] = layout(s["lens_after"])
            s["rotary"] = ts.make_rotary(s["table"], interleaved=c["interleaved"], q_norm=s["q_norm"],
                                         k_norm=s["k_norm"], norm_eps=EPS)
        if c["op"] in ("step", "dense"):
            s["workspace"] = ts.new_dense_workspace(s["layout"], DEVICE)
        elif c["op"] == "aware":
            s["workspace"] = ts.new_workspace(s["layout"], s["most"], DEVICE)
    return s


def _outwards_as(v, dtype, up):
    """16-bit pools: their own numbers.  4 bits: rounded outwards to bf16."""
    return v.to(dtype) if dtype == torch.float16 else _outwards(v, up)


# -------------------------------------------------------------------------------------- plain forms
def _rotated(x, norm, cos, sin, interleaved):
    """16-bit rows [n][H][d] -> the same, normed and rotated: fp32, one rounding at the end."""
    y = x.float()
    if norm is not None:
        square = y.double().square().mean(-1, keepdim=True)
        y = y * (1.0 / torch.sqrt(square + EPS)).float() * norm
    half = cos.shape[-1]
    c, s = cos[:, None], sin[:, None]
    turned, rest = y[..., :2 * half], y[..., 2 * half:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, rest], dim=-1).to(x.dtype)


def _angles(table, positions, axis):
    """cos, sin [n][rot / 2] for positions [axes][n]."""
    half = table.shape[1] // 2
    if positions.shape[0] == 1:
        rows = table[positions[0].long()]
        return rows[:, :half], rows[:, half:]
    pair = torch.arange(half, device=table.device)
    at = positions.long()[torch.tensor(axis, device=table.device)].t()       # [n][rot / 2]
    return table[at, pair], table[at, pair + half]


def _token_places(s):
    """Sequence and position of every new token."""
    count = (s["cu"][1:] - s["cu"][:-1]).long()
    n = s["q"].shape[0]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEVICE), count, output_size=n)
    pos = s["lens"].long()[seq] + torch.arange(n, device=DEVICE) - s["cu"].long()[seq]
    return seq, pos


def _widen(s, seq, pos, lo, hi):
    """The boxes of the pages that the new tokens [n][Hkv][d] lie in."""
    S = s["case"]["S"]
    B, Hkv, wide, d = s["page_min"].shape
    key = seq * wide + torch.div(pos, S, rounding_mode="floor")
    opened = torch.where(pos % S == 0, key, B * wide)
    for box, rows, fill, how in ((s["page_min"], lo, math.inf, "amin"), (s["page_max"], hi, -math.inf, "amax")):
        flat = torch.empty((B * wide + 1, Hkv, d), dtype=torch.float32, device=DEVICE)
        flat[:-1] = box.transpose(1, 2).reshape(-1, Hkv, d)
        flat[opened] = fill
        flat.index_reduce_(0, key, rows.float(), how)
        box.copy_(flat[:-1].view(B, wide, Hkv, d).transpose(1, 2))


def _plain_attention(s, q, pages, tokens_in):
    """Attention of one query a sequence over the listed pages of the 4-bit cache.  pages: physical ids
    [B][Hkv][n]; tokens_in: how many tokens of each count."""
    c = s["case"]
    B, Hkv, n = pages.shape
    S, d, G = c["S"], c["d"], c["Hq"] // c["Hkv"]
    out = s["out"]
    step = max(1, (1 << 30) // max(1, Hkv * n * S * d))                  # sequences at a time
    head = torch.arange(Hkv, device=DEVICE)[None, :, None]
    for at in range(0, B, step):
        to = min(B, at + step)
        blocks = s["pool"][pages[at:to], head.expand(to - at, Hkv, n)]                    # [b][Hkv][n][bytes]
        k, v = _unpack_pages(blocks.view((to - at) * Hkv, n, -1), S, d)
        k, v = k.view(to - at, Hkv, n * S, d), v.view(to - at, Hkv, n * S, d)
        w = torch.matmul(q[at:to].float().view(to - at, Hkv, G, d), k.transpose(2, 3).contiguous()) * s["scale"]
        there = (torch.arange(S, device=DEVICE) < tokens_in[at:to, :, :, None]).view(to - at, Hkv, 1, n * S)
        w = w.masked_fill(~there, -math.inf)
        w = torch.exp(w - w.amax(-1, keepdim=True))
        o = torch.matmul(w, v) / w.sum(-1, keepdim=True)
        out[at:to] = o.view(to - at, c["Hq"], d).to(out.dtype)
    return out


def _plain_dense(s, q, lens):
    wide, S = s["block_table"].shape[1], s["case"]["S"]
    Hkv = s["case"]["Hkv"]
    left = lens[:, None] - torch.arange(wide, device=DEVICE) * S
    pages = s["block_table"].clamp(min=0).long()[:, None].expand(-1, Hkv, -1)
    return _plain_attention(s, q, pages, left.clamp(0, S)[:, None].expand(-1, Hkv, -1))


def _plain_append(s):
    c = s["case"]
    S = c["S"]
    seq, pos = _token_places(s)
    cos, sin = _angles(s["table"], pos[None], s["axis"])
    s["q_out"].copy_(_rotated(s["q"], s["q_norm"], cos, sin, c["interleaved"]))
    k = _rotated(s["k"], s["k_norm"], cos, sin, c["interleaved"])
    phys, slot = s["block_table"].long()[seq, torch.div(pos, S, rounding_mode="floor")], pos % S
    if c["op"] == "append":
        s["k_pool"][phys, :, slot] = k
        s["v_pool"][phys, :, :, slot] = s["v"]
        _widen(s, seq, pos, k, k)
        return
    d, Hkv = c["d"], c["Hkv"]
    (kc, ks), (vc, vs) = _fp4_codes(k.float()), _fp4_codes(s["v"].float())
    half = S * d // 2
    pool, head, n = s["pool"], torch.arange(Hkv, device=DEVICE), k.shape[0]
    row = (phys[:, None] * Hkv + head) * _block_bytes(S, d)                               # [n][Hkv]
    flat = pool.view(-1)
    byte = torch.arange(d // 2, device=DEVICE)
    flat[(row[..., None] + slot[:, None, None] * (d // 2) + byte).view(-1)] = (kc[..., 0::2] | kc[..., 1::2] << 4).view(-1)
    ch = torch.arange(d, device=DEVICE)
    place = (torch.div(ch, 64, rounding_mode="floor") * 16 + ch % 16) * 4 + torch.div(ch, 16, rounding_mode="floor") % 4
    octet, pair = torch.div(slot, 8, rounding_mode="floor"), torch.div(slot, 2, rounding_mode="floor") % 4
    at = row[..., None] + half + (octet[:, None, None] * d + place) * 4 + pair[:, None, None]
    at, odd, code = at.view(-1), (slot % 2 * 4)[:, None, None].expand(at.shape).reshape(-1).to(torch.uint8), vc.reshape(-1)
    # (two tokens share a byte: each adds what its own half of it changes by)
    flat.index_add_(0, at, (code - (flat[at] >> odd & 15)) << odd)
    for x, base in ((ks, 2 * half), (vs, 2 * half + 2 * S)):
        two = x.contiguous().view(torch.uint8).view(n, Hkv, 2)
        flat[(row[..., None] + base + slot[:, None, None] * 2 + torch.arange(2, device=DEVICE)).view(-1)] = two.view(-1)
    table = torch.tensor(FP4 + [-x for x in FP4], device=DEVICE)
    value = table[kc.long()] * ks.float()[..., None]
    _widen(s, seq, pos, _outwards(value, False), _outwards(value, True))


def _plain_aware(s):
    c = s["case"]
    S, Hkv, d, G = c["S"], c["Hkv"], c["d"], c["Hq"] // c["Hkv"]
    B, wide = s["block_table"].shape
    lens = s["lens"]
    q = s["query"].view(B, Hkv, G, d).double()
    score = torch.matmul(s["page_max"].double(), q.clamp(min=0).sum(2)[..., None]) \
        + torch.matmul(s["page_min"].double(), q.clamp(max=0).sum(2)[..., None])
    page = torch.arange(wide, device=DEVICE)
    there = (page * S < lens[:, None])[:, None]
    scores = score[..., 0].float().masked_fill(~there, -math.inf)
    s["scores"].copy_(scores)
    order = torch.sort(scores, dim=-1, descending=True, stable=True).indices[..., :s["most"]]
    mine = torch.arange(s["most"], device=DEVICE) < s["kept"][:, None, None]
    chosen = torch.sort(torch.where(mine, order, wide), dim=-1).values
    s["sel"].copy_(torch.where(mine, chosen, -1))
    s["count"].copy_(s["kept"])
    at = chosen.clamp(max=wide - 1)
    phys = torch.gather(s["block_table"].long()[:, None].expand(-1, Hkv, -1), 2, at).clamp(min=0)
    tokens = torch.where(mine, (lens.long()[:, None, None] - at * S).clamp(0, S), 0)
    _plain_attention(s, s["query"], phys, tokens)


def run(state):
    s = state
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2509_12211_amd import tinyserve as ts
        if op == "rotate":
            ts.rotate_rows(s["rotary"], s["q"], s["k"], s["q_out"], s["k_out"])
            return s["q_out"], s["k_out"]
        if op in ("append", "step"):
            ts.append_rows(s["layout"], s["k"], s["v"], rotary=s["rotary"], q=s["q"], q_out=s["q_out"],
                           cu_tokens=None if c["new"] == 1 else s["cu"], advance_seq_lens=False)
            if op == "append":
                return s["q_out"], s["k_pool"], s["v_pool"], s["page_min"], s["page_max"]
            last = s["q_out"] if c["new"] == 1 else s["q_out"][s["last"]]
            ts.dense_decode_attention(s["layout_after"], last, s["scale"], s["out"], s["workspace"])
            return s["out"], s["q_out"], s["page_min"], s["page_max"]
        if op == "dense":
            ts.dense_decode_attention(s["layout"], s["query"], s["scale"], s["out"], s["workspace"])
            return s["out"]
        ts.query_aware_decode(s["layout"], s["query"], s["most"], s["most"], s["scale"], s["out"], s["workspace"],
                              topk_per_seq=s["kept"], scores_out=s["scores"], sel_out=s["sel"], sel_count_out=s["count"])
        return s["out"], s["scores"], s["sel"], s["count"]
    if op == "rotate":
        cos, sin = _angles(s["table"], s["positions"], s["axis"])
        for x in ("q", "k"):
            s[x + "_out"].copy_(_rotated(s[x], s[x + "_norm"], cos, sin, c["interleaved"]))
        return s["q_out"], s["k_out"]
    if op in ("append", "step"):
        _plain_append(s)
        if op == "append":
            return s["q_out"], s["k_pool"], s["v_pool"], s["page_min"], s["page_max"]
        _plain_dense(s, s["q_out"][s["last"]], s["lens_after"])
        return s["out"], s["q_out"], s["page_min"], s["page_max"]
    if op == "dense":
        return _plain_dense(s, s["query"], s["lens"])
    _plain_aware(s)
    return s["out"], s["scores"], s["sel"], s["count"]


# -------------------------------------------------------- the definitions, in 64 bits, one by one
def _exact_turn(x, w, table, at, interleaved):
    """One token's rows [H][d] by complex numbers; at: the table's row of every pair."""
    y = x.double()
    if w is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + EPS).sqrt() * w.double()
    half = table.shape[1] // 2
    pair = torch.arange(half, device=x.device)
    turn = torch.complex(table[at, pair].double(), table[at, pair + half].double())
    first = 2 * pair if interleaved else pair
    second = 2 * pair + 1 if interleaved else pair + half
    z = torch.complex(y[..., first], y[..., second]) * turn[..., None, :]
    y = y.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_block(block, S, d):
    """Keys and values [..., S, d] of blocks [..., bytes], by the byte and nibble each lies in."""
    t, ch = torch.meshgrid(torch.arange(S, device=block.device), torch.arange(d, device=block.device), indexing="ij")
    k_at = t * (d // 2) + ch // 2
    v_at = S * d // 2 + ((((t // 8) * (d // 64) + ch // 64) * 16 + ch % 16) * 4 + ch // 16 % 4) * 4 + t % 8 // 2
    sign_of = lambda n: 1.0 - 2.0 * (n // 8)  # noqa: E731
    tokens = torch.arange(S, device=block.device)

    def value(at, odd, scale_at):
        n = (block[..., at].int() >> (4 * odd).int()) & 15
        e, m = (n & 7) // 2, n & 1
        x = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e.double() - 1))
        bits = block[..., scale_at + 2 * tokens].int() | block[..., scale_at + 2 * tokens + 1].int() << 8
        return sign_of(n) * x * (bits << 16).view(torch.float32).double()[..., None]

    return value(k_at, ch % 2, S * d), value(v_at, t % 2, S * d + 2 * S)


def _exact_attention(q, k, v, scale):
    """q [H][d] against k, v [Hkv][n][d]."""
    G = q.shape[0] // k.shape[0]
    w = torch.softmax(torch.matmul(q.double().view(k.shape[0], G, -1), k.transpose(1, 2).contiguous()) * scale, dim=-1)
    return torch.matmul(w, v).reshape(q.shape)


def _exact_cached(s, b, n):
    S, d = s["case"]["S"], s["case"]["d"]
    ids = s["block_table"][b, :-(-n // S)].long()
    k, v = _exact_block(s["pool"][ids], S, d)
    return (x.transpose(0, 1).reshape(x.shape[1], -1, d)[:, :n] for x in (k, v))


def _nearest_fp4(x):
    """A row as its 4-bit numbers: values and nothing else.  Ties go to the code with an even last bit."""
    most = x.abs().amax(-1, keepdim=True)
    up = (torch.ceil((most / 6).float().double() / torch.exp2(torch.floor(torch.log2(most / 6)) - 7)))
    scale = torch.where(most > 0, up * torch.exp2(torch.floor(torch.log2(most / 6)) - 7), 1.0)
    grid = torch.tensor(FP4, dtype=torch.float64, device=x.device)
    r = (x.abs() / scale).clamp(max=6.0)
    above = torch.searchsorted(grid, r.contiguous()).clamp(max=7)
    below = (above - 1).clamp(min=0)
    up_by, down_by = grid[above] - r, r - grid[below]
    pick = torch.where((up_by < down_by) | ((up_by == down_by) & (above % 2 == 0)), above, below)
    return torch.sign(x) * grid[pick] * scale


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, Hq, Hkv, d, S = c["B"], c["Hq"], c["Hkv"], c["d"], c["S"]
    if c["op"] == "rotate":
        at = s["positions"].long()[torch.tensor(s["axis"], device=DEVICE)].t()
        return [_exact_turn(s[x], s[x + "_norm"], s["table"], at, c["interleaved"]) for x in ("q", "k")]
    lens = s["lens"].tolist()
    if c["op"] == "dense":
        return torch.stack([_exact_attention(s["query"][b], *_exact_cached(s, b, n), s["scale"]) for b, n in enumerate(lens)])
    if c["op"] == "aware":
        # its attention goes by the selection, which is whole numbers; scores and the attention have values
        lo, hi, G = s["page_min"].double(), s["page_max"].double(), Hq // Hkv
        score, out = torch.full(s["scores"].shape, -math.inf, dtype=torch.float64, device=DEVICE), []
        for b, n in enumerate(lens):
            pages = -(-n // S)
            q = s["query"][b].double().view(Hkv, G, 1, d)
            for h in range(Hkv):
                score[b, h, :pages] = torch.maximum(q[h] * lo[b, h, :pages], q[h] * hi[b, h, :pages]).sum(dim=(0, 2))
            k, v = _exact_cached(s, b, n)
            rows = []
            for h in range(Hkv):
                best = torch.sort(score[b, h, :pages].float(), descending=True, stable=True).indices[:int(s["kept"][b])]
                pick = (best[:, None] * S + torch.arange(S, device=DEVICE)).view(-1)
                pick = pick[pick < n]
                rows.append(_exact_attention(s["query"][b, h * G:(h + 1) * G], k[h:h + 1, pick], v[h:h + 1, pick], s["scale"]))
            out.append(torch.cat(rows))
        return torch.stack(out), score, None, None
    cu = s["cu"].tolist()
    half = c["rot"] // 2
    q_out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lo, hi = s["page_min"].double(), s["page_max"].double()
    out = []
    pools = [s["k_pool"].double(), s["v_pool"].double()] if c["op"] == "append" else None
    for b, n in enumerate(lens):
        a, z = cu[b], cu[b + 1]
        pos = torch.arange(n, n + z - a, device=DEVICE)
        at = pos[:, None].expand(-1, half)
        q_out[a:z] = _exact_turn(s["q"][a:z], s["q_norm"], s["table"], at, c["interleaved"])
        k = _exact_turn(s["k"][a:z], s["k_norm"], s["table"], at, c["interleaved"])
        v = s["v"][a:z].double()
        if c["op"] == "append":
            ids = s["block_table"][b].long()[pos // S]
            pools[0][ids, :, pos % S] = k
            pools[1][ids, :, :, pos % S] = v
            kept = k
        else:
            # (the cache holds the 4-bit numbers of the rotated keys rounded to bf16)
            kept, v = _nearest_fp4(k.bfloat16().double()), _nearest_fp4(v)
            k0, v0 = _exact_cached(s, b, n) if n else (kept.new_empty(Hkv, 0, d),) * 2
            query = q_out[z - 1].bfloat16()
            out.append(_exact_attention(query, torch.cat([k0, kept.transpose(0, 1)], 1), torch.cat([v0, v.transpose(0, 1)], 1), s["scale"]))
        for j in range(n // S, -(-(n + z - a) // S)):
            mine = kept[max(0, j * S - n):max(0, (j + 1) * S - n)]
            fresh = j * S >= n
            lo[b, :, j] = mine.amin(0) if fresh else torch.minimum(lo[b, :, j], mine.amin(0))
            hi[b, :, j] = mine.amax(0) if fresh else torch.maximum(hi[b, :, j], mine.amax(0))
    if c["op"] == "append":
        return q_out, pools[0], pools[1], lo, hi
    return torch.stack(out), q_out, lo, hi
