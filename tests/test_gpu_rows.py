"""ts_rotate_rows and ts_append_rows on the GPU against plain 64-bit forms (row_reference.py)."""
import math

import pytest
import torch

import row_reference as ref
from paper_2509_12211_amd import tinyserve as ts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = float(torch.tensor(1e-6, dtype=torch.float32))
BF, HF = torch.bfloat16, torch.float16


def rows_of(n, heads, d, dtype, g, fused=False):
    if fused:
        return list(torch.randn((n, sum(heads), d), generator=g).to(dtype).to(DEV).split(heads, dim=1))
    return [torch.randn((n, h, d), generator=g).to(dtype).to(DEV) for h in heads]


def gains(d, g):
    return (1.0 + 0.2 * torch.randn((2, d), generator=g)).to(DEV).unbind(0)


def assert_rows(got, x, norm, table, at, interleaved, what):
    exact, slack = ref.rotated(x.cpu(), None if norm is None else norm.cpu(), EPS, None if table is None else table.cpu(),
                               at, interleaved)
    bound = ref.row_bound(exact, slack, got.dtype)
    off = (got.cpu().double() - exact).abs()
    assert (off <= bound).all(), f"{what}: {(off / bound).max():.3f} of the bound"


@pytest.mark.parametrize("n,Hq,Hkv,d,dtype,rot,interleaved,norm,fused", [
    (1, 32, 4, 64, BF, 64, False, True, False),
    (1, 1, 1, 128, HF, 128, True, False, False),
    (7, 8, 8, 64, BF, 32, True, True, True),
    (33, 12, 4, 128, BF, 96, False, True, True),
    (129, 5, 1, 64, HF, 24, False, False, False),
    (257, 40, 8, 128, HF, 8, True, True, True),
    (1000, 16, 2, 64, BF, 64, False, False, True),
    (600, 64, 8, 128, BF, 128, False, True, False),
])
def test_rows_match_the_formula(n, Hq, Hkv, d, dtype, rot, interleaved, norm, fused):
    g = torch.Generator().manual_seed(n + d)
    q, k, _ = rows_of(n, [Hq, Hkv, Hkv], d, dtype, g, fused)
    table = ts.rotary_table(5000, rot, device=DEV)
    pos = torch.randint(0, 5000, (n,), generator=g, dtype=torch.int32)
    qn, kn = gains(d, g) if norm else (None, None)
    r = ts.make_rotary(table, positions=pos.to(DEV), interleaved=interleaved, q_norm=qn, k_norm=kn, norm_eps=EPS)
    qo, ko = torch.full_like(q, math.nan), torch.full((n + 1, Hkv, d), 7.0, dtype=dtype, device=DEV)
    ts.rotate_rows(r, q, k, qo, ko[:n])
    at = pos.long()[:, None].expand(-1, rot // 2)
    assert_rows(qo, q, qn, table, at, interleaved, "q")
    assert_rows(ko[:n], k, kn, table, at, interleaved, "k")
    assert (ko[n] == 7.0).all(), "a row behind the last was written"
    # one of the two alone, and in place: the same bits
    alone = q.clone(memory_format=torch.preserve_format)
    ts.rotate_rows(r, alone, None)
    assert torch.equal(alone, qo)
    inplace = torch.cat([q, k], dim=1)
    ts.rotate_rows(r, inplace[:, :Hq], inplace[:, Hq:])
    assert torch.equal(inplace, torch.cat([qo, ko[:n]], dim=1))


@pytest.mark.parametrize("axes,rot,interleaved", [(2, 64, False), (3, 96, True), (3, 128, False), (4, 128, True)])
def test_each_pair_turns_by_its_own_axis(axes, rot, interleaved):
    n, d = 150, 128
    g = torch.Generator().manual_seed(axes)
    q, k, _ = rows_of(n, [6, 2, 2], d, BF, g)
    table = ts.rotary_table(300, rot, device=DEV)
    pos = torch.randint(0, 300, (axes, n), generator=g, dtype=torch.int32)
    axis = torch.randint(0, axes, (rot // 2,), generator=g)
    r = ts.make_rotary(table, positions=pos.to(DEV), interleaved=interleaved, axis_of_pair=axis.tolist())
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ts.rotate_rows(r, q, k, qo, ko)
    at = pos.long()[axis].t()
    assert_rows(qo, q, None, table, at, interleaved, "q")
    assert_rows(ko, k, None, table, at, interleaved, "k")


def test_rows_at_the_edges_of_their_type():
    """Zero rows, the largest and the smallest numbers, positions at and outside the table's ends."""
    d = 64
    big, small = torch.finfo(BF).max, torch.finfo(BF).smallest_normal
    x = torch.zeros((5, 1, d), dtype=BF, device=DEV)
    x[1] = small
    x[2] = 1e18
    x[3, 0, ::2] = big / 4
    x[4, 0, 5] = -3.0
    table = ts.rotary_table(50, d, device=DEV)
    w = torch.ones(d, device=DEV)
    pos = torch.tensor([0, 49, 50, -3, 2 ** 31 - 1], dtype=torch.int32)
    out = torch.empty_like(x)
    ts.rotate_rows(ts.make_rotary(table, positions=pos.to(DEV), q_norm=w, norm_eps=EPS), x, None, out)
    at = pos.long().clamp(0, 49)[:, None].expand(-1, d // 2)
    assert_rows(out, x, w, table, at, False, "edges")
    assert (out[0] == 0).all()
    # neither norm nor rotation: the same bits, NaN among them
    x[1, 0, 3] = math.nan
    ts.rotate_rows(ts.make_rotary(), x, None, out)
    assert torch.equal(out.view(torch.int16), x.view(torch.int16))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_hold_infinities_and_what_is_not_a_number(d, dtype):
    """By the formula: an infinity's row is zero but for the infinity itself, 0 / 0 and NaN go where they go."""
    x = torch.randn((4, 2, d), generator=torch.Generator().manual_seed(d)).to(dtype)
    x[0, 0, 9] = math.inf
    x[1, 1, 2], x[1, 1, 40] = -math.inf, math.inf
    x[2, 0, 5] = math.nan
    x[3, 0] = 0
    for table in (None, ts.rotary_table(10, 32, device=DEV)):
        pos = torch.tensor([3, 0, 9, 4], dtype=torch.int32)
        w, out = torch.ones(d, device=DEV), torch.empty((4, 2, d), dtype=dtype, device=DEV)
        r = ts.make_rotary(table, positions=None if table is None else pos.to(DEV), q_norm=w, norm_eps=0.0)
        ts.rotate_rows(r, x.to(DEV), None, out)
        exact, slack = ref.rotated(x, w.cpu(), 0.0, None if table is None else table.cpu(),
                                   pos.long()[:, None].expand(-1, 16), False)
        got = out.cpu().double()
        assert torch.equal(got.isnan(), exact.isnan())
        on = ~exact.isnan()
        assert ((got - exact).abs() <= ref.row_bound(exact, slack, dtype))[on].all()


# ------------------------------------------------------------------------------------------- append
class Cache:
    """A paged cache of any format with its boxes, what it holds, and room for more."""

    def __init__(self, fmt, B, Hkv, d, S, wide, g, Hq=None, stride_pad=0):
        self.fmt, self.B, self.Hkv, self.d, self.S, self.wide = fmt, B, Hkv, d, S, wide
        n = B * wide + 3
        self.dtype = HF if fmt == "fp16" else BF
        self.v_pool = self.ks = self.vs = None
        if fmt == "fp4":
            self.k_pool = torch.randint(0, 256, (n, Hkv, S * (d + 4) + stride_pad), generator=g, dtype=torch.uint8).to(DEV)
        elif fmt == "int8":
            kv = torch.randint(-127, 128, (n, Hkv, 2, S * d), generator=g, dtype=torch.int8).to(DEV)
            self.k_pool, self.v_pool = kv[:, :, 0].view(n, Hkv, S, d), kv[:, :, 1].view(n, Hkv, d, S)
            self.ks = torch.full((n, Hkv, S), math.nan, device=DEV)
            self.vs = torch.full((n, Hkv, S), math.nan, device=DEV)
        else:
            kv = torch.full((n, Hkv, 2, S * d), math.nan, dtype=self.dtype, device=DEV)
            self.k_pool, self.v_pool = kv[:, :, 0].view(n, Hkv, S, d), kv[:, :, 1].view(n, Hkv, d, S)
        self.table = torch.randperm(n, generator=g)[:B * wide].view(B, wide).int().to(DEV)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.lo = torch.full((B, Hkv, wide, d), 7.0, dtype=self.dtype, device=DEV)
        self.hi = torch.full_like(self.lo, -7.0)
        self.layout = ts.make_layout(B, Hq or 2 * Hkv, Hkv, d, S, wide, self.k_pool, self.v_pool, self.table, self.lens,
                                     self.lo, self.hi, k_scale=self.ks, v_scale=self.vs)

    def state(self):
        """Everything a call may change, as bytes."""
        return [None if t is None else t.clone() for t in (self.k_pool, self.v_pool, self.ks, self.vs, self.lo, self.hi, self.lens)]

    def held(self, b, n):
        """Keys and values of the first n tokens of sequence b as fp64 [Hkv][n][d] (and their raw codes)."""
        pages = -(-n // self.S)
        at = self.table[b, :pages].long()
        if self.fmt == "fp4":
            kc, ks, vc, vs = ref.fp4_unpacked(self.k_pool[at].cpu(), self.S, self.d)
            k, v = (ref.fp4_values(c) * s[..., None] for c, s in ((kc, ks), (vc, vs)))
        else:
            k, v = self.k_pool[at].cpu().double(), self.v_pool[at].cpu().double().transpose(2, 3)
            if self.fmt == "int8":
                k, v = k * self.ks[at].cpu().double()[..., None], v * self.vs[at].cpu().double()[..., None]
        return (x.transpose(0, 1).reshape(self.Hkv, -1, self.d)[:, :n] for x in (k, v))


def stored(x, fmt):
    """What a cache of this format holds of 16-bit rows [n][Hkv][d]: fp64 values."""
    if fmt == "fp4":
        c, s = ref.fp4_quantised(x)
        return ref.fp4_values(c) * s[..., None]
    if fmt == "int8":
        c, s = ref.int8_quantised(x)
        return c.double() * s[..., None]
    return x.double()


def assert_cache(c, tokens, what):
    """tokens: for each sequence (keys, values) [n][Hkv][d] as rows; the cache and its boxes hold just these."""
    for b, (k, v) in enumerate(tokens):
        n = k.shape[0]
        if n == 0:
            continue
        gk, gv = c.held(b, n)
        wk, wv = (stored(x, c.fmt).transpose(0, 1) for x in (k, v))
        assert torch.equal(gk, wk), f"{what}: keys of sequence {b}"
        assert torch.equal(gv, wv), f"{what}: values of sequence {b}"
        for j in range(-(-n // c.S)):
            page = wk[:, j * c.S:(j + 1) * c.S]
            lo, hi = page.amin(1), page.amax(1)
            if c.fmt in ("fp4", "int8"):
                lo, hi = ref.outwards(lo, False), ref.outwards(hi, True)
            assert torch.equal(c.lo[b, :, j].cpu().double(), lo), f"{what}: lower box {b}, {j}"
            assert torch.equal(c.hi[b, :, j].cpu().double(), hi), f"{what}: upper box {b}, {j}"
        assert (c.lo[b, :, -(-n // c.S):] == 7.0).all() and (c.hi[b, :, -(-n // c.S):] == -7.0).all(), f"{what}: boxes behind {b}"


FORMATS = [("bf16", 4), ("bf16", 16), ("fp16", 8), ("fp16", 64), ("int8", 4), ("int8", 16), ("int8", 64), ("fp4", 8),
           ("fp4", 16), ("fp4", 32), ("fp4", 64)]


@pytest.mark.parametrize("fmt,S", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_ragged_appends_in_several_rounds(fmt, S, d):
    """Prompts of any length, none and one among them, then more of them behind: rows, slots, boxes, lengths."""
    g = torch.Generator().manual_seed(S + d)
    B, Hq, Hkv, wide = 5, 6, 2, 12 if S <= 16 else 4
    c = Cache(fmt, B, Hkv, d, S, wide, g, Hq, stride_pad=48)
    cap = wide * S
    table = ts.rotary_table(cap, d, device=DEV)
    qn, kn = gains(d, g)
    r = ts.make_rotary(table, q_norm=qn, k_norm=kn, norm_eps=EPS)
    held = [[torch.zeros((0, Hkv, d), dtype=c.dtype)] * 2 for _ in range(B)]
    for rnd, counts in enumerate([[S + 1, 0, 1, 2 * S, S - 1], [1, 1, 1, 1, 1], [0, 2, S + 3, 1, 2 * S + 5 if S < 64 else 30]]):
        n, extra = sum(counts), 2
        q, k, v = rows_of(n + extra, [Hq, Hkv, Hkv], d, c.dtype, g, fused=rnd != 1)
        before = c.lens.cpu()
        cu = torch.tensor([0] + counts).cumsum(0).int().to(DEV)
        qo = torch.full((n + extra, Hq, d), 3.0, dtype=c.dtype, device=DEV)
        ts.append_rows(c.layout, k, v, rotary=r, q=q, q_out=qo, cu_tokens=cu)
        # the rows themselves: the same bits as the rotation alone gives
        pos = torch.cat([int(before[b]) + torch.arange(m) for b, m in enumerate(counts)]).int()
        alone = ts.make_rotary(table, positions=pos.to(DEV), q_norm=qn, k_norm=kn, norm_eps=EPS)
        wq, wk = torch.empty((n, Hq, d), dtype=c.dtype, device=DEV), torch.empty((n, Hkv, d), dtype=c.dtype, device=DEV)
        ts.rotate_rows(alone, q[:n], k[:n], wq, wk)
        assert torch.equal(qo[:n], wq), f"round {rnd}: queries"
        assert (qo[n:] == 3.0).all(), f"round {rnd}: rows behind the last sequence"
        assert c.lens.cpu().tolist() == [int(a) + m for a, m in zip(before, counts)]
        for b in range(B):
            a, z = int(cu[b]), int(cu[b + 1])
            held[b] = [torch.cat([held[b][0], wk[a:z].cpu()]), torch.cat([held[b][1], v[a:z].cpu()])]
        assert_cache(c, held, f"round {rnd}")


@pytest.mark.parametrize("fmt,S", [("bf16", 16), ("fp16", 32), ("int8", 16), ("fp4", 16)])
def test_one_token_each_without_offsets(fmt, S):
    """The decode form, all three ways of counting lengths, against the form with offsets."""
    g = torch.Generator().manual_seed(S)
    B, Hq, Hkv, d, wide = 70, 8, 2, 64, 3
    caches = [Cache(fmt, B, Hkv, d, S, wide, torch.Generator().manual_seed(1), Hq) for _ in range(4)]
    start = torch.randint(0, 2 * S, (B,), generator=g).int()
    start[:3] = torch.tensor([0, S - 1, S])
    q, k, v = rows_of(B, [Hq, Hkv, Hkv], d, caches[0].dtype, g, fused=True)
    prompt = rows_of(int(start.sum()), [Hkv, Hkv], d, caches[0].dtype, g)
    cu0 = torch.cat([torch.zeros(1), start.cumsum(0)]).int().to(DEV)
    r = ts.make_rotary(ts.rotary_table(wide * S, d, device=DEV))
    outs = []
    for i, c in enumerate(caches):
        ts.append_rows(c.layout, prompt[0], prompt[1], rotary=r, cu_tokens=cu0)
        assert torch.equal(c.lens.cpu(), start)
        qo = torch.empty_like(q)
        one = torch.arange(B + 1, dtype=torch.int32, device=DEV)
        if i == 2:
            c.lens += 1
        ts.append_rows(c.layout, k, v, rotary=r, q=q, q_out=qo, cu_tokens=one if i == 3 else None,
                       advance_seq_lens=i != 1, lens_include_new=i == 2)
        assert torch.equal(c.lens.cpu(), start + (i != 1))
        c.lens.copy_(start)
        outs.append([qo] + c.state())
    for other in outs[1:]:
        for x, y in zip(outs[0], other):
            assert (x is None and y is None) or torch.equal(x.nan_to_num(9.0) if x.is_floating_point() else x,
                                                            y.nan_to_num(9.0) if y.is_floating_point() else y)


@pytest.mark.parametrize("fmt,S", [("bf16", 16), ("int8", 8), ("fp4", 32)])
def test_lengths_that_count_the_new_tokens_already(fmt, S):
    """Ragged appends with the lengths before and after give the same cache; positions by several axes."""
    g = torch.Generator().manual_seed(S)
    B, Hq, Hkv, d, wide = 3, 2, 1, 64, 5
    before, after = (Cache(fmt, B, Hkv, d, S, wide, torch.Generator().manual_seed(4), Hq) for _ in range(2))
    table = ts.rotary_table(40, d, device=DEV)
    axis = [i % 3 for i in range(d // 2)]
    outs = {}
    for counts in ([S + 3, 1, 0], [2, S, 2 * S + 1]):
        n = sum(counts)
        q, k, v = rows_of(n, [Hq, Hkv, Hkv], d, before.dtype, g, fused=True)
        pos = torch.randint(0, 40, (3, n), generator=g, dtype=torch.int32).to(DEV)
        r = ts.make_rotary(table, positions=pos, interleaved=True, axis_of_pair=axis)
        cu = torch.tensor([0] + counts).cumsum(0).int().to(DEV)
        for c in (before, after):
            if c is after:
                c.lens += cu[1:] - cu[:-1]
            outs[c] = torch.empty_like(q)
            ts.append_rows(c.layout, k, v, rotary=r, q=q, q_out=outs[c], cu_tokens=cu, lens_include_new=c is after)
        wq = torch.empty_like(q)
        ts.rotate_rows(r, q, None, wq)
        assert torch.equal(outs[before], wq) and torch.equal(outs[after], wq)
        for x, y in zip(before.state(), after.state()):
            assert (x is None and y is None) or torch.equal(x.nan_to_num(9.0) if x.is_floating_point() else x,
                                                            y.nan_to_num(9.0) if y.is_floating_point() else y)


@pytest.mark.parametrize("fmt,S", FORMATS)
def test_boxes_and_slots_as_token_by_token(fmt, S):
    """Without rotation: the same cache as ts_append_token_meta leaves, called once for each token."""
    g = torch.Generator().manual_seed(S)
    B, Hkv, d, wide, n = 3, 2, 128, 3, 2 * S + 3
    one, all_ = (Cache(fmt, B, Hkv, d, S, wide, torch.Generator().manual_seed(2)) for _ in range(2))
    k, v = rows_of(B * n, [Hkv, Hkv], d, one.dtype, g)
    k, v = k.view(B, n, Hkv, d), v.view(B, n, Hkv, d)
    for t in range(n):
        ts.append_token_meta(one.layout, k[:, t].contiguous(), v[:, t].contiguous())
    cu = (torch.arange(B + 1) * n).int().to(DEV)
    ts.append_rows(all_.layout, k.view(B * n, Hkv, d), v.view(B * n, Hkv, d), cu_tokens=cu)
    for x, y in zip(one.state(), all_.state()):
        assert (x is None and y is None) or torch.equal(x.nan_to_num(9.0) if x.is_floating_point() else x,
                                                        y.nan_to_num(9.0) if y.is_floating_point() else y)
    if fmt != "fp4":
        return
    # boxes alone (no values): widened by the key as it would be stored
    boxes = Cache(fmt, B, Hkv, d, S, wide, torch.Generator().manual_seed(2))
    pool = boxes.k_pool.clone()
    for t in range(n):
        ts.append_token_meta(boxes.layout, k[:, t].contiguous())
    assert torch.equal(boxes.lo, one.lo) and torch.equal(boxes.hi, one.hi) and torch.equal(boxes.lens, one.lens)
    assert torch.equal(boxes.k_pool, pool)


@pytest.mark.parametrize("fmt", ["bf16", "int8", "fp4"])
def test_sequences_that_do_not_fit_and_bad_pages(fmt):
    """A sequence without room stays as it is, a page without an entry is left out, the others go on."""
    g = torch.Generator().manual_seed(5)
    B, Hq, Hkv, d, S, wide = 4, 4, 2, 64, 16, 2
    c = Cache(fmt, B, Hkv, d, S, wide, g, Hq)
    c.table[2, 1] = -1
    c.table[3, 0] = 10 ** 6
    counts = [2 * S + 1, 2 * S, 2 * S, 5]
    n = sum(counts)
    q, k, v = rows_of(n, [Hq, Hkv, Hkv], d, c.dtype, g)
    cu = torch.tensor([0] + counts).cumsum(0).int().to(DEV)
    before = c.state()
    qo = torch.full_like(q, math.nan)
    ts.append_rows(c.layout, k, v, q=q, q_out=qo, cu_tokens=cu)
    assert torch.equal(qo, q)                                  # neither norm nor rotation: copied
    assert c.lens.cpu().tolist() == [0, 2 * S, 2 * S, 5]
    after = c.state()
    bits = lambda t: t.contiguous().view(torch.uint8).view(*t.shape, -1)  # noqa: E731
    touched = torch.zeros(c.k_pool.shape[0], dtype=torch.bool)
    touched[torch.stack([c.table[1, 0], c.table[1, 1], c.table[2, 0]]).long().cpu()] = True
    for x, y in zip(before[:4], after[:4]):
        if x is not None:
            same = (bits(x) == bits(y)).flatten(1).all(1).cpu()
            assert same[~touched].all() and not same[touched].any()
    assert (c.lo[0] == 7.0).all() and (c.lo[2, :, 1] == 7.0).all() and (c.lo[3] == 7.0).all()
    assert_cache_pages = [(1, 2 * S), (2, S)]
    for b, m in assert_cache_pages:
        a = int(cu[b])
        gk, gv = c.held(b, m)
        assert torch.equal(gk, stored(k[a:a + m].cpu(), fmt).transpose(0, 1))
        assert torch.equal(gv, stored(v[a:a + m].cpu(), fmt).transpose(0, 1))


@pytest.mark.parametrize("one_each", [False, True])
def test_four_bit_numbers_at_their_borders(one_each):
    """Rows whose numbers lie on the borders between codes, just beside them, and on either side of zero, at
    scales from the smallest to the largest; a row of infinities and NaN."""
    d, S, wide = 64, 8, 9
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = []
    for scale in (1.0, 1.5, 2.0 ** -100, 3 * 2.0 ** -120, 1.25 * 2.0 ** 90, 2.0 ** 125, 2.0 ** -133):
        x = torch.cat([border, -border, torch.tensor([6.0, -6.0, 0.0, -0.0])]).double() * scale
        up, down = (x.to(BF).view(torch.int16) + 1).view(BF), (x.to(BF).view(torch.int16) - 1).view(BF)
        row = torch.cat([x.to(BF), up[:14], down[:14], torch.zeros(18).to(BF)])
        rows.append(torch.where(row.abs().double() <= 6 * scale, row, torch.zeros_like(row)))
    k = torch.stack(rows)[:, None].contiguous()
    B, n = (k.shape[0], 1) if one_each else (1, k.shape[0])
    v = (k * 1).flip(-1).contiguous()
    c = Cache("fp4", B, 1, d, S, wide, torch.Generator().manual_seed(1))
    cu = None if one_each else torch.tensor([0, n], dtype=torch.int32, device=DEV)
    ts.append_rows(c.layout, k.to(DEV), v.to(DEV), cu_tokens=cu)
    held = [[k[b:b + 1], v[b:b + 1]] for b in range(B)] if one_each else [[k, v]]
    assert_cache(c, held, "borders")
    # not finite: the largest number of the row's scale, and zero
    x = torch.zeros((B if one_each else 1, 1, d), dtype=BF)
    x[..., 0], x[..., 1], x[..., 2], x[..., 3] = math.inf, -math.inf, math.nan, 1.0
    c.lens.zero_()
    ts.append_rows(c.layout, x.to(DEV), x.to(DEV), cu_tokens=None if one_each else torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    for held in c.held(0, 1):
        assert torch.isfinite(held).all() and held[0, 0, 0] == -held[0, 0, 1] > 3e38 and (held[0, 0, 2:] == 0).all()


def test_many_sequences_of_few_tokens():
    """More sequences than a wave has lanes, most of them without a new token."""
    g = torch.Generator().manual_seed(9)
    B, Hkv, d, S, wide = 200, 1, 64, 16, 4
    c = Cache("bf16", B, Hkv, d, S, wide, g)
    held = [[torch.zeros((0, Hkv, d), dtype=BF)] * 2 for _ in range(B)]
    for _ in range(3):
        counts = torch.randint(0, 20, (B,), generator=g) * (torch.rand(B, generator=g) < 0.3)
        n = int(counts.sum())
        k, v = rows_of(n, [Hkv, Hkv], d, BF, g)
        cu = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).int().to(DEV)
        ts.append_rows(c.layout, k, v, cu_tokens=cu)
        for b in range(B):
            a, z = int(cu[b]), int(cu[b + 1])
            held[b] = [torch.cat([held[b][i], x[a:z].cpu()]) for i, x in enumerate((k, v))]
    assert_cache(c, held, "few tokens")


def test_more_pages_than_one_side_of_a_grid_holds():
    """40000 sequences of three tokens that get none, one or two: half of them reach into a second page."""
    g = torch.Generator().manual_seed(40)
    B, S, d = 40000, 4, 64
    n = torch.randint(0, 3, (B,), generator=g)
    cu = torch.zeros(B + 1, dtype=torch.int64)
    cu[1:] = n.cumsum(0)
    T = int(cu[-1])
    table = torch.randperm(2 * B, generator=g).view(B, 2)
    k, v = (torch.randn((T, 1, d), generator=g).to(BF) for _ in range(2))
    kp, vp = (torch.zeros((2 * B, 1, S * d), dtype=BF, device=DEV) for _ in range(2))
    box = [torch.zeros((B, 1, 2, d), dtype=BF, device=DEV) for _ in range(2)]
    lens = torch.full((B,), 3, dtype=torch.int32, device=DEV)
    on_gpu = table.int().to(DEV)       # (held: a layout has addresses)
    lay = ts.make_layout(B, 1, 1, d, S, 2, kp, vp, on_gpu, lens, *box)
    ts.append_rows(lay, k.to(DEV), v.to(DEV), cu_tokens=cu.int().to(DEV))
    seq = torch.repeat_interleave(torch.arange(B), n)
    at = 3 + torch.arange(T) - cu[seq]
    page, slot = table[seq, at // S], at % S
    want_k, want_v = torch.zeros((2 * B, S, d), dtype=BF), torch.zeros((2 * B, d, S), dtype=BF)
    want_k[page, slot], want_v[page, :, slot] = k[:, 0], v[:, 0]
    assert torch.equal(kp.cpu().view(2 * B, S, d), want_k) and torch.equal(vp.cpu().view(2 * B, d, S), want_v)
    assert torch.equal(lens.cpu(), (3 + n).int())
    new = slot == 0                                            # (a page of one token: its box is the token)
    for side in box:
        assert torch.equal(side.cpu()[seq[new], 0, 1], k[new, 0])


def test_appends_on_another_stream_and_captured():
    """A captured append replayed with other rows in the same buffers, eager work between the replays."""
    g = torch.Generator().manual_seed(11)
    B, Hq, Hkv, d, S, wide = 3, 4, 2, 64, 16, 8
    c, e = (Cache("fp4", B, Hkv, d, S, wide, torch.Generator().manual_seed(1), Hq) for _ in range(2))
    r = ts.make_rotary(ts.rotary_table(wide * S, d, device=DEV))
    q, k, v = rows_of(B, [Hq, Hkv, Hkv], d, BF, g)
    qo = torch.empty_like(q)
    ts.append_rows(e.layout, k, v, rotary=r, q=q, q_out=torch.empty_like(q))      # (loads the code)
    e.lens.zero_()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ts.append_rows(c.layout, k, v, rotary=r, q=q, q_out=qo)
    for i in range(2 * S + 3):
        x = [t.to(DEV) for t in (torch.randn((B, h, d), generator=g).to(BF) for h in (Hq, Hkv, Hkv))]
        for dst, src in zip((q, k, v), x):
            dst.copy_(src)
        graph.replay()
        want = torch.empty_like(q)
        with torch.cuda.stream(stream):
            stream.wait_stream(torch.cuda.default_stream())
            ts.append_rows(e.layout, x[1], x[2], rotary=r, q=x[0], q_out=want)
        torch.cuda.synchronize()
        assert torch.equal(qo, want), i
    for b in range(B):
        for x, y in zip(c.held(b, 2 * S + 3), e.held(b, 2 * S + 3)):
            assert torch.equal(x, y)
    assert torch.equal(c.lo, e.lo) and torch.equal(c.hi, e.hi) and torch.equal(c.lens, e.lens)
