"""The 4-bit cache on the GPU against plain 64-bit forms (row_reference.py)."""
import math

import pytest
import torch

import row_reference as ref
from paper_2509_12211_amd import tinyserve as ts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


class Fp4:
    """A 4-bit cache filled by the tests' own quantiser: blocks beyond a sequence's tokens, and slots behind
    its last, hold anything (scales of NaN among it)."""

    def __init__(self, lens, Hq, Hkv, d, S, g, room=0, pad=0, wider=0, out="f32", offset=0.0):
        self.lens_l, self.Hq, self.Hkv, self.d, self.S = lens, Hq, Hkv, d, S
        B = len(lens)
        need = [-(-(n + room) // S) for n in lens]
        self.wide = max(max(need), 1) + wider
        n_phys = sum(need) + 2
        stride = S * (d + 4) + pad
        perm = torch.randperm(n_phys, generator=g)
        table = torch.full((B, self.wide), -1, dtype=torch.int32)
        pool = torch.randint(0, 256, (n_phys, Hkv, stride), generator=g, dtype=torch.uint8)
        pool[:, :, S * d:S * (d + 4)] = 255                        # NaN scales
        self.k, self.v = [], []
        at = 0
        for b, n in enumerate(lens):
            ids = perm[at:at + need[b]]
            table[b, :need[b]] = ids.int()
            at += need[b]
            pages = -(-n // S)
            x = torch.randn((2, Hkv, pages * S, d), generator=g) + offset * torch.randn((2, Hkv, 1, d), generator=g)
            (kc, ks), (vc, vs) = (ref.fp4_quantised(t.to(BF)) for t in x)
            self.k.append((ref.fp4_values(kc) * ks[..., None])[:, :n])
            self.v.append((ref.fp4_values(vc) * vs[..., None])[:, :n])
            behind = torch.arange(pages * S) >= n
            ks[:, behind] = math.nan
            vs[:, behind] = math.nan
            paged = [t.view(Hkv, pages, S, *t.shape[2:]).transpose(0, 1) for t in (kc, ks, vc, vs)]
            if pages:
                pool[ids[:pages]] = ref.fp4_packed(*paged, stride)
        self.pool, self.table = pool.to(DEV), table.to(DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.lo = torch.full((B, Hkv, self.wide, d), 7.0, dtype=BF, device=DEV)
        self.hi = torch.full_like(self.lo, -7.0)
        fmt = ts.TS_OUT_BF16 if out == "bf16" else ts.TS_OUT_F32
        self.layout = ts.make_layout(B, Hq, Hkv, d, S, self.wide, self.pool, None, self.table, self.lens, self.lo, self.hi,
                                     out_format=fmt)
        self.q = torch.randn((B, Hq, d), generator=g).to(BF).to(DEV)
        self.out = torch.full((B, Hq, d), math.nan, dtype=BF if out == "bf16" else torch.float32, device=DEV)
        self.lse = torch.full((B, Hq), math.nan, device=DEV)

    def check(self, out, lse, scale, tokens=None, q=None, what=""):
        """tokens[b][h]: which tokens count (None: all)."""
        q = self.q if q is None else q
        G = self.Hq // self.Hkv
        for b in range(len(self.lens_l)):
            for h in range(self.Hkv):
                pick = slice(None) if tokens is None else tokens[b][h]
                k, v = self.k[b][h:h + 1, pick], self.v[b][h:h + 1, pick]
                heads = slice(h * G, (h + 1) * G)
                want, wlse, bound = ref.attention(q[b, heads].cpu(), k, v, scale)
                got = out[b, heads].cpu()
                if got.dtype == BF:
                    bound = bound + ref.step(BF) * (want.abs() + bound)
                off = (got.double() - want).abs()
                assert (off <= bound).all(), f"{what} sequence {b} head {h}: {(off / bound.clamp(min=1e-300)).max():.3f} of the bound"
                if lse is not None:
                    g_ = lse[b, heads].cpu().double()
                    if k.shape[1] == 0:
                        assert torch.isneginf(g_).all()
                    else:
                        # the logits' bound, sums of n weights, and the logarithm's own last bits
                        tol = 1e-5 + (k.shape[1] + 64) * 2.0 ** -23 + (self.d + 8) * 2.0 ** -24 * abs(scale) * float(
                            torch.matmul(q[b, heads].cpu().double().abs(), k[0].abs().t()).amax())
                        assert ((g_ - wlse).abs() <= tol + 2.0 ** -22 * wlse.abs()).all(), f"{what} lse of {b}, {h}"


SHAPES = [
    # lens, Hq, Hkv, d, S
    ([1], 1, 1, 64, 16), ([33], 16, 1, 128, 8), ([0, 5, 0, 64], 8, 4, 64, 16), ([31, 32, 33], 4, 4, 128, 32),
    ([700, 1, 63], 12, 4, 64, 64), ([2111], 32, 4, 128, 16), ([500, 3000, 20, 1999], 16, 2, 64, 32),
    ([4097, 129], 5, 1, 128, 64), ([16, 8, 1000], 40, 8, 128, 8), ([0, 0], 2, 1, 64, 8),
]


@pytest.mark.parametrize("lens,Hq,Hkv,d,S", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_dense_attention(lens, Hq, Hkv, d, S, out):
    c = Fp4(lens, Hq, Hkv, d, S, torch.Generator().manual_seed(len(lens) + Hq), pad=16, wider=3, out=out, offset=1.0)
    ws = ts.new_dense_workspace(c.layout, DEV)
    scale = 1.0 / math.sqrt(d)
    ts.dense_decode_attention(c.layout, c.q, scale, c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, scale, what="dense")
    # the same again, on the workspace that the call before has left, without the denominators: the same bits
    again = torch.full_like(c.out, math.nan)
    ts.dense_decode_attention(c.layout, c.q, scale, again, ws)
    assert torch.equal(again, c.out)
    assert ts.workspace_status(ws) == 0


@pytest.mark.parametrize("lens,Hq,Hkv,d,S", SHAPES)
def test_sparse_attention_over_lists(lens, Hq, Hkv, d, S):
    """Lists of any length, none and all pages, the partly filled one somewhere in the middle or left out."""
    g = torch.Generator().manual_seed(7 * len(lens) + Hq)
    c = Fp4(lens, Hq, Hkv, d, S, g, wider=1)
    B = len(lens)
    pages = [-(-n // S) for n in lens]
    most = max(max(pages), 1) + 2
    counts = [p if b % 3 == 0 else max(0, p // 2 - (b % 2)) for b, p in enumerate(pages)]
    sel = torch.full((B, Hkv, most), -1, dtype=torch.int32)
    tokens = []
    for b in range(B):
        tokens.append([])
        for h in range(Hkv):
            ids = torch.randperm(pages[b], generator=g)[:counts[b]].sort().values
            sel[b, h, :counts[b]] = ids.int()
            t = (ids[:, None] * S + torch.arange(S)).view(-1)
            tokens[-1].append(t[t < lens[b]])
    ws = ts.new_workspace(c.layout, most, DEV)
    scale = 0.3
    ts.sparse_decode_attention(c.layout, c.q, sel.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV), most, scale,
                               c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, scale, tokens, what="sparse")


@pytest.mark.parametrize("lens,Hq,Hkv,d,S", SHAPES)
def test_boxes_are_rebuilt(lens, Hq, Hkv, d, S):
    c = Fp4(lens, Hq, Hkv, d, S, torch.Generator().manual_seed(3), pad=32, wider=2, offset=1.0)
    ts.build_page_meta(c.layout)
    for b, n in enumerate(lens):
        pages = -(-n // S)
        for j in range(pages):
            k = c.k[b][:, j * S:(j + 1) * S]
            assert torch.equal(c.lo[b, :, j].cpu().double(), ref.outwards(k.amin(1), False))
            assert torch.equal(c.hi[b, :, j].cpu().double(), ref.outwards(k.amax(1), True))
        assert (c.lo[b, :, pages:] == 7.0).all() and (c.hi[b, :, pages:] == -7.0).all()


@pytest.mark.parametrize("lens,Hq,Hkv,d,S", [s for s in SHAPES if max(s[0]) > 1])
@pytest.mark.parametrize("append", [False, True])
def test_query_aware_decode(lens, Hq, Hkv, d, S, append):
    """Scores, selection and attention in one call; with the append, the state that two calls leave."""
    g = torch.Generator().manual_seed(13)
    c = Fp4(lens, Hq, Hkv, d, S, g, room=1, offset=1.0)
    B = len(lens)
    ts.build_page_meta(c.layout)
    k, v = torch.randn((2, B, Hkv, d), generator=g).to(BF).to(DEV).unbind(0)
    most = max(1, c.wide // 3)
    budget = torch.tensor([max(1, most - b) for b in range(B)], dtype=torch.int32, device=DEV)
    ws = ts.new_workspace(c.layout, most, DEV)
    scores = torch.empty((B, Hkv, c.wide), device=DEV)
    sel = torch.empty((B, Hkv, most), dtype=torch.int32, device=DEV)
    count = torch.empty(B, dtype=torch.int32, device=DEV)
    kw = dict(topk_per_seq=budget, scores_out=scores, sel_out=sel, sel_count_out=count)
    scale = 1.0 / math.sqrt(d)
    if append:
        pool, lo, hi, n = c.pool.clone(), c.lo.clone(), c.hi.clone(), c.lens.clone()
        ts.append_and_decode(c.layout, k, v, c.q, most, most, scale, c.out, ws, **kw)
        after = [t.clone() for t in (c.pool, c.lo, c.hi, c.lens)]
        for t, was in zip((c.pool, c.lo, c.hi, c.lens), (pool, lo, hi, n)):
            t.copy_(was)
        ts.append_token_meta(c.layout, k, v)
        assert all(torch.equal(x, y) for x, y in zip(after, (c.pool, c.lo, c.hi, c.lens)))
        assert ts.append_and_decode_launches(c.layout, most) == 5
        for b in range(B):
            for have, x in ((c.k, k), (c.v, v)):
                code, s = ref.fp4_quantised(x[b].cpu())
                have[b] = torch.cat([have[b], (ref.fp4_values(code) * s[..., None])[:, None]], dim=1)
    else:
        ts.query_aware_decode(c.layout, c.q, most, most, scale, c.out, ws, **kw)
    # the same from the calls of each stage
    s2, sel2, count2 = torch.empty_like(scores), torch.empty_like(sel), torch.empty_like(count)
    ts.score_pages(c.layout, c.q, s2)
    ts.select_topk_pages(c.layout, s2, most, most, sel2, count2, topk_per_seq=budget)
    assert torch.equal(scores, s2) and torch.equal(sel, sel2) and torch.equal(count, count2)
    # a page's score is no less than any of its tokens' summed products
    G = Hq // Hkv
    tokens = []
    for b in range(B):
        tokens.append([])
        for h in range(Hkv):
            qk = torch.matmul(c.q[b, h * G:(h + 1) * G].cpu().double(), c.k[b][h].t()).sum(0)
            for j in range(-(-qk.numel() // S)):
                top = qk[j * S:(j + 1) * S].max()
                assert float(scores[b, h, j]) >= top - 1e-5 * abs(top) - 1e-6
            ids = sel[b, h, :int(count[b])].cpu().long()
            t = (ids[:, None] * S + torch.arange(S)).view(-1)
            tokens[-1].append(t[t < c.k[b].shape[1]])
    c.check(c.out, None, scale, tokens, what="aware")
    # without the optional outputs: the same
    again = torch.full_like(c.out, math.nan)
    ts.query_aware_decode(c.layout, c.q, most, most, scale, again, ws, topk_per_seq=budget)
    assert torch.equal(again, c.out)


def test_extreme_logits_and_scales():
    """Logits far apart, one token that outweighs all, scales from the smallest to the largest."""
    d, S = 64, 16
    for mult in (1e-30, 1.0, 3e4):
        c = Fp4([300, 45], 8, 2, d, S, torch.Generator().manual_seed(1))
        x = c.pool.clone()
        sc = x[:, :, S * d:].contiguous().view(BF)
        sc[:, :, :S] = (sc[:, :, :S].float() * mult).to(BF)
        x[:, :, S * d:] = sc.view(torch.uint8).view(*x.shape[:2], -1)
        c.pool.copy_(x)
        for b in range(2):
            n = c.lens_l[b]
            _, ks, _, _ = ref.fp4_unpacked(c.pool[c.table[b, :-(-n // S)].long()].cpu(), S, d)
            kc = ref.fp4_unpacked(c.pool[c.table[b, :-(-n // S)].long()].cpu(), S, d)[0]
            c.k[b] = (ref.fp4_values(kc) * ks[..., None]).transpose(0, 1).reshape(2, -1, d)[:, :n]
        ws = ts.new_dense_workspace(c.layout, DEV)
        ts.dense_decode_attention(c.layout, c.q, 1.0, c.out, ws)
        if mult <= 1.0:
            c.check(c.out, None, 1.0, what=f"scales times {mult}")
        else:       # one token has all the weight
            for b in range(2):
                for h in range(8):
                    best = torch.matmul(c.q[b, h].cpu().double(), c.k[b][h // 4].t()).argmax()
                    want = c.v[b][h // 4, best]
                    assert torch.allclose(c.out[b, h].cpu().double(), want, rtol=2.0 ** -17, atol=1e-30)


def test_pages_without_a_valid_entry_count_as_absent():
    c = Fp4([100, 40], 4, 2, 64, 16, torch.Generator().manual_seed(2))
    c.table[0, 3] = -1
    c.table[1, 0] = 10 ** 7
    tokens = [[torch.cat([torch.arange(48), torch.arange(64, 100)])] * 2, [torch.arange(16, 40)] * 2]
    ws = ts.new_dense_workspace(c.layout, DEV)
    ts.dense_decode_attention(c.layout, c.q, 0.125, c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, 0.125, tokens, what="bad pages")


def test_rows_into_the_cache_and_decode_steps():
    """As a serving engine uses them together: prompts appended with norm and rotation, then steps that
    append a token for each sequence and attend, over all tokens and over selected pages."""
    g = torch.Generator().manual_seed(21)
    B, Hq, Hkv, d, S, wide = 3, 8, 2, 128, 16, 20
    pool = ts.new_fp4_pool(B * wide, Hkv, S, d, DEV)
    table = torch.randperm(B * wide, generator=g).view(B, wide).int().to(DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    lo = torch.zeros((B, Hkv, wide, d), dtype=BF, device=DEV)
    hi = torch.zeros_like(lo)
    lay = ts.make_layout(B, Hq, Hkv, d, S, wide, pool, None, table, lens, lo, hi)
    tab = ts.rotary_table(wide * S, d, device=DEV)
    qn, kn = (1 + 0.1 * torch.randn((2, d), generator=g)).to(DEV).unbind(0)
    rot = ts.make_rotary(tab, q_norm=qn, k_norm=kn)
    eps = float(torch.tensor(1e-6))
    held = [[torch.zeros((Hkv, 0, d), dtype=torch.float64)] * 2 for _ in range(B)]
    dense_ws, ws = ts.new_dense_workspace(lay, DEV), ts.new_workspace(lay, 4, DEV)
    out, scale = torch.empty((B, Hq, d), device=DEV), 1.0 / math.sqrt(d)
    for rnd, counts in enumerate([[130, 1, 47]] + [[1] * B] * 20):
        n = sum(counts)
        qkv = torch.randn((n, Hq + 2 * Hkv, d), generator=g).to(BF).to(DEV)
        q, k, v = qkv.split([Hq, Hkv, Hkv], dim=1)
        before = lens.tolist()
        cu = torch.tensor([0] + counts).cumsum(0).int().to(DEV)
        ts.append_rows(lay, k, v, rotary=rot, q=q, cu_tokens=None if rnd else cu)        # queries in place
        last = q[(cu[1:] - 1).long()].contiguous()
        ts.dense_decode_attention(lay, last, scale, out, dense_ws)
        for b in range(B):
            a, z = int(cu[b]), int(cu[b + 1])
            at = (before[b] + torch.arange(z - a))[:, None].expand(-1, d // 2)
            # (the plain form rotates from the rows as they were; what the cache rounds to bf16 is taken from the
            # library's own rotation of the same rows, tested elsewhere)
            pos = (before[b] + torch.arange(z - a)).int().to(DEV)
            kr = torch.empty((z - a, Hkv, d), dtype=BF, device=DEV)
            ts.rotate_rows(ts.make_rotary(tab, positions=pos, k_norm=kn), None, k[a:z], None, kr)
            exact, slack = ref.rotated(k[a:z].cpu(), kn.cpu(), eps, tab.cpu(), at, False)
            assert ((kr.cpu().double() - exact).abs() <= ref.row_bound(exact, slack, BF)).all()
            for i, x in enumerate((kr, v[a:z])):
                code, s = ref.fp4_quantised(x.cpu())
                held[b][i] = torch.cat([held[b][i], (ref.fp4_values(code) * s[..., None]).transpose(0, 1)], dim=1)
            want, _, bound = ref.attention(last[b].cpu(), held[b][0], held[b][1], scale)
            assert ((out[b].cpu().double() - want).abs() <= bound).all(), f"round {rnd}, sequence {b}"
        sel = torch.empty((B, Hkv, 4), dtype=torch.int32, device=DEV)
        cnt = torch.empty(B, dtype=torch.int32, device=DEV)
        ts.query_aware_decode(lay, last, 4, 4, scale, out, ws, sel_out=sel, sel_count_out=cnt)
        for b in range(B):
            for h in range(Hkv):
                t = (sel[b, h, :int(cnt[b])].cpu().long()[:, None] * S + torch.arange(S)).view(-1)
                t = t[t < held[b][0].shape[1]]
                heads = slice(h * 4, h * 4 + 4)
                want, _, bound = ref.attention(last[b, heads].cpu(), held[b][0][h:h + 1, t], held[b][1][h:h + 1, t], scale)
                assert ((out[b, heads].cpu().double() - want).abs() <= bound).all(), f"round {rnd}, pages of {b}, {h}"


def test_long_sequences_shared_by_many_workgroups():
    """Several workgroups to a unit, units that end inside a workgroup's share, one very long sequence."""
    for lens, Hq, Hkv, d, S in (([40000, 7, 9000, 0, 333], 8, 2, 64, 16), ([100, 70000], 4, 1, 128, 32)):
        g = torch.Generator().manual_seed(4)
        c = Fp4(lens, Hq, Hkv, d, S, g)
        ws = ts.new_dense_workspace(c.layout, DEV)
        scale = 1.0 / math.sqrt(d)
        first = None
        for _ in range(3):
            ts.dense_decode_attention(c.layout, c.q, scale, c.out, ws, lse_out=c.lse)
            assert first is None or torch.equal(first, c.out)        # the order of arrival changes nothing
            first = c.out.clone()
        c.check(c.out, c.lse, scale, what="long")


def test_batches_of_several_shapes_take_turns_on_one_workspace():
    """Counts and partial results of one batch never stand where another's counts do."""
    g = torch.Generator().manual_seed(8)
    batches = [Fp4([9000, 40], 8, 2, 64, 16, g), Fp4([700] * 40, 4, 4, 128, 32, g), Fp4([30] * 300, 2, 2, 64, 8, g),
               Fp4([20000], 16, 1, 128, 64, g)]
    size = max(ts.new_dense_workspace(c.layout, DEV).numel() for c in batches)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    ts.workspace_init(ws)
    for rnd in range(2):
        for c in batches + batches[::-1]:
            c.out.fill_(math.nan)
            ts.dense_decode_attention(c.layout, c.q, 0.125, c.out, ws, lse_out=c.lse)
            if rnd == 0:
                c.first = c.out.clone()
            assert torch.equal(c.first, c.out)
    for c in batches:
        c.check(c.out, c.lse, 0.125, what="turns")


@pytest.mark.parametrize("B,lens,Hq,Hkv,d", [(70, (1, 90), 4, 2, 64), (100, (1, 2500), 16, 8, 128), (130, (0, 40), 32, 8, 64),
                                             (3, (6000, 9000), 64, 64, 64)])
def test_many_units(B, lens, Hq, Hkv, d):
    """More sequences than a wave has lanes, more units than workgroups at once, whole units and shares."""
    g = torch.Generator().manual_seed(B)
    n = torch.randint(lens[0], lens[1] + 1, (B,), generator=g).tolist()
    c = Fp4(n, Hq, Hkv, d, 16, g)
    ws = ts.new_dense_workspace(c.layout, DEV)
    ts.dense_decode_attention(c.layout, c.q, 0.2, c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, 0.2, what="many")


@pytest.mark.parametrize("B,top,Hq,Hkv,d,S,out", [
    (103, 1024, 5, 5, 64, 16, "f32"), (111, 300, 14, 7, 128, 8, "bf16"), (111, 90, 70, 7, 128, 32, "f32"),
    (33, 200, 40, 40, 64, 64, "bf16"), (103, 31, 80, 5, 64, 8, "f32"), (111, 1024, 7, 7, 128, 64, "f32"),
    (111, 190, 7, 7, 128, 8, "f32"), (111, 192, 112, 7, 128, 16, "bf16"), (410, 1024, 10, 10, 64, 8, "f32"),
])
def test_more_short_units_than_workgroups(B, top, Hq, Hkv, d, S, out):
    """Every length from none to as many tokens as a wave takes by itself (and more), whole caches and lists of pages."""
    g = torch.Generator().manual_seed(B + top)
    n = (torch.randint(0, top + 1, (B,), generator=g) // (8 if B > 200 else 1)).tolist()
    n[3], n[B // 2], n[B - 1], n[7], n[8] = 0, top, top, 1, 32
    c = Fp4(n, Hq, Hkv, d, S, g, pad=16, out=out, offset=0.5)
    scale = 1.0 / math.sqrt(d)
    ws = ts.new_dense_workspace(c.layout, DEV)
    ts.dense_decode_attention(c.layout, c.q, scale, c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, scale, what="short")
    again = torch.full_like(c.out, math.nan)
    ts.dense_decode_attention(c.layout, c.q, scale, again, ws)
    assert torch.equal(again, c.out)
    # every other page, and of some sequences none
    pages = [-(-x // S) for x in n]
    most = max(-(-x // 2) for x in pages)
    sel = torch.full((B, Hkv, most), -1, dtype=torch.int32)
    counts = [0 if b % 9 == 4 else x // 2 for b, x in enumerate(pages)]
    tokens = [[torch.zeros(0, dtype=torch.long)] * Hkv for _ in n]
    for b, k in enumerate(counts):
        for h in range(Hkv):
            ids = 2 * torch.arange(k) + (h & 1)
            sel[b, h, :k] = ids.int()
            at = (ids[:, None] * S + torch.arange(S)).view(-1)
            tokens[b][h] = at[at < n[b]]
    c.out.fill_(math.nan)
    c.lse.fill_(math.nan)
    ws = ts.new_workspace(c.layout, most, DEV)
    ts.sparse_decode_attention(c.layout, c.q, sel.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV), most, scale,
                               c.out, ws, lse_out=c.lse)
    c.check(c.out, c.lse, scale, tokens=tokens, what="lists")


def test_equal_shares_of_more_long_units_than_workgroups():
    """800 units of some 190 fragments: workgroups that reach over several units' ends.  The sequences'
    tables are permutations of the same pages, so that the cache and its plain form stay small."""
    g = torch.Generator().manual_seed(12)
    B, Hq, Hkv, d, S, pages = 100, 16, 8, 64, 16, 400
    one = Fp4([pages * S], Hq, Hkv, d, S, g)
    perm = torch.stack([torch.randperm(pages, generator=g) for _ in range(B)])
    table = one.table.cpu()[0].long()[perm].int().to(DEV)
    n = torch.randint(5900, pages * S + 1, (B,), generator=g).int()
    n[1], n[50] = 0, 1
    lens = n.to(DEV)
    box = torch.zeros((B, Hkv, pages, d), dtype=BF, device=DEV)
    lay = ts.make_layout(B, Hq, Hkv, d, S, pages, one.pool, None, table, lens, box, box)
    q = torch.randn((B, Hq, d), generator=g).to(BF).to(DEV)
    out = torch.full((B, Hq, d), math.nan, device=DEV)
    ws = ts.new_dense_workspace(lay, DEV)
    ts.dense_decode_attention(lay, q, 0.125, out, ws)
    assert torch.isfinite(out).all() and (out[1] == 0).all()
    for b in (0, 1, 2, 33, 50, 51, 98, 99):
        at = (perm[b][:, None] * S + torch.arange(S)).view(-1)[:int(n[b])]
        want, _, bound = ref.attention(q[b].cpu(), one.k[0][:, at], one.v[0][:, at], 0.125)
        assert ((out[b].cpu().double() - want).abs() <= bound).all(), b
    again = torch.full_like(out, math.nan)
    ts.dense_decode_attention(lay, q, 0.125, again, ws)
    assert torch.equal(again, out)


def test_what_is_not_a_number_stays_with_its_head():
    c = Fp4([3000, 17], 8, 2, 64, 16, torch.Generator().manual_seed(9))
    ws = ts.new_dense_workspace(c.layout, DEV)
    clean = torch.empty_like(c.out)
    ts.dense_decode_attention(c.layout, c.q, 0.125, clean, ws)
    c.q[0, 5, 3] = math.nan
    c.q[1, 0, :] = math.nan
    ts.dense_decode_attention(c.layout, c.q, 0.125, c.out, ws)
    bad = torch.zeros(c.out.shape[:2], dtype=torch.bool)
    bad[0, 5] = bad[1, 0] = True
    assert c.out.cpu()[bad].isnan().all() and torch.equal(c.out.cpu()[~bad], clean.cpu()[~bad])


def test_captured_attention_is_replayed():
    c = Fp4([5000, 100, 1], 8, 2, 64, 16, torch.Generator().manual_seed(6))
    scale = 0.125
    ws, ws2 = ts.new_dense_workspace(c.layout, DEV), ts.new_dense_workspace(c.layout, DEV)
    want = torch.empty_like(c.out)
    ts.dense_decode_attention(c.layout, c.q, scale, want, ws2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ts.dense_decode_attention(c.layout, c.q, scale, c.out, ws)
    for i in range(5):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(i)).to(BF))
        graph.replay()
        ts.dense_decode_attention(c.layout, c.q, scale, want, ws2)
        torch.cuda.synchronize()
        assert torch.equal(c.out, want), i
