"""CPU-only: what ts_rotate_rows, ts_append_rows and the 4-bit cache turn away on the host, the C structs
against their ctypes mirrors, and the plain forms that the GPU tests compare with."""
import ctypes
import os
import subprocess

import pytest
import torch

import row_reference as ref
from paper_2509_12211_amd import tinyserve as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000


def rotary(**kw):
    base = dict(rot_dim=64, interleaved=0, num_axes=1, num_positions=100, cos_sin=P, positions=P, q_norm=P, k_norm=P,
                norm_eps=1e-6)
    axis = kw.pop("axis", None)
    base.update(kw)
    r = ts.TsRotary(**base)
    if axis is not None:
        r.axis_of_pair[:len(axis)] = axis
    return r


def rows(**kw):
    base = dict(num_tokens=2, format=ts.TS_KV_BF16, q=P, k=P, v=P, q_out=P, k_out=P, q_stride=512, k_stride=128,
                v_stride=128, q_out_stride=512, k_out_stride=128)
    base.update(kw)
    return ts.TsRows(**base)


def layout(**kw):
    base = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_pages_per_seq=64,
                num_phys_pages=128, kv_tile_stride=0, k_pool=P, v_pool=P, block_table=P, seq_lens=P, page_min=P,
                page_max=P)
    base.update(kw)
    return ts.TsLayout(**base)


def fp4(**kw):
    return layout(**dict(dict(kv_format=ts.TS_KV_FP4, v_pool=None), **kw))


def rotate(r, w, Hq=8, Hkv=2, d=64):
    return ts.lib().ts_rotate_rows(None if r is None else ctypes.byref(r), None if w is None else bytes(w), Hq, Hkv, d,
                                   None)


def append(lay, r, w, cu=P, lens=0):
    return ts.lib().ts_append_rows(None if lay is None else ctypes.byref(lay), None if r is None else ctypes.byref(r),
                                   None if w is None else bytes(w), cu, lens, None)


@pytest.mark.parametrize("struct,mirror", [("ts_rotary", ts.TsRotary), ("ts_rows", ts.TsRows)])
def test_struct_layouts_match_the_header(tmp_path, struct, mirror):
    fields = [n for n, _ in mirror._fields_]
    src = tmp_path / "lay.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tinyserve.h"\n'
                   f'int main(void) {{\n  printf("%zu", sizeof({struct}));\n'
                   + "".join(f'  printf(" %zu", offsetof({struct}, {n}));\n' for n in fields) + "  return 0;\n}\n")
    exe = tmp_path / "lay"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(mirror)] + [getattr(mirror, n).offset for n in fields]


def test_the_packed_rows_are_the_struct():
    values = list(range(3, 15))
    assert ts._pack_rows(*values) == bytes(ts.TsRows(*values))


BAD_ROTARY = [
    (dict(rot_dim=-8), ts.TS_ERR_SHAPE), (dict(rot_dim=72), ts.TS_ERR_SHAPE), (dict(rot_dim=12), ts.TS_ERR_SHAPE),
    (dict(num_axes=0), ts.TS_ERR_SHAPE), (dict(num_axes=5), ts.TS_ERR_UNSUPPORTED),
    (dict(num_positions=0), ts.TS_ERR_SHAPE), (dict(cos_sin=None), ts.TS_ERR_NULL), (dict(cos_sin=P + 8), ts.TS_ERR_SHAPE),
    (dict(q_norm=P + 4), ts.TS_ERR_SHAPE), (dict(k_norm=P + 8), ts.TS_ERR_SHAPE), (dict(norm_eps=-1e-6), ts.TS_ERR_SHAPE),
    (dict(norm_eps=float("nan")), ts.TS_ERR_SHAPE), (dict(num_axes=3, axis=[0, 1, 3]), ts.TS_ERR_SHAPE),
    (dict(num_axes=2, positions=None), ts.TS_ERR_NULL),
]


@pytest.mark.parametrize("kw,code", BAD_ROTARY)
def test_a_rotary_out_of_range_is_refused(kw, code):
    assert rotate(rotary(**kw), rows()) == code
    assert append(layout(), rotary(**kw), rows()) == code


@pytest.mark.parametrize("kw,code", [
    (dict(num_tokens=-1), ts.TS_ERR_SHAPE), (dict(format=ts.TS_KV_INT8), ts.TS_ERR_UNSUPPORTED),
    (dict(format=ts.TS_KV_FP4), ts.TS_ERR_UNSUPPORTED), (dict(q=None, k=None), ts.TS_ERR_NULL),
    (dict(q_out=None), ts.TS_ERR_NULL), (dict(k_out=None), ts.TS_ERR_NULL), (dict(q_stride=511), ts.TS_ERR_SHAPE),
    (dict(q_stride=508), ts.TS_ERR_SHAPE), (dict(k_out_stride=124), ts.TS_ERR_SHAPE), (dict(k_stride=-128), ts.TS_ERR_SHAPE),
    (dict(q=P + 4), ts.TS_ERR_SHAPE), (dict(k_out=P + 2), ts.TS_ERR_SHAPE),
])
def test_rows_out_of_range_are_refused_by_the_rotation(kw, code):
    assert rotate(rotary(), rows(**kw)) == code


def test_rotation_refuses_other_shapes():
    assert rotate(None, rows()) == ts.TS_ERR_NULL
    assert rotate(rotary(), None) == ts.TS_ERR_NULL
    assert rotate(rotary(positions=None), rows()) == ts.TS_ERR_NULL     # (no sequence to count places in)
    assert rotate(rotary(), rows(), Hq=0) == ts.TS_ERR_SHAPE
    assert rotate(rotary(), rows(), d=96) == ts.TS_ERR_UNSUPPORTED
    assert rotate(rotary(), rows(), d=0) == ts.TS_ERR_SHAPE
    # no tokens: nothing to do, whatever the positions
    assert rotate(rotary(positions=None), rows(num_tokens=0)) == ts.TS_OK


@pytest.mark.parametrize("kw,code", [
    (dict(num_tokens=-1), ts.TS_ERR_SHAPE), (dict(k=None), ts.TS_ERR_NULL), (dict(v=None), ts.TS_ERR_NULL),
    (dict(q_out=None), ts.TS_ERR_NULL), (dict(v_stride=126), ts.TS_ERR_SHAPE), (dict(v_stride=120), ts.TS_ERR_SHAPE),
    (dict(q_out_stride=256), ts.TS_ERR_SHAPE), (dict(v=P + 4), ts.TS_ERR_SHAPE),
])
def test_rows_out_of_range_are_refused_by_the_append(kw, code):
    assert append(layout(), rotary(), rows(**kw)) == code


def test_append_refuses_other_arguments():
    assert append(None, rotary(), rows()) == ts.TS_ERR_NULL
    assert append(layout(), rotary(), None) == ts.TS_ERR_NULL
    assert append(layout(), rotary(), rows(), lens=3) == ts.TS_ERR_SHAPE
    assert append(layout(), rotary(), rows(), lens=-1) == ts.TS_ERR_SHAPE
    assert append(layout(), rotary(), rows(num_tokens=3), cu=None) == ts.TS_ERR_SHAPE    # one token for each of two
    assert append(layout(page_min=None), rotary(), rows()) == ts.TS_ERR_NULL
    assert append(layout(v_pool=None), rotary(), rows()) == ts.TS_ERR_NULL
    assert append(layout(block_table=None), rotary(), rows()) == ts.TS_ERR_NULL
    assert append(layout(kv_format=ts.TS_KV_INT8, kv_tile_stride=1024), rotary(), rows()) == ts.TS_ERR_NULL   # scales
    assert append(layout(head_dim=96), rotary(), rows()) == ts.TS_ERR_UNSUPPORTED
    assert append(fp4(page_size=4), rotary(), rows()) == ts.TS_ERR_UNSUPPORTED
    assert append(layout(), rotary(), rows(num_tokens=0)) == ts.TS_OK


@pytest.mark.parametrize("kw,code", [
    (dict(page_size=4), ts.TS_ERR_UNSUPPORTED), (dict(page_size=12), ts.TS_ERR_UNSUPPORTED),
    (dict(kv_tile_stride=1072), ts.TS_ERR_SHAPE),       # less than a block of 16 * 68 bytes
    (dict(kv_tile_stride=1096), ts.TS_ERR_SHAPE),       # blocks must stay 16-byte aligned
    (dict(head_dim=96), ts.TS_ERR_UNSUPPORTED), (dict(kv_format=4), ts.TS_ERR_UNSUPPORTED),
    (dict(k_pool=P + 8), ts.TS_ERR_SHAPE),              # and so must their pool
])
def test_four_bit_layouts_out_of_range_are_refused(kw, code):
    lay, L = fp4(**kw), ts.lib()
    ref_ = ctypes.byref(lay)
    assert L.ts_build_page_meta(ref_, None) == code
    assert L.ts_append_token_meta(ref_, P, P, 1, None) == code
    assert L.ts_dense_decode_attention(ref_, P, 1.0, P, None, P, 1 << 30, None) == code
    assert L.ts_query_aware_decode(ref_, P, 4, None, 4, 1.0, P, None, None, None, P, 1 << 30, None) == code
    if "k_pool" not in kw:      # (these two look at the shape alone)
        assert L.ts_append_and_decode_launches(ref_, 4) == code
        assert ts.workspace_bytes(lay, 4) == 0


def test_four_bit_calls_check_their_pointers_and_workspaces():
    L, big = ts.lib(), 1 << 30
    for kw in (dict(k_pool=None), dict(block_table=None), dict(seq_lens=None)):
        lay = ctypes.byref(fp4(**kw))
        assert L.ts_dense_decode_attention(lay, P, 1.0, P, None, P, big, None) == ts.TS_ERR_NULL
        assert L.ts_sparse_decode_attention(lay, P, P, P, 8, 1.0, P, None, P, big, None) == ts.TS_ERR_NULL
        assert L.ts_append_token_meta(lay, P, P, 1, None) == ts.TS_ERR_NULL
        assert L.ts_build_page_meta(lay, None) == ts.TS_ERR_NULL
    lay = fp4()
    by = ctypes.byref(lay)
    dense = L.ts_dense_workspace_bytes(by)
    aware = ts.workspace_bytes(lay, 8)
    assert dense > 0 and aware > 0
    assert L.ts_dense_decode_attention(by, P, 1.0, P, None, P, dense - 1, None) == ts.TS_ERR_WORKSPACE
    assert L.ts_query_aware_decode(by, P, 8, None, 8, 1.0, P, None, None, None, P, aware - 1, None) == ts.TS_ERR_WORKSPACE
    assert L.ts_append_and_decode(by, P, P, P, 8, None, 8, 1.0, P, None, None, None, P, aware - 1, None) == ts.TS_ERR_WORKSPACE
    assert L.ts_sparse_decode_attention(by, P, P, P, 8, 1.0, P, None, P, 16, None) == ts.TS_ERR_WORKSPACE
    assert L.ts_query_aware_decode_static(by, P, 8, None, 8, 1.0, P, None, None, None, None) == ts.TS_ERR_UNSUPPORTED
    for q, out, bf16 in ((P + 8, P, 0), (P, P + 8, 0), (P, P + 4, 1)):       # rows that do not lie on their bytes
        by_ = ctypes.byref(fp4(out_format=bf16))
        assert L.ts_dense_decode_attention(by_, q, 1.0, out, None, P, big, None) == ts.TS_ERR_SHAPE
        assert L.ts_sparse_decode_attention(by_, q, P, P, 8, 1.0, out, None, P, big, None) == ts.TS_ERR_SHAPE
        assert L.ts_append_and_decode(by_, P, P, q, 8, None, 8, 1.0, out, None, None, None, P, big, None) == ts.TS_ERR_SHAPE
    assert L.ts_query_aware_decode(by, P, 9, None, 8, 1.0, P, None, None, None, P, big, None) == ts.TS_ERR_SHAPE


def test_four_bit_workspace_grows_with_the_batch_and_the_list():
    sizes = [ts.workspace_bytes(fp4(num_seqs=b), k) for b, k in ((1, 1), (1, 8), (2, 8), (16, 8), (16, 64))]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_binding_refuses_tensors_that_do_not_fit():
    bf = torch.zeros((4, 8, 64), dtype=torch.bfloat16)
    kv = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    table = ts.rotary_table(10, 64, device="cpu")
    assert table.shape == (10, 64) and table[0, :32].eq(1).all() and table[0, 32:].eq(0).all()
    r = ts.make_rotary(table, positions=torch.zeros(3, dtype=torch.int32))
    for call in (lambda: ts.rotate_rows(r, bf, kv),                                    # positions of three tokens
                 lambda: ts.rotate_rows(ts.make_rotary(), bf, kv.half()),
                 lambda: ts.rotate_rows(ts.make_rotary(), bf, kv[:3]),
                 lambda: ts.rotate_rows(ts.make_rotary(), bf, kv, bf[:, :4], kv),
                 lambda: ts.rotate_rows(ts.make_rotary(), bf.transpose(0, 1), None),
                 lambda: ts.rotate_rows(ts.make_rotary(), bf.float(), None),
                 lambda: ts.rotate_rows(ts.make_rotary(), None, None),
                 lambda: ts.rotate_rows(ts.make_rotary(q_norm=torch.ones(128)), bf, None),
                 lambda: ts.make_rotary(table.double()),
                 lambda: ts.make_rotary(table, positions=torch.zeros((3, 4), dtype=torch.int32)),
                 lambda: ts.append_rows(layout(), kv.half(), kv),
                 lambda: ts.append_rows(layout(), kv[:, :1], kv[:, :1]),
                 lambda: ts.append_rows(layout(), kv, kv, q=bf[:, :4]),
                 lambda: ts.append_rows(layout(), kv, kv, cu_tokens=torch.zeros(4, dtype=torch.int32)),
                 lambda: ts.append_rows(layout(), kv, kv, cu_tokens=torch.zeros(3)),
                 lambda: ts.append_rows(layout(), kv, kv),                             # four tokens, two sequences
                 lambda: ts.append_rows(layout(num_seqs=4), kv, kv),                   # tensors that no GPU can read
                 lambda: ts.rotate_rows(ts.make_rotary(), bf, kv)):
        with pytest.raises(ts.TinyServeError):
            call()


def test_rows_of_no_tokens_are_no_work():
    """(An empty tensor has no address, and nothing is enqueued: this runs where there is no GPU.)"""
    none = torch.empty((0, 8, 64), dtype=torch.bfloat16)
    ts.rotate_rows(ts.make_rotary(), none, none[:, :2])
    ts.append_rows(layout(), none[:, :2], none[:, :2], q=none[:, :8], cu_tokens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ts.TinyServeError):
        ts.rotate_rows(ts.make_rotary(), none, none.half())


def test_reference_four_bit_numbers():
    """The plain form itself: every code is its own nearest, ties go to even codes, the largest number of
    a row is kept by the scale that it sets, and packing is undone by unpacking."""
    codes = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11, 12, 13, 14, 15])
    x = ref.fp4_values(codes)
    got, scale = ref.fp4_quantised(x.bfloat16())
    assert scale == 1.0 and torch.equal(got, codes)
    ties = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -5])
    assert ref.fp4_quantised(ties.bfloat16())[0].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 0, 10, 14]
    g = torch.Generator().manual_seed(0)
    for S, d in ((8, 64), (16, 128), (64, 64)):
        kc, vc = torch.randint(0, 16, (2, 3, S, d), generator=g).unbind(0)
        ks, vs = (torch.rand((2, 3, S), generator=g) + 0.5).bfloat16().double().unbind(0)
        block = ref.fp4_packed(kc, ks, vc, vs, S * (d + 4) + 16)
        for a, b in zip(ref.fp4_unpacked(block, S, d), (kc, ks, vc, vs)):
            assert torch.equal(a, b)
    y = torch.randn((1000,), generator=g).double()
    lo, hi = ref.outwards(y, False), ref.outwards(y, True)
    assert (lo < y).all() and (hi > y).all() and ((hi - lo) <= y.abs() * 2.0 ** -6).all()
    b = y.bfloat16().double()
    assert torch.equal(ref.outwards(b, False), b) and torch.equal(ref.outwards(b, True), b)
