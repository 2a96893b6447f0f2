"""Orthogonalised updates that lie among others in memory: against the iteration in 64
bits with the tolerance of test_gpu_orthogonalize_spectra, and what lies between stays
as it was."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2011_12025_amd as sb
from paper_2011_12025_amd import _binding as b
from parity_util import log
from test_gpu_orthogonalize_spectra import ABC, iteration, off_before_rounding

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    b.lib()


def orders(t):
    """A batch [B, m, n] with the same values in other orders of memory."""
    yield "matrix after matrix", t.contiguous()
    yield "rows in turn", t.transpose(0, 1).contiguous().transpose(0, 1)
    yield "columns in turn", t.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    yield "rows in turn in a wider buffer", torch.nn.functional.pad(t.transpose(0, 1), (3, 5, 1, 0)).transpose(0, 1)[1:, :, 3:-5]
    yield "columns, matrix after matrix", t.transpose(1, 2).contiguous().transpose(1, 2)


def near_exact(got, g, what):
    """got against the iteration of g in 64 bits, matrix by matrix."""
    for i in range(g.shape[0]):
        one = g[i].cpu()
        exact = iteration(one, ABC)
        size = exact.norm().item()
        allowed = (exact.to(g.dtype).double() - exact).norm().item() / size + off_before_rounding(one, ABC)
        off = (got[i].double().cpu() - exact).norm().item() / size
        assert off <= allowed, f"{what}, matrix {i}: {off:.2e} off, {allowed:.2e} allowed"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,m,n", [(3, 20, 40), (4, 70, 33), (2, 130, 130), (1, 5, 9), (5, 1, 16), (5, 16, 1)])
def test_batches_in_any_order(_gpu, B, m, n, dtype):
    log(f"[orthogonalize] batches of {B} x {m} x {n} {dtype}")
    t = torch.randn(B, m, n, generator=torch.Generator().manual_seed(B + m)).to(DT[dtype]).cuda()
    for name, x in orders(t):
        assert torch.equal(x, t)
        near_exact(sb.orthogonalize(x), t, name)
    # into rows that are taken in turn, among others
    buf = torch.full((m, B + 2, n + 4), 7.0, dtype=DT[dtype], device="cuda")
    out = buf[:, 1:-1, 2:-2].transpose(0, 1)
    sb.orthogonalize(t, out=out)
    near_exact(out, t, "among others")
    out.fill_(7.0)
    assert bool((buf == 7.0).all())


def entry(**kw):
    q = b.Matrix(batch=3, rows=8, cols=10, ld=10, ld_out=10, batch_stride=80, batch_stride_out=80)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(ld_out=30, batch_stride_out=10), 0), (dict(ld_out=33, batch_stride_out=11), 0),
    (dict(ld_out=29, batch_stride_out=10), -1), (dict(ld_out=30, batch_stride_out=9), -1),
    (dict(ld_out=10, batch_stride_out=79), -1), (dict(ld_out=30, batch_stride_out=220), 0),
    (dict(ld_out=30, batch_stride_out=40), -1), (dict(ld_out=30, batch_stride_out=-10), -1),
    (dict(rows=1, ld_out=10, batch_stride_out=10), 0), (dict(rows=1, batch_stride_out=9), -1),
    (dict(ld=30, batch_stride=10), 0), (dict(batch_stride=0), 0),
    # extents past 64 bits, which would wrap to a few elements
    (dict(rows=1, cols=1, ld=1, ld_out=1, batch=(1 << 20) + 1, batch_stride=1 << 44, batch_stride_out=1), -1),
    (dict(rows=1, cols=1, ld=1, ld_out=1, batch=(1 << 20) + 1, batch_stride=1, batch_stride_out=1 << 44), -1),
    (dict(rows=1, cols=1, ld=1, ld_out=1, batch=(1 << 20) + 1, batch_stride=1 << 24, batch_stride_out=1 << 24), 0),
    (dict(batch=2, batch_stride=1 << 44, batch_stride_out=1 << 44), 0),
])
def test_results_of_a_batch_may_interleave_but_not_overlap(kw, code):
    n = ctypes.c_size_t(0)
    assert b.lib().segblocks_orthogonalize_workspace_size(ctypes.pointer(entry(**kw)), 1, 0, ctypes.byref(n)) == code
    if code:
        assert "strides" in b.lib().segblocks_last_error().decode()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_updates_and_results_in_columns_of_one_buffer(_gpu, dtype):
    log(f"[orthogonalize] columns of one buffer {dtype}")
    gen = torch.Generator().manual_seed(11)
    cols = [40, 24, 1, 130, 8]
    buf = torch.randn(70, 2 * sum(cols) + 6, generator=gen).to(DT[dtype]).cuda()
    before, at, updates, outs = buf.clone(), 3, [], []
    for n in cols:  # an update, its result, the next update
        updates.append(buf[:, at:at + n])
        outs.append(buf[:, at + n:at + 2 * n])
        at += 2 * n
    sb.orthogonalize(updates, out=outs)
    for g, o in zip(updates, outs):
        near_exact(o[None], g[None], f"{g.shape[1]} columns")
    for o in outs:
        o.copy_(before[:, o.storage_offset():o.storage_offset() + o.shape[1]])
    assert torch.equal(buf, before)
    # a batch in the rows of one buffer with another one's columns, and single rows between them
    many = torch.zeros(4, 30, 50, dtype=DT[dtype], device="cuda")
    rows = many.view(120, 50)
    batch = torch.randn(4, 30, 20, generator=gen).to(DT[dtype]).cuda()
    row = torch.randn(1, 10, generator=gen).to(DT[dtype]).cuda()
    whole = torch.randn(120, 15, generator=gen).to(DT[dtype]).cuda()
    sb.orthogonalize([batch, row, whole], out=[many[:, :, :20], rows[7:8, 20:30], rows[:, 30:45]])
    near_exact(many[:, :, :20], batch, "a batch")
    near_exact(rows[7:8, 20:30][None], row[None], "a row")
    near_exact(rows[:, 30:45][None], whole[None], "all rows")
    assert int((many != 0).sum()) <= 120 * 35 + 10


def at_bytes(offset):
    return 0x100000000 + 2 * offset  # (fp16; never read or written)


@pytest.mark.parametrize("entries", [
    # (update, out, rows, cols, ld_out, batch, batch_stride_out) in elements from one place
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 9, 8, 10, 64, 1, 0)],           # columns that share one
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 60, 8, 5, 64, 1, 0)],           # columns past the end of a row
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 128 + 9, 8, 10, 64, 1, 0)],     # two rows on
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 20, 8, 10, 63, 1, 0)],          # rows at other distances
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 20, 1, 45, 45, 1, 0)],          # a row that reaches into the next
    [(1 << 20, 0, 8, 10, 64, 1, 0), (15, 1 << 21, 8, 50, 64, 1, 0)],          # an update on a result
    [(1 << 20, 0, 8, 10, 64, 2, 16), (1 << 21, 20, 8, 10, 64, 1, 0)],         # rows of a batch in turn
    [(1 << 20, 0, 8, 10, 64, 2, 640), (1 << 21, 9 + 704, 8, 10, 64, 1, 0)],   # matrix after matrix
    [(1 << 20, 0, 8, 10, 64, 1, 0), (1 << 21, 20, 8, 10, 64, 1, 0), (1 << 22, 512 - 40, 2, 8, 8, 1, 0)],  # a third one
])
def test_results_that_overlap_in_one_buffer_are_refused(entries):
    for order in (entries, entries[::-1]):
        mats = (b.Matrix * len(order))()
        for q, (u, o, m, n, ld, batch, stride) in zip(mats, order):
            q.batch, q.rows, q.cols, q.ld, q.ld_out = batch, m, n, 64 if n <= 64 else n, ld
            q.batch_stride, q.batch_stride_out = 1 << 14, stride
            q.update, q.out = at_bytes(u), at_bytes(o)
        c = (ctypes.c_double * 3)(1.0, 0.0, 0.0)
        n = ctypes.c_size_t(0)
        assert b.lib().segblocks_orthogonalize_workspace_size(mats, len(order), 1, ctypes.byref(n)) == 0
        code = b.lib().segblocks_orthogonalize(mats, len(order), 1, 1, c, 0.0, ctypes.c_void_p(0x900000000), n.value, None)
        assert code == -1 and "overlap" in b.lib().segblocks_last_error().decode()


@pytest.mark.parametrize("m,n", [(64, 1 << 20), (4096, 4096), (4096, 16384), (32768, 1 << 18)])
def test_workspace_takes_twelve_bytes_an_element(m, n):
    """X and two transposes in pairs, five matrices of the shorter side, sums of tiles (up to 128 KB a CU) and 8 KB."""
    size = ctypes.c_size_t(0)
    for dtype in (0, 1, 2):
        for rows, cols in ((m, n), (n, m)):
            q = b.Matrix(batch=1, rows=rows, cols=cols, ld=cols, ld_out=cols)
            assert b.lib().segblocks_orthogonalize_workspace_size(ctypes.pointer(q), 1, dtype, ctypes.byref(size)) == 0
            assert size.value <= 12 * m * n + 20 * m * m + 512 * 65536 + 8192 + 256
