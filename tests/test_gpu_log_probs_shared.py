"""The gradient of class scores written to other channels of the buffer that holds the
scores: bit for bit what a buffer of its own gets, and nothing else changes."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2011_12025_amd as sb
from paper_2011_12025_amd import _binding as b
from parity_util import log

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["nhwc", "nchw", "rows"])
@pytest.mark.parametrize("C,at,of,many", [(19, 24, 48, 900), (19, 20, 41, 70000), (7, 7, 14, 333), (150, 160, 320, 500),
                                          (5000, 5008, 10016, 9)])
def test_scores_and_gradient_in_one_buffer(C, at, of, many, layout, dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    log(f"[log_probs] scores and gradient in one buffer: {C} at {at} of {of}, {many} {layout} {dtype}")
    gen = torch.Generator().manual_seed(C + many)
    shape = (many, of) if layout == "rows" else (2, of, many // 5, 5) if many < 60000 else (1, of, many // 200, 200)
    buf = (torch.randn(shape, generator=gen) * 2.5).to(DT[dtype]).cuda()
    if layout == "nhwc":
        buf = buf.contiguous(memory_format=torch.channels_last)
    rows = (many,) if layout == "rows" else (shape[0], *shape[2:])
    labels = torch.randint(0, C, rows, generator=gen).cuda()
    for first, second in ((0, at), (at, 0)):
        z = buf.narrow(1, first, C)
        keep = buf.clone(memory_format=torch.preserve_format)
        _, lse, H, _, ti = sb.log_probs(z, labels, topk=2)
        kw = dict(d_logp=torch.randn(rows, generator=gen).cuda(), entropy=H, d_entropy=torch.randn(rows, generator=gen).cuda(),
                  top_index=ti, d_top=torch.randn(ti.shape, generator=gen).cuda())
        # (at an address with the same alignment: vectors begin at the same classes)
        own = keep.clone(memory_format=torch.preserve_format).narrow(1, second, C)
        sb.log_probs_backward(keep.narrow(1, first, C), labels, lse, out=own, **kw)
        out = buf.narrow(1, second, C)
        assert sb.log_probs_backward(z, labels, lse, out=out, **kw) is out
        assert torch.equal(out, own)
        out.copy_(keep.narrow(1, second, C))
        assert torch.equal(buf, keep), "other channels were written"


@pytest.mark.parametrize("offset,C_dbuf", [
    (0, 48), (18, 48), (30, 48), (48, 48), (24, 47), (24, 40), (24 - 48, 47),
])
@pytest.mark.parametrize("layout", [0, 1])
def test_channels_that_overlap_are_refused(offset, C_dbuf, layout):
    """19 scores of 48 channels, fp16, 4 images of 8 x 8 pixels; gradients that share some of them."""
    per = 64 if layout == 0 else 1
    z, dz = 0x100000000, 0x100000000 + 2 * offset * per
    at = lambda i: ctypes.c_void_p(0x200000000 + i * 0x10000000)  # noqa: E731
    code = b.lib().segblocks_log_probs_backward(ctypes.c_void_p(z), 1, layout, 4, 19, 8, 8, 48, at(1), 255, at(2), at(3), None,
                                                None, 0, None, None, C_dbuf, ctypes.c_void_p(dz), None)
    assert code == -1 and "overlaps" in b.lib().segblocks_last_error().decode()
