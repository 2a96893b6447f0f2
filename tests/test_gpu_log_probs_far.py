"""Gradients of rows whose |lse| is past 256, where p comes from the row's own maximum
and sum, taken anew by every workgroup or range of classes of the row: rows of
several of them, with near, empty and far rows side by side.  Tolerance of
test_gpu_log_probs (2^-16 of what a class's gradient is made of, and the result's
rounding), and 2^-126 of what multiplies p: the exponential gives 0 below the
smallest normal number of 32 bits (differences of 88 and more, which these rows
have), so p is off by that much at most.  Where one class has nearly all of a row,
ln p + H is small, and what counts is the absolute error of its terms: ln p = z - lse
has half a step of lse, 2^-24 |lse|, and the entropy that the forward call gives is
off by 2^-18 (1 + 2 H + 2 ln C) at most (test_gpu_log_probs), both times |g_H| p."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2011_12025_amd as sb
from parity_util import log
from test_gpu_log_probs import DT, IGNORE, close, grad_reference, labels_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2011_12025_amd._binding as b
    b.lib()


def far_scores(R, C, dtype, gen):
    """Rows around 0, 3000 and -3000 (300 and -700 in 16 bits, which are coarse up there) and at one value."""
    z = torch.randn(R, C, generator=gen) * 2.5
    if dtype != "f32":
        z = (z * 2).round() * 2  # (steps that bf16 has up to 512)
    up, down = (3000.0, -3000.0) if dtype == "f32" else (300.0, -700.0)
    z[0::4] += up
    z[1::4] += down
    z[2::4, C // 3:] = -math.inf
    z[2::4] += up
    return z.to(DT[dtype])


def check_grad(z, labels, topk):
    """All gradients given; z in rows or as a map."""
    rows = (lambda x: x.movedim(1, -1).reshape(-1, x.shape[1])) if z.dim() == 4 else (lambda x: x)
    gen = torch.Generator().manual_seed(11)
    _, lse, H, _, ti = sb.log_probs(z, labels, topk=topk, ignore=IGNORE)
    g, gh = (torch.randn(labels.shape, generator=gen).cuda() for _ in range(2))
    gt = torch.randn(ti.shape, generator=gen).cuda() if topk else None
    dz = sb.log_probs_backward(z, labels, lse, d_logp=g, entropy=H, d_entropy=gh, top_index=ti, d_top=gt, ignore=IGNORE)
    one = lambda x: x.reshape(-1).double().cpu()  # noqa: E731
    z64, lab = rows(z).double().cpu(), labels.reshape(-1).cpu()
    ref, size = grad_reference(z64, lab, one(g), one(gh), rows(ti).cpu().long() if topk else None,
                               rows(gt).double().cpu() if topk else None)
    by = 2 * (one(g).abs() + (rows(gt).double().cpu().abs().sum(1) if topk else 0)) + one(gh).abs() * (1000 + one(H))
    l64 = torch.logsumexp(z64, 1)
    p64 = torch.where(l64[:, None] == -math.inf, 0.0, (z64 - l64[:, None]).exp())
    of_terms = one(gh).abs() * (2.0 ** -24 * torch.where(l64 == -math.inf, 0.0, l64.abs()) +
                                2.0 ** -18 * (1 + 2 * one(H) + 2 * math.log(z64.shape[1])))
    eps = torch.finfo(z.dtype).eps / 2
    tiny = torch.finfo(z.dtype).smallest_normal * 2 * eps  # half the least step
    tol = eps * ref.abs() * (1 + 2.0 ** -8) + tiny + (1 + eps) * (2.0 ** -16 * size + 2.0 ** -126 * by[:, None] + p64 * of_terms[:, None])
    close(rows(dz), ref, tol, "dlogits")
    assert dz.dtype == z.dtype and dz.shape == z.shape


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,C,of,topk", [(7, 70001, 70001, 3), (5, 9000, 9004, 0), (3, 131072, 131072, 20), (600, 20001, 20008, 2),
                                         (200, 100, 104, 12)])
def test_rows(R, C, of, topk, dtype):
    log(f"[log_probs] far rows {R} x {C} of {of} {dtype}, top {topk}")
    gen = torch.Generator().manual_seed(C)
    z = torch.zeros(R, of, dtype=DT[dtype])
    z[:, :C] = far_scores(R, C, dtype, gen)
    lab = torch.randint(0, C // 3, (R,), generator=gen)
    lab[1::5] = IGNORE
    check_grad(z.cuda()[:, :C], lab.cuda(), topk)


@pytest.mark.parametrize("layout", ["nhwc", "nchw"])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("N,C,H,W,topk", [(1, 1000, 8, 9, 2), (2, 150, 33, 17, 0), (1, 37, 5, 130, 12), (1, 500, 40, 40, 4)])
def test_maps(N, C, H, W, topk, dtype, layout):
    log(f"[log_probs] far maps {N} x {C} x {H} x {W} {layout} {dtype}, top {topk}")
    gen = torch.Generator().manual_seed(C + H)
    z = far_scores(N * H * W, C, dtype, gen).reshape(N, H, W, C).permute(0, 3, 1, 2).cuda()
    z = z.contiguous(memory_format=torch.channels_last if layout == "nhwc" else torch.contiguous_format)
    lab = labels_of((N, H, W), C // 3, gen)
    check_grad(z, lab, topk)


def test_a_far_row_without_a_class():
    """Every class at -inf beside far rows, in several ranges: gradient 0."""
    z = torch.full((3, 30000), -math.inf, device="cuda")
    z[1] = torch.randn(30000) + 2000.0
    lab = torch.zeros(3, dtype=torch.int64, device="cuda")
    _, lse, H, _, _ = sb.log_probs(z, lab)
    dz = sb.log_probs_backward(z, lab, lse, d_logp=torch.ones(3, device="cuda"), entropy=H, d_entropy=torch.ones(3, device="cuda"))
    assert bool((dz[0] == 0).all()) and bool((dz[2] == 0).all()) and bool(dz[1].isfinite().all()) and bool((dz[1] != 0).any())
