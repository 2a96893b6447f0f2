"""GPU parity of the log probabilities of class scores and of their gradient
against a plain implementation in 64 bits on the CPU.

Tolerances.  The results are fp32 sums of rounded terms: exp and log are good to
two units in the last place (2^-22 relative), a term's exponent z - m carries
half a step of |z - m| (at most 30 in these inputs where the term counts:
2^-25 * 30), and the sum of C terms of one sign at most adds its own roundings
in the order of log2(C) + 32 (lanes, vectors, waves): below 2^-18 relative in
all for s and t.  logp = (z - m) - ln s then is off by 2^-18 + 2^-24 |z - m|,
lse by the same plus 2^-24 |lse|, the entropy by 2^-18 (1 + H + |t / s|).  A
gradient's p is off by that relative 2^-18 and by 2^-25 |lse| <= 2^-17 (past
|lse| = 256 the row's maximum takes its place), times |G| + |g_H| (|ln p| + H),
and is rounded once to its type (half a step).
"""
from __future__ import annotations

import math

import pytest
import torch

import paper_2011_12025_amd as sb
from parity_util import log

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
REL = 2.0 ** -18
IGNORE = 255


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2011_12025_amd._binding as b
    b.lib()


def reference(z, labels, topk, ignore=IGNORE):
    """z [R, C] in 64 bits -> logp, lse, entropy, top_logp, top_index (lists of rows)."""
    C = z.shape[1]
    m = z.max(1, keepdim=True)[0]
    empty = (m == -math.inf).squeeze(1)
    m = torch.where(m == -math.inf, 0.0, m)
    ln_s = (z - m).exp().sum(1, keepdim=True).log()
    lse = (m + ln_s).squeeze(1)
    # (the difference first: the lowest value of fp32 swallows ln s in 64 bits too)
    logq = torch.where(empty[:, None], -math.inf, (z - m) - ln_s)
    q = logq.exp()
    H = -(q * torch.where(q > 0, logq, 0.0)).sum(1)
    bad = (labels != ignore) & ((labels < 0) | (labels >= C))
    t = torch.where((labels == ignore) | bad, 0, labels)
    logp = logq.gather(1, t[:, None]).squeeze(1)
    logp = torch.where(labels == ignore, 0.0, torch.where(bad, math.nan, logp))
    order = torch.sort(torch.where(z.isnan(), math.inf, z), dim=1, descending=True, stable=True)[1][:, :topk]
    return logp, lse, torch.where(empty, 0.0, H), logq.gather(1, order), order


def close(got, ref, tol, what):
    got = got.double().cpu().reshape(ref.shape)
    same = (got == ref) | (got.isnan() & ref.isnan())
    off = torch.where(same, 0.0, (got - ref).abs() - tol)
    assert bool((same | (off <= 0)).all()), (
        f"{what}: {got[~(same | (off <= 0))][:4].tolist()} vs {ref[~(same | (off <= 0))][:4].tolist()}, "
        f"past the tolerance by up to {off.max().item():.2e}")


def check(z, labels, topk, entropy=True, ignore=IGNORE):
    """z: the scores on the GPU in any of the accepted forms."""
    d = z.dim()
    rows = z.permute(0, 2, 3, 1) if d == 4 else z
    C = rows.shape[-1]
    r64 = rows.reshape(-1, C).double().cpu()
    lab = labels.reshape(-1).cpu()
    logp, lse, H, tl, ti = sb.log_probs(z, labels, topk=topk, entropy=entropy, ignore=ignore)
    torch.cuda.synchronize()
    e_logp, e_lse, e_H, e_tl, e_ti = reference(r64, lab, topk, ignore)
    fin = torch.where(e_lse.isfinite(), e_lse.abs(), 0.0)
    top = torch.where(r64 == -math.inf, 0.0, r64).abs().max(1)[0]  # bounds |z - m| together with m
    far = REL + 2.0 ** -23 * (top + fin)
    close(logp, e_logp, far, "logp")
    close(lse, e_lse, far, "lse")
    assert logp.shape == labels.shape and lse.shape == labels.shape
    if entropy:
        close(H, e_H, REL * (1 + 2 * e_H + 2 * math.log(C)), "entropy")
    else:
        assert H is None
    if topk:
        want = (*z.shape[:1], topk, *z.shape[2:]) if d == 4 else (*z.shape[:-1], topk)
        assert tuple(tl.shape) == want and tuple(ti.shape) == want and ti.dtype == torch.int32
        flat = (lambda x: x.permute(0, 2, 3, 1).reshape(-1, topk)) if d == 4 else (lambda x: x.reshape(-1, topk))
        assert torch.equal(flat(ti).cpu().long(), e_ti), "top_index"
        close(flat(tl).contiguous(), e_tl, far[:, None], "top_logp")
    else:
        assert tl is None and ti is None
    return lse, H, tl, ti


def tokens(R, C, dtype, gen, of=None, skip=0):
    z = (torch.randn(R, (of or C) + skip, generator=gen) * 2.5).to(DT[dtype]).cuda()
    return z[:, skip:skip + C]


def labels_of(shape, C, gen, ignored=0.1):
    lab = torch.randint(0, C, shape, generator=gen)
    lab[torch.rand(shape, generator=gen) < ignored] = IGNORE
    return lab.cuda()


ROWS = [  # rows, classes, buffer, skipped classes before, topk
    (1, 1, 1, 0, 1), (1, 2, 2, 0, 0), (3, 7, 7, 0, 7), (2, 64, 64, 0, 64), (70, 19, 24, 0, 3), (300, 65, 72, 3, 5),
    (1, 1000, 1000, 0, 20), (5, 1023, 1024, 1, 64), (9, 1025, 1030, 0, 8), (257, 333, 340, 4, 9), (33, 5003, 5003, 0, 4),
    (2, 16385, 16400, 7, 33), (20000, 30, 31, 0, 1), (17000, 100, 200, 0, 2), (17000, 67, 135, 0, 10),
    (16500, 130, 130, 0, 64), (3, 70001, 70001, 0, 20), (1, 131072, 131072, 0, 64), (65, 66000, 66001, 0, 5),
    (600, 20000, 20000, 0, 3),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,C,of,skip,topk", ROWS)
def test_rows(R, C, of, skip, topk, dtype):
    log(f"[log_probs] rows {R} x {C} of {of} from {skip}, {dtype}, top {topk}")
    gen = torch.Generator().manual_seed(R + 7 * C)
    z, lab = tokens(R, C, dtype, gen, of, skip), labels_of((R,), C, gen)
    check(z, lab, topk)


MAPS = [  # N, C, H, W, buffer, topk
    (1, 19, 16, 32, 24, 1), (2, 5, 7, 9, 5, 3), (1, 150, 33, 47, 152, 10), (2, 1, 4, 4, 1, 1), (3, 300, 5, 3, 304, 20),
    (1, 1000, 7, 7, 1000, 5), (1, 40, 300, 301, 40, 0), (2, 8, 1, 1, 8, 2), (1, 70, 1, 40, 70, 64), (1, 129, 64, 65, 130, 8),
    (2, 13, 25, 44, 13, 13), (1, 60, 9, 11, 64, 16), (1, 532, 9, 4, 532, 20),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("layout", ["nhwc", "nchw"])
@pytest.mark.parametrize("N,C,H,W,of,topk", MAPS)
def test_maps(N, C, H, W, of, topk, layout, dtype):
    log(f"[log_probs] map {N} x {C} of {of} x {H} x {W} {layout} {dtype}, top {topk}")
    gen = torch.Generator().manual_seed(C + H)
    z = (torch.randn(N, of, H, W, generator=gen) * 2.5).to(DT[dtype]).cuda()
    z = z.contiguous(memory_format=torch.channels_last if layout == "nhwc" else torch.contiguous_format)[:, :C]
    check(z, labels_of((N, H, W), C, gen), topk, entropy=C != 40)


@pytest.mark.parametrize("form", ["short", "rows", "parts", "planes", "planes16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_masks_and_odd_values(form, dtype):
    """Equal scores, -inf, the type's lowest value, an empty row, NaN, infinities,
    signed zeros, labels outside the classes; every kernel form."""
    log(f"[log_probs] odd values, {form}, {dtype}")
    C, R = {"short": (21, 12), "rows": (1500, 12), "parts": (70000, 12), "planes": (21, 12), "planes16": (400, 12)}[form]
    low = torch.finfo(DT[dtype]).min
    gen = torch.Generator().manual_seed(3)
    z = torch.randint(-2, 3, (R, C), generator=gen).float()        # many ties
    z[1, :] = -math.inf                                            # empty
    z[2, 1:] = -math.inf                                           # one class
    z[3, :] = low                                                  # a mask of the lowest value everywhere: uniform
    z[4, ::2] = low
    z[5, C // 2] = math.inf
    z[6, C // 3] = math.nan
    z[7, :] = 0.0
    z[7, ::2] = -0.0
    z[8, :C - 3] = -math.inf
    z[9, :] = torch.linspace(-30, 30, C)
    z[10, :] = 300.0 + z[10, :]                                    # a large log-sum-exp
    lab = torch.randint(0, C, (R,), generator=gen)
    lab[0], lab[11], lab[2] = -7, C, 0
    z = z.to(DT[dtype])
    if form.startswith("planes"):
        zd = z.reshape(1, R, 1, C).permute(0, 3, 1, 2).contiguous().cuda()
        ld = lab.reshape(1, R, 1).cuda()
    else:
        zd, ld = z.cuda(), lab.cuda()
    # NaN and infinite rows apart: their statistics are NaN, the order still holds
    logp, lse, H, tl, ti = (x.reshape(R, -1) if x.dim() < 3 else x.movedim(1, -1).reshape(R, -1)
                            for x in sb.log_probs(zd, ld, topk=min(C, 20)))
    for r in (5, 6):
        assert all(bool(x[r].isnan().all()) for x in (logp, lse, H, tl))
    assert ti[5, 0] == C // 2 and ti[6, 0] == C // 3
    fine = [r for r in range(R) if r not in (5, 6)]
    lp, ls, h, etl, eti = reference(z.double()[fine], lab[fine], 20)
    big = 2.0 ** -23 * torch.where(ls.isfinite(), ls.abs(), 0.0)
    tol = torch.where(ls.abs() < 1e30, REL + big, REL)
    close(logp[fine].squeeze(1), lp, tol, "logp")
    close(lse[fine].squeeze(1), ls, REL + big, "lse")
    close(H[fine].squeeze(1), h, REL * (1 + 2 * h + 2 * math.log(C)), "entropy")
    assert torch.equal(ti[fine].cpu().long(), eti)
    keep = ls.abs() < 1e30
    close(tl[fine][keep.cuda()], etl[keep], (tol[keep])[:, None], "top_logp")
    # a row of nothing but the lowest value is uniform
    assert abs(H[3, 0].item() - math.log(C)) < REL * (1 + 4 * math.log(C)) and abs(tl[3, 0].item() + math.log(C)) < 1e-5
    assert H[1, 0].item() == 0.0 and lse[1, 0].item() == -math.inf


def grad_reference(z, labels, g, gh, top, gt, ignore=IGNORE):
    """[R, C] gradient in 64 bits by the softmax's Jacobian, and what its error scales with."""
    m = z.max(1, keepdim=True)[0]
    empty = m == -math.inf
    z = torch.where(empty, 0.0, z)
    d = z - z.max(1, keepdim=True)[0]
    logq = d - d.exp().sum(1, keepdim=True).log()
    q = logq.exp()
    lq = torch.where(q > 0, logq, 0.0)
    H = -(q * lq).sum(1, keepdim=True)
    u = torch.zeros_like(z)
    size = torch.zeros_like(z)
    if g is not None:
        w = torch.where(labels == ignore, 0.0, g)[:, None]
        t = torch.where(labels == ignore, 0, labels)[:, None]
        u.scatter_add_(1, t, w)
    if gt is not None:
        u.scatter_add_(1, top, gt)
    G = u.sum(1, keepdim=True)
    A = u.abs().sum(1, keepdim=True)
    if gt is not None:
        A = A + gt.abs().sum(1, keepdim=True)
    d = u - q * G
    size = q * (A + 0 * G)
    if gh is not None:
        d = d - gh[:, None] * q * (lq + H)
        size = size + q * gh.abs()[:, None] * (lq.abs() + H)
    return torch.where(empty, 0.0, d), size + u.abs()


def check_grad(z, labels, topk, use, dz_of=None):
    d = z.dim()
    C = z.shape[1] if d == 4 else z.shape[-1]
    flat = (lambda x: x.permute(0, 2, 3, 1).reshape(-1, x.shape[1])) if d == 4 else (lambda x: x.reshape(-1, x.shape[-1]))
    lse, H, tl, ti = sb.log_probs(z, labels, topk=topk, ignore=IGNORE)[1:]
    gen = torch.Generator().manual_seed(11)
    g = torch.randn(labels.shape, generator=gen).cuda() if "g" in use else None
    gh = torch.randn(labels.shape, generator=gen).cuda() if "h" in use else None
    gt = torch.randn(ti.shape, generator=gen).cuda() if topk and "t" in use else None
    kw = dict(d_logp=g, entropy=H if gh is not None else None, d_entropy=gh, top_index=ti if gt is not None else None,
              d_top=gt, ignore=IGNORE)
    if dz_of:
        wide = torch.full((*z.shape[:1], dz_of, *z.shape[2:]) if d == 4 else (*z.shape[:-1], dz_of), 7.0, dtype=z.dtype,
                          device="cuda")
        if d == 4 and z.stride(1) == 1:
            wide = wide.contiguous(memory_format=torch.channels_last)
        out = wide.narrow(1 if d == 4 else -1, 0, C)
        kw["out"] = out
    dz = sb.log_probs_backward(z, labels, lse, **kw)
    torch.cuda.synchronize()
    if dz_of:
        assert bool((wide.narrow(1 if d == 4 else -1, C, dz_of - C) == 7.0).all()), "channels past the classes were written"
    one = lambda x: None if x is None else x.reshape(-1).double().cpu()  # noqa: E731
    ref, size = grad_reference(flat(z).double().cpu(), labels.reshape(-1).cpu(), one(g), one(gh),
                               None if gt is None else flat(ti).cpu().long(), None if gt is None else flat(gt).double().cpu())
    eps = torch.finfo(z.dtype).eps / 2
    tiny = torch.finfo(z.dtype).smallest_normal * 2 * eps  # half the least step
    got = flat(dz).double().cpu()
    # p: 2^-18 and 2^-17 (lse) and 2^-23 |z - lse| for its exponent
    tol = eps * ref.abs() * (1 + 2.0 ** -8) + tiny + (1 + eps) * (2.0 ** -16) * size
    close(got, ref, tol, "dlogits")
    assert dz.dtype == z.dtype and dz.shape == z.shape


GRADS = [(R, C, of, skip, min(topk, 9)) for R, C, of, skip, topk in ROWS]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("R,C,of,skip,topk", GRADS)
def test_grad_rows(R, C, of, skip, topk, dtype):
    log(f"[log_probs] gradient, rows {R} x {C} of {of} from {skip}, {dtype}, top {topk}")
    gen = torch.Generator().manual_seed(R + 5 * C)
    z, lab = tokens(R, C, dtype, gen, of, skip), labels_of((R,), C, gen)
    check_grad(z, lab, topk, "ght", dz_of=of if of > C else None)


@pytest.mark.parametrize("use", ["g", "h", "t", "gh"])
@pytest.mark.parametrize("layout", ["nhwc", "nchw"])
@pytest.mark.parametrize("N,C,H,W,of,topk", MAPS)
def test_grad_maps(N, C, H, W, of, topk, layout, use):
    if use == "t" and topk == 0:
        topk = 2
    log(f"[log_probs] gradient, map {N} x {C} of {of} x {H} x {W} {layout}, {use}, top {topk}")
    gen = torch.Generator().manual_seed(C + H)
    z = (torch.randn(N, of, H, W, generator=gen) * 2.5).half().cuda()
    z = z.contiguous(memory_format=torch.channels_last if layout == "nhwc" else torch.contiguous_format)[:, :C]
    check_grad(z, labels_of((N, H, W), C, gen), topk, use, dz_of=of if of > C else None)


@pytest.mark.parametrize("form", ["short", "rows", "planes"])
def test_grad_odd_rows(form):
    """Empty rows, masked classes, the lowest value everywhere, a large lse, ignored
    and bad labels, an alternative that is the label."""
    log(f"[log_probs] gradient, odd rows, {form}")
    C, R = (21, 7) if form != "rows" else (3000, 7)
    gen = torch.Generator().manual_seed(4)
    z = torch.randn(R, C, generator=gen)
    z[0] = -math.inf
    z[1, 2:] = -math.inf
    z[2] = torch.finfo(torch.float32).min
    z[3] += 3000.0
    z[4, 5] = 40.0
    lab = torch.tensor([1, 0, 2, 3, 5, IGNORE, C + 4])
    if form == "planes":
        zd, ld = z.reshape(1, R, 1, C).permute(0, 3, 1, 2).contiguous().cuda(), lab.reshape(1, R, 1).cuda()
    else:
        zd, ld = z.cuda(), lab.cuda()
    logp, lse, H, tl, ti = sb.log_probs(zd, ld, topk=2, ignore=IGNORE)
    g, gh, gt = torch.ones_like(logp), torch.full_like(H, 0.5), torch.full_like(tl, 0.25)
    dz = sb.log_probs_backward(zd, ld, lse, d_logp=g, entropy=H, d_entropy=gh, top_index=ti, d_top=gt, ignore=IGNORE)
    rows = (lambda x: x.movedim(1, -1).reshape(R, -1)) if form == "planes" else (lambda x: x.reshape(R, -1))
    dz, ti = rows(dz).cpu(), rows(ti).cpu()
    assert bool((dz[0] == 0).all()), "an empty row"
    assert bool(dz[6].isnan().all()), "a label outside the classes"
    keep = [1, 2, 3, 4, 5]
    k = lambda v: torch.full((5,), v, dtype=torch.float64)  # noqa: E731
    ref, size = grad_reference(z.double()[keep], lab[keep], k(1.0), k(0.5), ti[keep].long(),
                               torch.full((5, 2), 0.25, dtype=torch.float64))
    close(dz[keep], ref, 2.0 ** -16 * size + 2.0 ** -23 * ref.abs() + 1e-38, "dlogits")


@pytest.mark.parametrize("topk", [3, 8, 12])
@pytest.mark.parametrize("form", ["short", "rows", "planes"])
def test_grad_of_a_class_named_twice(form, topk):
    """Indices that name a class more than once, the label's among them: their gradients add up."""
    log(f"[log_probs] gradient, a class named twice, {form}, top {topk}")
    C, R = (21, 70) if form != "rows" else (3000, 5)
    gen = torch.Generator().manual_seed(topk)
    z, lab = torch.randn(R, C, generator=gen), torch.randint(0, C, (R,), generator=gen)
    ti = torch.randint(0, 4, (R, topk), generator=gen).int()
    ti[:, 1], ti[:, -1] = lab, lab
    g, gt = torch.randn(R, generator=gen), torch.randn(R, topk, generator=gen)
    ref, size = grad_reference(z.double(), lab, g.double(), None, ti.long(), gt.double())
    up = (lambda x: x.reshape(1, R, 1, -1).permute(0, 3, 1, 2).contiguous().cuda()) if form == "planes" else (lambda x: x.cuda())
    one = (lambda x: x.reshape(1, R, 1).cuda()) if form == "planes" else (lambda x: x.cuda())
    lse = sb.log_probs(up(z))[1]
    dz = sb.log_probs_backward(up(z), one(lab), lse, d_logp=one(g), top_index=up(ti), d_top=up(gt)).cpu()
    dz = dz.movedim(1, -1).reshape(R, C) if form == "planes" else dz
    # fp32: a sum of up to 14 terms, each sum rounded, beside what grad_reference's size allows for
    many = gt.abs().sum(1, keepdim=True).double() + g.abs()[:, None]
    close(dz, ref, 2.0 ** -16 * size + 14 * 2.0 ** -24 * many + 1e-38, "dlogits")


def test_gradient_by_differences():
    gen = torch.Generator().manual_seed(8)
    z = torch.randn(6, 40, generator=gen).cuda()
    lab = torch.randint(0, 40, (6,), generator=gen).cuda()
    wl, wh, wt = (torch.randn(s, generator=gen).double() for s in ((6,), (6,), (6, 3)))

    def value(x):
        logp, _, H, tl, _ = reference(x, lab.cpu(), 3)
        return (wl * logp).sum() + (wh * H).sum() + (wt * tl).sum()
    _, lse, H, _, ti = sb.log_probs(z, lab, topk=3)
    dz = sb.log_probs_backward(z, lab, lse, d_logp=wl.float().cuda(), entropy=H, d_entropy=wh.float().cuda(), top_index=ti,
                               d_top=wt.float().cuda()).double().cpu()
    x, h = z.double().cpu(), 1e-5
    for r, c in [(0, 0), (1, 7), (2, int(lab[2])), (3, int(ti[3, 0])), (5, 39)]:
        step = torch.zeros_like(x)
        step[r, c] = h
        d = (value(x + step) - value(x - step)) / (2 * h)
        # differences are good to h^2 and 1e-16 / h, the gradient to 2^-16 of its terms (at most 20 here)
        assert abs(d.item() - dz[r, c].item()) < 20 * 2.0 ** -16


def test_batches_of_sequences_strides_and_nothing():
    gen = torch.Generator().manual_seed(9)
    z = (torch.randn(3, 5, 50, generator=gen)).cuda()
    check(z, labels_of((3, 5), 50, gen), 4)
    check(z[:, :, 3:40], labels_of((3, 5), 37, gen), 4)
    check(z[1:2, :, :], labels_of((1, 5), 50, gen), 1)
    out = sb.log_probs(z[:0], labels_of((0, 5), 50, gen), topk=2)
    assert [tuple(x.shape) for x in out] == [(0, 5), (0, 5), (0, 5), (0, 5, 2), (0, 5, 2)]
    lse, H = sb.log_probs(z)[1:3]  # no labels
    dz = sb.log_probs_backward(z, None, lse, entropy=H, d_entropy=torch.ones_like(H))
    assert dz.shape == z.shape
    # gradients broadcast from one value, as the mean of a loss gives them
    lab = labels_of((3, 5), 50, gen, ignored=0.0)
    a = sb.log_probs_backward(z, lab, lse, d_logp=torch.full((1, 1), -0.1, device="cuda").expand(3, 5))
    b = sb.log_probs_backward(z, lab, lse, d_logp=torch.full((3, 5), -0.1, device="cuda"))
    assert torch.equal(a, b)


def test_rows_past_32_bits():
    """More rows than threads of one launch, and offsets past 2^32 elements: the last rows, forward and backward."""
    R, C = (1 << 25) + 70, 132
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free memory")
    log(f"[log_probs] {R} rows of {C}")
    z = torch.empty(R, C, dtype=torch.float16, device="cuda").normal_(0, 2.5)
    lab = torch.zeros(R, dtype=torch.int64, device="cuda")
    lab[-200:] = torch.arange(200, device="cuda") % C
    logp, lse, H, tl, ti = sb.log_probs(z, lab, topk=2)
    dz = sb.log_probs_backward(z, lab, lse, d_logp=torch.ones_like(logp))
    torch.cuda.synchronize()
    for at in (slice(0, 200), slice(R // 2, R // 2 + 200), slice(R - 200, R)):
        r64, l64 = z[at].double().cpu(), lab[at].cpu()
        e_logp, e_lse, e_H, e_tl, e_ti = reference(r64, l64, 2, -100)
        close(logp[at], e_logp, 1e-4, "logp")
        close(H[at], e_H, 1e-4, "entropy")
        assert torch.equal(ti[at].cpu().long(), e_ti)
        ref, size = grad_reference(r64, l64, torch.ones(200, dtype=torch.float64), None, None, None, -100)
        close(dz[at], ref, 2.0 ** -11 * ref.abs() * (1 + 2.0 ** -8) + 2.0 ** -25 + 2.0 ** -16 * size, "dlogits")


@pytest.mark.parametrize("bad", ["labels type", "labels shape", "topk", "topk classes", "columns", "rows", "overlap",
                                 "no gradient", "entropy", "workspace", "dtype", "cpu"])
def test_refusals(bad):
    z = torch.randn(4, 30, device="cuda")
    lab = torch.zeros(4, dtype=torch.int64, device="cuda")
    lse = torch.zeros(4, device="cuda")
    with pytest.raises((ValueError, TypeError, RuntimeError)):
        if bad == "labels type":
            sb.log_probs(z, lab.int())
        elif bad == "labels shape":
            sb.log_probs(z, lab[:3])
        elif bad == "topk":
            sb.log_probs(torch.randn(2, 100, device="cuda"), topk=65)
        elif bad == "topk classes":
            sb.log_probs(z, topk=31)
        elif bad == "columns":
            sb.log_probs(z.t().contiguous().t())
        elif bad == "rows":
            sb.log_probs(z[:1].expand(4, 30))
        elif bad == "overlap":
            sb.log_probs_backward(z, lab, lse, d_logp=lse, out=z)
        elif bad == "no gradient":
            sb.log_probs_backward(z, lab, lse)
        elif bad == "entropy":
            sb.log_probs_backward(z, lab, lse, d_entropy=lse)
        elif bad == "workspace":
            sb.log_probs(torch.randn(1, 131072, device="cuda"), topk=5,
                         workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
        elif bad == "dtype":
            sb.log_probs(z.double())
        elif bad == "cpu":
            sb.log_probs(z.cpu())


def test_stream_capture_and_reproducibility():
    """A side stream, a captured graph replayed among eager work, and the same bits each time."""
    gen = torch.Generator().manual_seed(10)
    z, lab = tokens(2, 70001, "bf16", gen), labels_of((2,), 70001, gen, ignored=0.0)
    m = (torch.randn(1, 24, 32, 64, generator=gen)).half().cuda().contiguous(memory_format=torch.channels_last)[:, :19]
    ml = labels_of((1, 32, 64), 19, gen)

    def work():
        a = sb.log_probs(z, lab, topk=7)
        b = sb.log_probs(m, ml, topk=1, ignore=IGNORE)
        c = sb.log_probs_backward(m, ml, b[1], d_logp=torch.ones_like(b[1]), entropy=b[2], d_entropy=b[2], ignore=IGNORE)
        return [*a, *b, c]
    first = [x.clone() for x in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    keep = z.clone()
    for i in range(4):
        z.copy_(keep if i % 2 == 0 else -keep)
        graph.replay()
        torch.cuda.synchronize()
        eager = work()
        torch.cuda.synchronize()
        for x, y, w in zip(out, eager, first):
            assert torch.equal(x, y)
            assert i % 2 or torch.equal(x, w)
