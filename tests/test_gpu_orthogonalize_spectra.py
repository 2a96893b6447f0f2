"""GPU parity of the Newton-Schulz orthogonalisation where its rounding counts
most: flat, Gaussian, trained-like and steeply falling spectra, one to eight active
rows of equal norm or directions of equal weight, and coefficients with steep slopes, against the iteration in
64 bits on the CPU.

Tolerance (2-norms over that of the result).  The result's own rounding to its type
is computed from the exact result.  Before it, X after step k is off by what
matrices of 22 bits and a sign (2^-22 with what products drop and sums round) make
of a X + b A X + c A A X, whose terms have norms of at most |a|, |b| l, |c| l^2
times that of X (l the largest eigenvalue of A), and every later step multiplies an
error by at most the largest of its slopes: |f'(s)|, and the divided differences
|f(s) - f(t)| / |s - t| and (f(s) + f(t)) / (s + t) between the singular values s, t
(0 among them, for the directions that X has not), f(s) = a s + b s^3 + c s^5:
  2^-22 sum_k (|a_k| + |b_k| l_k + |c_k| l_k^2) |X_k| prod_{j > k} slope_j.
Nothing else is allowed for: no factor for random signs, none for a type.
"""
from __future__ import annotations

import pytest
import torch

import paper_2011_12025_amd as sb
from parity_util import log

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ABC = [(3.4445, -4.7750, 2.0315)] * 5
# a step of its own each, which begins with a slope of 8.3 at 0 and 24 at 1
STEEP = [(8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.5100),
         (2.3007, -1.6689, 0.4188)]
EPS = 1e-7


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2011_12025_amd._binding as b
    b.lib()


def iteration(g, coef, dtype=torch.float64):
    x = g.to(dtype)
    flip = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if flip else x
    x = x / (x.norm() + EPS)
    for a, b, c in coef:
        A = x @ x.t()
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.t() if flip else x


def off_before_rounding(g, coef):
    s = torch.linalg.svdvals(g.double())
    s = torch.cat([s / (s.norm() + EPS), torch.zeros(1, dtype=torch.float64)])
    made, slopes = [], []
    for a, b, c in coef:
        f = s * (a + s ** 2 * (b + c * s ** 2))
        top = s.max().item() ** 2
        made.append((abs(a) + abs(b) * top + abs(c) * top ** 2) * s.norm().item())
        apart, both = (s[:, None] - s[None]).abs(), s[:, None] + s[None]
        steep = (a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max()
        for num, den in (((f[:, None] - f[None]).abs(), apart), ((f[:, None] + f[None]).abs(), both)):
            steep = torch.maximum(steep, torch.where(den > 1e-9, num / den.clamp_min(1e-9), 0.0).max())
        slopes.append(steep.item())
        s = f
    total = 0.0
    for k, term in enumerate(made):
        for d in slopes[k + 1:]:
            term *= d
        total += term
    return 2.0 ** -22 * total / s.norm().item()


def spectra(m, n, gen):
    r, s = max(1, min(m, n) // 8), min(m, n)
    yield "gaussian", torch.randn(m, n, generator=gen)
    yield "trained", ((torch.randn(m, r, generator=gen) * torch.arange(1, r + 1).rsqrt()) @ torch.randn(r, n, generator=gen) +
                      0.5 * torch.randn(m, n, generator=gen))
    u, v = (torch.linalg.qr(torch.randn(k, s, generator=gen))[0] for k in (m, n))
    yield "flat", u @ v.t()
    yield "falling", (u * torch.logspace(0, -4, s)) @ v.t()
    for k in (1, 2, 4, 8):
        g = torch.zeros(m, n)
        rows = torch.randn(k, n, generator=gen)
        g[torch.randperm(m, generator=gen)[:k]] = rows / rows.norm(dim=1, keepdim=True)
        yield f"{k} rows", g
        yield f"{k} directions", u[:, :k] @ v[:, :k].t()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("coef", [ABC, STEEP, ABC[:3]], ids=["default", "steep", "three"])
@pytest.mark.parametrize("m,n", [(64, 576), (100, 90), (256, 256), (200, 700), (1030, 515), (1200, 1300)])
def test_spectra(m, n, coef, dtype):
    log(f"[orthogonalize] spectra of {m} x {n} {dtype}, {len(coef)} steps")
    for name, g in spectra(m, n, torch.Generator().manual_seed(m + n)):
        g = g.to(DT[dtype])
        exact = iteration(g, coef)
        got = sb.orthogonalize(g.cuda(), steps=len(coef), coefficients=coef, eps=EPS).double().cpu()
        size = exact.norm().item()
        allowed = (exact.to(DT[dtype]).double() - exact).norm().item() / size + off_before_rounding(g, coef)
        off = (got - exact).norm().item() / size
        assert off <= allowed, f"{name}: {off:.2e} off, {allowed:.2e} allowed"


@pytest.mark.parametrize("m,n", [(64, 576), (512, 1024), (300, 900)])
def test_bf16_results_are_the_exact_ones_rounded(m, n):
    """An iteration in 32 bits is off by d, and four times that where matrices have two bits fewer.  A value
    whose rounding that changes lies within d of a border of its step of 2 h, in d / h of all places: at most the
    mean of that share differs from the exact result rounded (twice what errors of either sign give)."""
    log(f"[orthogonalize] rounded results of {m} x {n}")
    for name, g in spectra(m, n, torch.Generator().manual_seed(7 * m + n)):
        if name[0].isdigit():  # (of few directions: their errors are no sample)
            continue
        g = g.bfloat16()
        exact = iteration(g, ABC)
        d = 4 * (iteration(g, ABC, torch.float32).double() - exact).norm().item() / exact.numel() ** 0.5
        half = torch.ldexp(torch.ones_like(exact), torch.frexp(exact)[1] - 9)  # (frexp: [0.5, 1), steps of 2^-8 of 1)
        share = (d / half).clamp_max(1.0).mean().item()
        got = sb.orthogonalize(g.cuda(), eps=EPS).cpu()
        differ = (got != exact.bfloat16()).double().mean().item()
        assert differ <= share, f"{name}: {differ:.2e} of the values differ, {share:.2e} allowed"


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_an_update_among_others(dtype):
    """The same update alone and beside smaller, larger, longer and many others: within the same tolerance
    (sums are split by the sizes of the call), and the others' values have no part in it."""
    log(f"[orthogonalize] one update in lists {dtype}")
    gen = torch.Generator().manual_seed(21)
    def random(m, n):
        return torch.randn(m, n, generator=gen).to(DT[dtype]).cuda()
    for m, n in [(64, 576), (40, 50), (200, 190), (512, 512)]:
        for name, g in spectra(m, n, gen):
            if name not in ("gaussian", "falling", "1 directions", "4 rows"):
                continue
            g = g.to(DT[dtype])
            exact = iteration(g, ABC)
            size = exact.norm().item()
            allowed = (exact.to(DT[dtype]).double() - exact).norm().item() / size + off_before_rounding(g, ABC)
            g = g.cuda()
            for others in ([], [(8, 20)], [(900, 900)], [(64, 9000)], [(1500, 1500), (70, 4000)], [(30, 40)] * 40):
                mats = [random(*s) for s in others]
                got = sb.orthogonalize([g] + mats, eps=EPS)[0]
                off = (got.double().cpu() - exact).norm().item() / size
                assert off <= allowed, f"{m} x {n} {name} beside {others}: {off:.2e} off, {allowed:.2e} allowed"
                assert torch.equal(got, sb.orthogonalize([g] + [2 * t + 1 for t in mats], eps=EPS)[0])
