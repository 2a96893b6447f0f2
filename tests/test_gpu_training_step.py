"""A training step through the framework's own calls: a block layer writes class
scores, their log probabilities are the loss, its gradient goes back through the
layer, and the filter is updated by its orthogonalised gradient.  Each link is
compared with 64 bits on the inputs that it had on the GPU, and the filter's
gradient as a whole with the CPU oracle's chain.

Tolerances: the links' own (tests of the single operators); the convolution and
its gradients meet 1e-4 of the largest value in fp32 (the library's bound for
them), and the softmax between them is a map of slope at most 1 with weights that
add up to at most 2 a pixel, so the chain's gradient is off by at most that bound
for the scores, once more for the gradient itself, and its share of the sum:
4e-4 of the largest value."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2011_12025_amd as sb
from paper_2011_12025_amd import inputs
from parity_util import log

pytestmark = pytest.mark.gpu

VOID, CLASSES, CHANNELS = 255, 19, 24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2011_12025_amd._binding as b
    b.lib()
    oracle.set_threads(0)


def step(x, mask, bs, w, bias, labels, rate=0.02):
    """Loss, gradients and the updated filter."""
    y = sb.layer(x, mask, bs, w, bias)
    scores = y[:, :CLASSES]
    logp, lse, H, _, best = sb.log_probs(scores, labels, topk=1, ignore=VOID)
    n = (labels != VOID).sum()
    g = torch.full_like(logp, -1.0) / n
    gh = torch.full_like(H, -0.05) / n  # a little entropy is kept
    dy = torch.zeros_like(y)
    sb.log_probs_backward(scores, labels, lse, d_logp=g, entropy=H, d_entropy=gh, ignore=VOID, out=dy[:, :CLASSES])
    dx, dw, db = sb.layer_backward(x, mask, bs, w, dy)
    update = sb.orthogonalize(dw)
    loss = -(logp.sum() + 0.05 * H.sum()) / n
    return dict(y=y, loss=loss, dy=dy, dx=dx, dw=dw, update=update, w=w - rate * update, best=best)


def softmax_gradient(y, labels):
    """d loss / d y in 64 bits (pixels last): the labels' log probabilities and 0.05 of the entropy."""
    z = y[:, :CLASSES]
    logq = z - z.max(1, keepdims=True)
    logq = logq - np.log(np.exp(logq).sum(1, keepdims=True))
    q = np.exp(logq)
    H = -(q * logq).sum(1, keepdims=True)
    keep = labels != VOID
    n = keep.sum()
    hot = np.zeros_like(z)
    np.put_along_axis(hot, np.where(keep, labels, 0)[:, None], 1.0, 1)
    d = np.zeros_like(y)
    d[:, :CLASSES] = (-(hot - q) * keep[:, None] + 0.05 * q * (logq + H)) / n
    loss = -((logq * hot).sum(1) * keep).sum() / n - 0.05 * H.sum() / n
    return loss, d


@pytest.mark.parametrize("layout", ["nhwc", "nchw"])
def test_step_against_the_oracle(layout):
    log(f"[training step] {layout}")
    N, C, Hh, Ww, bs = 2, 16, 32, 48, 8
    fmt = torch.channels_last if layout == "nhwc" else torch.contiguous_format
    mask = inputs.mask_bernoulli(3, N, Hh // bs, Ww // bs, 0.5)
    x = inputs.feature_map(3, N, C, Hh, Ww, "f32")
    w = inputs.conv_weight(3, CHANNELS, C, 3, "f32") * 3
    bias = inputs.conv_bias(3, CHANNELS, 9 * C, "f32")
    labels = np.random.default_rng(3).integers(0, CLASSES, (N, Hh, Ww))
    labels[np.random.default_rng(4).random(labels.shape) < 0.2] = VOID
    got = step(x.cuda().contiguous(memory_format=fmt), torch.from_numpy(mask).cuda(), bs,
               w.cuda().contiguous(memory_format=fmt), bias.cuda(), torch.from_numpy(labels).cuda())
    torch.cuda.synchronize()
    host = {k: v.detach().double().cpu() for k, v in got.items()}
    assert all(bool(v.isfinite().all()) for v in host.values())
    # the loss's gradient on the scores as the layer wrote them
    loss, d = softmax_gradient(host["y"].numpy(), labels)
    assert abs(loss - host["loss"].item()) < 1e-5 * (1 + abs(loss))
    n = (labels != VOID).sum()
    # (terms below 2 / n a pixel and 2^-16 of them, as in the operator's tests)
    assert np.abs(host["dy"].numpy() - d).max() < 2.0 ** -16 * 2.5 / n
    assert bool((host["dy"][:, CLASSES:] == 0).all())
    best = host["y"][:, :CLASSES].max(1)[0]
    assert torch.equal(host["y"].gather(1, host["best"].long()).squeeze(1), best)
    # the chain as a whole
    y = oracle.layer(x.numpy(), mask, bs, w.numpy(), bias.numpy(), "f32")
    _, d = softmax_gradient(np.asarray(y, dtype=np.float64), labels)
    rdx, rdw, _ = oracle.layer_backward(x.numpy(), mask, bs, w.numpy(), bias.numpy(), d.astype(np.float32), "f32")
    for name, ref in (("dx", rdx), ("dw", rdw)):
        assert np.abs(host[name].numpy() - ref).max() < 4e-4 * np.abs(ref).max(), name
    # the update of that gradient, and the filter
    g = host["dw"].reshape(CHANNELS, -1)
    u = g / (g.norm() + 1e-7)
    for _ in range(5):
        A = u @ u.t()
        u = 3.4445 * u + (-4.7750 * A + 2.0315 * (A @ A)) @ u
    off = (host["update"].reshape(CHANNELS, -1) - u).norm() / u.norm()
    assert off < 2e-5, off
    torch.testing.assert_close(host["w"], w.double() - 0.02 * host["update"], rtol=0, atol=1e-6)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_step_in_sixteen_bits(dtype):
    """The same calls in 16 bits on a stage-1 map: gradients finite, channels that are no classes without one, and
    the filter's update orthogonal up to what five steps leave (singular values in [0.6, 1.25])."""
    log(f"[training step] {dtype}")
    N, C, Hh, Ww, bs = 1, 64, 128, 256, 32
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(N, C, Hh, Ww, generator=gen).to(dtype).cuda().contiguous(memory_format=torch.channels_last)
    mask = (torch.rand(N, Hh // bs, Ww // bs, generator=gen) > 0.5).to(torch.uint8).cuda()
    w = (torch.randn(CHANNELS, C, 3, 3, generator=gen) * 0.1).to(dtype).cuda().contiguous(memory_format=torch.channels_last)
    labels = torch.randint(0, CLASSES, (N, Hh, Ww), generator=gen).cuda()
    # (a mean over 32768 pixels would be near the least value of fp16, so the loss is scaled as training does)
    y = sb.layer(x, mask, bs, w)
    scores = y[:, :CLASSES]
    logp, lse, H, _, _ = sb.log_probs(scores, labels, ignore=VOID)
    dy = torch.zeros_like(y)
    sb.log_probs_backward(scores, labels, lse, d_logp=torch.full_like(logp, -1 / 64), ignore=VOID, out=dy[:, :CLASSES])
    dx, dw, _ = sb.layer_backward(x, mask, bs, w, dy)
    update = sb.orthogonalize(dw)
    torch.cuda.synchronize()
    assert all(bool(v.isfinite().all()) for v in (logp, dy, dx, dw, update))
    assert bool((dw[CLASSES:] == 0).all()) and bool((update[CLASSES:] == 0).all())
    s = torch.linalg.svdvals(update[:CLASSES].reshape(CLASSES, -1).double().cpu())
    g = torch.linalg.svdvals(dw[:CLASSES].reshape(CLASSES, -1).double().cpu())
    # (directions below 1e-2 of the norm are not brought up to 1 by five steps)
    s = s[g > 1e-2 * g.norm()]
    assert s.numel() and s.min() > 0.6 and s.max() < 1.25
