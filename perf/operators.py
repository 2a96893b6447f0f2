"""The two ends of a training step around the block convolutions, and their serving forms.

Each case is one pass through an operator:

  log_probs   log probabilities of given labels, log-sum-exp, entropy and the top alternatives of every row of
              class scores (``log_probs``): rows are tokens [R, V] or the pixels of a map [N, C, H, W]
  log_grad    the gradient of those results with respect to the scores (``log_probs_backward``)
  orth        a filter's gradient orthogonalised by Newton-Schulz products (``orthogonalize``): one filter, a
              batch of matrices, or all filters of an encoder in one call

A case is a dict of plain values.  ``of`` is the number of channels (or vocabulary entries) of the buffer whose
first C are the classes: a convolution writes multiples of eight channels, a vocabulary is padded.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def _tokens(kind, dtype, rows, classes, **more):
    return dict({"kind": kind, "dtype": dtype, "form": "tokens", "rows": rows, "classes": classes, "of": classes, "top": 0,
                 "entropy": True, "ignored": 0.0, "masked": 0.0}, **more)


def _pixels(kind, dtype, N, classes, H, W, layout, **more):
    return dict({"kind": kind, "dtype": dtype, "form": "map", "N": N, "classes": classes, "of": classes, "H": H, "W": W,
                 "layout": layout, "top": 0, "entropy": True, "ignored": 0.1, "masked": 0.0}, **more)


def _orth(dtype, m, n, **more):
    return dict({"kind": "orth", "dtype": dtype, "m": m, "n": n, "k": 0, "batch": 0, "steps": 5, "set": "one"}, **more)


def listed():
    return [
        # one generated token and its five best alternatives: latency counts
        dict(_tokens("log_probs", "f32", 1, 32000, top=5), name="token_f32"),
        # a decoding batch whose grammar masks a third of the vocabulary, 20 alternatives, an odd vocabulary
        dict(_tokens("log_probs", "bf16", 64, 50001, top=20, masked=0.33), name="decode_top20_bf16"),
        # a training batch over a large vocabulary
        dict(_tokens("log_probs", "bf16", 2048, 131072, ignored=0.05), name="train_bf16"),
        # the classes of every pixel of a 1024x2048 image: the prediction and how sure it is, 19 classes in 24 channels
        dict(_pixels("log_probs", "f16", 1, 19, 1024, 2048, "nhwc", of=24, top=1), name="pixels_nhwc_f16"),
        # training maps at a quarter of the resolution in torch's own format and type, three alternatives
        dict(_pixels("log_probs", "f32", 4, 19, 256, 512, "nchw", top=3), name="pixels_nchw_f32"),
        # the loss's gradient on the map that the last block convolution wrote
        dict(_pixels("log_grad", "f16", 1, 19, 256, 512, "nhwc", of=24, entropy=False), name="pixels_grad_f16"),
        # the gradient of a training batch with an entropy term
        dict(_tokens("log_grad", "bf16", 2048, 131072, ignored=0.05), name="train_grad_bf16"),
        # a distillation step: gradients of the alternatives too, odd sizes, 32 bits
        dict(_tokens("log_grad", "f32", 333, 5003, top=4), name="ragged_grad_f32"),
        # one filter of the first stage: latency counts
        dict(_orth("f16", 64, 64, k=3), name="filter_stage1_f16"),
        # every filter of the ResNet-18 encoder, as one optimiser step has them
        dict(_orth("bf16", 0, 0, set="encoder"), name="encoder_filters_bf16"),
        # a large square matrix
        dict(_orth("bf16", 4096, 4096), name="square_bf16"),
        # a tall matrix with odd sides and a 32-bit gradient
        dict(_orth("f32", 3001, 701), name="tall_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["log_probs", "log_probs", "log_grad", "orth"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind == "orth":
        s = _log_int(rng, 1, 2048)
        # at most the work of the largest listed case
        n = min(_log_int(rng, s, 16 * s + 64), 16384)
        m, n = (s, n) if rng.random() < 0.6 else (n, s)
        batch = rng.choice([0, 0, 1, 3, 8]) if s <= 512 else 0
        return _orth(dtype, m, n, batch=batch, steps=rng.choice([3, 5, 5, 6]))
    entropy, ignored, masked = rng.random() < 0.7, rng.choice([0.0, 0.1, 0.5]), rng.choice([0.0, 0.0, 0.3, 0.9])
    if rng.random() < 0.5:
        classes = _log_int(rng, 2, 200000)
        rows = _log_int(rng, 1, min(4096, max(1, 120_000_000 // classes)))
        c = _tokens(kind, dtype, rows, classes)
    else:
        classes = _log_int(rng, 2, 1000)
        H, W = _log_int(rng, 1, 512), _log_int(rng, 1, 512)
        N = max(1, min(rng.choice([1, 2, 4]), 60_000_000 // (classes * H * W)))
        c = _pixels(kind, dtype, N, classes, H, W, rng.choice(["nhwc", "nchw"]))
        if classes * H * W > 60_000_000:
            c["classes"] = c["of"] = classes = 60_000_000 // (H * W)
    of = classes if rng.random() < 0.6 else (classes + 7) // 8 * 8
    return dict(c, of=of, top=min(classes, rng.choice([0, 0, 1, 3, 20])), entropy=entropy, ignored=ignored, masked=masked)


IGNORE = 255  # the label of a pixel or token that does not count; no case has that class drawn as a label


def _shape(case):
    """(shape of the scores' buffer, dimension of the classes)."""
    if case["form"] == "tokens":
        return (case["rows"], case["of"]), 1
    return (case["N"], case["of"], case["H"], case["W"]), 1


def _encoder_shapes():
    shapes, cin = [], 64
    for width in (64, 128, 256, 512):
        for i in range(4):
            shapes.append((width, cin if i == 0 else width, 3, 3))
        if cin != width:
            shapes.append((width, cin, 1, 1))
        cin = width
    return shapes


def _gradient(shape, gen, dtype):
    """A gradient as training gives it: a few strong directions over noise, small values."""
    m, n = shape[0], math.prod(shape[1:])
    r = max(1, min(m, n) // 8)
    g = torch.randn(m, r, generator=gen, device="cuda") * torch.arange(1, r + 1, device="cuda").rsqrt()
    g = g @ torch.randn(r, n, generator=gen, device="cuda") + 0.5 * torch.randn(m, n, generator=gen, device="cuda")
    return (g * 1e-3).reshape(shape).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    state = {"case": case}
    if own:
        import paper_2011_12025_amd as sb
        state["sb"] = sb
    if case["kind"] == "orth":
        if case["set"] == "encoder":
            state["updates"] = [_gradient(s, gen, dtype).contiguous(memory_format=torch.channels_last)
                                for s in _encoder_shapes()]
        elif case["k"]:
            g = _gradient((case["m"], case["n"], case["k"], case["k"]), gen, dtype)
            state["updates"] = [g.contiguous(memory_format=torch.channels_last)]
        elif case["batch"]:
            state["updates"] = [torch.stack([_gradient((case["m"], case["n"]), gen, dtype) for _ in range(case["batch"])])]
        else:
            state["updates"] = [_gradient((case["m"], case["n"]), gen, dtype)]
        return state
    shape, dim = _shape(case)
    C = case["classes"]
    z = torch.empty(shape, dtype=dtype, device="cuda",
                    memory_format=torch.channels_last if case.get("layout") == "nhwc" else torch.contiguous_format)
    z.normal_(0.0, 2.5, generator=gen)
    if case["masked"]:  # a grammar's or a task's forbidden classes, other ones in every row
        hide = torch.zeros(shape, dtype=torch.uint8, device="cuda").bernoulli_(case["masked"], generator=gen)
        hide.select(dim, 0).zero_()
        z.masked_fill_(hide.bool(), -math.inf)
        del hide
    z = z.narrow(dim, 0, C)
    rows = z.shape[:1] + z.shape[2:]
    labels = torch.randint(0, C, rows, generator=gen, device="cuda")
    if case["masked"]:  # what was sampled was allowed
        labels = torch.where(z.gather(dim, labels.unsqueeze(dim)).squeeze(dim) == -math.inf, 0, labels)
    labels = torch.where(labels == IGNORE, 0, labels)
    if case["ignored"]:
        labels[torch.zeros(rows, device="cuda").bernoulli_(case["ignored"], generator=gen).bool()] = IGNORE
    state.update(z=z, labels=labels)
    if case["kind"] == "log_grad":
        with torch.no_grad():
            _, lse, H, _, index = _log_probs(z, labels, case["top"], True)
        state["lse"] = lse
        state["d_logp"] = torch.randn(rows, generator=gen, device="cuda") * 0.1 - 1.0
        if case["entropy"]:
            state.update(H=H, d_H=torch.randn(rows, generator=gen, device="cuda") * 0.1)
        if case["top"]:
            state.update(index=index, d_top=torch.randn(index.shape, generator=gen, device="cuda") * 0.1)
    return state


def _log_probs(z, labels, top, entropy):
    z = z.float()
    m = z.amax(1, keepdim=True)
    d = z - m
    e = d.exp()
    s = e.sum(1, keepdim=True)
    logs = s.log()
    ignored = labels == IGNORE
    t = d.gather(1, torch.where(ignored, 0, labels).unsqueeze(1)) - logs
    logp = torch.where(ignored, 0.0, t.squeeze(1))
    H = None
    if entropy:
        # a class of probability zero adds nothing
        H = (logs - (e * torch.where(e > 0, d, 0.0)).sum(1, keepdim=True) / s).squeeze(1)
    top_logp = index = None
    if top:
        # equal scores: the lower class first
        index = d.argmax(1, keepdim=True) if top == 1 else d.sort(dim=1, descending=True, stable=True)[1].narrow(1, 0, top)
        top_logp = d.gather(1, index) - logs
        index = index.int()
    return logp, (m + logs).squeeze(1), H, top_logp, index


def _log_grad(state):
    z, labels, dtype = state["z"].float(), state["labels"], state["z"].dtype
    ignored = labels == IGNORE
    d = z - state["lse"].unsqueeze(1)
    p = d.exp()
    g_l = torch.where(ignored, 0.0, state["d_logp"]).unsqueeze(1)
    G = g_l + state["d_top"].sum(1, keepdim=True) if "d_top" in state else g_l
    if "d_H" in state:
        G = G + state["d_H"].unsqueeze(1) * (torch.where(p > 0, d, 0.0) + state["H"].unsqueeze(1))
    dz = -p * G
    dz.scatter_add_(1, torch.where(ignored, 0, labels).unsqueeze(1), g_l)
    if "d_top" in state:
        dz.scatter_add_(1, state["index"].long(), state["d_top"])
    return dz.to(dtype)


def _orthogonalize(g, steps):
    a, b, c = COEFFICIENTS
    x = (g if g.dim() == 3 else g.reshape(1, g.shape[0], -1)).float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):  # the iteration itself
        A = x @ x.transpose(1, 2).contiguous()
        x = a * x + (b * A + c * (A @ A)) @ x
    if tall:
        x = x.transpose(1, 2)
    return x.reshape(g.shape).to(g.dtype)


def run(state):
    case = state["case"]
    if case["kind"] == "log_probs":
        if own:
            return state["sb"].log_probs(state["z"], state["labels"], topk=case["top"], entropy=case["entropy"], ignore=IGNORE)
        return _log_probs(state["z"], state["labels"], case["top"], case["entropy"])
    if case["kind"] == "log_grad":
        if own:
            return state["sb"].log_probs_backward(state["z"], state["labels"], state["lse"], d_logp=state["d_logp"],
                                                  entropy=state.get("H"), d_entropy=state.get("d_H"),
                                                  top_index=state.get("index"), d_top=state.get("d_top"), ignore=IGNORE)
        return _log_grad(state)
    if own:
        return state["sb"].orthogonalize(state["updates"], steps=case["steps"], coefficients=COEFFICIENTS, eps=EPS)
    return [_orthogonalize(g, case["steps"]) for g in state["updates"]]


def _matrices(case):
    """(rows, columns) of every matrix of an orth case."""
    if case["set"] == "encoder":
        return [(s[0], math.prod(s[1:])) for s in _encoder_shapes()]
    return [(case["m"], case["n"] * max(1, case["k"]) ** 2)] * max(1, case["batch"])


def work(case):
    es, k = SIZES[case["dtype"]], case.get("top", 0)
    if case["kind"] == "orth":
        # with X = Q X0, Q a polynomial of A = X0 X0^T: A once and Q X0 once on the long side, four products a step on
        # the short one (A A, P Q, P A, P A P; fewer in the first and the last step); half of a symmetric product
        nbytes = flops = 0
        for m, n in _matrices(case):
            s, L = min(m, n), max(m, n)
            nbytes += 2 * m * n * es
            flops += 3 * s * s * L + max(1, 4 * case["steps"] - 3) * s ** 3
        return {"bytes": nbytes, "flops": flops}
    rows = case["rows"] if case["form"] == "tokens" else case["N"] * case["H"] * case["W"]
    values = rows * case["classes"]
    if case["kind"] == "log_probs":
        return {"bytes": values * es + rows * (8 + 8 + 4 * case["entropy"] + 8 * k), "flops": 6 * values}
    return {"bytes": 2 * values * es + rows * (16 + 8 * case["entropy"] + 8 * k), "flops": 6 * values}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "orth":
        return [_exact_orth(g, case["steps"]) for g in state["updates"]]
    # the classes last, in pieces of rows that 64 bits have room for
    z = state["z"].movedim(1, -1)
    C, lead = z.shape[-1], z.shape[:-1]
    z, labels = z.reshape(-1, C), state["labels"].reshape(-1)
    step = max(1, 100_000_000 // C)
    parts = [_exact_rows(case, state, z, labels, slice(i, i + step)) for i in range(0, z.shape[0], step)]

    def whole(k):
        if parts[0][k] is None:
            return None
        x = torch.cat([p[k] for p in parts])
        x = x.reshape(lead + x.shape[1:])
        return x if x.dim() == len(lead) else x.movedim(-1, 1)
    if case["kind"] == "log_grad":
        return whole(0)
    return whole(0), whole(1), whole(2), whole(3), None


def _exact_rows(case, state, z, labels, at):
    z, labels = z[at].double(), labels[at]
    n = torch.arange(z.shape[0], device=z.device)
    lse = torch.logsumexp(z, 1)
    logq = z - lse[:, None]
    q = logq.exp()
    counts = labels != IGNORE
    t = labels.masked_fill(~counts, 0)
    entropy = torch.special.entr(q).sum(1)
    if case["kind"] == "log_probs":
        top = logq.topk(case["top"], 1)[0] if case["top"] else None
        return logq[n, t] * counts if not case["masked"] else torch.where(counts, logq[n, t], 0.0), lse, (
            entropy if case["entropy"] else None), top

    # the definition: the gradient of  sum g_l log q_t + sum g_H H + sum g_i log q_i  by the softmax's Jacobian
    def rows_of(x):
        x = x if x.dim() == labels.dim() or x.dim() < 3 else x.movedim(1, -1) if x.dim() == 4 else x
        return x.reshape(-1, *x.shape[len(state["labels"].shape):])[at]
    u = torch.zeros_like(z)  # the derivative with respect to log q, weighted
    u[n, t] += rows_of(state["d_logp"]).double() * counts
    if "d_top" in state:
        for i in range(case["top"]):
            u[n, rows_of(state["index"])[:, i].long()] += rows_of(state["d_top"])[:, i].double()
    dz = u - q * u.sum(1, keepdim=True)
    if "d_H" in state:
        dz -= rows_of(state["d_H"]).double()[:, None] * (q * entropy[:, None] - torch.special.entr(q))
    return (dz,)


def _exact_orth(g, steps):
    a, b, c = COEFFICIENTS
    y = (g if g.dim() == 3 else g.reshape(1, g.shape[0], -1)).double()
    flip = y.shape[1] > y.shape[2]
    y = y.transpose(1, 2) if flip else y
    y = y / (torch.linalg.vector_norm(y, dim=(1, 2), keepdim=True) + EPS)
    out = []
    for x in y:
        # through the smaller side alone: X = Q X0, where Q and A = X X^T are polynomials of X0 X0^T
        x0, A, Q = x, x @ x.t(), torch.eye(x.shape[0], dtype=x.dtype, device=x.device)
        for _ in range(steps):
            P = c * (A @ A) + b * A
            P.diagonal().add_(a)
            Q, A = P @ Q, P @ A @ P
        out.append(Q @ x0)
    y = torch.stack(out)
    return (y.transpose(1, 2) if flip else y).reshape(g.shape)
