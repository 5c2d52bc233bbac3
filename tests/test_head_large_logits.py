"""Gradients of the classifier-head operators where a row's logits are large: log-sum-exp in float32 no longer holds the
logarithm of the sum beside them.  References take the largest logit out first, in 64 bits.  Run with -m gpu."""
import math

import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1909_11985_amd as E
    return E


def softmax64(z):
    """(z - max, log p, p, entropy) of float64 rows; a class at -inf has p = 0 and log p = 0 here."""
    d = z - z.amax(1, keepdim=True)
    log_s = d.exp().sum(1, keepdim=True).log()
    masked = z == -math.inf
    lp = torch.where(masked, torch.zeros_like(z), d - log_s)
    p = torch.where(masked, torch.zeros_like(z), lp.exp())
    return d, lp, p, -(p * lp).sum(1)


def gradient64(z, t, g, h):
    """dz of float64 logits, and how far float32 arithmetic from the largest logit on may be off.

    log p = (z - m) - log s: a step of 2^-24 for the difference (|d|) and for log s; s itself is off by 2^-24 for about
    sqrt(n / 64) of the additions that follow each other, the logarithm, the exponential and its argument's factor by a few
    steps.  That is p's relative error; entropy has the same relative to log n.  Rows whose lse is below 128 take their log p
    from it: half a step of it, 2^-24 x 64, more."""
    n = z.shape[1]
    d, lp, p, H = softmax64(z)
    hot = torch.zeros_like(z)
    has = (t >= 0) & (t < n)
    hot[has.nonzero()[:, 0], t[has].long()] = 1.0
    g = torch.where(has, g.double(), torch.zeros_like(H))[:, None]
    h, H = h.double()[:, None], H[:, None]
    dz = g * (hot - p) - h * p * (lp + H)
    dz = torch.where((g == 0) & (h == 0), torch.zeros_like(dz), dz)
    lse = (z.amax(1) + d.exp().sum(1).log())[:, None]
    step = 2.0 ** -24
    eps = step * (torch.where(z == -math.inf, torch.zeros_like(d), d.abs()).clamp(max=200.0) * 2 + 3 * math.log(n) + math.sqrt(n / 64) + 16 +
                  torch.where(lse.abs() < 128, torch.full_like(lse, 64.0), torch.zeros_like(lse)))
    parts = g.abs() * (hot + p) + h.abs() * p * (lp.abs() + H + 1)
    return dz, parts, eps


def rows_like(kind, rows, classes, dtype, gen):
    big = torch.finfo(DT[dtype]).max
    if kind == "lowest":
        z = torch.full((rows, classes), -big)
    elif kind == "largest":
        z = torch.full((rows, classes), big)
    elif kind == "few_of_largest":         # the rest at the other end
        z = torch.full((rows, classes), -big)
        z[:, ::3] = big
    elif kind == "mixed":                  # ordinary rows between large ones, masked classes, rows that count for nothing
        z = torch.randn(rows, classes, generator=gen) * 2
        z[::2] += 5000.0
        z[::3, 1::2] = -math.inf
        z[1::4] = -70000.0
    elif kind == "border":                 # lse on both sides of 128
        z = torch.randn(rows, classes, generator=gen) * 0.5
        z += (128.0 - math.log(classes) + torch.linspace(-2, 2, rows))[:, None]
        z[1::2] = -z[1::2] - 2 * math.log(classes)
    else:
        z = torch.full((rows, classes), float(kind))
        z[1::2] += torch.randn(z[1::2].shape, generator=gen)
    return z.to(DT[dtype])


KINDS = ["lowest", "largest", "few_of_largest", "mixed", "border", "1e4", "-1e5", "1e6"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,classes,pad", [(5, 1, 0), (6, 70, 3), (8, 1024, 0), (8, 1025, 1), (7, 9001, 0), (2, 200003, 5)])
def test_gradient_of_large_logits(E, dtype, kind, rows, classes, pad):
    gen = torch.Generator().manual_seed(classes + rows)
    z = rows_like(kind, rows, classes, dtype, gen)
    t = torch.randint(0, classes, (rows,), generator=gen, dtype=torch.int32)
    t[rows // 2] = -1
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    g[1] = h[1] = 0.0
    buf = torch.full((rows, classes + pad), 7.0, dtype=DT[dtype]).cuda()
    zd = buf[:, :classes]
    zd.copy_(z)
    r = E.edl_log_probs(zd, t.cuda())
    want, parts, eps = gradient64(z.double(), t, g, h)
    got = E.edl_log_probs_backward(zd, t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda())
    off = (got.cpu().double() - want).abs() - R.EPS[DT[dtype]] * want.abs() - parts * eps
    assert float(off.max()) <= 1e-37, float(off.max())
    assert bool((got[1] == 0).all())
    again = E.edl_log_probs_backward(zd, t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda(), out=zd)       # in place
    assert again is zd and torch.equal(zd, got) and bool((buf[:, classes:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(9000, 40), (2300, 1700), (70001, 9), (700, 3001)])
def test_gradient_of_many_rows_of_large_logits(E, dtype, rows, classes):
    """More rows than there are blocks for them."""
    gen = torch.Generator().manual_seed(classes)
    z = rows_like("mixed", rows, classes, dtype, gen)
    t = torch.randint(-1, classes, (rows,), generator=gen, dtype=torch.int32)
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    zd = z.cuda()
    r = E.edl_log_probs(zd, t.cuda())
    want, parts, eps = gradient64(z.double(), t, g, h)
    got = E.edl_log_probs_backward(zd, t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda())
    off = (got.cpu().double() - want).abs() - R.EPS[DT[dtype]] * want.abs() - parts * eps
    assert float(off.max()) <= 1e-37, float(off.max())
    assert torch.equal(E.edl_log_probs_backward(zd, t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda(), out=zd), got)


def test_gradient_of_large_logits_in_a_replayed_graph(E):
    """Which rows are large is found on the device: replays follow it."""
    gen = torch.Generator().manual_seed(8)
    z = (torch.randn(6, 3000, generator=gen) * 2).cuda()
    t = torch.tensor([0, 5, -1, 2999, 7, 8], dtype=torch.int32).cuda()
    g, h = torch.randn(6, generator=gen).cuda(), torch.randn(6, generator=gen).cuda()

    def call():
        r = E.edl_log_probs(z, t)
        return E.edl_log_probs_backward(z, t, r.lse, r.entropy, g, h)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(4):
        z[i] += (-1.0) ** i * 10.0 ** (i + 3)
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want), i
        exact, parts, eps = gradient64(z.cpu().double(), t.cpu(), g.cpu(), h.cpu())
        assert bool(((held.cpu().double() - exact).abs() <= parts * (eps + 2.0 ** -24) + 1e-37).all()), i


# Features and weights of small whole numbers, so that x w^T is exact, and with it z = x w^T + b for a whole b of up to 2^23;
# a bias of the type's lowest value takes x w^T in.
def whole_case(seed, dtype, rows, dim, classes):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randint(-1, 2, (rows, dim), generator=gen).to(DT[dtype])
    w = torch.randint(-1, 2, (classes, dim), generator=gen).to(DT[dtype])
    t = torch.randint(-1, classes, (rows,), generator=gen, dtype=torch.int32)
    return x, w, t, gen


def check_grads(E, x, w, b, t, z, g, h):
    """z: the exact logits, in float64; the reference is formed where it lies."""
    dev, back = (lambda v: v.cuda()), (lambda v: v.to(z.device).double())         # noqa: E731
    r = E.edl_classifier_log_probs(dev(x), dev(w), dev(b), dev(t))
    dx, dw, db = E.edl_classifier_log_probs_backward(dev(x), dev(w), dev(b), dev(t), r.lse, r.entropy, dev(g), dev(h))
    dz, parts, eps = gradient64(z, t.to(z.device), g.to(z.device), h.to(z.device))
    rows, classes = z.shape
    xc, wc = back(x), back(w)
    # dz is stored as three bf16 numbers (2^-24), of which dx of bf16 takes two (2^-16); sums of n float32 terms
    sums = lambda n: 2.0 ** -24 * (math.sqrt(n) + 8)            # noqa: E731
    two = 2.0 ** -16 if x.dtype == torch.bfloat16 else 0.0
    lost = parts * eps
    want = dz @ wc
    assert bool(((back(dx) - want).abs() <= lost @ wc.abs() + (parts @ wc.abs()) * (two + sums(classes)) + R.EPS[x.dtype] * want.abs() + 1e-36).all())
    want = dz.t() @ xc
    assert bool(((back(dw) - want).abs() <= lost.t() @ xc.abs() + (parts.t() @ xc.abs()) * sums(rows) + 1e-36).all())
    assert bool(((back(db) - dz.sum(0)).abs() <= lost.sum(0) + parts.sum(0) * sums(rows) + 1e-36).all())


WHOLE = [(3, 8, 40001), (1, 8, 5), (8, 64, 10), (3, 16, 3000), (31, 40, 24001), (100, 64, 1000), (40, 8, 5000), (5000, 8, 12), (300, 64, 8300), (129, 24, 12500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bias", [1e4, -1e5, 1e6, -4e6, "lowest", "half_lowest"])
@pytest.mark.parametrize("rows,dim,classes", WHOLE)
def test_classifier_gradients_of_large_logits(E, dtype, bias, rows, dim, classes):
    x, w, t, gen = whole_case(rows + classes, dtype, rows, dim, classes)
    lowest = torch.finfo(torch.float32).min
    z = x.double() @ w.double().t()
    if isinstance(bias, float):
        b = bias + torch.randint(-4, 5, (classes,), generator=gen).float()
        z = z + b.double()
    else:
        b = torch.full((classes,), lowest)
        if bias == "half_lowest":
            b[1::2] = -math.inf
        z = b.double().expand(rows, classes).clone()
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    if bias == "half_lowest":
        t = torch.where((t >= 0) & (t % 2 == 1), t - 1, t)
    check_grads(E, x, w, b, t, z, g, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes", [c for c in WHOLE if c[0] > 1] + [(32, 8, 33000)])
def test_classifier_gradients_of_some_rows_of_large_logits(E, dtype, rows, dim, classes):
    """A feature that some rows have lifts all of their logits; the others stay as small as they were."""
    x, w, t, gen = whole_case(rows * 3 + classes, dtype, rows, dim, classes)
    x[:, 0] = 0
    x[::5, 0] = 1
    w[:, 0] = 131072
    b = torch.randint(-4, 5, (classes,), generator=gen).float()
    z = x.double() @ w.double().t() + b.double()
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    check_grads(E, x, w, b, t, z, g, h)       # (131,072 stands in w: dx's first column is a sum of parts as large)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes,every", [(1100, 64, 13000, 1), (1100, 64, 13000, 300), (16400, 24, 11003, 1), (16400, 24, 11003, 1000)])
def test_classifier_gradients_of_large_logits_on_large_tiles_and_in_pieces(E, dtype, rows, dim, classes, every):
    """256x256 tiles, and more of dz than is held at a time; all rows or few of them have large logits.  The reference is formed on the GPU."""
    x, w, t, gen = whole_case(rows + every, dtype, rows, dim, classes)
    x[:, 0] = 0
    x[every // 2::every, 0] = 1
    w[:, 0] = -65536
    b = torch.randint(-4, 5, (classes,), generator=gen).float()
    z = x.cuda().double() @ w.cuda().double().t() + b.cuda().double()
    check_grads(E, x, w, b, t, z, torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3)
