"""The operators of a classifier's head on an MI355X against plain references in 64 bits.  Run with -m gpu."""
import math

import numpy as np
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


def rows_of(gen, rows, cols, pad, dtype, size=1.0, offset=0):
    """A [rows][cols] view on the GPU whose rows lie cols + pad apart and start `offset` elements into their buffer, and the
    buffer: what lies between the rows must stay as it is."""
    buf = (torch.randn(offset + rows * (cols + pad), generator=gen) * size).to(DT[dtype]).cuda()
    return buf[offset:].view(rows, cols + pad)[:, :cols] if rows else buf[:0].view(0, cols), buf


def same_bits(a, b):
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.contiguous().view(kind).cpu(), b.contiguous().view(kind).cpu())


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,offset,rate,first", [
    (1, 1, 0, 0, 0.5, 0), (3, 2, 0, 0, 0.5, 7), (1, 7, 0, 0, 0.25, 0), (5, 8, 0, 0, 0.1, 0), (64, 9, 3, 1, 0.9, 1 << 40),
    (1000, 1, 2, 3, 0.5, 5), (37, 255, 1, 0, 0.3, 0), (300, 24, 0, 0, 0.5, 0), (33, 2047, 0, 1, 0.5, 2 ** 62), (32, 4096, 0, 0, 0.5, 0),
    (7, 8193, 5, 1, 0.2, 11), (700, 2048, 0, 0, 0.75, 3), (2100, 1000, 24, 0, 0.5, 9), (600, 4097, 1, 1, 0.1, 0), (140000, 16, 0, 0, 0.5, 0)])
def test_dropout_is_its_definition_to_the_bit(E, dtype, rows, cols, pad, offset, rate, first):
    """Small calls (one piece per lane) and large ones (four), rows shorter and longer than a block, unaligned ones; the same
    into a padded result and in place."""
    gen = torch.Generator().manual_seed(rows * 131 + cols)
    x, buf = rows_of(gen, rows, cols, pad, dtype, offset=offset)
    key = R.draw(99, rows + cols)
    want = R.dropout(x.cpu(), rate, key, first)
    assert same_bits(E.edl_dropout(x, rate, key, first_row=first), want)
    out, obuf = rows_of(gen, rows, cols, 5, dtype, offset=1)
    before = obuf.clone()
    assert E.edl_dropout(x, rate, key, first_row=first, out=out) is out
    assert same_bits(out, want)
    out.copy_(before[1:].view(rows, cols + 5)[:, :cols])
    assert same_bits(obuf, before)                  # nothing beside the rows was touched
    before = buf.clone()
    E.edl_dropout(x, rate, key, first_row=first, out=x)
    assert same_bits(x, want)
    x.copy_(before[offset:].view(rows, cols + pad)[:, :cols])
    assert same_bits(buf, before)


def test_dropout_keeps_its_share_and_rate_zero_everything(E):
    x = torch.ones(512, 4096, device="cuda")
    for rate in (0.1, 0.5, 0.9):
        n = int((E.edl_dropout(x, rate, E.edl_dropout_key(3, 4, 5)) != 0).sum())
        want, spread = x.numel() * (1 - rate), (x.numel() * rate * (1 - rate)) ** 0.5
        assert abs(n - want) < 6 * spread, (rate, n)
    y = torch.randn(3, 5, device="cuda")
    assert same_bits(E.edl_dropout(y, 0.0, 1), y)


def test_dropout_drops_what_is_not_finite(E):
    """A dropped element is +0 whatever it held; a kept one stays what it is."""
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    x[1::4] = -1e30
    y = E.edl_dropout(x, 0.5, 12345).cpu()
    assert same_bits(y, R.dropout(x.cpu(), 0.5, 12345))
    assert not torch.isnan(y[torch.from_numpy(~R.kept(64, 64, 0.5, 12345))]).any()


def test_dropout_of_rows_in_parts_has_the_masks_of_the_whole(E):
    x = torch.randn(100, 333, device="cuda")
    whole = E.edl_dropout(x, 0.5, 77, first_row=10)
    parts = [E.edl_dropout(x[a:b], 0.5, 77, first_row=10 + a) for a, b in ((0, 1), (1, 40), (40, 100))]
    assert same_bits(torch.cat(parts), whole)


def test_dropout_on_another_stream_and_in_a_replayed_graph(E):
    x = torch.randn(257, 1025, device="cuda")
    want = R.dropout(x.cpu(), 0.5, 5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = E.edl_dropout(x, 0.5, 5, stream=side.cuda_stream)
    side.synchronize()
    assert same_bits(y, want)
    with torch.cuda.stream(side):
        E.edl_dropout(x, 0.5, 5)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = E.edl_dropout(x, 0.5, 5)
    for i in range(3):
        x.mul_(-2.0)
        y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same_bits(y, R.dropout(x.cpu(), 0.5, 5)), i


def test_dropout_of_nothing(E):
    for shape in ((0, 5), (5, 0), (0, 0)):
        assert E.edl_dropout(torch.empty(*shape, device="cuda"), 0.5, 1).shape == shape


# ---------------------------------------------------------------- log probabilities
# Float32 sums of n terms each: an absolute error of the logit's rounding, 2^-24 (|z| + |lse|) for the difference z - lse, and
# of the sum's relative error.  Terms are joined over lanes of at most ~n / 64 / parts sequential additions of 2^-24 each, plus
# the exponential's 2 ulp and its argument's 2^-24 |z - m|: (n / 64 + 2 + |z - m|) 2^-24, n <= 200,000 -> 2e-4 worst case of
# all errors aligned; they are not, their signs alternate, and the root of n / 64 stands for n / 64.
def stat_tolerance(z, classes):
    finite = torch.where(torch.isfinite(z), z.abs(), torch.zeros_like(z))
    return 2.0 ** -24 * (4 + (classes / 64) ** 0.5 + 4 * float(finite.max()))


def logits_of(gen, rows, classes, pad, dtype, size=3.0, masked=0.0, offset=0):
    z, buf = rows_of(gen, rows, classes, pad, dtype, size, offset)
    if masked:
        z[torch.rand(rows, classes, generator=gen).cuda() < masked] = -float("inf")
    return z, buf


def targets_of(gen, rows, classes):
    t = torch.randint(0, classes, (rows,), generator=gen, dtype=torch.int32)
    t[torch.rand(rows, generator=gen) < 0.2] = -1
    return t


def check_stats(r, want, tol, top):
    log_prob, entropy, lse, top_lp, top_cls = want
    for got, ref in ((r.log_prob, log_prob), (r.entropy, entropy), (r.lse, lse)) + (((r.top_log_prob, top_lp),) if top else ()):
        if got is None:
            assert ref is None
            continue
        got = got.cpu().double()
        fine = torch.isfinite(ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[got.isinf()], ref[ref.isinf()])
        assert torch.equal(torch.isfinite(got), fine)
        if fine.any():
            assert float((got - ref)[fine].abs().max()) <= tol
    if top:
        assert torch.equal(r.top_class.cpu(), top_cls)


SHAPES = [(1, 1, 0, 0, 1, 0), (1, 2, 0, 0, 2, 0), (5, 3, 0, 0, 1, 1), (9, 10, 0, 0, 0, 0), (256, 1000, 0, 0, 5, 0), (3, 1023, 1, 1, 64, 0.3), (6, 1024, 0, 0, 3, 0),
          (6, 1025, 0, 1, 3, 0.9), (2, 4097, 3, 1, 20, 0), (1, 32000, 0, 0, 5, 0), (3, 50001, 5, 1, 40, 0.3), (700, 2051, 0, 0, 7, 0), (65, 8200, 8, 0, 64, 0),
          (1, 200003, 0, 1, 64, 0), (1030, 1500, 0, 0, 0, 0.5), (4, 4096, 0, 0, 10, 0), (2, 262150, 0, 0, 1, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,pad,offset,top,masked", SHAPES)
def test_log_probs(E, dtype, rows, classes, pad, offset, top, masked):
    """A wave per row, a block per row, rows in parts; odd lengths, unaligned rows, masked classes, rows without a target."""
    gen = torch.Generator().manual_seed(rows * 7 + classes)
    z, _ = logits_of(gen, rows, classes, pad, dtype, masked=min(masked, 0.95), offset=offset)
    t = targets_of(gen, rows, classes)
    zc = z.cpu().double()
    r = E.edl_log_probs(z, t.cuda(), top=top)
    check_stats(r, R.log_probs(zc, t, top), stat_tolerance(zc, classes), top)
    again = E.edl_log_probs(z, t.cuda(), top=top)
    for a, b in zip(r, again):
        assert a is None or torch.equal(a.view(torch.int32), b.view(torch.int32))
    if top < 2:
        q = E.edl_log_probs(z, None, top=top)
        assert q.log_prob is None and torch.equal(q.lse, r.lse) and torch.equal(q.entropy, r.entropy)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(8, 100), (8, 3000), (8, 20000)])
def test_log_probs_of_rows_at_their_edges(E, dtype, rows, classes):
    """One class left; all masked; all equal (ties by the lower number); the type's lowest value as a mask; NaN; +inf; large
    values that differ little; signed zeros."""
    gen = torch.Generator().manual_seed(classes)
    z = (torch.randn(rows, classes, generator=gen) * 2).to(DT[dtype])
    lowest = torch.finfo(DT[dtype]).min
    z[0] = -float("inf")
    z[0, classes // 2] = 1.5
    z[1] = -float("inf")
    z[2] = 0.25
    z[3, : classes - 3] = lowest
    z[4, classes - 1] = float("nan")
    z[5, 3] = float("inf")
    z[6] = 1000.0
    z[7] = -0.0
    z[7, 1::2] = 0.0
    t = torch.tensor([classes // 2, 0, classes - 1, 2, 0, 3, -5, classes], dtype=torch.int32)
    top = 20
    r = E.edl_log_probs(z.cuda(), t.cuda(), top=top)
    zc = z.double()
    fine = torch.where(zc <= lowest, torch.full_like(zc, -1e30), zc)      # the lowest value's log probability is itself: checked apart
    want = R.log_probs(torch.where(zc == -float("inf"), zc, fine), t, top)
    got = E.LogProbs(r.log_prob.clone(), r.entropy, r.lse, r.top_log_prob.clone(), r.top_class)
    assert float(r.log_prob[3]) == float(lowest) and bool((r.top_log_prob[3, 3:] == lowest).all())
    want[0][3] = 0.0
    want[3][3, 3:] = 0.0
    got.log_prob[3] = 0.0
    got.top_log_prob[3, 3:] = 0.0
    check_stats(got, want, 2.0 ** -24 * (4 + classes ** 0.5 / 8 + 4 * 1000.0), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_log_probs_of_the_types_largest_values(E, dtype):
    """Rows of nothing but the lowest value (every class masked alike: all equally likely), of the largest, and of both."""
    big = torch.finfo(DT[dtype]).max
    for classes in (70, 1500, 9001):
        z = torch.full((3, classes), -big, dtype=DT[dtype])
        z[1] = big
        z[2, 5] = big
        r = E.edl_log_probs(z.cuda(), torch.tensor([3, 4, 5], dtype=torch.int32).cuda(), top=1)
        assert r.lse.cpu().tolist() == [-big, big, big]          # log(classes) is far below a step
        H, lp = r.entropy.cpu(), r.log_prob.cpu()
        assert r.top_class[:, 0].tolist() == [0, 0, 5] and torch.equal(lp, r.top_log_prob[:, 0].cpu())
        assert abs(float(lp[0]) + np.log(classes)) < 1e-5 and abs(float(lp[1]) + np.log(classes)) < 1e-5 and float(lp[2]) == 0.0
        assert abs(float(H[0]) - np.log(classes)) < 1e-5 and abs(float(H[1]) - np.log(classes)) < 1e-5 and float(H[2]) == 0.0


def test_log_probs_in_rising_order_and_of_equal_logits(E):
    """Every class beats all before it (the list of the best changes with each), and falling and equal ones."""
    for dtype in (torch.float32, torch.bfloat16):
        up = torch.arange(9000, dtype=torch.float32).mul(0.001).to(dtype)
        z = torch.stack([up, up.flip(0), torch.zeros_like(up), up.abs().sub(4).abs()])
        r = E.edl_log_probs(z.cuda(), None, top=64)
        zc = z.double()
        check_stats(r, R.log_probs(zc, None, 64), stat_tolerance(zc, 9000), 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,pad,offset,top,masked", SHAPES)
def test_log_probs_backward(E, dtype, rows, classes, pad, offset, top, masked):
    """Against the formula; padded, in place, and with either gradient missing.  Tolerance: half a step of the result, and the
    float32 error of p (that of z - lse) times the gradients."""
    gen = torch.Generator().manual_seed(rows * 11 + classes)
    z, buf = logits_of(gen, rows, classes, pad, dtype, masked=min(masked, 0.95), offset=offset)
    t = targets_of(gen, rows, classes)
    r = E.edl_log_probs(z, t.cuda())
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    g[rows // 2] = 0.0
    h[rows // 2] = 0.0
    zc = z.cpu().double()
    alive = torch.isfinite(R.log_probs(zc, None)[2])
    for dg, dh in ((g, h), (g, None), (None, h)):
        want = R.log_probs_backward(zc, t, dg, dh)
        want = torch.where(alive[:, None] | (want == 0), want, torch.nan_to_num(want))
        d = E.edl_log_probs_backward(z, t.cuda(), r.lse, r.entropy, None if dg is None else dg.cuda(), None if dh is None else dh.cuda())
        got = d.cpu().double()
        size = (0 if dg is None else g.abs()) + (0 if dh is None else h.abs() * 15)     # p (log p + H): H and -p log p stay below 13
        tol = R.EPS[DT[dtype]] * want.abs() + (size[:, None] * stat_tolerance(zc, classes))
        assert bool(((got - want).abs() <= tol)[alive].all())
        assert bool((got[rows // 2] == 0).all())
    before = buf.clone()
    assert E.edl_log_probs_backward(z, t.cuda(), r.lse, r.entropy, None, h.cuda(), out=z) is z
    assert same_bits(z, d)
    z.copy_(before[offset:].view(rows, classes + pad)[:, :classes])
    assert same_bits(buf, before)


def test_log_probs_backward_against_differences(E):
    """Central differences of the loss g log_prob + h entropy in float64 at a few classes of every row."""
    gen = torch.Generator().manual_seed(3)
    z = (torch.randn(6, 40, generator=gen) * 2)
    t = torch.tensor([0, 39, -1, 7, 8, 20], dtype=torch.int32)
    g, h = torch.randn(6, generator=gen), torch.randn(6, generator=gen)
    r = E.edl_log_probs(z.cuda(), t.cuda())
    d = E.edl_log_probs_backward(z.cuda(), t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda()).cpu().double()

    def loss(zz):
        lp, H, *_ = R.log_probs(zz, t)
        return g.double() * lp + h.double() * H
    step = 1e-5
    for c in (0, 7, 8, 20, 39, 11):
        e = torch.zeros(6, 40, dtype=torch.float64)
        e[:, c] = step
        diff = (loss(z.double() + e) - loss(z.double() - e)) / (2 * step)
        # the difference quotient's error: step^2 times third derivatives (of size |g| + 6 |h|), and 2^-52 x 20 / step
        assert float((diff - d[:, c]).abs().max()) <= 1e-6


def test_log_probs_backward_of_rows_without_a_distribution(E):
    """All masked: zeros (and the target's g).  NaN rows: NaN, unless nothing is wanted of them."""
    z = torch.full((4, 1500), -float("inf"))
    z[2:] = float("nan")
    t = torch.tensor([-1, 5, -1, -1], dtype=torch.int32)
    r = E.edl_log_probs(z.cuda(), t.cuda())
    h = torch.tensor([1.0, 1.0, 0.0, 1.0])
    d = E.edl_log_probs_backward(z.cuda(), t.cuda(), r.lse, r.entropy, torch.full((4,), 2.0).cuda(), h.cuda()).cpu()
    assert bool((d[0] == 0).all()) and float(d[1, 5]) == 2.0 and float(d[1].abs().sum()) == 2.0
    assert bool((d[2] == 0).all()) and bool(torch.isnan(d[3]).all())


def test_log_probs_in_a_replayed_graph_and_on_another_stream(E):
    gen = torch.Generator().manual_seed(5)
    z = (torch.randn(4, 20000, generator=gen) * 3).cuda()
    t = torch.tensor([1, 2, -1, 19999], dtype=torch.int32).cuda()
    g = torch.randn(4, generator=gen).cuda()

    def call(stream=None):
        r = E.edl_log_probs(z, t, top=9, stream=stream)
        return (*r, E.edl_log_probs_backward(z, t, r.lse, r.entropy, g, g, stream=stream))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    on_side = call(side.cuda_stream)
    side.synchronize()
    eager = call()
    for a, b in zip(on_side, eager):
        assert torch.equal(a, b)
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(3):
        z.add_(torch.randn(4, 20000, generator=gen).cuda())
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), i


def test_log_probs_of_no_rows(E):
    z = torch.empty(0, 7, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    r = E.edl_log_probs(z, t, top=3)
    assert r.lse.shape == (0,) and r.top_class.shape == (0, 3)
    assert E.edl_log_probs_backward(z, t, r.lse, r.entropy, r.lse, r.lse).shape == (0, 7)


# ---------------------------------------------------------------- classifier
# Per element, of float32 sums of n products whose errors do not all point one way: 2^-24 (sqrt(n) + 4) sum |a b|.  z: that of
# its own sum.  dz: p's relative error is z - lse's absolute one.  dx in bf16: dz as two bf16 numbers (2^-16) and half a step.
def classifier_case(seed, dtype, rows, dim, classes, bias=True, pads=(0, 0), offsets=(0, 0), size=1.0):
    gen = torch.Generator().manual_seed(seed)
    x, _ = rows_of(gen, rows, dim, pads[0], dtype, size, offsets[0])
    w, _ = rows_of(gen, classes, dim, pads[1], dtype, size * (2.0 / dim) ** 0.5, offsets[1])
    b = torch.randn(classes, generator=gen) * 0.3 if bias else None
    t = targets_of(gen, rows, classes)
    return x, w, b, t, gen


def classifier_reference(x, w, b, t):
    xc, wc = x.cpu().double(), w.cpu().double()
    z = xc @ wc.t() + (0 if b is None else b.double())
    spread = (xc.abs() @ wc.abs().t() + (0 if b is None else b.double().abs())).max()
    tol = 2.0 ** -24 * (x.shape[1] ** 0.5 + 4) * float(torch.nan_to_num(spread, posinf=0.0)) + stat_tolerance(z, z.shape[1])
    return z, R.log_probs(z, t), tol


def check_classifier_grads(E, x, w, b, t, r, z, tol, g, h, **kw):
    rows, dim = x.shape
    dev = lambda v: None if v is None else v.cuda()         # noqa: E731
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, dev(b), dev(t), r.lse, r.entropy, dev(g), dev(h), **kw)
    dz = R.log_probs_backward(z, t, g, h)
    xc, wc = x.cpu().double(), w.cpu().double()
    size = torch.zeros(rows, dtype=torch.float64)
    if g is not None:
        size = size + torch.where((t >= 0) & (t < z.shape[1]), g.abs().double(), size)
    lp = z - torch.logsumexp(z, 1)[:, None]
    p = lp.exp()
    # |dz|'s parts before they cancel
    parts = size[:, None] * p + dz.abs()
    if h is not None:
        parts = parts + h.abs().double()[:, None] * p * (lp.abs().clamp(max=1e3) + 15)
    e = 2 * tol
    two = 2.0 ** -16 if x.dtype == torch.bfloat16 else 0.0
    sums = lambda n: 2.0 ** -24 * (n ** 0.5 + 6)            # noqa: E731
    want = dz @ wc
    assert bool(((dx.cpu().double() - want).abs() <= (parts @ wc.abs()) * (e + two + sums(z.shape[1])) + R.EPS[x.dtype] * want.abs() + 1e-37).all())
    want = dz.t() @ xc
    assert dw.dtype == torch.float32
    assert bool(((dw.cpu().double() - want).abs() <= (parts.t() @ xc.abs()) * (e + sums(rows)) + 1e-37).all())
    if b is not None or kw.get("dbias") is not None:
        assert bool(((db.cpu().double() - dz.sum(0)).abs() <= parts.sum(0) * (e + sums(rows)) + 1e-37).all())
    return dx, dw, db


CLASSIFIERS = [  # rows, dim, classes, bias, pads, offsets
    (1, 1, 1, True, (0, 0), (0, 0)), (1, 16, 2, False, (0, 0), (0, 0)), (3, 7, 5, True, (1, 2), (1, 0)), (8, 64, 10, True, (0, 0), (0, 0)),
    (33, 100, 40, True, (0, 0), (0, 0)), (8, 4096, 1000, True, (0, 0), (0, 0)), (256, 512, 1000, True, (0, 0), (0, 0)), (130, 72, 129, False, (8, 8), (0, 0)),
    (65, 1000, 333, True, (0, 0), (8, 0)), (1, 256, 20000, True, (0, 0), (0, 0)), (2, 48, 24000, True, (0, 3), (0, 0)), (5000, 24, 12, True, (0, 0), (0, 0)),
    # tiles enough for the sums of whole tiles
    (300, 64, 8300, True, (0, 0), (0, 0)), (129, 200, 12500, False, (0, 0), (0, 0)), (257, 33, 8192, True, (0, 0), (0, 0)), (1, 40, 24600, True, (0, 0), (0, 0)),
    (3300, 16, 1000, True, (8, 0), (0, 8)), (640, 130, 5121, True, (0, 0), (1, 1)), (24700, 8, 100, True, (0, 0), (0, 0)), (1030, 320, 3000, True, (0, 0), (0, 0))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes,bias,pads,offsets", CLASSIFIERS)
def test_classifier_log_probs(E, dtype, rows, dim, classes, bias, pads, offsets):
    x, w, b, t, _ = classifier_case(rows + dim, dtype, rows, dim, classes, bias, pads, offsets)
    z, want, tol = classifier_reference(x, w, b, t)
    dev = lambda v: None if v is None else v.cuda()         # noqa: E731
    r = E.edl_classifier_log_probs(x, w, dev(b), t.cuda())
    check_stats(r, want, tol, 0)
    again = E.edl_classifier_log_probs(x, w, dev(b), t.cuda())
    assert all(torch.equal(a, c) for a, c in zip(r[:3], again[:3]))
    q = E.edl_classifier_log_probs(x, w, dev(b))
    assert q.log_prob is None and torch.equal(q.lse, r.lse) and torch.equal(q.entropy, r.entropy)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes,bias,pads,offsets", CLASSIFIERS)
def test_classifier_backward(E, dtype, rows, dim, classes, bias, pads, offsets):
    x, w, b, t, gen = classifier_case(rows + dim + 1, dtype, rows, dim, classes, bias, pads, offsets)
    z, want, tol = classifier_reference(x, w, b, t)
    dev = lambda v: None if v is None else v.cuda()         # noqa: E731
    r = E.edl_classifier_log_probs(x, w, dev(b), t.cuda())
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3
    first = check_classifier_grads(E, x, w, b, t, r, z, tol, g, h)
    again = check_classifier_grads(E, x, w, b, t, r, z, tol, g, h)
    assert all(a is None or torch.equal(a, c) for a, c in zip(first, again))
    check_classifier_grads(E, x, w, b, t, r, z, tol, g, None)
    check_classifier_grads(E, x, w, b, t, r, z, tol, None, h)


def test_classifier_backward_in_several_pieces_of_the_classes(E):
    """dz of more rows and classes than are held at a time: two pieces, the second of another size."""
    rows, dim, classes = 16400, 24, 11003
    x, w, b, t, gen = classifier_case(31, "bf16", rows, dim, classes)
    assert rows * classes * 6 > 1 << 30
    z, want, tol = classifier_reference(x, w, b, t)
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    check_stats(r, want, tol, 0)
    check_classifier_grads(E, x, w, b, t, r, z, tol, torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3)


@pytest.mark.parametrize("dtype,rows,dim,classes", [("bf16", 70001, 9, 7000), ("f32", 70001, 9, 7000), ("bf16", 9000, 300, 40003)])
def test_classifier_backward_in_many_pieces_adds_dx_up(E, dtype, rows, dim, classes):
    """Three pieces of the classes: dx is the sum of their parts, of which few rows have several."""
    x, w, b, t, gen = classifier_case(33, dtype, rows, dim, classes)
    assert rows * classes * 6 > 2 << 30
    g = torch.randn(rows, generator=gen).cuda()
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g)
    again = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1]) and torch.equal(db, again[2])
    # of some rows, in 64 bits
    some = torch.cat([torch.arange(0, 40), torch.arange(rows - 40, rows)])
    x64, w64 = x.cpu().double()[some], w.cpu().double()
    z = x64 @ w64.t() + b.double()
    p = torch.softmax(z, 1)
    hot = torch.zeros_like(p)
    mine = (t[some] >= 0) & (t[some] < classes)
    hot[mine.nonzero()[:, 0], t[some][mine].long()] = 1
    gs = torch.where(mine, g.cpu().double()[some], torch.zeros(80, dtype=torch.float64))[:, None]
    want = (gs * (hot - p)) @ w64
    parts = (gs.abs() * (hot + p)) @ w64.abs()              # before they cancel
    # a probability is off by the logit's error (dim products and sums of float32 and those of log-sum-exp, a rounding each, of
    # terms as large as |x| |w|) and a few steps of its own, and every sum of classes by a step for each of its additions
    size = (x64.abs() @ w64.abs().t() + b.double().abs()).amax(1, keepdim=True) + math.log(classes)
    eps = 2.0 ** -24
    tol = parts * eps * ((dim + 40) * size + 40 + math.sqrt(classes) + 3)
    if dtype == "bf16":
        tol = tol + parts * 2.0 ** -16 + want.abs() * 2.0 ** -8           # (two planes of dz; the result's rounding)
    assert bool(((dx.cpu().double()[some] - want).abs() <= tol).all())


@pytest.mark.parametrize("rows,dim,classes,bias", [(1100, 1024, 13000, True), (1085, 1001, 13003, False)])
def test_classifier_of_large_tiles(E, rows, dim, classes, bias):
    """Sizes whose products run on 256x256 tiles, the one for dx with its reduction cut: even ones, and odd ones throughout."""
    x, w, b, t, gen = classifier_case(37, "bf16", rows, dim, classes, bias)
    z, want, tol = classifier_reference(x, w, b, t)
    dev = lambda v: None if v is None else v.cuda()         # noqa: E731
    r = E.edl_classifier_log_probs(x, w, dev(b), t.cuda())
    check_stats(r, want, tol, 0)
    check_classifier_grads(E, x, w, b, t, r, z, tol, torch.randn(rows, generator=gen), torch.randn(rows, generator=gen) * 0.3)


def test_classifier_outputs_in_wider_matrices(E):
    """Gradients into views of wider matrices: what lies beside their rows stays."""
    x, w, b, t, gen = classifier_case(5, "bf16", 70, 40, 300)
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    g = torch.randn(70, generator=gen).cuda()
    plain = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g)
    bx, bw = torch.full((70, 43), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((300, 47), 7.0, device="cuda")
    bb = torch.full((302,), 7.0, device="cuda")
    E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g, dx=bx[:, 1:41], dw=bw[:, 2:42], dbias=bb[1:301])
    assert torch.equal(bx[:, 1:41], plain[0]) and torch.equal(bw[:, 2:42], plain[1]) and torch.equal(bb[1:301], plain[2])
    assert bool((bx[:, 0] == 7).all() and (bx[:, 41:] == 7).all() and (bw[:, :2] == 7).all() and (bw[:, 42:] == 7).all() and bb[0] == 7 and bb[301] == 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes", [(40, 64, 500), (300, 64, 8300)])
def test_classifier_masked_classes_and_rows_that_count_for_nothing(E, dtype, rows, dim, classes):
    """A bias of -inf takes a class out; targets that are no class; rows with zero gradients leave no trace."""
    x, w, b, t, gen = classifier_case(9, dtype, rows, dim, classes)
    b[::3] = -float("inf")
    t = torch.where(t % 3 == 0, t + 1, t)
    t[0], t[1], t[2] = classes, -7, 2 ** 31 - 1
    z, want, tol = classifier_reference(x, w, b, t)
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    check_stats(r, want, tol, 0)
    assert r.log_prob[:3].tolist() == [0.0, 0.0, 0.0]
    g, h = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    g[5:9] = 0
    h[5:9] = 0
    dx, dw, db = check_classifier_grads(E, x, w, b, t, r, torch.where(z == -float("inf"), torch.full_like(z, -1e4), z), tol, g, h)
    assert bool((dx[5:9] == 0).all() and (dw[::3] == 0).all() and (db[::3] == 0).all())
    everything = torch.full((classes,), -float("inf"))
    r = E.edl_classifier_log_probs(x, w, everything.cuda(), t.cuda())
    assert bool((r.lse == -float("inf")).all() and (r.entropy == 0).all())
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, everything.cuda(), t.cuda(), r.lse, r.entropy, None, h.cuda())
    assert bool((dx == 0).all() and (dw == 0).all() and (db == 0).all())


def test_classifier_is_log_probs_of_its_logits(E):
    """The same head with and without logits in memory, and finite differences of the loss along a random direction."""
    x, w, b, t, gen = classifier_case(13, "f32", 50, 96, 700)
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    z = (x.double() @ w.double().t() + b.cuda().double())
    q = E.edl_log_probs(z.float(), t.cuda())
    for a, c in zip(r[:3], q[:3]):
        assert float((a - c).abs().max()) <= 2e-5
    g, h = torch.randn(50, generator=gen).cuda(), torch.randn(50, generator=gen).cuda()
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g, h)
    ux, uw, ub = (torch.randn(*v.shape, generator=gen).double() for v in (x, w, b))

    def loss(s):
        zz = (x.cpu().double() + s * ux) @ (w.cpu().double() + s * uw).t() + b.double() + s * ub
        lp, H, *_ = R.log_probs(zz, t)
        return float((g.cpu().double() * lp + h.cpu().double() * H).sum())
    slope = (loss(1e-6) - loss(-1e-6)) / 2e-6
    mine = float((dx.cpu().double() * ux).sum() + (dw.cpu().double() * uw).sum() + (db.cpu().double() * ub).sum())
    assert abs(slope - mine) <= 1e-4 * max(1.0, abs(slope))


def test_classifier_in_a_replayed_graph_and_on_another_stream(E):
    x, w, b, t, gen = classifier_case(17, "bf16", 300, 64, 8300)
    b, t, g = b.cuda(), t.cuda(), torch.randn(300, generator=gen).cuda()

    def call(stream=None):
        r = E.edl_classifier_log_probs(x, w, b, t, stream=stream)
        return (*r[:3], *E.edl_classifier_log_probs_backward(x, w, b, t, r.lse, r.entropy, g, g, stream=stream))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    on_side = call(side.cuda_stream)
    side.synchronize()
    for a, c in zip(on_side, call()):
        assert torch.equal(a, c)
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(3):
        x.copy_(torch.randn(300, 64, generator=gen).to(x.dtype).cuda())
        want = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(held, want):
            assert torch.equal(a, c), i


def test_classifier_workspace_from_the_caller(E):
    x, w, b, t, gen = classifier_case(19, "f32", 300, 30, 8300)
    need = E.edl_classifier_workspace(x, w), E.edl_classifier_workspace(x, w, backward=True)
    assert min(need) > 0
    work = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda")       # NaN all over
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda(), work=work)
    want = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    assert all(torch.equal(a, c) for a, c in zip(r[:3], want[:3]))
    work.fill_(255)
    g = torch.randn(300, generator=gen).cuda()
    a = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g, work=work)
    c = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g)
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    with pytest.raises(E.EdlError) as ei:
        E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda(), work=work[:need[0] - 1])
    assert ei.value.code == -3


def test_classifier_of_no_rows(E):
    x, w = torch.empty(0, 24, device="cuda"), torch.randn(10, 24, device="cuda")
    t, e = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    assert E.edl_classifier_log_probs(x, w, None, t).lse.shape == (0,)
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, torch.zeros(10, device="cuda"), t, e, e, e, e)
    assert dx.shape == (0, 24) and bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_head_as_it_is_trained(E, dtype):
    """The operators together: dropout of hidden features, the loss over many classes, its gradient back through the dropout,
    and the update of the weights (Adam, with its bf16 copy), against the same in float64."""
    x, w, b, t, gen = classifier_case(23, dtype, 96, 64, 9000)
    master = w.float().contiguous() if dtype == "bf16" else w
    n = 9000 * 64
    m, s = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    key = E.edl_dropout_key(1, 2, 3)
    y = E.edl_dropout(x, 0.25, key)
    r = E.edl_classifier_log_probs(y, w, b.cuda(), t.cuda())
    g = torch.full((96,), -1.0 / 96)
    z, want, tol = classifier_reference(y, w, b, t)
    check_stats(r, want, tol, 0)
    dy, dw, db = check_classifier_grads(E, y, w, b, t, r, z, tol, g, None)
    dx = E.edl_dropout(dy, 0.25, key)
    assert same_bits(dx, R.dropout(dy.cpu(), 0.25, key))
    assert bool((dx[~torch.from_numpy(R.kept(96, 64, 0.25, key)).cuda()] == 0).all())
    before = master.cpu().double().flatten()
    w16 = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    E.edl_adam_update([dw.flatten()], master.view(-1), m, s, w16, 0.01, 0.9, 0.999, 1e-8, 0.0, 1)
    step = 0.01 * torch.sign(dw.cpu().double().flatten()) * (dw.cpu().double().flatten().abs() / (dw.cpu().double().flatten().abs() + 1e-8))
    # the first step of Adam: lr g / (|g| + eps); half a step of the weight, and the moments' roundings (a few 2^-24 of lr)
    assert bool(((master.cpu().double().flatten() - (before - step)).abs() <= 2.0 ** -24 * before.abs() + 2e-7).all())
    assert same_bits(w16, master.flatten().to(torch.bfloat16))


# ---------------------------------------------------------------- dropout inside a job
def _net(model, arch, x, params, table, masks, rate, stored):
    """Logits of MLP, VGG and AlexNet jobs in float64 on the CPU; masks: which elements the hidden layers keep.  Activations
    are what the job's type stores (a ReLU's sign is taken from those); their rounding passes gradients through."""
    import torch.nn.functional as F
    r = lambda t: t + (t.detach().to(stored).double() - t.detach())        # noqa: E731
    at = {name: (off, size) for name, off, size, _ in table}
    take = lambda name: params[at[name][0]:at[name][0] + at[name][1]]      # noqa: E731

    def conv(t, name, k, size, stride, pad):
        w = take(name + ".w").view(k, size, size, t.shape[1]).permute(0, 3, 1, 2)
        return r(F.relu(F.conv2d(t, w, take(name + ".b"), stride=stride, padding=pad)))

    if model == "vgg16":
        t, i = x.permute(0, 3, 1, 2), 0
        for width, times in zip((1, 2, 4, 8, 8), arch[2:7]):
            for _ in range(times):
                i += 1
                t = conv(t, "conv%d" % i, arch[0] * width, 3, 1, 1)
            t = F.max_pool2d(t, 2, 2)
        t = t.permute(0, 2, 3, 1)
    else:
        t = x
    t = t.reshape(t.shape[0], -1)
    for name, mask in zip(("fc1", "fc2"), masks):
        t = r(F.relu(t @ take(name + ".w").view(-1, t.shape[1]).t() + take(name + ".b")))
        t = r(torch.where(mask, t / (1.0 - rate), torch.zeros_like(t)))
    return t @ take("fc3.w").view(-1, t.shape[1]).t() + take("fc3.b")


JOBS = {
    # fully connected nets of vector widths (the small layers' kernels, the classifier's launch) and of odd ones
    "mlp": dict(model="mlp", geom=dict(H=1, W=1, C_=784, classes=10), arch=(256, 256), N=128, B=64),
    "mlp_odd": dict(model="mlp", geom=dict(H=1, W=1, C_=37, classes=5), arch=(29, 51), N=48, B=24),
    "vgg": dict(model="vgg16", geom=dict(H=32, W=32, C_=3, classes=10), arch=(8, 64, 1, 1, 1, 1, 1), N=32, B=16),
}


def _job(E, which, dtype, p_max=4, seed=11, **kw):
    from paper_1909_11985_amd.binding import make_config
    import synth_inputs
    c = JOBS[which]
    g = c["geom"]
    x, y = synth_inputs.dataset(2, c["N"], g["H"], g["W"], g["C_"], g["classes"])
    cfg = make_config(c["model"], dtype=dtype, N=c["N"], B=c["B"], p_max=p_max, lr=0.05, arch=c["arch"], **g, **kw)
    job = E.Job(cfg, seed)
    job.bind_dataset(torch.from_numpy(x).cuda(), torch.from_numpy(y).cuda())
    return job, torch.from_numpy(x).double(), torch.from_numpy(y).long(), E.edl_tensor_table(cfg)


def _layers(E, job):
    """Places of fc1 and fc2 in the layer list: the third and second convolution from its end."""
    ops = job.debug_op_count()          # ..., fc1, fc2, fc3, loss
    return ops - 4, ops - 3


def _reference(E, job, which, x, y, table, idx, rate, step, seed=11):
    c = JOBS[which]
    widths = c["arch"][:2] if c["model"] == "mlp" else (c["arch"][1],) * 2
    masks = [torch.from_numpy(R.kept(len(idx), n, rate, E.edl_dropout_key(seed, step, layer)))
             for n, layer in zip(widths, _layers(E, job))]
    w = torch.from_numpy(job.params()).double().requires_grad_()
    if job.cfg.dtype == 1:
        wl = w + (w.detach().to(torch.bfloat16).double() - w.detach())     # what the products read; biases stay float32
        keep = torch.zeros_like(w, dtype=torch.bool)
        for name, off, size, _ in table:
            if name.endswith(".b"):
                keep[off:off + size] = True
        wl = torch.where(keep, w, wl)
        xs = x[idx].to(torch.bfloat16).double()
    else:
        wl, xs = w, x[idx]
    logits = _net(c["model"], c["arch"], xs, wl, table, masks, rate, torch.bfloat16 if job.cfg.dtype == 1 else torch.float32)
    rows = torch.nn.functional.cross_entropy(logits, y[idx], reduction="none")
    return rows, w


@pytest.mark.parametrize("which,dtype,p,rate", [("mlp", "f32", 1, 0.5), ("mlp", "f32", 4, 0.5), ("mlp_odd", "f32", 3, 0.25), ("mlp", "bf16", 2, 0.5),
                                                ("vgg", "f32", 2, 0.5), ("vgg", "bf16", 4, 0.3)])
def test_job_dropout_gradients_are_the_definitions(E, which, dtype, p, rate):
    """Loss and every worker's gradient at two consecutive steps, against float64 with the masks from the host."""
    job, x, y, table = _job(E, which, dtype)
    job.set_dropout(rate)
    tol = 1e-4 if dtype == "f32" else 2e-2      # what layer-by-layer parity of these jobs is held to
    for step in range(2):
        idx, off = job.shard(job.cfg.B, p, *job.progress()[1:])
        loss = job.gradients(p)
        rows, w = _reference(E, job, which, x, y, table, idx, rate, step)
        assert abs(loss - float(rows.detach().mean())) <= tol * max(1.0, abs(loss))
        for k in range(p):
            (want,) = torch.autograd.grad(rows[off[k]:off[k + 1]].mean(), w, retain_graph=True)
            got = torch.from_numpy(job.grad(k)).double()
            assert float((got - want).norm() / want.norm()) <= tol, (step, k)
        job.apply(p)


@pytest.mark.parametrize("which,dtype", [("mlp", "f32"), ("vgg", "bf16")])
def test_job_dropout_does_not_depend_on_the_cut(E, which, dtype):
    """One mini-batch as 1, 2 and 4 shards and as an uneven cut (with an empty shard): the same masks, so the same aggregate."""
    job, *_ = _job(E, which, dtype)
    job.set_dropout(0.5)
    B = job.cfg.B
    idx, _ = job.shard(B, 1, 0, 0)
    means = []
    for off in ([0, B], [0, B // 2, B], [0, B // 4, B // 2, 3 * B // 4, B], [0, 3, 3, B]):
        off = np.array(off, dtype=np.int64)
        job.gradients(len(off) - 1, idx, off)
        share = np.diff(off) / B
        means.append(sum(s * job.grad(k).astype(np.float64) for k, s in enumerate(share) if s > 0))
    for m in means[1:]:
        err = np.linalg.norm(m - means[0]) / np.linalg.norm(means[0])
        assert err <= (1e-5 if dtype == "f32" else 1e-2), err


def test_job_dropout_zero_is_the_job_without_it(E):
    """Rate 0 takes the launches of a job that never heard of dropout, bit for bit; a rate set and taken back as well."""
    a, *_ = _job(E, "mlp", "f32")
    b, *_ = _job(E, "mlp", "f32")
    b.set_dropout(0.5)
    b.set_dropout(0.0)
    for p in (1, 4):
        assert a.step(p) == b.step(p)
    assert np.array_equal(a.params(), b.params())


def test_job_dropout_travels_with_the_state_image(E):
    """A joiner created without dropout continues exactly as the job it joined; so does the step without an arena's scratch."""
    a, *_ = _job(E, "mlp", "f32")
    a.set_dropout(0.5)
    a.step(2)
    b, *_ = _job(E, "mlp", "f32", seed=99)
    b.restore(a.snapshot())
    c, *_ = _job(E, "mlp", "f32", seed=98)
    c.restore(a.snapshot())
    for p in (4, 1, 2):
        loss = a.step(p)
        assert loss == b.step(p) and loss == c.step_static_scratch(p)
    assert np.array_equal(a.params(), b.params()) and np.array_equal(a.params(), c.params())


def test_job_dropout_refusals(E):
    from paper_1909_11985_amd.binding import make_config
    job, *_ = _job(E, "mlp", "f32")
    for rate in (-0.1, 1.0, float("nan")):
        with pytest.raises(E.EdlError) as ei:
            job.set_dropout(rate)
        assert ei.value.code == -1
    res = E.Job(make_config("resnet20", N=16, B=8, p_max=1, H=16, W=16, C_=3, classes=4, arch=(8, 2, 1)), 1)
    with pytest.raises(E.EdlError):
        res.set_dropout(0.5)
    res.set_dropout(0.0)
