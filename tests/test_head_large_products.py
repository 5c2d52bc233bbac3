"""The classifier operators at sizes whose products run on 256x256 tiles, with and without their reductions cut, and whose dz comes in
several pieces of the classes: every element of every result against a reference in 64 bits, formed on the GPU.  Run with -m gpu."""
import math

import pytest
import torch

import head_reference as R

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1909_11985_amd as E
    return E


def off_by(got, want, most):
    """How much further than `most` elements are off, relative to `most` (at most 0: none)."""
    return float((((got.double() - want).abs() - most) / most.clamp(min=1e-30)).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,dim,classes,bias", [
    (4096, 4096, 1000, True),          # dx whole, dw cut in four
    (256, 512, 32768, False),          # dw whole
    (8192, 2048, 1000, True),          # dx whole, dw cut in eight
    (2085, 2051, 5501, True),          # odd throughout: dx cut in three, dw whole
    (2048, 1024, 6000, True),          # dw cut in two
    (1500, 4100, 1900, True),          # logits in float32 parts, of four cuts
    # several pieces of the classes
    (4096, 4096, 50000, True),         # dx added up on whole tiles
    (8201, 701, 45003, False),         # odd: dx added up in two cuts, the last piece shorter
    (70001, 9, 7000, True), (9000, 300, 40003, True)])
def test_products_on_large_tiles_and_in_pieces(E, dtype, rows, dim, classes, bias):
    gen = torch.Generator(device="cuda").manual_seed(rows + classes)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")         # noqa: E731
    x, w = rand(rows, dim).to(DT[dtype]), (rand(classes, dim) * (2.0 / dim) ** 0.5).to(DT[dtype])
    b = rand(classes) * 0.3 if bias else None
    t = torch.randint(-1, classes, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    g, h = rand(rows), rand(rows) * 0.3
    g[3] = h[3] = 0.0
    r = E.edl_classifier_log_probs(x, w, b, t)
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b, t, r.lse, r.entropy, g, h)

    xd, wd = x.double(), w.double()
    z = xd @ wd.t()
    size = xd.abs() @ wd.abs().t()
    if bias:
        z += b.double()
        size += b.double().abs()
    # a logit: dim products and sums in float32; z - lse and its sums as in test_head_operators.py
    off = STEP * ((math.sqrt(dim) + 4) * size.amax(1) + 4 + math.sqrt(classes / 64) + 4 * z.abs().amax(1))
    del size
    lse = torch.logsumexp(z, 1)
    z -= lse[:, None]                  # log p
    p = z.exp()
    H = -(p * z).sum(1)
    has = t >= 0
    at = t.clamp(min=0).long()[:, None]
    assert off_by(r.lse, lse, off) <= 0
    assert off_by(r.entropy, H, off * (1 + H)) <= 0            # (p is off by `off` of itself, and -log p by `off`)
    assert off_by(r.log_prob, torch.where(has, z.gather(1, at)[:, 0], torch.zeros_like(lse)), 2 * off) <= 0
    gd, hd = torch.where(has, g.double(), torch.zeros_like(lse)), h.double()
    dz = -gd[:, None] * p - hd[:, None] * p * (z + H[:, None])
    # what float32 may leave of dz: its parts before they cancel, times twice the error of log p
    parts = (gd.abs()[:, None] * p + hd.abs()[:, None] * p * (z.abs() + H[:, None] + 1)).mul_(2 * off[:, None])
    del z, p
    dz.scatter_add_(1, at, gd[:, None])
    # a sum of n float32 terms, and dz as three bf16 numbers; dx of bf16 takes two of them and is rounded
    sums = lambda n: STEP * (math.sqrt(n) + 6)            # noqa: E731
    two = 2.0 ** -16 if dtype == "bf16" else 0.0
    mag = dz.abs()
    want = dz @ wd
    assert off_by(dx, want, parts @ wd.abs() + (mag @ wd.abs()) * (two + sums(classes)) + R.EPS[DT[dtype]] * want.abs() + 1e-36) <= 0
    assert bool((dx[3] == 0).all())
    want = dz.t() @ xd
    assert off_by(dw, want, parts.t() @ xd.abs() + (mag.t() @ xd.abs()) * sums(rows) + 1e-36) <= 0
    if bias:
        assert off_by(db, dz.sum(0), parts.sum(0) + mag.sum(0) * sums(rows) + 1e-36) <= 0
    else:
        assert db is None
