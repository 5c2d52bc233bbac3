"""The classifier operators where a bias is not a number or infinite, on every path that forms their logits.  Run with -m gpu."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1909_11985_amd as E
    return E


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
# rows read by a wave, the same in parts of many classes, logits in float32 parts from tiles, sums of whole tiles
@pytest.mark.parametrize("rows,dim,classes", [(7, 24, 100), (3, 8, 40001), (100, 64, 1000), (300, 64, 8300), (1100, 64, 13000)])
def test_a_bias_that_is_no_number_leaves_no_distribution(E, dtype, bad, rows, dim, classes):
    """Everything of every row is NaN, but what nothing is wanted of: rows with zero gradients, log probabilities without a target."""
    gen = torch.Generator().manual_seed(rows)
    x, w = (torch.randn(*s, generator=gen).to(DT[dtype]).cuda() for s in ((rows, dim), (classes, dim)))
    b = torch.randn(classes, generator=gen)
    b[classes // 3] = bad
    t = torch.randint(0, classes, (rows,), generator=gen, dtype=torch.int32)
    t[1] = -1
    r = E.edl_classifier_log_probs(x, w, b.cuda(), t.cuda())
    assert bool(torch.isnan(r.lse).all() and torch.isnan(r.entropy).all())
    assert torch.isnan(r.log_prob).tolist() == [i != 1 for i in range(rows)] and float(r.log_prob[1]) == 0.0
    g, h = torch.ones(rows), torch.zeros(rows)
    g[2] = 0.0
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, g.cuda(), h.cuda())
    assert bool((dx[1:3] == 0).all() and torch.isnan(dx[0]).all() and torch.isnan(dx[3:]).all())
    assert bool(torch.isnan(dw).all() and torch.isnan(db).all())
    only = torch.zeros(rows)
    dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b.cuda(), t.cuda(), r.lse, r.entropy, only.cuda(), only.cuda())
    assert bool((dx == 0).all() and (dw == 0).all() and (db == 0).all())
