"""The classifier-head operators beside autograd: inside its functions, and what they write to.  Run with -m gpu."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1909_11985_amd as E
    return E


def test_head_as_an_autograd_function(E):
    """Parameters that require gradients go through a function whose forward and backward make the calls; vectors that require
    one are refused outside."""
    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b, t):
            r = E.edl_classifier_log_probs(x, w, b, t)
            ctx.save_for_backward(x, w, b, t, r.lse, r.entropy)
            return -r.log_prob.mean()

        @staticmethod
        def backward(ctx, g):
            x, w, b, t, lse, entropy = ctx.saved_tensors
            dx, dw, db = E.edl_classifier_log_probs_backward(x, w, b, t, lse, entropy, (-g / x.shape[0]).expand(x.shape[0]).contiguous())
            return dx, dw, db, None
    gen = torch.Generator().manual_seed(4)
    x, w, b = (torch.randn(*s, generator=gen).cuda().requires_grad_() for s in ((20, 30), (50, 30), (50,)))
    t = torch.randint(0, 50, (20,), generator=gen, dtype=torch.int32).cuda()
    Loss.apply(x, w, b, t).backward()
    want = torch.autograd.grad(torch.nn.functional.cross_entropy(x.double() @ w.double().t() + b.double(), t.long()), (x, w, b))
    for v, g in zip((x, w, b), want):
        # float32 sums of 30 to 50 terms of a gradient below 1 / 20
        assert float((v.grad - g).abs().max()) <= 1e-6
    with pytest.raises(E.EdlError, match="bias requires a gradient"):
        E.edl_classifier_log_probs(x.detach(), w.detach(), b, t)
    with torch.no_grad():
        assert E.edl_classifier_log_probs(x, w, b, t).lse.shape == (20,)


def test_what_a_call_writes_to_counts_as_changed(E):
    """Autograd refuses to go back through a tensor that was saved and then overwritten."""
    a, p = torch.randn(6, 40, device="cuda"), torch.ones(6, 40, device="cuda", requires_grad=True)
    t, g = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.ones(6, device="cuda")
    w = torch.randn(5, 40, device="cuda")

    def classifier(out):
        x = torch.randn(6, 40, device="cuda")
        r = E.edl_classifier_log_probs(x, w, None, t)
        E.edl_classifier_log_probs_backward(x, w, None, t, r.lse, r.entropy, g, dx=out)

    def logits(out):
        r = E.edl_log_probs(out, t)
        E.edl_log_probs_backward(out, t, r.lse, r.entropy, g, out=out)
    for write in (lambda out: E.edl_dropout(out, 0.5, 1, out=out), logits, classifier):
        y = (p * a).sum()           # saves a
        write(a)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
