"""CPU-only checks of what the binding of the classifier-head operators refuses before the library sees it."""
import pytest
import torch


@pytest.fixture(scope="module")
def E():
    import paper_1909_11985_amd as E
    return E


@pytest.mark.parametrize("args,names", [((2 ** 64, 0, 0), "seed"), ((-2 ** 63 - 1, 0, 0), "seed"), ((0, 2 ** 63, 0), "step"), ((0, 2 ** 64 + 3, 0), "step"),
                                        ((0, 0, 2 ** 31), "layer"), ((0, 0, 2 ** 32), "layer")])
def test_dropout_keys_of_more_bits_are_refused(E, args, names):
    """Not cut to the bits that the library's types have: (0, 2^64 + 3, 0) would have the masks of step 3."""
    with pytest.raises(E.EdlError, match=names) as ei:
        E.edl_dropout_key(*args)
    assert ei.value.code == -1
    assert E.edl_dropout_key(-1, 5, 1) == E.edl_dropout_key(2 ** 64 - 1, 5, 1)      # the same 64 bits


@pytest.mark.parametrize("key,first_row,names", [(2 ** 64, 0, "key"), (-2 ** 63 - 1, 0, "key"), (1, 2 ** 63, "first_row"), (1, 2 ** 64 + 5, "first_row")])
def test_dropout_numbers_of_more_bits_are_refused(E, key, first_row, names):
    with pytest.raises(E.EdlError, match=names) as ei:
        E.edl_dropout(torch.zeros(2, 2), 0.5, key, first_row=first_row)
    assert ei.value.code == -1


def test_numbers_of_alternatives_of_more_bits_are_refused(E):
    for call in (lambda: E.edl_log_probs_workspace(1, 100, 2 ** 32), lambda: E.edl_log_probs_workspace(1, 2 ** 64 + 100, 1),
                 lambda: E.edl_log_probs_workspace(2 ** 64 + 1, 100, 1)):
        with pytest.raises(E.EdlError, match="top|rows|classes") as ei:
            call()
        assert ei.value.code == -1


def test_tensors_that_require_a_gradient_are_refused_while_autograd_records(E):
    x, w = (torch.zeros(*s, requires_grad=True) for s in ((2, 3), (4, 3)))
    t, f = torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    calls = [lambda: E.edl_dropout(x, 0.5, 1), lambda: E.edl_log_probs(x), lambda: E.edl_log_probs_backward(x, t, f, f, f), lambda: E.edl_classifier_log_probs(x, w)]
    for call in calls:
        with pytest.raises(E.EdlError, match="requires a gradient") as ei:
            call()
        assert ei.value.code == -1
        with torch.no_grad(), pytest.raises(E.EdlError, match="must be on a GPU"):      # (what else is wrong with them)
            call()
    with pytest.raises(E.EdlError, match="must be on a GPU"):
        E.edl_dropout(x.detach(), 0.5, 1)
