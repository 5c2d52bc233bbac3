"""CPU-only checks of the classifier-head operators: host functions, and every refusal of the C boundary and the binding.
No call here reaches a launch."""
import ctypes as C

import numpy as np
import pytest
import torch

import head_reference as R


@pytest.fixture(scope="module")
def E():
    import paper_1909_11985_amd as E
    return E


GOLDEN = R.GOLDEN
SOME = 1 << 20       # stands for device memory that no refused call looks at


def test_dropout_keys_are_draws(E):
    seen = set()
    for seed in (0, 7, 2 ** 63 + 5):
        for step in (0, 1, 2, 10 ** 9):
            for layer in (0, 1, 17):
                k = E.edl_dropout_key(seed, step, layer)
                assert k == R.draw(R.draw(seed ^ 0x5D6C1F3A9B27E841, step), layer)
                seen.add(k)
    assert len(seen) == 36
    for bad in ((0, -1, 0), (0, 0, -1)):
        with pytest.raises(E.EdlError) as ei:
            E.edl_dropout_key(*bad)
        assert ei.value.code == -1


def test_reference_masks_agree_with_the_scalar_generator():
    m = R.kept(3, 5, 0.5, 42, first_row=2 ** 61)
    for r in range(3):
        for c in range(5):
            d = R.draw(42, ((2 ** 61 + r) * 3 + c // 2) & R.M64)
            assert m[r, c] == (((d >> 32) if c & 1 else (d & 0xFFFFFFFF)) >= 2 ** 31)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), -1), (dict(x=None), -1), (dict(y=None), -1), (dict(rows=-1), -1), (dict(cols=-1), -1), (dict(first=-1), -1),
    (dict(rate=1.0), -1), (dict(rate=-0.01), -1), (dict(rate=float("nan")), -1), (dict(ldx=15), -1), (dict(ldy=15), -1),
    (dict(ldx=2 ** 31), -1), (dict(x=SOME + 2), -1), (dict(y=SOME + 1, dtype=1), -1), (dict(y=SOME, ldy=17), -1),
    (dict(rows=2 ** 38, cols=24, ldx=24, ldy=24), -4)])
def test_dropout_refusals(E, change, code):
    a = dict(dtype=0, x=SOME, ldx=16, y=2 * SOME, ldy=16, rows=4, cols=16, rate=0.5, first=0)
    a.update(change)
    rc = E.lib.edl_dropout(a["dtype"], a["x"], a["ldx"], a["y"], a["ldy"], a["rows"], a["cols"], a["rate"], 1, a["first"], None)
    assert rc == code and E.lib.edl_last_error()


def test_binding_refuses_what_is_no_matrix_on_a_gpu(E):
    for x in (torch.zeros(2, 2), torch.zeros(4), torch.zeros(2, 2, dtype=torch.float16), torch.zeros(2, 2, dtype=torch.float64)):
        with pytest.raises(E.EdlError) as ei:
            E.edl_dropout(x, 0.5, 1)
        assert ei.value.code == -1
