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
    (dict(rows=2 ** 33, cols=24, ldx=24, ldy=24), -4)])
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


LOG_PROBS = dict(dtype=0, z=SOME, ld=100, rows=4, classes=100, t=SOME, k=3, lp=SOME, ent=SOME, lse=SOME, tv=SOME, tc=SOME, work=None, bytes=0)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-1), -1), (dict(z=None), -1), (dict(z=SOME + 2), -1), (dict(ld=99), -1), (dict(rows=-1), -1), (dict(classes=0), -1),
    (dict(k=-1), -1), (dict(k=65), -1), (dict(k=4, classes=3, ld=3), -1), (dict(lp=None), -1), (dict(ent=None), -1), (dict(lse=None), -1),
    (dict(tv=None), -1), (dict(tc=None), -1), (dict(lse=SOME + 2), -1), (dict(t=SOME + 1), -1), (dict(classes=20000, ld=20000), -3),
    (dict(classes=20000, ld=20000, work=None, bytes=1 << 20), -1), (dict(classes=20000, ld=20000, work=SOME + 8, bytes=1 << 20), -1),
    (dict(rows=2 ** 23 + 1), -4), (dict(rows=2 ** 22, classes=2 ** 20, ld=2 ** 20), -4)])
def test_log_probs_refusals(E, change, code):
    a = dict(LOG_PROBS)
    a.update(change)
    rc = E.lib.edl_log_probs(a["dtype"], a["z"], a["ld"], a["rows"], a["classes"], a["t"], a["k"], a["lp"], a["ent"], a["lse"], a["tv"], a["tc"],
                             a["work"], a["bytes"], None)
    assert rc == code and E.lib.edl_last_error()


@pytest.mark.parametrize("change,code", [
    (dict(dtype=7), -1), (dict(z=None), -1), (dict(d=None), -1), (dict(ldd=99), -1), (dict(lse=None), -1), (dict(ent=None), -1), (dict(t=None), -1),
    (dict(d=SOME, ldd=101), -1), (dict(d=SOME + 1, dtype=1), -1), (dict(g=SOME + 2), -1), (dict(classes=-3), -1), (dict(rows=2 ** 30), -4)])
def test_log_probs_backward_refusals(E, change, code):
    a = dict(dtype=0, z=SOME, ld=100, rows=4, classes=100, t=SOME, lse=SOME, ent=SOME, g=SOME, h=SOME, d=2 * SOME, ldd=100)
    a.update(change)
    rc = E.lib.edl_log_probs_backward(a["dtype"], a["z"], a["ld"], a["rows"], a["classes"], a["t"], a["lse"], a["ent"], a["g"], a["h"], a["d"], a["ldd"], None)
    assert rc == code and E.lib.edl_last_error()


def test_log_probs_workspace(E):
    assert E.edl_log_probs_workspace(256, 1000, 5) == 0 and E.edl_log_probs_workspace(5000, 100000, 64) == 0 and E.edl_log_probs_workspace(0, 10, 0) == 0
    assert E.edl_log_probs_workspace(1, 32000, 5) == 8 * (16 + 5 * 8)          # eight parts of 4,000
    for bad in ((1, 0, 0), (-1, 5, 0), (1, 5, 6), (1, 100, 65)):
        with pytest.raises(E.EdlError) as ei:
            E.edl_log_probs_workspace(*bad)
        assert ei.value.code == -1


def test_parts_of_a_row_cover_it(E):
    """What the plan promises: no part empty, none beyond 64, workspace whole parts."""
    for rows in (1, 2, 17, 63, 300, 1023, 1024, 5000):
        for classes in (1, 8, 1024, 1025, 4096, 4097, 8193, 49999, 200000, 262145, 10 ** 7):
            n = E.edl_log_probs_workspace(rows, classes, 0)
            assert n % (16 * rows) == 0 and n // (16 * rows) <= 64 and n // (16 * rows) != 1


CLASSIFIER = dict(dtype=0, x=SOME, ldx=64, w=SOME, ldw=64, b=SOME, rows=4, dim=64, classes=100, t=SOME, lp=SOME, ent=SOME, lse=SOME, work=SOME, bytes=1 << 30)
CLASSIFIER_BAD = [
    (dict(dtype=2), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(ldx=63), -1), (dict(ldw=63), -1), (dict(rows=-1), -1), (dict(dim=0), -1),
    (dict(classes=0), -1), (dict(lse=None), -1), (dict(b=SOME + 2), -1), (dict(t=SOME + 1), -1), (dict(x=SOME + 2), -1), (dict(work=None), -1),
    (dict(work=SOME + 16), -1), (dict(bytes=16), -3), (dict(rows=2 ** 23 + 1), -4), (dict(dim=2 ** 16 + 1, ldx=2 ** 17, ldw=2 ** 17), -4),
    (dict(classes=2 ** 24 + 1), -4), (dict(rows=2 ** 14, dim=2 ** 16, ldx=2 ** 16, ldw=2 ** 16), -4), (dict(rows=2 ** 22, classes=2 ** 24), -4),
    (dict(classes=2 ** 22, dim=2 ** 13, ldx=2 ** 13, ldw=2 ** 13), -4)]


@pytest.mark.parametrize("change,code", CLASSIFIER_BAD + [(dict(lp=None), -1), (dict(ent=None), -1)])
def test_classifier_refusals(E, change, code):
    a = dict(CLASSIFIER)
    a.update(change)
    rc = E.lib.edl_classifier_log_probs(a["dtype"], a["x"], a["ldx"], a["w"], a["ldw"], a["b"], a["rows"], a["dim"], a["classes"], a["t"], a["lp"],
                                        a["ent"], a["lse"], a["work"], a["bytes"], None)
    assert rc == code and E.lib.edl_last_error()


@pytest.mark.parametrize("change,code", CLASSIFIER_BAD + [
    (dict(t=None), -1), (dict(ent=None), -1), (dict(dx=None), -1), (dict(lddx=63), -1), (dict(dw=None), -1), (dict(lddw=63), -1), (dict(dw=SOME + 2), -1),
    (dict(db=SOME + 1), -1), (dict(rows=0, dw=None), -1), (dict(dx=2 * SOME), -1), (dict(dx=3 * SOME), -1), (dict(dw=3 * SOME), -1)])
def test_classifier_backward_refusals(E, change, code):
    a = dict(CLASSIFIER, x=2 * SOME, w=3 * SOME, g=SOME, h=SOME, dx=4 * SOME, lddx=64, dw=5 * SOME, lddw=64, db=SOME)
    if "ldx" in change and change["ldx"] > 64:
        a.update(lddx=change["ldx"], lddw=change["ldx"])
    a.update(change)
    rc = E.lib.edl_classifier_log_probs_backward(a["dtype"], a["x"], a["ldx"], a["w"], a["ldw"], a["b"], a["rows"], a["dim"], a["classes"], a["t"], a["lse"],
                                                 a["ent"], a["g"], a["h"], a["dx"], a["lddx"], a["dw"], a["lddw"], a["db"], a["work"], a["bytes"], None)
    assert rc == code and E.lib.edl_last_error()


def test_classifier_workspace_does_not_grow_with_the_pieces_of_the_classes(E):
    """dx is one float32 sum (of a few cuts at most), however many pieces dz comes in."""
    n = C.c_int64()
    for rows, dim, classes in ((65536, 4096, 131072), (65536, 4096, 32768), (8192, 512, 500000)):
        assert E.lib.edl_classifier_workspace(1, SOME, dim, SOME, dim, rows, dim, classes, 1, C.byref(n)) == 0
        assert n.value <= (1 << 30) + 512 * 128 * 128 * 4 + rows * dim * 4 + (1 << 26), (rows, dim, classes, n.value)


def test_classifier_workspace_grows_with_what_it_holds(E):
    def need(x, ldx, w, ldw, rows, dim, classes, backward, dtype=1):
        n = C.c_int64()
        assert E.lib.edl_classifier_workspace(dtype, x, ldx, w, ldw, rows, dim, classes, backward, C.byref(n)) == 0
        return n.value
    aligned = need(SOME, 1024, SOME, 1024, 4096, 1024, 32768, 1)
    assert aligned <= (1 << 30) + 8 * 4096 * 1024 * 4 + (1 << 20)               # dz a piece at a time, and parts of dx
    copied = need(SOME + 2, 1024, SOME, 1025, 4096, 1024, 32768, 1)
    assert copied == aligned + 2 * 1024 * (4096 + 32768) == need(None, 0, None, 0, 4096, 1024, 32768, 1)
    assert need(SOME, 1024, SOME, 1024, 4096, 1024, 32768, 0) < 20 << 20
    assert need(SOME, 1024, SOME, 1024, 0, 1024, 32768, 1) == 0
    for rows in (1, 31, 500, 4097):
        for classes in (1, 100, 5000, 100001):
            for dim in (1, 64, 4096):
                for dtype in (0, 1):
                    for backward in (0, 1):
                        any_way = need(None, 0, None, 0, rows, dim, classes, backward, dtype)
                        ways = [need(SOME + a, dim + b, SOME + c, dim + d, rows, dim, classes, backward, dtype)
                                for a in (0, 4) for b in (0, 1) for c in (0, 4) for d in (0, 1)]
                        assert 0 < max(ways) <= any_way
