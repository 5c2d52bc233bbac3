"""Dropout inside AlexNet jobs: loss and every worker's gradient against float64 with the masks from the host.  Run with -m gpu."""
import pytest
import torch
import torch.nn.functional as F

import head_reference as R
import synth_inputs

pytestmark = pytest.mark.gpu

BASE, WIDE, CLASSES, SIDE, N, B, SEED = 8, 64, 10, 67, 32, 16, 11


@pytest.fixture(scope="module")
def E():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1909_11985_amd as E
    return E


def losses(x, y, params, table, masks, rate, stored):
    """Each sample's loss, in float64 over activations of the type that the job stores (whose rounding lets gradients through)."""
    r = lambda t: t + (t.detach().to(stored).double() - t.detach())        # noqa: E731
    at = {name: (off, size) for name, off, size, _ in table}
    take = lambda name: params[at[name][0]:at[name][0] + at[name][1]]      # noqa: E731
    t = x.permute(0, 3, 1, 2)
    for i, (k, size, stride, pad, pool) in enumerate([(1, 11, 4, 2, True), (3, 5, 1, 2, True), (6, 3, 1, 1, False), (4, 3, 1, 1, False), (4, 3, 1, 1, True)], 1):
        w = take("conv%d.w" % i).view(k * BASE, size, size, t.shape[1]).permute(0, 3, 1, 2)
        t = r(F.relu(F.conv2d(t, w, take("conv%d.b" % i), stride=stride, padding=pad)))
        if pool:
            t = F.max_pool2d(t, 3, 2)
    t = t.permute(0, 2, 3, 1).reshape(t.shape[0], -1)
    for name, mask in zip(("fc1", "fc2"), masks):
        t = r(F.relu(t @ take(name + ".w").view(-1, t.shape[1]).t() + take(name + ".b")))
        t = r(torch.where(mask, t / (1.0 - rate), torch.zeros_like(t)))
    return F.cross_entropy(t @ take("fc3.w").view(-1, t.shape[1]).t() + take("fc3.b"), y, reduction="none")


@pytest.mark.parametrize("dtype,p,rate", [("f32", 1, 0.5), ("f32", 4, 0.25), ("bf16", 2, 0.5)])
def test_alexnet_dropout_gradients_are_the_definitions(E, dtype, p, rate):
    from paper_1909_11985_amd.binding import make_config
    cfg = make_config("alexnet", dtype=dtype, N=N, B=B, p_max=4, lr=0.01, H=SIDE, W=SIDE, C_=3, classes=CLASSES, arch=(BASE, WIDE))
    x, y = synth_inputs.dataset(2, N, SIDE, SIDE, 3, CLASSES)
    job = E.Job(cfg, SEED)
    job.bind_dataset(torch.from_numpy(x).cuda(), torch.from_numpy(y).cuda())
    job.set_dropout(rate)
    table, ops = E.edl_tensor_table(cfg), job.debug_op_count()              # the list ends in fc1, fc2, fc3, loss
    stored = torch.float32 if dtype == "f32" else torch.bfloat16
    tol = 1e-4 if dtype == "f32" else 2e-2      # what layer-by-layer parity of these jobs is held to
    for step in range(2):
        idx, off = job.shard(B, p, *job.progress()[1:])
        loss = job.gradients(p)
        masks = [torch.from_numpy(R.kept(B, WIDE, rate, E.edl_dropout_key(SEED, step, layer))) for layer in (ops - 4, ops - 3)]
        params = torch.from_numpy(job.params()).double().requires_grad_()
        read = params
        if dtype == "bf16":                     # products read bf16 weights; biases stay float32
            bias = torch.zeros_like(params, dtype=torch.bool)
            for name, at, size, _ in table:
                bias[at:at + size] = name.endswith(".b")
            read = torch.where(bias, params, params + (params.detach().to(stored).double() - params.detach()))
        rows = losses(torch.from_numpy(x[idx]).to(stored).double(), torch.from_numpy(y[idx]).long(), read, table, masks, rate, stored)
        assert abs(loss - float(rows.detach().mean())) <= tol * max(1.0, abs(loss))
        for k in range(p):
            (want,) = torch.autograd.grad(rows[off[k]:off[k + 1]].mean(), params, retain_graph=True)
            got = torch.from_numpy(job.grad(k)).double()
            assert float((got - want).norm() / want.norm()) <= tol, (step, k)
        job.apply(p)
