"""Values that the operators on real weights have to keep apart: NaN and infinities in the gradient's inputs, rows of very different size,
columns of one wide buffer, no rows at all."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def nm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2009_05766_b200 import binding
    binding.lib()
    return binding


def normal(seed, *shape, std=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std).to(dtype).cuda()


def backward(nm, dy, x, w, z, activation):
    storage = "f32" if x.dtype == torch.float32 else "bf16"
    M, n, n_in = x.shape
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(M, w.shape[1], dtype=x.dtype, device="cuda")
    ws = torch.full((nm.netmax_layer_workspace_size(M, n, n_in, w.shape[1], storage),), 0x7F, dtype=torch.uint8, device="cuda")
    nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=db, z=z if activation != "none" else None, activation=activation, workspace=ws)
    nm.netmax_workspace_status(ws)
    return dx, dw, db


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 12, 90])
@pytest.mark.parametrize("activation", ["none", "relu", "gelu", "silu"])
def test_what_is_not_finite_spreads_as_far_as_it_counts(nm, activation, n, storage):
    """A NaN or an infinity among dy, z, x or the weights makes those sums infinite or NaN that it enters, and leaves all others as they were.  (relu's
    slope at an infinite z is 0 or 1.)"""
    t, M, n_in, n_out, worker, row, out, col = TYPES[storage], 2, 70, 90, 1, 2, 17, 5
    sources = {"dy": normal(1, M, n, n_out, dtype=t), "z": normal(2, M, n, n_out, dtype=t), "x": normal(3, M, n, n_in, dtype=t), "w": normal(4, M, n_out, n_in, dtype=t)}
    places = {"dy": (worker, row, out), "z": (worker, row, out), "x": (worker, row, col), "w": (worker, out, col)}
    for name, at in places.items():
        sources[name][at] = 0.25        # (the largest of no matrix)
    call = lambda s: backward(nm, s["dy"], s["x"], s["w"], s["z"], activation)  # noqa: E731
    clean = call(sources)
    for name, at in places.items():
        for value in (float("nan"), float("inf"), float("-inf")):
            if name == "z" and (activation == "none" or (activation == "relu" and value == value)):
                continue
            changed = dict(sources)
            changed[name] = sources[name].clone()
            changed[name][at] = value
            touched = [torch.zeros_like(v, dtype=torch.bool) for v in clean]
            if name in ("dy", "z"):
                touched[0][worker, row] = touched[1][worker, out] = touched[2][worker, out] = True
            elif name == "x":
                touched[1][worker, :, col] = True
            else:
                touched[0][worker, :, col] = True
            for got, want, where in zip(call(changed), clean, touched):
                assert not torch.isfinite(got[where]).any(), (name, value)
                assert torch.equal(got[~where], want[~where]), (name, value)


@pytest.mark.parametrize("n", [12, 40, 300])
def test_gradients_of_rows_of_different_size(nm, n):
    """fp32: rows of dy from 1 down to 2^-40.  Up to 16 rows every value counts in full; beyond, factors keep 22 bits and no less than 2^-38 of their
    matrix's largest, so that |dx| and |dW| are off by at most (3 2^-22 + (K/16 + 4) 2^-23) sum |a||b| + 2^-37 sum (max |a| |b| + |a| max |b|):
    each factor's rounding, the product of the two low parts that is left out, and the sum's."""
    M, n_in, n_out = 2, 72, 104
    x, w = normal(1, M, n, n_in), normal(2, M, n_out, n_in)
    dy = normal(3, M, n, n_out) * 2.0 ** torch.linspace(0, -40, n).cuda()[None, :, None]
    dx, dw, db = backward(nm, dy, x, w, None, "none")
    for got, a, b in ((dx, dy, w.mT), (dw, dy.mT, x.mT)):
        a, b = a.double(), b.double()
        K = a.shape[-1]
        want, size = a @ b.mT, a.abs() @ b.abs().mT
        top = lambda v: v.abs().amax((1, 2), keepdim=True)  # noqa: E731
        floor = 0.0 if n <= 16 else 2.0 ** -37 * (top(a) * b.abs().sum(2)[:, None, :] + top(b) * a.abs().sum(2)[:, :, None])
        assert ((got.double() - want).abs() <= (3 * 2.0 ** -22 + (K / 16 + 4) * 2.0 ** -23) * size + floor + 1e-37).all()
    want = dy.double().sum(1)
    assert ((db.double() - want).abs() <= (n + 4) * 2.0 ** -24 * dy.double().abs().sum(1) + 1e-37).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("M", [1, 3])
@pytest.mark.parametrize("n", [3, 40, 150])
def test_columns_of_one_wide_buffer(nm, n, M, storage):
    """Inputs and outputs side by side in the rows of one buffer (one worker's rows behind another's, and workers woven into one another)."""
    t, n_in, n_out = TYPES[storage], 40, 64
    width = 2 * n_in + 4 * n_out
    x, w, dy, r = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, dtype=t), normal(3, M, n, n_out, dtype=t), normal(4, M, n, n_out, dtype=t)
    ws = torch.full((nm.netmax_layer_workspace_size(M, n, n_in, n_out, storage),), 0x7F, dtype=torch.uint8, device="cuda")
    want_y, want_z, want_dx = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(x)
    dw = torch.empty_like(w)
    nm.netmax_layer_forward(x, w, want_y, residual=r, z=want_z, activation="silu", workspace=ws)
    nm.netmax_layer_backward(dy, x, w, dx=want_dx, dweight=dw, z=want_z, activation="silu", workspace=ws)
    unit = 2.0 ** -7 if storage == "bf16" else 2.0 ** -18
    for buffer in (torch.full((M, n, width), 7.0, dtype=t, device="cuda"), torch.full((n, M, width), 7.0, dtype=t, device="cuda").transpose(0, 1)):
        ends = torch.tensor([n_in, n_out, n_out, n_out, n_out, n_in]).cumsum(0).tolist()
        vx, vy, vz, vr, vdy, vdx = (buffer[:, :, a:b] for a, b in zip([0] + ends[:-1], ends))
        vx.copy_(x), vr.copy_(r), vdy.copy_(dy)
        nm.netmax_layer_forward(vx, w, vy, residual=vr, z=vz, activation="silu", workspace=ws)
        nm.netmax_workspace_status(ws)
        for got, want in ((vy, want_y), (vz, want_z)):
            assert (got.double() - want.double()).norm() <= unit * want.double().norm()
        vz.copy_(want_z)
        nm.netmax_layer_backward(vdy, vx, w, dx=vdx, dweight=dw, z=vz, activation="silu", workspace=ws)
        nm.netmax_workspace_status(ws)
        assert (vdx.double() - want_dx.double()).norm() <= unit * want_dx.double().norm()
        assert torch.equal(vx, x) and torch.equal(vr, r) and torch.equal(vdy, dy)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_no_rows_and_gradients_far_apart(nm, storage):
    """A batch without rows clears dweight, whatever its row stride: of one row (where it counts for nothing) and of rows more than 2^31 bytes apart."""
    t = TYPES[storage]
    apart = 2 ** 30 + 8
    room = torch.full((apart + 64,), 5.0, dtype=t, device="cuda")
    for n_out, row in ((1, 1 << 36), (2, apart)):
        ws = torch.full((nm.netmax_layer_workspace_size(1, 0, 7, n_out, storage),), 0x7F, dtype=torch.uint8, device="cuda")
        room[:64], room[apart:] = 5.0, 5.0
        a = nm.Layer()
        a.M, a.n, a.n_in, a.n_out, a.storage, a.activation, a.device = 1, 0, 7, n_out, nm.STORAGE[storage], 0, 0
        a.dweight = nm.View(room.data_ptr(), row, 0)
        a.stream, a.workspace, a.workspace_bytes = torch.cuda.current_stream().cuda_stream, ws.data_ptr(), ws.numel()
        nm._check(nm.lib().netmax_layer_backward(C.addressof(a)))
        torch.cuda.synchronize()
        assert (room[:7] == 0).all() and (room[7:64] == 5).all()
        assert (room[apart:apart + 7] == (0 if n_out == 2 else 5)).all() and (room[apart + 7:] == 5).all() and (room[apart - 64:apart] == 5).all()
