"""Layers and their gradients (netmax_layer_forward, netmax_layer_backward) against the formulas in 64 bits.

Tolerances, with u the type's half unit (bf16 2^-8, the fp16 pairs of fp32 2^-22, fp32 2^-24) and S = sum |x||w| the sum of a product's
magnitudes:
  fp32: each factor is off by at most 2^-22 of itself or 2^-38 of its matrix's largest; products are summed in fp32 by the tensor
        cores, whose steps may drop bits below 2^-23 of the running sum of magnitudes for each of K/16 steps: |dz| <= (2^-21 + (K/16 + 4)
        2^-23) S + 2^-36 K max max;
  bf16: factors are exact, but for dz, which is rounded to bf16 (2^-8 of itself), and the result is rounded once (2^-8).
The activations' slopes are below 1.13 and their own errors a few fp32 units."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ACTIVATIONS = ["none", "relu", "gelu", "silu"]
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


def act(z, name):
    return {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v), "silu": lambda v: v * torch.sigmoid(v)}[name](z)


def product_bound(a, b, storage, rounded=0.0):
    """Error of a @ b^T over the last dimension of both, (M, r, k) x (M, c, k), before the result is rounded; `rounded`: the
    relative error of a factor that was rounded beforehand."""
    K = a.shape[-1]
    S = a.double().abs() @ b.double().abs().mT
    factors = 2.0 ** -21 if storage == "f32" else 0.0
    tiny = 2.0 ** -36 * K * a.double().abs().amax() * b.double().abs().amax() if storage == "f32" else 0.0
    return (factors + rounded + (K / 16 + 4) * 2.0 ** -23) * S + tiny


def rounded(v, storage):
    return (2.0 ** -8 if storage == "bf16" else 2.0 ** -23) * v.abs() + 1e-37


def workspace(nm, M, n, n_in, n_out, storage):
    return torch.full((nm.netmax_layer_workspace_size(M, n, n_in, n_out, storage),), 0x7F, dtype=torch.uint8, device="cuda")


def check(got, want, bound, what):
    excess = (got.double() - want).abs() - bound
    assert not torch.isnan(excess).any(), what
    assert excess.max().item() <= 0, f"{what}: {excess.max().item():.3e} beyond the bound ({(got.double() - want).abs().max().item():.3e} off)"


SIZES = [  # M, n, n_in, n_out
    (1, 1, 1, 1), (2, 1, 5, 3), (4, 1, 512, 10), (3, 7, 64, 64), (2, 64, 64, 128), (1, 130, 129, 131), (5, 77, 1001, 333), (2, 300, 72, 520),
    (1, 2, 4100, 17), (2, 513, 8, 264), (1, 1024, 768, 1280), (3, 2, 16, 2050), (37, 3, 24, 40),
    (2, 11, 520, 1300), (3, 16, 130, 77), (150, 8, 40, 33), (160, 4, 72, 48), (2, 5, 1001, 600), (1, 9, 64, 5000),
]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(nm, size, storage):
    M, n, n_in, n_out = size
    t = TYPES[storage]
    x, w = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, std=n_in ** -0.5, dtype=t)
    b, r = normal(3, M, n_out, dtype=t), normal(4, M, n, n_out, dtype=t)
    ws = workspace(nm, M, n, n_in, n_out, storage)
    raw = x.double() @ w.double().mT
    bound = product_bound(x, w, storage)
    for name in ACTIVATIONS if n * n_out < 10000 else ["gelu"]:
        for bias, residual, keep in ((True, True, True), (False, False, False), (True, False, True)):
            y = torch.full((M, n, n_out), float("nan"), dtype=t, device="cuda")
            z = torch.full_like(y, float("nan")) if keep else None
            nm.netmax_layer_forward(x, w, y, bias=b if bias else None, residual=r if residual else None, z=z, activation=name, workspace=ws)
            nm.netmax_workspace_status(ws)
            want_z = raw + b.double()[:, None] if bias else raw
            off = bound + 2.0 ** -22 * (raw.abs() + want_z.abs())
            if keep:
                check(z, want_z, off + rounded(want_z, storage), "z")
            want = act(want_z, name)
            off = 1.13 * off + 2.0 ** -20 * want_z.abs()
            if residual:
                want = want + r.double()
                off = off + 2.0 ** -23 * want.abs()
            check(y, want, off + rounded(want.abs() + off, storage), f"y {name}")


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(nm, size, storage):
    M, n, n_in, n_out = size
    t = TYPES[storage]
    x, w = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, std=n_in ** -0.5, dtype=t)
    dy, z = normal(5, M, n, n_out, dtype=t), normal(6, M, n, n_out, std=2.0, dtype=t)
    ws = workspace(nm, M, n, n_in, n_out, storage)
    for name in ACTIVATIONS if n * n_out < 10000 else ["gelu"]:
        dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
        db = torch.full((M, n_out), float("nan"), dtype=t, device="cuda")
        nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=db, z=z if name != "none" else None, activation=name, workspace=ws)
        nm.netmax_workspace_status(ws)
        dz = dy.double()
        if name != "none":
            v = z.double().requires_grad_(True)
            dz, = torch.autograd.grad(act(v, name), v, dz)
        slope = 2.0 ** -20 * dy.double().abs() * (1 + z.double().abs())   # the slope's own error, fp32 units
        if name == "none":
            slope = torch.zeros_like(slope)
        before = (2.0 ** -8 if storage == "bf16" and name != "none" else 0.0)
        want = dz @ w.double()
        off = product_bound(dz, w.mT, storage, before) + slope @ w.double().abs()
        check(dx, want, off + rounded(want.abs() + off, storage), f"dx {name}")
        want = dz.mT @ x.double()
        off = product_bound(dz.mT, x.mT, storage, before) + slope.mT @ x.double().abs()
        check(dw, want, off + rounded(want.abs() + off, storage), f"dweight {name}")
        want = dz.sum(1)
        off = (n + 4) * 2.0 ** -24 * dz.abs().sum(1) + slope.sum(1)
        check(db, want, off + rounded(want.abs() + off, storage), f"dbias {name}")


def forward(nm, x, w, **kw):
    storage = "f32" if x.dtype == torch.float32 else "bf16"
    M, n, n_in = x.shape
    y = torch.full((M, n, w.shape[1]), float("nan"), dtype=x.dtype, device="cuda")
    ws = workspace(nm, M, n, n_in, w.shape[1], storage)
    nm.netmax_layer_forward(x, w, y, workspace=ws, **kw)
    nm.netmax_workspace_status(ws)
    return y


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 40, 150])
def test_views(nm, storage, n):
    """Weights inside replicas, workers woven into one another, odd offsets, one matrix for all: the results of dense copies, bit for bit
    where the same path is taken, and nothing outside the outputs written."""
    t, M, n_in, n_out = TYPES[storage], 5, 72, 88
    dense_x, dense_w, dense_dy = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, dtype=t), normal(3, M, n, n_out, dtype=t)

    def embed(v, kind):
        M, r, c = v.shape
        if kind == "replica":       # behind 3 elements of a row as long as the matrix and 13 more
            base = torch.full((M, r * c + 16), 7.0, dtype=t, device="cuda")
            view = base.as_strided((M, r, c), (r * c + 16, c, 1), 3)
        elif kind == "woven":
            base = torch.full((r, M, c), 7.0, dtype=t, device="cuda")
            view = base.transpose(0, 1)
        else:
            base = torch.full((M, r, c + 24), 7.0, dtype=t, device="cuda")
            view = base[:, :, 8:8 + c]
        view.copy_(v)
        return base, view

    want_y, want_z = torch.empty(M, n, n_out, dtype=t, device="cuda"), torch.empty(M, n, n_out, dtype=t, device="cuda")
    ws = workspace(nm, M, n, n_in, n_out, storage)
    nm.netmax_layer_forward(dense_x, dense_w, want_y, z=want_z, activation="silu", workspace=ws)
    want_dx, want_dw, want_db = torch.empty_like(dense_x), torch.empty_like(dense_w), torch.empty(M, n_out, dtype=t, device="cuda")
    nm.netmax_layer_backward(dense_dy, dense_x, dense_w, dx=want_dx, dweight=want_dw, dbias=want_db, z=want_z, activation="silu", workspace=ws)
    unit = 2.0 ** -7 if storage == "bf16" else 2.0 ** -18
    near = lambda got, want: ((got.double() - want.double()).norm() <= unit * want.double().norm()).item()  # noqa: E731
    for kind in ("replica", "woven", "padded"):
        (_, x), (_, w), (_, dy) = embed(dense_x, kind), embed(dense_w, kind), embed(dense_dy, kind)
        (by, y), (bz, z) = embed(torch.zeros_like(want_y), kind), embed(torch.zeros_like(want_z), kind)
        nm.netmax_layer_forward(x, w, y, z=z, activation="silu", workspace=ws)
        assert near(y, want_y) and near(z, want_z), kind
        (bx, dx), (bw, dw) = embed(torch.zeros_like(dense_x), kind), embed(torch.zeros_like(dense_w), kind)
        bb = torch.full((M, n_out + 5), 7.0, dtype=t, device="cuda")
        z.copy_(want_z)
        nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=bb[:, 2:2 + n_out], z=z, activation="silu", workspace=ws)
        nm.netmax_workspace_status(ws)
        assert near(dx, want_dx) and near(dw, want_dw) and near(bb[:, 2:2 + n_out], want_db), kind
        assert (bb[:, :2] == 7).all() and (bb[:, 2 + n_out:] == 7).all()
        for base, view in ((by, y), (bz, z), (bx, dx), (bw, dw)):
            view.fill_(7.0)
            assert (base == 7).all(), kind      # (what was outside the view still is as it was)
    one = dense_x[:1].expand(M, n, n_in)
    assert near(forward(nm, one, dense_w), forward(nm, one.contiguous(), dense_w))
    same = dense_w[:1].expand(M, n_out, n_in)
    assert near(forward(nm, dense_x, same), forward(nm, dense_x, same.contiguous()))


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 60, 300])
def test_the_residual_as_the_output(nm, storage, n):
    t = TYPES[storage]
    x, w, r = normal(1, 3, n, 64, dtype=t), normal(2, 3, 96, 64, dtype=t), normal(3, 3, n, 96, dtype=t)
    want = torch.empty_like(r)
    ws = workspace(nm, 3, n, 64, 96, storage)
    nm.netmax_layer_forward(x, w, want, residual=r, activation="gelu", workspace=ws)
    nm.netmax_layer_forward(x, w, r, residual=r, activation="gelu", workspace=ws)
    assert torch.equal(r, want)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_no_rows(nm, storage):
    t = TYPES[storage]
    w = normal(2, 3, 9, 7, dtype=t)
    x, y = torch.empty(3, 0, 7, dtype=t, device="cuda"), torch.empty(3, 0, 9, dtype=t, device="cuda")
    ws = workspace(nm, 3, 0, 7, 9, storage)
    nm.netmax_layer_forward(x, w, y, workspace=ws)
    dw, db = torch.full((3, 9, 12), 5.0, dtype=t, device="cuda"), torch.full((3, 9), 5.0, dtype=t, device="cuda")
    nm.netmax_layer_backward(y, x, w, dweight=dw[:, :, 2:9], dbias=db, workspace=ws)
    nm.netmax_workspace_status(ws)
    assert (dw[:, :, 2:9] == 0).all() and (dw[:, :, :2] == 5).all() and (dw[:, :, 9:] == 5).all() and (db == 0).all()


@pytest.mark.parametrize("n", [2, 50, 200])
def test_each_row_for_itself(nm, n):
    """fp32: rows of x and of the weights from 1e-18 to 1e18 in one call are each as exact as alone; a row with a NaN or an infinity makes
    nothing else other than finite."""
    x, w = normal(1, 2, n, 70), normal(2, 2, 90, 70)
    a = 10.0 ** torch.linspace(-18, 18, n).cuda().float()
    b = 10.0 ** torch.linspace(18, -18, 90).cuda().float()
    xs, wsd = x * a[None, :, None], w * b[None, :, None]
    y = forward(nm, xs, wsd).double()
    want = xs.double() @ wsd.double().mT
    bound = (2.0 ** -21 + (70 / 16 + 4) * 2.0 ** -23) * (xs.double().abs() @ wsd.double().abs().mT) + 2.0 ** -34 * 70 * xs.double().abs().amax(2)[:, :, None] * wsd.double().abs().amax(2)[:, None]
    assert ((y - want).abs() <= bound + 2.0 ** -23 * want.abs()).all()
    bad = x.clone()
    bad[0, 1, 3], bad[1, 0, 5] = float("nan"), float("inf")
    y, clean = forward(nm, bad, w), forward(nm, x, w)
    assert not torch.isfinite(y[0, 1]).any() and not torch.isfinite(y[1, 0]).any()
    y[0, 1], y[1, 0] = clean[0, 1], clean[1, 0]
    assert torch.equal(y, clean)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 200])
def test_in_a_graph_and_on_another_stream(nm, storage, n):
    t, M, n_in, n_out = TYPES[storage], 4, 96, 160
    x, w, dy = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, dtype=t), normal(3, M, n, n_out, dtype=t)
    y, z = torch.empty(M, n, n_out, dtype=t, device="cuda"), torch.empty(M, n, n_out, dtype=t, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(M, n_out, dtype=t, device="cuda")
    ws = workspace(nm, M, n, n_in, n_out, storage)

    def run(stream):
        nm.netmax_layer_forward(x, w, y, z=z, activation="gelu", workspace=ws, stream=stream)
        nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=db, z=z, activation="gelu", workspace=ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(side.cuda_stream)
    side.synchronize()
    first = [v.clone() for v in (y, dx, dw, db)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(torch.cuda.current_stream().cuda_stream)
    for v in (y, z, dx, dw, db):
        v.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for got, want in zip((y, dx, dw, db), first):
        assert torch.equal(got, want)


def test_two_streams_at_once(nm):
    """Calls with workspaces of their own on two streams, products in pairs of CTAs beside clusters and small matrices."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    x, w = normal(1, 8, 700, 320), normal(2, 8, 640, 320)
    u, v = normal(3, 12, 60, 1500), normal(4, 40, 64, 64)
    y, ou, ov = torch.empty(8, 700, 640, device="cuda"), torch.empty_like(u), torch.empty_like(v)
    wy = workspace(nm, 8, 700, 320, 640, "f32")
    wu = torch.empty(nm.netmax_orthogonalise_workspace_size(12, 60, 1500), dtype=torch.uint8, device="cuda")
    wv = torch.empty(nm.netmax_orthogonalise_workspace_size(40, 64, 64), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    nm.netmax_layer_forward(x, w, y, workspace=wy)
    nm.netmax_orthogonalise(u, ou, workspace=wu)
    nm.netmax_orthogonalise(v, ov, workspace=wv)
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, ou, ov)]
    for t in (y, ou, ov):
        t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        nm.netmax_layer_forward(x, w, y, workspace=wy, stream=a.cuda_stream)
        nm.netmax_orthogonalise(u, ou, workspace=wu, stream=b.cuda_stream)
        nm.netmax_orthogonalise(v, ov, workspace=wv, stream=b.cuda_stream)
    torch.cuda.synchronize()
    for ws in (wy, wu, wv):
        nm.netmax_workspace_status(ws)
    for got, w_ in zip((y, ou, ov), want):
        assert torch.equal(got, w_)


@pytest.mark.parametrize("n", [2, 12, 40])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_workers_further_apart_than_32_bits(nm, storage, n):
    """Two workers' views 2^31 + 64 elements apart: every entry's offsets are 64 bits wide."""
    t, n_in, n_out, apart = TYPES[storage], 40, 72, 2 ** 31 + 64
    used = 3 * n * n_out + 2 * n * n_in + 2 * n_out * n_in  # of all views, x, w, z, y, dy, dx and dw, in one worker
    room = torch.empty(apart + used, dtype=t, device="cuda")
    at = 0
    def far(seed, rows, cols):  # the two matrices of a view, each in its worker's part of the room
        nonlocal at
        v = room.as_strided((2, rows, cols), (apart, cols, 1), at)
        at += rows * cols
        if seed:
            v.copy_(normal(seed, 2, rows, cols, dtype=t))
        return v
    x, w, z = far(1, n, n_in), far(2, n_out, n_in), far(0, n, n_out)
    y = far(0, n, n_out)
    ws = workspace(nm, 2, n, n_in, n_out, storage)
    nm.netmax_layer_forward(x, w, y, z=z, activation="silu", workspace=ws)
    nm.netmax_workspace_status(ws)
    want = x.double() @ w.double().mT
    off = product_bound(x, w, storage) + 2.0 ** -22 * want.abs()
    check(z, want, off + rounded(want, storage), "z")
    value = act(want, "silu")
    check(y, value, 1.13 * off + 2.0 ** -20 * want.abs() + rounded(value.abs() + off, storage), "y")
    dy, dx, dw = far(3, n, n_out), far(0, n, n_in), far(0, n_out, n_in)
    nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, workspace=ws)
    nm.netmax_workspace_status(ws)
    for got, a, b, what in ((dx, dy, w.mT, "dx"), (dw, dy.mT, x.mT, "dw")):
        true = a.double() @ b.mT.double()
        check(got, true, product_bound(a, b, storage) + rounded(true, storage), what)
