"""The operators on real weights at sizes that take the kernels of large problems (on 148 SMs: pairs of CTAs, three and more tiles a pair, Gram
matrices in parts of k by pairs, more shapes than a launch has groups), against 64 bits; and how exact fp32 sums are, whatever their length."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_layers import TYPES, act, check as check_layer, normal, product_bound, rounded, workspace  # noqa: E402
from test_gpu_orthogonalise import check as check_orthogonal, exact_step, orthogonalise, step_case, update  # noqa: E402


@pytest.fixture(scope="module")
def nm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2009_05766_b200 import binding
    binding.lib()
    return binding


LARGE = [(8, 1024, 320, 2048), (8, 1001, 200, 2041), (3, 2560, 72, 1800), (40, 300, 136, 512)]      # M, n, n_in, n_out


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large_layers(nm, size, storage):
    M, n, n_in, n_out = size
    t = TYPES[storage]
    x, w = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, std=n_in ** -0.5, dtype=t)
    b, r = normal(3, M, n_out, dtype=t), normal(4, M, n, n_out, dtype=t)
    ws = workspace(nm, M, n, n_in, n_out, storage)
    raw = x.double() @ w.double().mT
    bound = product_bound(x, w, storage)
    for name, extras in (("gelu", True), ("none", False)):
        y = torch.full((M, n, n_out), float("nan"), dtype=t, device="cuda")
        z = torch.full_like(y, float("nan")) if extras else None
        nm.netmax_layer_forward(x, w, y, bias=b if extras else None, residual=r if extras else None, z=z, activation=name, workspace=ws)
        nm.netmax_workspace_status(ws)
        want_z = raw + b.double()[:, None] if extras else raw
        off = bound + 2.0 ** -22 * (raw.abs() + want_z.abs())
        if extras:
            check_layer(z, want_z, off + rounded(want_z, storage), "z")
        want = act(want_z, name)
        off = 1.13 * off + 2.0 ** -20 * want_z.abs()
        if extras:
            want = want + r.double()
            off = off + 2.0 ** -23 * want.abs()
        check_layer(y, want, off + rounded(want.abs() + off, storage), "y")


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_gradients_of_large_layers(nm, size, storage):
    M, n, n_in, n_out = size
    t = TYPES[storage]
    x, w = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, std=n_in ** -0.5, dtype=t)
    dy = normal(5, M, n, n_out, dtype=t)
    dx, dw, db = torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full((M, n_out), float("nan"), dtype=t, device="cuda")
    ws = workspace(nm, M, n, n_in, n_out, storage)
    nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=db, workspace=ws)
    nm.netmax_workspace_status(ws)
    dz = dy.double()
    want = dz @ w.double()
    off = product_bound(dy, w.mT, storage)
    check_layer(dx, want, off + rounded(want.abs() + off, storage), "dx")
    want = dz.mT @ x.double()
    off = product_bound(dy.mT, x.mT, storage)
    check_layer(dw, want, off + rounded(want.abs() + off, storage), "dweight")
    want = dz.sum(1)
    off = (n + 4) * 2.0 ** -24 * dz.abs().sum(1)
    check_layer(db, want, off + rounded(want.abs() + off, storage), "dbias")


# Relative error in the 2-norm for factors that are normal noise.  A part of 256 k is 16 steps of products of the high parts (those with a low part come
# first and are 2^-11 of them); each drops less than 2^-23 of the running sum, which is at most the part's in the root mean square: 2^-19 of
# a part.  Parts are independent of one another, so the same holds for their sum.  Factors: 2^-22 each, and 2^-22 for the product of the low
# parts.  Up to 32 parts are added in fp32, each addition off by 2^-24 of the sum so far, independently: 6 2^-24; the result's own rounding 2^-24.
FLAT = 2.0 ** -19 + 3 * 2.0 ** -22 + 7 * 2.0 ** -24


@pytest.mark.parametrize("K", [512, 2048, 8192])
def test_fp32_sums_are_as_exact_when_they_are_long(nm, K):
    side = 256
    error = lambda got, want: ((got.double() - want).norm() / want.norm()).item()  # noqa: E731
    x, w = normal(1, 2, side, K), normal(2, 2, side, K)
    y = torch.full((2, side, side), float("nan"), device="cuda")
    ws = workspace(nm, 2, side, K, side, "f32")
    nm.netmax_layer_forward(x, w, y, workspace=ws)
    assert error(y, x.double() @ w.double().mT) <= FLAT
    dy, wide = normal(3, 2, side, K), normal(4, 2, K, side)     # dx sums over K outputs
    dx = torch.full((2, side, side), float("nan"), device="cuda")
    ws = workspace(nm, 2, side, side, K, "f32")
    nm.netmax_layer_backward(dy, x[:, :, :side], wide, dx=dx, workspace=ws)
    assert error(dx, dy.double() @ wide.double()) <= FLAT
    dy, x = normal(5, 2, K, side), normal(6, 2, K, side)        # dW sums over K rows
    dw = torch.full((2, side, side), float("nan"), device="cuda")
    ws = workspace(nm, 2, K, side, side, "f32")
    nm.netmax_layer_backward(dy, x, wide[:, :side], dweight=dw, workspace=ws)
    assert error(dw, dy.double().mT @ x.double()) <= FLAT
    nm.netmax_workspace_status(ws)


# ---- Newton-Schulz
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(24, 512, 600), (22, 600, 500), (8, 512, 1536), (9, 1500, 510), (6, 512, 1536)], ids=str)
def test_large_batches_orthogonalised(nm, size, storage):
    """Gram matrices and polynomials by pairs of CTAs; Gram matrices in parts of k (bfloat16: eight of 512 x 1536, fp32: six)."""
    u = update(1, *size, dtype=TYPES[storage])
    check_orthogonal(orthogonalise(nm, u), u)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_a_step_of_more_shapes_than_a_launch_has_groups(nm, storage):
    """Fourteen shapes of eight workers: twelve in one launch, by pairs of CTAs, and two in another."""
    M, matrices, at = 8, [], 5
    for k in range(14):
        rows, cols = (256, 480 + 8 * k) if k % 2 else (480 + 9 * k, 256)
        matrices.append((at, rows, cols, 1.0 + 0.1 * k))
        at += rows * cols + k % 3
    d = at + 11
    x, m, grad, peers, weights = step_case(3, M, d, matrices, storage)
    want, off, want_m = exact_step(x, m, grad, matrices, peers, weights, 0.05, 0.9, True, 0.01, 5)
    ws = torch.full((nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage),), 0x7F, dtype=torch.uint8, device="cuda")
    new, m_next = torch.full_like(x, float("nan")), torch.full_like(m, float("nan"))
    nm.netmax_orthogonalised_step(x, new, grad, m, m_next, matrices, peers, weights, lr=0.05, mu=0.9, decay=0.01, workspace=ws)
    nm.netmax_workspace_status(ws)
    assert ((new.double() - want).abs() - off).max().item() <= 0
    assert ((m_next.double() - want_m).abs() <= 2.0 ** -23 * (want_m.abs() + m.double().abs()) + 1e-30).all()
    # 2-norms of what the matrices' updates add, for all but a rounding of the replicas
    moved, true = new.double() - x.double(), want - x.double()
    unit = 2.0 ** -8 if storage == "bf16" else 2.0 ** -23
    for at, rows, cols, scale in matrices:
        part = slice(at, at + rows * cols)
        assert (moved[:, part] - true[:, part]).norm() <= 2.0 ** -7 * true[:, part].norm() + 2 * unit * want[:, part].norm()
