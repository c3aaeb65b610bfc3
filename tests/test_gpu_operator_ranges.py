"""The operators on real weights at the ends of their ranges: sums as long as a view may be, rows of very different size, what is not a
number, no rows at all, streams and workspaces."""
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
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def layer_workspace(nm, M, n, n_in, n_out, storage):
    return torch.full((nm.netmax_layer_workspace_size(M, n, n_in, n_out, storage),), 0x7F, dtype=torch.uint8, device="cuda")


# ---- long sums
# All values lie in [0.5, 1.5), so that nothing cancels.  An accumulator of the tensor cores holds at most 2^15 k of a sum, and what its
# 2^11 steps of 16 k drop is less than 2^-23 of the running sum each: 2^-12 in all; parts of such a sum are added in fp32, fewer than
# 2^11 of them here, each addition off by 2^-24: 2^-13.  The result is rounded to bfloat16, 2^-8.
LONG = 2.0 ** -12 + 2.0 ** -13 + 2.0 ** -8


def positive(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (0.5 + torch.rand(*shape, generator=g, device="cuda")).to(torch.bfloat16)


def long_product(a, b):
    """a (r, k) times b (c, k) transposed, in 64 bits, a stretch of k at a time."""
    total = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], 1 << 20):
        total += a[:, k:k + (1 << 20)].double() @ b[:, k:k + (1 << 20)].double().T
    return total


@pytest.mark.parametrize("activation", ["none", "relu"])
@pytest.mark.parametrize("size", [(1, 1 << 23, 16, 24), (1, (1 << 23) + 77, 9, 5), (2, 300_000, 200, 136)], ids=str)
def test_gradients_of_many_rows(nm, size, activation):
    """bfloat16: the sums of dW run over all rows of the batch."""
    M, n, n_in, n_out = size
    x, dy, w = positive(1, M, n, n_in), positive(2, M, n, n_out), positive(3, M, n_out, n_in)
    z = torch.ones_like(dy)
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    ws = layer_workspace(nm, M, n, n_in, n_out, "bf16")
    nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, z=z if activation != "none" else None, activation=activation, workspace=ws)
    nm.netmax_workspace_status(ws)
    for i in range(M):
        want = long_product(dy[i].T, x[i].T)
        assert ((dw[i].double() - want).abs() <= LONG * want).all(), ((dw[i].double() - want) / want).abs().max().item()
        rows = slice(0, n, 997)
        want = dy[i, rows].double() @ w[i].double()
        assert ((dx[i, rows].double() - want).abs() <= LONG * want).all()


def test_layers_of_many_inputs(nm):
    n, n_in, n_out = 24, (1 << 22) + 8, 40
    x, w = positive(1, 1, n, n_in), positive(2, 1, n_out, n_in)
    y = torch.full((1, n, n_out), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = layer_workspace(nm, 1, n, n_in, n_out, "bf16")
    nm.netmax_layer_forward(x, w, y, workspace=ws)
    nm.netmax_workspace_status(ws)
    want = long_product(x[0], w[0])
    assert ((y[0].double() - want).abs() <= LONG * want).all(), ((y[0].double() - want) / want).abs().max().item()


def test_long_matrices_orthogonalised(nm):
    """bfloat16: S = X X^T sums over the longer side, here 74,899 columns in a part.  The rows are Walsh functions, orthogonal to one another, so
    every step is the quintic of one number; the result is rounded to bfloat16 (2^-8), S and the polynomial to fp16 (2^-11 each, at most |b| + 2 |c| S = 8
    times as much of X a step, carried on by at most 3.4445 a step over two steps); LONG's first two parts enter as S's roundings do."""
    count, rows, cols = 10, 130, 1 << 19
    r, c = torch.arange(rows, device="cuda")[:, None], torch.arange(256, device="cuda")[None]
    common, sign = r & c, torch.zeros(rows, 256, dtype=torch.int64, device="cuda")
    for bit in range(8):
        sign ^= common >> bit & 1
    u = (1 - 2 * sign).to(torch.bfloat16).repeat(1, cols // 256).expand(count, rows, cols).contiguous()
    out = torch.full_like(u, float("nan"))
    ws = torch.full((nm.netmax_orthogonalise_workspace_size(count, rows, cols, "bf16"),), 0x7F, dtype=torch.uint8, device="cuda")
    nm.netmax_orthogonalise(u, out, steps=2, workspace=ws)
    nm.netmax_workspace_status(ws)
    s = rows ** -0.5
    for _ in range(2):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    s /= cols ** 0.5
    off = (2.0 ** -8 + 16 * (2.0 ** -11 + 2.0 ** -12 + 2.0 ** -13)) * s
    for k in range(count):
        assert ((out[k].double() - u[k].double() * s).abs() <= off).all()
