"""Calls of the operators on real weights that their documentation allows: any subset of a gradient's outputs, one matrix for all workers, the
longest and thinnest sizes, as many matrices as a step takes, peers that are no workers, and a context's rounds across its trace ring."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_layers import TYPES, check as check_layer, normal, product_bound, rounded, workspace  # noqa: E402
from test_gpu_orthogonalise import check as check_orthogonal, exact_step, orthogonalise, step_case  # noqa: E402


@pytest.fixture(scope="module")
def nm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2009_05766_b200 import binding
    binding.lib()
    return binding


# ---- layers
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("activation", ["none", "silu"])
@pytest.mark.parametrize("n", [3, 14, 70])
def test_any_outputs_of_a_gradient(nm, n, activation, storage):
    t, M, n_in, n_out = TYPES[storage], 3, 72, 200
    x, w, dy, z = normal(1, M, n, n_in, dtype=t), normal(2, M, n_out, n_in, dtype=t), normal(3, M, n, n_out, dtype=t), normal(4, M, n, n_out, dtype=t)
    shapes = {"dx": x, "dweight": w, "dbias": dy[:, 0]}

    def call(names):
        ws = workspace(nm, M, n, n_in, n_out, storage)
        out = {k: torch.full_like(shapes[k], float("nan"), memory_format=torch.contiguous_format) for k in names}
        nm.netmax_layer_backward(dy, x, w, z=z if activation != "none" else None, activation=activation, workspace=ws, **out)
        nm.netmax_workspace_status(ws)
        return out

    want = call(shapes)
    unit = 2.0 ** -7 if storage == "bf16" else 2.0 ** -18
    for names in ((), ("dx",), ("dweight",), ("dbias",), ("dx", "dbias"), ("dweight", "dbias"), ("dx", "dweight")):
        for k, got in call(names).items():
            assert (got.double() - want[k].double()).norm() <= unit * want[k].double().norm(), (names, k)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("activation", ["none", "gelu"])
@pytest.mark.parametrize("n", [3, 14, 70])
def test_gradients_from_one_matrix_for_all_workers(nm, n, activation, storage):
    t, M, n_in, n_out = TYPES[storage], 4, 72, 136
    dense = {"x": normal(1, M, n, n_in, dtype=t), "weight": normal(2, M, n_out, n_in, dtype=t), "dy": normal(3, M, n, n_out, dtype=t), "z": normal(4, M, n, n_out, dtype=t)}

    def call(s):
        dx, dw, db = torch.full_like(dense["x"], float("nan")), torch.full_like(dense["weight"], float("nan")), torch.full((M, n_out), float("nan"), dtype=t, device="cuda")
        ws = workspace(nm, M, n, n_in, n_out, storage)
        nm.netmax_layer_backward(s["dy"], s["x"], s["weight"], dx=dx, dweight=dw, dbias=db, z=s["z"] if activation != "none" else None, activation=activation, workspace=ws)
        nm.netmax_workspace_status(ws)
        return dx, dw, db

    unit = 2.0 ** -7 if storage == "bf16" else 2.0 ** -18
    for shared in (("x",), ("weight",), ("dy",), ("z",), ("dy", "z"), ("x", "weight", "dy", "z")):
        repeated = {k: (v[:1].expand_as(v) if k in shared else v) for k, v in dense.items()}
        for got, want in zip(call(repeated), call({k: v.contiguous() for k, v in repeated.items()})):
            assert (got.double() - want.double()).norm() <= unit * want.double().norm(), shared


THIN = [(1, 1 << 22, 1, 1), (1, 17, 1, 1 << 22), (1, 17, 1 << 22, 1), (1, 2, 1, 1 << 22), (1, 2, 1 << 22, 1), (16384, 17, 8, 8), (16384, 3, 5, 9), (2, 1 << 20, 9, 3)]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", THIN, ids=str)
def test_the_longest_and_thinnest_layers(nm, size, storage):
    """Factors in [0.5, 1.5): nothing cancels.  Sums in parts (2^-12 of the whole) and 2^-22 for each factor; a batch of a few rows adds up to 2^17 products
    a thread, off by at most half a unit of the running sum each, independently: 2^-24 2^9."""
    M, n, n_in, n_out = size
    t = TYPES[storage]

    def positive(seed, *shape):
        g = torch.Generator(device="cuda").manual_seed(seed)
        return (0.5 + torch.rand(*shape, generator=g, device="cuda")).to(t)

    def near(got, want):
        off = (2.0 ** -12 + 2.0 ** -21 + 2.0 ** -14 + (2.0 ** -8 if storage == "bf16" else 0)) * want
        assert ((got.double() - want).abs() <= off).all(), ((got.double() - want) / want).abs().max().item()

    x, w, dy = positive(1, M, n, n_in), positive(2, M, n_out, n_in), positive(3, M, n, n_out)
    y, dx, dw, db = torch.full_like(dy, float("nan")), torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full((M, n_out), float("nan"), dtype=t, device="cuda")
    ws = workspace(nm, M, n, n_in, n_out, storage)
    nm.netmax_layer_forward(x, w, y, workspace=ws)
    nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, dbias=db, workspace=ws)
    nm.netmax_workspace_status(ws)
    near(y, x.double() @ w.double().mT)
    near(dx, dy.double() @ w.double())
    near(dw, dy.double().mT @ x.double())
    near(db, dy.double().sum(1))


# ---- Newton-Schulz
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1 << 20, 1, 1), (100_000, 3, 2), (1, 1, 1 << 22), (1, 1 << 22, 1), (3, 5, 300_001), (2, 70_000, 130)], ids=str)
def test_the_most_and_the_longest_matrices(nm, size, storage):
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.randn(*size, generator=g, device="cuda").to(TYPES[storage])
    got = orthogonalise(nm, u)
    if min(size[1:]) == 1:      # one singular value: the quintic of 1
        s = 1.0
        for _ in range(5):
            s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        want = s * u.double() / u.double().square().sum((1, 2), keepdim=True).sqrt()
        # S and the polynomial are off by 2^-10 of themselves where factors are fp16, 2^-19 elsewhere; |phi'(s)| carries on at most 3.4445 a step
        small = max(size[1:]) <= 8192
        off = 2.0 ** -8 + 40 * 2.0 ** -10 if storage == "bf16" and not small else 2.0 ** -8 if storage == "bf16" else 40 * 2.0 ** -19
        assert ((got.double() - want).abs() <= off * want.abs().amax((1, 2), keepdim=True) + 1e-30).all()
    else:
        check_orthogonal(got, u)


# ---- the step
def run_step(nm, M, d, matrices, storage, change=None):
    x, m, grad, peers, weights = step_case(7, M, d, matrices, storage)
    if change is not None:
        peers = torch.tensor(change, dtype=torch.int32, device="cuda")
    itself = torch.arange(M, dtype=torch.int32, device="cuda")
    known = torch.where((peers >= 0) & (peers < M), peers, itself)
    want, off, want_m = exact_step(x, m, grad, matrices, known, weights, 0.05, 0.9, True, 0.01, 5)
    ws = torch.full((nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage),), 0x7F, dtype=torch.uint8, device="cuda")
    new, m_next = torch.full_like(x, float("nan")), torch.full_like(m, float("nan"))
    nm.netmax_orthogonalised_step(x, new, grad, m, m_next, matrices, peers, weights, lr=0.05, mu=0.9, decay=0.01, workspace=ws)
    nm.netmax_workspace_status(ws)
    assert ((new.double() - want).abs() - off).max().item() <= 0
    assert ((m_next.double() - want_m).abs() <= 2.0 ** -23 * (want_m.abs() + m.double().abs()) + 1e-30).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(130, 133), (9, 14), (100, 40)], ids=str)
def test_a_step_of_as_many_matrices_as_it_takes(nm, shape, storage):
    rows, cols = shape
    matrices = [(3 + k * rows * cols + k // 2, rows, cols, 1.0 + k / 256) for k in range(256)]
    run_step(nm, 2, matrices[-1][0] + rows * cols + 5, matrices, storage)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_peers_that_are_no_workers_and_a_worker_alone(nm, storage):
    matrices = [(5, 40, 30, 1.0), (1300, 140, 150, 0.5)]
    run_step(nm, 5, 23000, matrices, storage, change=[-1, 5, 0, 2 ** 31 - 1, -2 ** 31])
    run_step(nm, 1, 23000, matrices, storage)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("trace_rounds,first_round", [(1, 0), (3, 0), (1024, 1000003)])
def test_rounds_across_the_trace_ring(nm, trace_rounds, first_round, storage):
    """The same draws as a context's ordinary rounds, whatever the ring's length, first rounds that are not 0, and rounds of both kinds in turn."""
    M, d, lr, t = 4, 3001, 0.05, TYPES[storage]
    matrices = [(8, 20, 30, 1.2), (700, 33, 33, 1.0)]
    make = lambda **kw: nm.Netmax(M=M, d=d, lr=lr, x0_std=1.0, seed=9, storage=storage, first_round=first_round, **kw)  # noqa: E731
    a, b = make(trace_rounds=trace_rounds), make()
    b.round(9)
    trace = b.peer_trace(first_round, 9)
    P, rho = a.get_policy()
    momentum, mine = torch.zeros(M, d, device="cuda"), torch.zeros(M, d, device="cuda")
    size = nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage)
    ws, ws2 = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda")
    done = 0
    for burst in (2, 1, 2):
        x = torch.from_numpy(a.read_replicas()).cuda().to(t)
        grad = step_case(20 + done, M, d, matrices, storage)[2]
        peers = trace[done]
        w = np.array([0.0 if peers[i] == i else lr * rho / P[i, peers[i]] for i in range(M)])
        new = torch.empty_like(x)
        nm.netmax_orthogonalised_step(x, new, grad, mine, mine, matrices, torch.from_numpy(peers.copy()).cuda(), torch.from_numpy(w).float().cuda(), lr=lr, mu=0.9, workspace=ws2)
        a.round_orthogonalised(grad, momentum, matrices, mu=0.9, workspace=ws)
        assert torch.equal(momentum, mine)
        got = torch.from_numpy(a.read_replicas()).cuda()
        assert ((got - new.float()).abs() <= (2.0 ** -7 if storage == "bf16" else 2.0 ** -21) * (new.float().abs() + x.float().abs() + 1e-6)).all()
        assert (a.peer_trace(first_round + done, 1)[0] == peers).all()
        if burst > 1:
            a.round(burst - 1)
        done += burst
    a.close()
    b.close()
