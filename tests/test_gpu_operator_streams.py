"""The operators on real weights beside torch's streams: a call without a stream runs on torch's current one, and a context's round is
ordered behind what that stream has queued and before what it queues next."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def nm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2009_05766_b200 import binding
    binding.lib()
    return binding


def normal(seed, *shape, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).cuda()


def calls(nm):
    """name: (call, outputs, input to be changed)"""
    M, n, n_in, n_out = 3, 40, 56, 72
    x, w, dy = normal(1, M, n, n_in), normal(2, M, n_out, n_in), normal(3, M, n, n_out)
    y, dx, dw = torch.zeros(M, n, n_out, device="cuda"), torch.zeros_like(x), torch.zeros_like(w)
    ws = torch.empty(nm.netmax_layer_workspace_size(M, n, n_in, n_out), dtype=torch.uint8, device="cuda")
    u, o = normal(4, 3, 130, 200), torch.zeros(3, 130, 200, device="cuda")
    wo = torch.empty(nm.netmax_orthogonalise_workspace_size(3, 130, 200), dtype=torch.uint8, device="cuda")
    d, table = 30000, nm.matrix_table([(0, 130, 140, 1.0), (18200, 20, 30, 1.0)])
    r, g, m = normal(5, M, d), normal(6, M, d), normal(7, M, d)
    r1, m1 = torch.zeros_like(r), torch.zeros_like(m)
    peers, weights = torch.tensor([1, 2, 0], dtype=torch.int32, device="cuda"), torch.full((M,), 0.25, device="cuda")
    wt = torch.empty(nm.netmax_orthogonalised_step_workspace_size(M, d, table), dtype=torch.uint8, device="cuda")
    return {
        "forward": (lambda: nm.netmax_layer_forward(x, w, y, workspace=ws), (y,), x),
        "backward": (lambda: nm.netmax_layer_backward(dy, x, w, dx=dx, dweight=dw, workspace=ws), (dx, dw), dy),
        "orthogonalise": (lambda: nm.netmax_orthogonalise(u, o, workspace=wo), (o,), u),
        "step": (lambda: nm.netmax_orthogonalised_step(r, r1, g, m, m1, table, peers, weights, lr=0.1, workspace=wt), (r1, m1), g),
    }


@pytest.mark.parametrize("name", ["forward", "backward", "orthogonalise", "step"])
def test_a_call_runs_on_the_current_stream(nm, name):
    call, outputs, changed = calls(nm)[name]
    other = normal(9, *changed.shape)
    changed.copy_(other)
    torch.cuda.synchronize()
    call()
    torch.cuda.synchronize()
    want = [v.clone() for v in outputs]
    changed.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)      # (a tenth of a second)
        changed.copy_(other)
        call()
        got = [v.clone() for v in outputs]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["forward", "backward", "orthogonalise", "step"])
def test_a_call_is_captured_from_the_current_stream(nm, name):
    call, outputs, _ = calls(nm)[name]
    call()
    torch.cuda.synchronize()
    want = [v.clone() for v in outputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for v in outputs:
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outputs, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("own_stream", [False, True])
def test_a_round_between_two_pieces_of_work_on_another_stream(nm, own_stream):
    M, d, matrices = 4, 40000, [(0, 130, 140, 1.0), (18200, 20, 30, 1.0)]
    ctx_stream = torch.cuda.Stream()
    make = lambda: nm.Netmax(M=M, d=d, lr=0.1, x0_std=1.0, seed=3, stream=ctx_stream.cuda_stream if own_stream else None)  # noqa: E731
    grad, table = normal(1, M, d, std=0.1), nm.matrix_table(matrices)
    ws = torch.empty(nm.netmax_orthogonalised_step_workspace_size(M, d, table), dtype=torch.uint8, device="cuda")
    a, b = make(), make()
    momentum = torch.zeros(M, d, device="cuda")
    torch.cuda.synchronize()
    a.round_orthogonalised(grad, momentum, table, workspace=ws)
    want_x = a.read_replicas()
    torch.cuda.synchronize()
    want = momentum.clone()
    late, momentum = torch.zeros(M, d, device="cuda"), torch.ones(M, d, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        late.copy_(grad)
        momentum.zero_()
        b.round_orthogonalised(late, momentum, table, workspace=ws)
        got = momentum.clone()
        late.zero_()
    side.synchronize()
    assert torch.equal(got, want)
    assert np.array_equal(b.read_replicas(), want_x)
    a.close()
    b.close()
