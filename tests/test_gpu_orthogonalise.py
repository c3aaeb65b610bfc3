"""Newton-Schulz orthogonalisation and the whole update (netmax_orthogonalise, netmax_orthogonalised_step, netmax_round_orthogonalised)
against their formulas in 64 bits.

How far an iterate may be off.  With singular values s the step is phi(s) = a s + b s^3 + c s^5 on them, and an error E of an iterate is
carried on entrywise in the basis of the singular vectors, by the divided differences (phi(s) -+ phi(t)) / (s -+ t), none above
a = 3.4445.  A step adds at most C u |X|_F itself, C = 40: |X|_2 <= 1.21, |S|_2 <= 1.46 and |P|_2 <= 2.81 bound the parts
(|b| + 2 |c| |S|) (2 |X| + |S| / |X|) |X| + |P| (1 + |X|) + |X'| of S = X X^T, P = b S + c S^2 and X' = a X + P X, each rounded by u.
The errors are spread like noise over the directions, so their factors are taken as the root mean square of the divided differences.
fp32: u = 2^-20 (22-bit factors; 48 steps between two fp32 sums, each of which drops less than 2^-24 of a running sum that is half the
final one on average and whose terms have both signs: at most 24 2^-24 = 1.5 2^-20 if they had one, and C, which takes every part at its
largest, has that much room).
Small matrices (see is_small) have 22-bit factors with bfloat16 storage as well: u = 2^-20, and the
result's rounding, 2^-8 of itself.
bfloat16, larger: the factors' rounding to fp16 is part of the definition (u = 2^-12); the emulation rounds at the same places in 64 bits, and the
kernel may differ from it by the rounding of the result (2^-8 of itself, and in the root mean square less than 0.6 of that, which leaves
room for factors that rounded the other way: one in a thousand, 2^-11 each)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

A, B, C = 3.4445, -4.7750, 2.0315
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def nm():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2009_05766_b200 import binding
    binding.lib()
    return binding


def update(seed, count, rows, cols, kind="training", dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    if kind == "noise":
        u = normal(count, rows, cols)
    elif kind == "rank 1":
        u = normal(count, rows, 1) @ normal(count, 1, cols)
    else:
        k = max(1, min(rows, cols) // 4)
        u = normal(count, rows, k) @ normal(count, k, cols) + 0.2 * normal(count, rows, cols)
    return (u * 0.01).to(dtype).cuda()


def iterates(u, steps, fp16=False):
    """The iterates in 64 bits, (count, rows, cols); fp16: with the factors of the products rounded as bfloat16 storage has them."""
    near = (lambda v: (v * 2.0 ** 14).to(torch.float16).double() / 2.0 ** 14) if fp16 else lambda v: v
    def both(v):  # the two planes
        hi = near(v)
        return hi + near(v - hi)
    x = u.double()
    n = x.square().sum((1, 2), keepdim=True).sqrt()
    x = torch.where(n > 0, x / torch.where(n > 0, n, torch.ones_like(n)), torch.zeros_like(x))
    tall = x.shape[1] > x.shape[2]
    found = []
    for _ in range(steps):
        found.append(x)
        if fp16:
            x = both(x)
        h = near(x)
        s = near(h.mT @ h if tall else h @ h.mT)
        p = near(B * s + C * (s @ s))
        x = A * x + (h @ p if tall else p @ h)
    return found + [x]


def bound(found, u):
    """2-norms (count,) of the error of the last iterate when every step adds 40 u |X|."""
    s = torch.linalg.svdvals(found[0])
    total = torch.zeros(s.shape[0], dtype=torch.float64, device=s.device)
    gain = torch.ones(s.shape[0], s.shape[1], s.shape[1], dtype=torch.float64, device=s.device)
    values = [s]
    for _ in found[1:]:
        s = A * s + B * s ** 3 + C * s ** 5
        values.append(s)
    for k in range(len(found) - 2, -1, -1):   # errors made by step k are carried on by the later ones
        total += 40 * u * found[k].norm(dim=(1, 2)) * gain.square().mean((1, 2)).sqrt()
        s, t = values[k], values[k + 1]
        d = (s[:, :, None] - s[:, None])
        near = d.abs() < 1e-6
        minus = torch.where(near, (A + 3 * B * s ** 2 + 5 * C * s ** 4)[:, :, None].expand_as(d), (t[:, :, None] - t[:, None]) / torch.where(near, torch.ones_like(d), d))
        plus = (t[:, :, None] + t[:, None]) / (s[:, :, None] + s[:, None]).clamp_min(1e-30)
        gain = gain * torch.maximum(minus.abs(), plus.abs())
    return total


def orthogonalise(nm, u, steps=5):
    storage = "f32" if u.dtype == torch.float32 else "bf16"
    out = torch.full(tuple(u.shape), float("nan"), dtype=u.dtype, device="cuda")
    ws = torch.full((nm.netmax_orthogonalise_workspace_size(*u.shape, storage),), 0x7F, dtype=torch.uint8, device="cuda")
    nm.netmax_orthogonalise(u, out, steps=steps, workspace=ws)
    nm.netmax_workspace_status(ws)
    return out


def is_small(rows, cols):
    side, length = min(rows, cols), max(rows, cols)
    return (side <= 64 and length <= 8192) or (side <= 128 and length <= 4096)


def is_narrow(rows, cols, matrices):
    """Whether a step rounds this one's factors to fp16 with bfloat16 storage."""
    larger = any(not is_small(r, c) for _, r, c, _ in matrices)
    return not is_small(rows, cols) or (larger and min(rows, cols) > 64 and max(rows, cols) > 256)


def check(got, u, steps=5):
    if u.dtype == torch.float32 or is_small(*u.shape[1:]):
        found = iterates(u, steps)
        off = bound(found, 2.0 ** -20) + (2.0 ** -23 if u.dtype == torch.float32 else 2.0 ** -8) * found[-1].norm(dim=(1, 2)) + 1e-30
    else:
        found = iterates(u, steps, fp16=True)
        off = 2.0 ** -8 * found[-1].norm(dim=(1, 2)) + 1e-30
    err = (got.double() - found[-1]).norm(dim=(1, 2))
    assert (err <= off).all(), f"{err.tolist()} beyond {off.tolist()}"


SIZES = [(1, 1, 1), (2, 1, 9), (2, 9, 1), (3, 5, 7), (4, 64, 64), (2, 64, 27), (1, 27, 64), (2, 130, 131), (3, 65, 300), (2, 300, 65), (1, 128, 128),
         (1, 129, 512), (2, 256, 256), (5, 257, 255), (2, 600, 520), (33, 40, 24), (1, 1003, 777), (2, 512, 1536), (3, 1100, 1100),
         (3, 27, 4024), (2, 3726, 11), (3, 97, 2513), (1, 128, 4096), (1, 8192, 64), (2, 64, 8191), (1, 8193, 64), (1, 128, 4097), (4, 64, 512), (40, 100, 256),
         (5, 65, 1025), (1, 1, 5000), (20, 31, 956), (7, 600, 128),
         (75, 70, 300), (74, 300, 70),
         (2, 200, 5000), (1, 5001, 300), (3, 513, 2100), (1, 140, 9000)]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_orthogonalise(nm, size, storage):
    u = update(1, *size, dtype=TYPES[storage])
    check(orthogonalise(nm, u), u)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["noise", "rank 1"])
@pytest.mark.parametrize("steps", [1, 2, 6])
def test_spectra_and_steps(nm, storage, kind, steps):
    for size in ((2, 96, 200), (2, 200, 96)):
        u = update(steps, *size, kind=kind, dtype=TYPES[storage])
        check(orthogonalise(nm, u, steps), u, steps)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_range_of_magnitudes(nm, storage):
    """Matrices from 1e-38 to 1e38, one of zeros and one with an infinity and a NaN, in one call: each for itself."""
    u = update(3, 7, 70, 90, dtype=torch.float32)
    for k, f in enumerate((1e-35, 1e-20, 1.0, 1e20, 1e36)):
        u[k] *= f
    u[5] = 0
    u = u.to(TYPES[storage])
    u[6, 3, 4], u[6, 60, 80] = float("inf"), float("nan")
    got = orthogonalise(nm, u)
    assert (got[5] == 0).all()
    assert torch.isnan(got[6]).all()
    check(got[:6], u[:6])


def test_strides(nm):
    """Matrices with gaps between rows, woven into one another, one for all: elements that no view names stay as they were."""
    base = update(4, 3, 50, 80)
    wide = torch.full((3, 50, 99), 7.0, device="cuda")
    wide[:, :, 5:85] = base
    out = torch.full((50, 3, 101), 7.0, device="cuda")
    ws = torch.empty(nm.netmax_orthogonalise_workspace_size(3, 50, 80), dtype=torch.uint8, device="cuda")
    view = out.transpose(0, 1)[:, :, 11:91]
    nm.netmax_orthogonalise(wide[:, :, 5:85], view, workspace=ws)
    want = orthogonalise(nm, base)
    assert torch.equal(view, want)
    assert (out[:, :, :11] == 7).all() and (out[:, :, 91:] == 7).all()
    same = base[:1].expand(3, 50, 80)
    got = torch.empty(3, 50, 80, device="cuda")
    nm.netmax_orthogonalise(same, got, workspace=ws)
    assert all(torch.equal(got[k], want[0]) for k in range(3))


def test_same_bits_again_in_a_graph_and_on_another_stream(nm):
    for storage in TYPES:
        u = update(5, 6, 300, 520, dtype=TYPES[storage])
        want = orthogonalise(nm, u)
        ws = torch.empty(nm.netmax_orthogonalise_workspace_size(6, 300, 520, storage), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(u)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        nm.netmax_orthogonalise(u, out, workspace=ws, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            nm.netmax_orthogonalise(u, out, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        v = update(6, 6, 300, 520, dtype=TYPES[storage])
        want_v = orthogonalise(nm, v)
        u.copy_(v)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want_v)


# ---- the whole update

def step_case(seed, M, d, matrices, storage):
    g = torch.Generator().manual_seed(seed)
    t = TYPES[storage]
    normal = lambda std, dtype: (torch.randn(M, d, generator=g, dtype=torch.float64) * std).to(dtype).cuda()  # noqa: E731
    x, m, grad = normal(0.5, t), normal(0.02, torch.float32), normal(0.1, t)
    peers = torch.randint(0, M, (M,), generator=g, dtype=torch.int32)
    peers[0] = 0
    weights = (0.05 + 0.4 * torch.rand(M, generator=g)).float()
    return x, m, grad, peers.cuda(), weights.cuda()


def exact_step(x, m, grad, matrices, peers, weights, lr, mu, nesterov, decay, steps):
    """(x', its tolerance, m') in 64 bits."""
    f16 = x.dtype == torch.bfloat16
    x64, g64 = x.double(), grad.double()
    m64 = float(np.float32(mu)) * m.double() + g64
    u = g64 + float(np.float32(mu)) * m64 if nesterov else m64
    o, off = u.clone(), 2.0 ** -22 * u.abs()
    for at, rows, cols, scale in matrices:
        part = u[:, at:at + rows * cols].reshape(-1, rows, cols)
        narrow = f16 and is_narrow(rows, cols, matrices)
        found = iterates(part, steps, fp16=narrow)
        o[:, at:at + rows * cols] = scale * found[-1].reshape(-1, rows * cols)
        # (the emulation's and the kernel's iterates differ by rounded factors: see above; 2-norms bound every element)
        e = bound(iterates(part, steps), 2.0 ** -20 if not narrow else 2.0 ** -12)
        off[:, at:at + rows * cols] = (scale * e[:, None]).expand(-1, rows * cols)
    lr, decay, w64 = float(np.float32(lr)), float(np.float32(decay)), weights.double()[:, None]
    h = x64 - lr * (o + decay * x64)
    off = lr * off + 2.0 ** -21 * (x64.abs() + lr * o.abs())
    itself = (peers == torch.arange(x.shape[0], device="cuda"))[:, None]
    new = torch.where(itself, h, h - w64 * (h - x64[peers.long()]))
    off = off + 2.0 ** -22 * (h.abs() + x64[peers.long()].abs())
    return new, off + (2.0 ** -8 if f16 else 2.0 ** -23) * (new.abs() + off), m64


CASES = [  # M, d, matrices
    (3, 130003, [(0, 70, 500, 1.0), (35003, 200, 300, 1.0), (95003, 60, 500, 2.0), (125003, 8, 600, 1.0)]), (3, 70002, [(1, 70, 500, 1.0), (35002, 500, 70, 1.0)]),
    (2, 1, []), (3, 5000, []), (4, 4096, [(0, 64, 48, 1.0)]), (3, 4097, [(1, 64, 64, 2.0)]), (5, 9001, [(3, 31, 77, 1.0), (2391, 77, 31, 0.5), (5000, 31, 77, 1.5), (7387, 1, 1614, 1.0)]),
    (2, 200000, [(0, 300, 300, 1.0), (90000, 300, 300, 1.0), (180001, 10, 512, 3.0)]),
]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{len(c[2])}")
def test_step(nm, case, storage):
    M, d, matrices = case
    for nesterov, mu, decay, in_place in ((True, 0.95, 0.01, False), (False, 0.0, 0.0, True)):
        x, m, grad, peers, weights = step_case(7, M, d, matrices, storage)
        want, off, want_m = exact_step(x, m, grad, matrices, peers, weights, 0.05, mu, nesterov, decay, 5)
        ws = torch.full((nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage),), 0x7F, dtype=torch.uint8, device="cuda")
        new = torch.full_like(x, float("nan"))
        m_next = m if in_place else torch.full_like(m, float("nan"))
        nm.netmax_orthogonalised_step(x, new, grad, m, m_next, matrices, peers, weights, lr=0.05, mu=mu, nesterov=nesterov, decay=decay, workspace=ws)
        nm.netmax_workspace_status(ws)
        excess = (new.double() - want).abs() - off
        assert excess.max().item() <= 0
        assert ((m_next.double() - want_m).abs() <= 2.0 ** -23 * (want_m.abs() + m.double().abs()) + 1e-30).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_round_of_a_context(nm, storage):
    """The context's round: the peers and weights of netmax_round's, the step's result, telemetry of the replicas before it."""
    M, d, lr = 5, 30011, 0.05
    matrices = [(8, 100, 90, 1.2), (9010, 33, 33, 1.0)]
    P = np.random.default_rng(3).random((M, M)) + 0.1
    P /= P.sum(1, keepdims=True)
    make = lambda: nm.Netmax(M=M, d=d, lr=lr, prob=P, x0_std=1.0, c_std=1.0, seed=9, storage=storage)  # noqa: E731
    a, b = make(), make()
    _, rho = a.get_policy()
    b.round(4)
    trace = b.peer_trace()
    t = TYPES[storage]
    momentum = torch.zeros(M, d, device="cuda")
    mine = torch.zeros(M, d, device="cuda")
    x = torch.from_numpy(a.read_replicas()).cuda().to(t)
    ws = torch.empty(nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage), dtype=torch.uint8, device="cuda")
    for r in range(4):
        grad = step_case(20 + r, M, d, matrices, storage)[2]
        cons, loss = a.measure()
        a.round_orthogonalised(grad, momentum, matrices, mu=0.9, decay=0.02, workspace=ws)
        peers = trace[r]
        w = np.array([0.0 if peers[i] == i else lr * rho / P[i, peers[i]] for i in range(M)])   # (d_im + d_mi) / 2 = 1
        new = torch.empty_like(x)
        ws2 = torch.empty_like(ws)
        torch.cuda.synchronize()
        nm.netmax_orthogonalised_step(x, new, grad, mine, mine, matrices, torch.from_numpy(peers).cuda(), torch.from_numpy(w).float().cuda(), lr=lr, mu=0.9,
                                      decay=0.02, workspace=ws2)
        assert torch.equal(momentum, mine)
        got = torch.from_numpy(a.read_replicas()).cuda()
        # (the context's weights are computed in another order: a few units of 2^-24 of a pull)
        assert ((got - new.float()).abs() <= (2.0 ** -7 if storage == "bf16" else 2.0 ** -21) * (new.float().abs() + x.float().abs() + 1e-6)).all()
        assert (a.peer_trace()[r] == trace[r]).all() and a.rounds_done == r + 1
        tel = a.telemetry(r, 1)
        assert tel[0][0] == pytest.approx(cons, rel=1e-4) and tel[1][0] == pytest.approx(loss, rel=1e-4)
        x = got.to(t)
    a.round(3)      # and the ordinary rounds go on from there
    assert a.rounds_done == 7
    a.close()
    b.close()


def test_a_round_after_a_capture_and_refusals_leave_the_context_as_it_was(nm):
    M, d = 4, 5000
    g = nm.Netmax(M=M, d=d, lr=0.1, x0_std=1.0, seed=2)
    before = g.read_replicas().copy()
    grad, momentum = torch.zeros(M, d, device="cuda"), torch.zeros(M, d, device="cuda")
    with pytest.raises(nm.NetmaxError):
        g.round_orthogonalised(grad, momentum, [(0, 64, 64, 1.0), (4000, 10, 10, 1.0)], workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
    with pytest.raises(nm.NetmaxError):
        size = nm.netmax_orthogonalised_step_workspace_size(M, d, [(0, 64, 64, 1.0)])
        g.round_orthogonalised(grad, momentum, [(0, 64, 64, 1.0)], workspace=torch.empty(size - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        g.round_orthogonalised(grad.bfloat16(), momentum, [], workspace=None)
    assert g.rounds_done == 0 and (g.read_replicas() == before).all()
    g.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_step_in_a_graph_and_from_one_replica(nm, storage):
    M, d, matrices = 4, 150001, [(5, 64, 64, 1.0), (4101, 300, 400, 1.0), (124101, 60, 420, 1.0)]
    x, m, grad, peers, weights = step_case(11, M, d, matrices, storage)
    ws = torch.empty(nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage), dtype=torch.uint8, device="cuda")
    table = nm.matrix_table(matrices)
    one = x[:1].expand(M, d)
    for source in (x, one):
        new, m_next, again, m_again = torch.empty_like(x), torch.empty_like(m), torch.empty_like(x), torch.empty_like(m)
        nm.netmax_orthogonalised_step(source, new, grad, m, m_next, table, peers, weights, lr=0.1, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            nm.netmax_orthogonalised_step(source, again, grad, m, m_again, table, peers, weights, lr=0.1, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        nm.netmax_workspace_status(ws)
        assert torch.equal(new, again) and torch.equal(m_next, m_again)
    dense = torch.empty_like(x)
    nm.netmax_orthogonalised_step(one.contiguous(), dense, grad, m, m_next, table, peers, weights, lr=0.1, workspace=ws)
    assert torch.equal(dense, new)


# ---- a run of all of them together

@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_workers_train_a_network(nm, storage):
    """M workers' two-layer networks live in their replicas: forward, gradient, orthogonalised update and pull, three rounds, against the
    same in 64 bits from the same replicas; the gradient also against differences of the loss."""
    M, n, n_in, hidden, n_out = 4, 96, 40, 72, 24
    t, lr = TYPES[storage], 0.05
    w1, b1, w2, b2 = 0, hidden * n_in, hidden * n_in + hidden, hidden * n_in + hidden + n_out * hidden
    d = b2 + n_out
    matrices = [(w1, hidden, n_in, 1.3), (w2, n_out, hidden, 1.0)]
    g = nm.Netmax(M=M, d=d, lr=lr, x0_std=0.2, seed=5, storage=storage)
    gen = torch.Generator().manual_seed(8)
    x = torch.randn(M, n, n_in, generator=gen, dtype=torch.float64).to(t).cuda()
    goal = torch.randn(M, n, n_out, generator=gen, dtype=torch.float64).to(t).cuda()
    grad, momentum = torch.zeros(M, d, dtype=t, device="cuda"), torch.zeros(M, d, device="cuda")
    z1, h1 = torch.empty(M, n, hidden, dtype=t, device="cuda"), torch.empty(M, n, hidden, dtype=t, device="cuda")
    y, dh = torch.empty(M, n, n_out, dtype=t, device="cuda"), torch.empty(M, n, hidden, dtype=t, device="cuda")
    size = max(nm.netmax_layer_workspace_size(M, n, n_in, hidden, storage), nm.netmax_layer_workspace_size(M, n, hidden, n_out, storage),
               nm.netmax_orthogonalised_step_workspace_size(M, d, matrices, storage))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    P, rho = g.get_policy()

    def parts(v):
        return (v[:, w1:b1].view(M, hidden, n_in), v[:, b1:w2], v[:, w2:b2].view(M, n_out, hidden), v[:, b2:])

    def loss(v):
        a, ab, b, bb = parts(v)
        out = act(x.double() @ a.mT + ab[:, None]) @ b.mT + bb[:, None]
        return 0.5 * (out - goal.double()).square().sum((1, 2)) / n

    def act(z):
        return z * torch.sigmoid(z)

    unit = 2.0 ** -8 if storage == "bf16" else 2.0 ** -20
    for r in range(3):
        now = torch.from_numpy(g.read_replicas()).cuda().to(t)
        a, ab, b, bb = parts(now)
        nm.netmax_layer_forward(x, a, h1, bias=ab, z=z1, activation="silu", workspace=ws)
        nm.netmax_layer_forward(h1, b, y, bias=bb, workspace=ws)
        dy = ((y.double() - goal.double()) / n).to(t)
        ga, gab, gb, gbb = parts(grad)
        nm.netmax_layer_backward(dy, h1, b, dx=dh, dweight=gb, dbias=gbb, workspace=ws)
        nm.netmax_layer_backward(dh, x, a, dweight=ga, dbias=gab, z=z1, activation="silu", workspace=ws)
        nm.netmax_workspace_status(ws)
        v = now.double().requires_grad_(True)
        want, = torch.autograd.grad(loss(v).sum(), v)
        # (a handful of roundings between the inputs and each gradient, each of a unit of sums over up to 96 rows of values near 1)
        for k, (p, q) in enumerate(zip(parts(grad), parts(want))):
            assert (p.double() - q).norm() <= 6 * unit * q.norm(), k
        h = 1e-4
        direction = torch.randn(M, d, generator=gen, dtype=torch.float64).cuda()
        slope = (loss(now.double() + h * direction) - loss(now.double() - h * direction)) / (2 * h)
        # the gradient's own error, and the third derivative's h^2 / 6 (well below 1e-5 of the slope's scale)
        scale = want.norm(dim=1) * direction.norm(dim=1)
        assert ((slope - (grad.double() * direction).sum(1)).abs() <= (6 * unit + 1e-5) * scale).all()
        kept = momentum.clone()
        g.round_orthogonalised(grad, momentum, matrices, mu=0.9, decay=0.01, workspace=ws)
        peers = g.peer_trace(r, 1)[0]
        weights = torch.tensor([0.0 if peers[i] == i else lr * rho / P[i, peers[i]] for i in range(M)]).cuda()
        new, off, want_m = exact_step(now, kept, grad, matrices, torch.from_numpy(peers).cuda(), weights.float(), lr, 0.9, True, 0.01, 5)
        got = torch.from_numpy(g.read_replicas()).cuda().double()
        assert ((got - new).abs() <= off + 2.0 ** -21 * new.abs()).all()
    g.close()


@pytest.mark.parametrize("shape", [(40, 24), (130, 200)], ids=str)
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_matrices_further_apart_than_32_bits(nm, storage, shape):
    """Two matrices 2^31 + 64 elements apart, on both paths."""
    t, (rows, cols), apart = {"f32": torch.float32, "bf16": torch.bfloat16}[storage], shape, 2 ** 31 + 64
    room = torch.empty(apart + 2 * rows * cols, dtype=t, device="cuda")
    u = room.as_strided((2, rows, cols), (apart, cols, 1), 0)
    out = room.as_strided((2, rows, cols), (apart, cols, 1), rows * cols)
    u.copy_(update(5, 2, rows, cols, dtype=t))
    ws = torch.full((nm.netmax_orthogonalise_workspace_size(2, rows, cols, storage),), 0x7F, dtype=torch.uint8, device="cuda")
    nm.netmax_orthogonalise(u, out, workspace=ws)
    nm.netmax_workspace_status(ws)
    check(out, u)
