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
