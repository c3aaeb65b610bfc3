"""Performance cases of the operators that train real weights in the replicas: what a user's program calls between rounds.

Three kinds of work, each batched over the M workers, whose weights are matrices inside their own replicas:
  forward   a layer, y = act(x W^T + b) + r, with the pre-activation z kept for the gradient where the layer has an activation;
  backward  its gradient: dz = dy act'(z), dx = dz W, dW = dz^T x, db = the column sums of dz;
  orth      matrices orthogonalised by five quintic Newton-Schulz steps, X <- a X + b (X X^T) X + c (X X^T)^2 X from U / |U|;
  step      a worker's whole update: momentum, its matrices orthogonalised, the local step, and the pull of the drawn peer.

Types are those of the replicas: "f32" or "bf16" for every array (momentum is fp32 in both).  Sizes: the M of
`paper_2009_05766_b200.workloads`, the matrices of its ResNet18-sized vector, and the ranges around them.
"""
import math

import torch

own = False

QUINTIC = (3.4445, -4.7750, 2.0315)
STEPS = 5
RESNET18 = 11_173_962   # parameters, in these matrices (a convolution's as outputs x inputs) and 9,610 others
RESNET18_MATRICES = ("64x27,64x576*4,128x576,128x1152*3,128x64,256x1152,256x2304*3,256x128,512x2304,512x4608*3,512x256,"
                     "10x512")
LR, MU, DECAY = 0.05, 0.95, 0.01

# the most that draw() gives
MAX_LAYER_FLOPS = 2 * 8 * 4096 ** 3
MAX_ORTH_FLOPS = 4 * STEPS * 4 * 4096 ** 3
MAX_STEP_ELEMENTS = 8 * RESNET18


def layer_case(kind, M, n, n_in, n_out, storage, activation="none", bias=True, residual=False):
    return {"kind": kind, "M": M, "n": n, "n_in": n_in, "n_out": n_out, "storage": storage, "activation": activation, "bias": bias,
            "residual": residual}


def orth_case(count, rows, cols, storage):
    return {"kind": "orth", "count": count, "rows": rows, "cols": cols, "storage": storage}


def step_case(M, matrices, rest, gap, storage, nesterov=True):
    """`matrices`: ROWSxCOLS[*COUNT],...; `gap` elements stand between two of them, `rest` behind the last."""
    return {"kind": "step", "M": M, "matrices": matrices, "rest": rest, "gap": gap, "storage": storage, "nesterov": nesterov}


def listed():
    return [
        # the smallest call: one sample per worker through the last layer of the ResNet18-sized vector
        dict(layer_case("forward", 4, 1, 512, 10, "f32"), name="forward_one_row"),
        # a batch of an ordinary hidden layer with the replicas' default type
        dict(layer_case("forward", 8, 512, 512, 2048, "f32", "gelu"), name="forward_f32"),
        # the largest: a wide layer, bfloat16 replicas, with its residual
        dict(layer_case("forward", 8, 4096, 4096, 4096, "bf16", "silu", residual=True), name="forward_large_bf16"),
        # nothing round about it
        dict(layer_case("backward", 5, 77, 1001, 333, "bf16", "relu"), name="backward_ragged_bf16"),
        dict(layer_case("backward", 8, 512, 512, 2048, "f32", "gelu"), name="backward_f32"),
        dict(layer_case("backward", 8, 4096, 4096, 2048, "bf16", "gelu"), name="backward_large_bf16"),
        # the smallest matrices, where launches count
        dict(orth_case(4, 64, 64, "f32"), name="orth_small"),
        # the largest convolution of the ResNet18-sized vector, 8 workers
        dict(orth_case(8, 512, 4608, "bf16"), name="orth_conv_bf16"),
        # taller than wide, odd
        dict(orth_case(6, 1003, 777, "f32"), name="orth_tall_f32"),
        # the largest square matrices
        dict(orth_case(4, 4096, 4096, "bf16"), name="orth_large_bf16"),
        # the whole update of four toy workers
        dict(step_case(4, "64x48", 1024, 0, "f32"), name="step_toy"),
        # the whole update of 8 ResNet18-sized replicas
        dict(step_case(8, RESNET18_MATRICES, 9610, 0, "f32"), name="step_resnet18_8"),
    ]


def _log(rng, lo, hi):
    """A whole number from [lo, hi], uniform over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["forward", "backward", "orth", "step"], weights=[3, 3, 4, 2])[0]
    storage = rng.choice(["f32", "bf16"])
    M = _log(rng, 2, 16)
    if kind in ("forward", "backward"):
        n_in, n_out, n = _log(rng, 16, 4096), _log(rng, 8, 4096), _log(rng, 1, 4096)
        if rng.random() < 0.5:      # half of the layers have the usual round sizes
            n_in, n_out = max(16, n_in // 16 * 16), max(16, n_out // 16 * 16)
        times = 1 if kind == "forward" else 2
        n = max(1, min(n, MAX_LAYER_FLOPS // (2 * times * M * n_in * n_out)))
        return layer_case(kind, M, n, n_in, n_out, storage, rng.choice(["none", "relu", "gelu", "silu"]), rng.random() < 0.8,
                          kind == "forward" and rng.random() < 0.4)
    if kind == "orth":
        rows, cols, count = _log(rng, 8, 4096), _log(rng, 8, 6000), _log(rng, 1, 32)
        if rng.random() < 0.5:
            rows, cols = max(8, rows // 8 * 8), max(8, cols // 8 * 8)
        count = max(1, min(count, MAX_ORTH_FLOPS // _orth_flops(rows, cols)))
        if _orth_flops(rows, cols) > MAX_ORTH_FLOPS:
            cols = min(cols, 4096)
        return orth_case(count, rows, cols, storage)
    rows, cols = _log(rng, 8, 512), _log(rng, 8, 1500)
    count = max(1, min(_log(rng, 1, 12), MAX_STEP_ELEMENTS // (2 * M * rows * cols)))
    return step_case(M, "%dx%d*%d,%dx%d" % (rows, cols, count, _log(rng, 8, 200), _log(rng, 8, 200)), _log(rng, 1, 20000),
                     rng.choice([0, 0, 3, 64]), storage, rng.random() < 0.8)


def _orth_flops(rows, cols):
    """Products of a matrix's five steps: the lower halves of X X^T and of its square, which are symmetric, and the last one whole."""
    r, c = min(rows, cols), max(rows, cols)
    return STEPS * (r * r * c + r * r * r + 2 * r * r * c)


def _matrices(case):
    """[(offset, rows, cols, scale)] of a step's replica, and its length."""
    at, found = 0, []
    for part in case["matrices"].split(","):
        shape, _, count = part.partition("*")
        rows, cols = (int(v) for v in shape.split("x"))
        for _ in range(int(count or 1)):
            found.append((at, rows, cols, math.sqrt(max(1.0, rows / cols))))
            at += rows * cols + case["gap"]
    return found, at + case["rest"]


def work(case):
    size = 4 if case["storage"] == "f32" else 2
    if case["kind"] == "orth":
        return {"bytes": 2 * size * case["count"] * case["rows"] * case["cols"], "flops": case["count"] * _orth_flops(case["rows"], case["cols"])}
    M = case["M"]
    if case["kind"] == "step":
        matrices, d = _matrices(case)
        # replicas and gradients read, replicas written; momentum read and written
        return {"bytes": M * d * (3 * size + 8), "flops": M * sum(_orth_flops(r, c) for _, r, c, _ in matrices) + 8 * M * d}
    x, w, y = case["n"] * case["n_in"], case["n_in"] * case["n_out"], case["n"] * case["n_out"]
    active = case["activation"] != "none"
    flops = 2 * M * case["n"] * case["n_in"] * case["n_out"]
    if case["kind"] == "forward":
        return {"bytes": M * size * (x + w + case["n_out"] * case["bias"] + y * (1 + active + case["residual"])), "flops": flops}
    return {"bytes": M * size * (2 * x + 2 * w + y * (1 + active) + case["n_out"] * case["bias"]), "flops": 2 * flops}


def _dtype(case):
    return torch.float32 if case["storage"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _dtype(case)

    def normal(*shape, std=1.0, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = {"case": case}
    if case["kind"] in ("forward", "backward"):
        M, n, n_in, n_out = case["M"], case["n"], case["n_in"], case["n_out"]
        s["x"], s["weight"] = normal(M, n, n_in), normal(M, n_out, n_in, std=n_in ** -0.5)
        active = case["activation"] != "none"
        if case["kind"] == "forward":
            s["bias"] = normal(M, n_out, std=0.1) if case["bias"] else None
            s["residual"] = normal(M, n, n_out) if case["residual"] else None
            s["y"] = torch.empty(M, n, n_out, device="cuda", dtype=t)
            s["z"] = torch.empty_like(s["y"]) if active else None
        else:
            s["dy"], s["z"] = normal(M, n, n_out, std=n ** -0.5), normal(M, n, n_out) if active else None
            s["dx"], s["dweight"] = torch.empty_like(s["x"]), torch.empty_like(s["weight"])
            s["dbias"] = torch.empty(M, n_out, device="cuda", dtype=t) if case["bias"] else None
        return s

    def gradient(count, rows, cols):
        """Updates as training gives them: most of a matrix lies in a quarter of its directions, the rest is noise."""
        k = max(1, min(rows, cols) // 4)
        u = torch.bmm(normal(count, rows, k, dtype=torch.float32), normal(count, k, cols, dtype=torch.float32)) / math.sqrt(k)
        return (u + 0.2 * normal(count, rows, cols, dtype=torch.float32)) * 0.01

    if case["kind"] == "orth":
        s["u"] = gradient(case["count"], case["rows"], case["cols"]).to(t)
        s["out"] = torch.empty_like(s["u"])
        return s
    M = case["M"]
    s["matrices"], d = _matrices(case)
    s["x"], s["momentum"] = normal(M, d, std=0.05), normal(M, d, std=0.002, dtype=torch.float32)
    s["gradient"] = normal(M, d, std=0.01)
    for at, rows, cols, _ in s["matrices"]:
        s["gradient"][:, at:at + rows * cols] = gradient(M, rows, cols).reshape(M, -1).to(t)
    s["x_next"], s["momentum_next"] = torch.empty_like(s["x"]), torch.empty_like(s["momentum"])
    # one peer of each worker, a few workers draw themselves; Eq. 16's weights are below a half
    s["peers"] = torch.randint(0, M, (M,), generator=g, device="cuda", dtype=torch.int32)
    s["weights"] = 0.05 + 0.4 * torch.rand(M, generator=g, device="cuda")
    return s


def _act(z, activation):
    if activation == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if activation == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if activation == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, activation):
    if activation == "relu":
        return (z > 0).to(z.dtype)
    if activation == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    sigmoid = 1 / (1 + torch.exp(-z))
    return sigmoid * (1 + z * (1 - sigmoid))


def _orthogonalise(u):
    """(count, rows, cols) in fp32.  The norm is a long sum that every step scales with: in 64 bits."""
    a, b, c = QUINTIC
    tall = u.shape[1] > u.shape[2]
    norm = u.double().square().sum(dim=(1, 2), keepdim=True).sqrt()
    x = torch.where(norm > 0, u.double() / norm, torch.zeros_like(norm)).float()
    for _ in range(STEPS):
        if tall:
            s = x.transpose(1, 2) @ x
            x = a * x + x @ (b * s + c * (s @ s))
        else:
            s = x @ x.transpose(1, 2)
            x = a * x + (b * s + c * (s @ s)) @ x
    return x


def _same_shapes(matrices):
    groups = {}
    for at, rows, cols, scale in matrices:
        groups.setdefault((rows, cols, scale), []).append(at)
    return groups.items()


def _plain(s):
    case, t = s["case"], _dtype(s["case"])
    if case["kind"] == "forward":
        z = s["x"].float() @ s["weight"].float().transpose(1, 2)
        if s["bias"] is not None:
            z = z + s["bias"].float()[:, None]
        y = _act(z, case["activation"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(t), z.to(t)) if s["z"] is not None else (y.to(t),)
    if case["kind"] == "backward":
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _act_slope(s["z"].float(), case["activation"])
        out = ((dz @ s["weight"].float()).to(t), (dz.transpose(1, 2) @ s["x"].float()).to(t))
        return out + ((dz.sum(dim=1)).to(t),) if case["bias"] else out
    if case["kind"] == "orth":
        return (_orthogonalise(s["u"].float()).to(t),)
    x, g = s["x"].float(), s["gradient"].float()
    m = MU * s["momentum"] + g
    u = g + MU * m if case["nesterov"] else m
    step = u.clone()
    for (rows, cols, scale), at in _same_shapes(s["matrices"]):
        block = torch.stack([u[:, k:k + rows * cols] for k in at])
        o = scale * _orthogonalise(block.reshape(-1, rows, cols)).reshape(len(at), u.shape[0], rows * cols)
        for k, part in zip(at, o):
            step[:, k:k + rows * cols] = part
    h = x - LR * (step + DECAY * x)
    itself = s["peers"] == torch.arange(x.shape[0], device=x.device)
    w = torch.where(itself, torch.zeros_like(s["weights"]), s["weights"])[:, None]
    return (h - w * (h - x[s["peers"].long()])).to(t), m


def _own(s):
    from paper_2009_05766_b200 import binding
    case = s["case"]
    if "workspace" not in s:    # a program keeps it, and the list of its matrices, from one call to the next
        if case["kind"] in ("forward", "backward"):
            size = binding.netmax_layer_workspace_size(case["M"], case["n"], case["n_in"], case["n_out"], case["storage"])
        elif case["kind"] == "orth":
            size = binding.netmax_orthogonalise_workspace_size(case["count"], case["rows"], case["cols"], case["storage"])
        else:
            s["table"] = binding.matrix_table(s["matrices"])
            size = binding.netmax_orthogonalised_step_workspace_size(case["M"], s["x"].shape[1], s["table"], case["storage"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if case["kind"] == "forward":
        binding.netmax_layer_forward(s["x"], s["weight"], s["y"], bias=s["bias"], residual=s["residual"], z=s["z"],
                                     activation=case["activation"], workspace=s["workspace"])
        return (s["y"], s["z"]) if s["z"] is not None else (s["y"],)
    if case["kind"] == "backward":
        binding.netmax_layer_backward(s["dy"], s["x"], s["weight"], dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"], z=s["z"],
                                      activation=case["activation"], workspace=s["workspace"])
        return (s["dx"], s["dweight"], s["dbias"]) if s["dbias"] is not None else (s["dx"], s["dweight"])
    if case["kind"] == "orth":
        binding.netmax_orthogonalise(s["u"], s["out"], steps=STEPS, workspace=s["workspace"])
        return (s["out"],)
    binding.netmax_orthogonalised_step(s["x"], s["x_next"], s["gradient"], s["momentum"], s["momentum_next"], s["table"], s["peers"],
                                       s["weights"], lr=LR, mu=MU, nesterov=case["nesterov"], decay=DECAY, steps=STEPS,
                                       workspace=s["workspace"])
    return s["x_next"], s["momentum_next"]


def run(state):
    return _own(state) if own else _plain(state)


def _exact_orthogonalise(u):
    """From the definition, in 64 bits: the odd polynomial by nested products with the matrix itself, wide as a tall one's transpose."""
    x = u.double()
    if x.shape[1] < x.shape[2]:
        return _exact_orthogonalise(x.transpose(1, 2)).transpose(1, 2)
    norm = torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True)
    x = x / torch.where(norm > 0, norm, torch.ones_like(norm))
    for _ in range(STEPS):
        cubed = x @ (x.mT @ x)
        x = QUINTIC[0] * x + QUINTIC[1] * cubed + QUINTIC[2] * (cubed @ (x.mT @ x))
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("forward", "backward"):
        x, weight = s["x"].double(), s["weight"].double()
        functions = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * torch.special.ndtr(v), "silu": lambda v: v * torch.sigmoid(v)}
        f = functions[case["activation"]]
        if case["kind"] == "forward":
            z = torch.einsum("mni,moi->mno", x, weight)
            z = z if s["bias"] is None else z + s["bias"].double().unsqueeze(1)
            y = f(z) if s["residual"] is None else f(z) + s["residual"].double()
            return (y, z) if s["z"] is not None else (y,)
        dz = s["dy"].double()
        if s["z"] is not None:
            z = s["z"].double().requires_grad_(True)
            dz, = torch.autograd.grad(f(z), z, dz)
        out = (torch.einsum("mno,moi->mni", dz, weight), torch.einsum("mno,mni->moi", dz, x))
        return out + (torch.einsum("mno->mo", dz),) if case["bias"] else out
    if case["kind"] == "orth":
        return (_exact_orthogonalise(s["u"]),)
    x, g = s["x"].double(), s["gradient"].double()
    m = s["momentum"].double() * MU + g
    u = MU * m + g if case["nesterov"] else m
    h = (1 - LR * DECAY) * x - LR * u
    for at, rows, cols, scale in s["matrices"]:
        part = slice(at, at + rows * cols)
        o = _exact_orthogonalise(u[:, part].reshape(-1, rows, cols)).reshape(-1, rows * cols)
        h[:, part] = (1 - LR * DECAY) * x[:, part] - LR * scale * o
    peers, w = s["peers"].tolist(), s["weights"].double().tolist()
    pulled = [h[i] if m_ == i else (1 - w[i]) * h[i] + w[i] * x[m_] for i, m_ in enumerate(peers)]
    return torch.stack(pulled), m
