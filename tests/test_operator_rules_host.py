"""More of what the operators on real weights accept and refuse, and rules of their sources that no run may be needed to see (no GPU needed)."""
import ctypes as C
import os
import re

import pytest

from paper_2009_05766_b200 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2009_05766_b200", "csrc")
BASE = 1 << 44      # an address that nothing is read from
NONE = b.View(None, 0, 0)


def no_gpu():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("would run")


# ---- views that lie between one another
M, N, N_IN, N_OUT = 3, 20, 8, 16
WIDE = 64     # columns of a buffer that x, y, z, the residual and dx share


def layer(**changes):
    ws = b.netmax_layer_workspace_size(M, N, N_IN, N_OUT)
    far = lambda k, row, worker: b.View(BASE + (k << 36), row, worker)  # noqa: E731
    a = b.Layer(M, N, N_IN, N_OUT, 0, 0, far(0, N_IN, N * N_IN), far(1, N_IN, N_IN * N_OUT), NONE, NONE, far(4, N_OUT, N * N_OUT), NONE,
                far(6, N_OUT, N * N_OUT), NONE, NONE, NONE, 0, None, BASE + (20 << 36), ws)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


def column(first, row=WIDE, worker=N * WIDE):
    return b.View(BASE + 4 * first, row, worker)


APART = [   # (changes of a forward call)
    dict(x=column(0), y=column(8)),
    dict(x=column(56), y=column(40)),
    dict(x=column(0), y=column(8), z=column(24), residual=column(40)),
    dict(M=1, x=column(0), y=column(8)),
    dict(x=column(0, M * WIDE, WIDE), y=column(8, M * WIDE, WIDE)),                 # workers woven into one another
    dict(x=column(0, WIDE, 0), y=column(8)),                                        # one input for all
    dict(x=column(0, WIDE, WIDE), y=column(8, M * WIDE, WIDE)),                     # sliding windows beside woven outputs
    dict(x=column(0, 2 * WIDE, 2 * N * WIDE), y=column(8)),                         # every second row
    dict(n=1, x=column(0, 0, WIDE), y=column(8, 0, WIDE)),
]
OVERLAPPING = [
    dict(x=column(0), y=column(7)),
    dict(x=column(56), y=column(41)),
    dict(x=column(0), y=column(49)),                                                # its last column is the next row's first
    dict(M=1, x=column(0), y=column(7)),
    dict(x=column(0, M * WIDE, WIDE), y=column(7, M * WIDE, WIDE)),
    dict(x=column(0, WIDE, 0), y=column(7)),
    dict(x=column(0), y=column(8), z=column(23)),
    dict(x=column(0, WIDE - 8, N * (WIDE - 8)), y=column(8)),                       # rows that drift against one another
    dict(n=1, x=column(0, 0, WIDE), y=column(7, 0, WIDE)),
]


@pytest.mark.parametrize("changes", APART)
def test_disjoint_columns_are_no_overlap(changes):
    no_gpu()
    assert b.lib().netmax_layer_forward(C.addressof(layer(**changes))) == -4


@pytest.mark.parametrize("changes", OVERLAPPING)
def test_shared_columns_are_an_overlap(changes):
    assert b.lib().netmax_layer_forward(C.addressof(layer(**changes))) == -1


@pytest.mark.parametrize("changes,code", [(dict(x=column(0), dy=column(8), dx=column(24)), -4), (dict(x=column(0), dy=column(8), dx=column(23)), -1),
                                          (dict(x=column(0), dy=column(8), dx=column(57), dweight=b.View(BASE + (8 << 36), N_IN, N_IN * N_OUT)), -1)])
def test_disjoint_columns_of_a_gradient(changes, code):
    if code == -4:
        no_gpu()
    assert b.lib().netmax_layer_backward(C.addressof(layer(**changes))) == code


def test_matrices_between_one_another():
    ws = b.netmax_orthogonalise_workspace_size(4, 20, 30)
    for first, code in ((30, -4), (29, -1), (71, -1), (70, -4)):
        if code == -4:
            no_gpu()
        a = b.Orthogonal(4, 20, 30, 0, 5, b.View(BASE, 100, 2000), b.View(BASE + 4 * first, 100, 2000), 0, None, BASE + (20 << 36), ws)
        assert b.lib().netmax_orthogonalise(C.addressof(a)) == code, first


# ---- numbers that fp32 does not hold
TABLE = b.matrix_table([(10, 20, 30, 1.0)])


@pytest.mark.parametrize("changes", [dict(lr=1e39), dict(mu=-1e39), dict(decay=1e300), dict(matrices=b.matrix_table([(10, 20, 30, 1e39)]))])
def test_a_step_refuses_what_is_infinite_in_fp32(changes):
    view = lambda k: b.View(BASE + (k << 36), 1000, 1000)  # noqa: E731
    ws = b.netmax_orthogonalised_step_workspace_size(3, 1000, TABLE)
    a = b.Step(3, 1000, 0, view(0), view(1), view(2), view(3), view(4), C.addressof(TABLE), 1, BASE + (9 << 36), BASE + (10 << 36), 0.1, 0.9, 0.0, 1, 5, 0, None,
               BASE + (20 << 36), ws)
    for k, v in changes.items():
        setattr(a, k, C.addressof(v) if k == "matrices" else v)
    assert b.lib().netmax_orthogonalised_step(C.addressof(a)) == -1


# ---- the binding
def test_a_workspace_has_all_the_bytes_that_it_counts():
    torch = pytest.importorskip("torch")
    like = torch.empty(1)
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 30), torch.empty(4096, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            b._workspace(bad, like)
    whole = torch.empty(4096, dtype=torch.uint8)
    assert b._workspace(whole, like) == (whole.data_ptr(), 4096)
    assert b._workspace(None, like) == (None, 0)


# ---- tensor memory
def test_a_kernel_lets_its_successor_start_only_once_it_holds_its_tensor_memory():
    """A CTA of the successor that takes an SM's tensor memory and waits for this grid, beside one of this grid that waits for tensor memory, would
    never end.  So every kernel that allocates some reads the address behind a barrier before it lets its successor start."""
    checked = 0
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for body in re.split(r"__global__", text)[1:]:
            body = body.split("\n}\n")[0]
            if "tmem_alloc<" not in body:
                continue
            checked += 1
            alloc, read, start = (body.index(s) for s in ("tmem_alloc<", "= tmem_at;", "let_successor_start()"))
            assert alloc < body.index("__syncthreads()", alloc) < read < start, name
    assert checked == 2
