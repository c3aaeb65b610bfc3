"""What the operators on real weights refuse, and their structs' layout: no kernel runs (no GPU needed)."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2009_05766_b200 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 1 << 44      # an address that nothing is read from: every call below is refused before


def view(k, row, worker):
    return b.View(BASE + (k << 36), row, worker)


def layer(**changes):
    M, n, n_in, n_out = 3, 20, 8, 16
    ws = b.netmax_layer_workspace_size(M, n, n_in, n_out)
    a = b.Layer(M, n, n_in, n_out, 0, 0, view(0, n_in, n * n_in), view(1, n_in, n_in * n_out), view(2, n_out, n_out), view(3, n_out, n * n_out),
                view(4, n_out, n * n_out), view(5, n_out, n * n_out), view(6, n_out, n * n_out), view(7, n_in, n * n_in),
                view(8, n_in, n_in * n_out), view(9, n_out, n_out), 0, None, BASE + (20 << 36), ws)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


def code_of(call, a):
    return call(C.addressof(a))


NONE = b.View(None, 0, 0)
LAYER_REFUSALS = [
    (dict(M=0), -1), (dict(M=16385), -1), (dict(n=-1), -1), (dict(n_in=0), -1), (dict(n_out=0), -1), (dict(n=1 << 30), -1), (dict(storage=2), -1),
    (dict(activation=4), -1), (dict(activation=-1), -1), (dict(x=NONE), -1), (dict(weight=NONE), -1), (dict(workspace=None), -1),
    (dict(workspace=BASE + (20 << 36) + 64), -1), (dict(workspace_bytes=100), -3), (dict(x=view(0, 7, 160)), -1), (dict(x=view(0, -8, 160)), -1),
    (dict(x=b.View(BASE + 2, 8, 160)), -1), (dict(weight=view(1, 1 << 39, 0)), -1),
]


@pytest.mark.parametrize("changes,code", LAYER_REFUSALS + [
    (dict(y=NONE), -1), (dict(y=view(4, 16, 0)), -1), (dict(y=view(4, 16, 319)), -1), (dict(y=view(0, 16, 320)), -1), (dict(y=view(1, 16, 320)), -1),
    (dict(y=view(2, 16, 320)), -1), (dict(y=b.View(BASE + (3 << 36) + 64, 16, 320)), -1), (dict(z=view(4, 16, 320)), -1), (dict(z=view(5, 16, 16)), -1),
    (dict(z=view(3, 16, 320)), -1), (dict(z=view(0, 16, 320)), -1)])
def test_forward_refuses(changes, code):
    assert code_of(b.lib().netmax_layer_forward, layer(**changes)) == code
    assert b.lib().netmax_last_error(None)


@pytest.mark.parametrize("changes,code", LAYER_REFUSALS + [
    (dict(dy=NONE), -1), (dict(activation=2, z=NONE), -1), (dict(dx=view(6, 8, 160)), -1), (dict(dx=view(7, 8, 8)), -1), (dict(dweight=view(0, 8, 128)), -1),
    (dict(dweight=view(8, 8, 0)), -1), (dict(dbias=view(9, 16, 8)), -1), (dict(dbias=view(7, 16, 16)), -1), (dict(dweight=view(7, 8, 128)), -1)])
def test_backward_refuses(changes, code):
    assert code_of(b.lib().netmax_layer_backward, layer(**changes)) == code


def test_what_is_allowed_reaches_the_device():
    """Woven outputs, shared inputs, the residual as the output, unused views: no argument is refused (without a GPU the call ends there)."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run")
    for changes in (dict(), dict(y=view(4, 48, 16), z=NONE), dict(x=view(0, 8, 0), weight=view(1, 8, 0)), dict(residual=view(4, 16, 320)), dict(bias=NONE, residual=NONE), dict(n=0)):
        assert code_of(b.lib().netmax_layer_forward, layer(**changes)) == -4
    for changes in (dict(), dict(dx=NONE, weight=NONE), dict(dweight=NONE, x=NONE), dict(dx=NONE, dweight=NONE), dict(z=NONE), dict(n=0, dy=NONE)):
        assert code_of(b.lib().netmax_layer_backward, layer(**changes)) == -4
    assert code_of(b.lib().netmax_orthogonalise, orthogonal()) == -4
    assert code_of(b.lib().netmax_orthogonalised_step, step()) == -4
    assert code_of(b.lib().netmax_orthogonalised_step, step(x=view(0, 1000, 0), momentum=view(3, 1000, 0))) == -4     # all workers from one replica


def orthogonal(**changes):
    ws = b.netmax_orthogonalise_workspace_size(4, 20, 30)
    a = b.Orthogonal(4, 20, 30, 0, 5, view(0, 30, 600), view(1, 30, 600), 0, None, BASE + (20 << 36), ws)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("changes,code", [
    (dict(count=0), -1), (dict(rows=0), -1), (dict(cols=0), -1), (dict(rows=1 << 20, cols=1 << 12), -1), (dict(storage=5), -1), (dict(steps=0), -1),
    (dict(steps=21), -1), (dict(u=NONE), -1), (dict(out=NONE), -1), (dict(out=view(0, 30, 600)), -1), (dict(out=view(1, 30, 0)), -1), (dict(u=view(0, 29, 600)), -1),
    (dict(workspace=None), -1), (dict(workspace_bytes=1000), -3), (dict(workspace=BASE + 8), -1)])
def test_orthogonalise_refuses(changes, code):
    assert code_of(b.lib().netmax_orthogonalise, orthogonal(**changes)) == code


TABLE = b.matrix_table([(10, 20, 30, 1.0), (700, 5, 5, 2.0)])


def step(**changes):
    ws = b.netmax_orthogonalised_step_workspace_size(3, 1000, TABLE)
    a = b.Step(3, 1000, 0, view(0, 1000, 1000), view(1, 1000, 1000), view(2, 1000, 1000), view(3, 1000, 1000), view(4, 1000, 1000), C.addressof(TABLE), 2,
               BASE + (9 << 36), BASE + (10 << 36), 0.1, 0.9, 0.0, 1, 5, 0, None, BASE + (20 << 36), ws)
    for k, v in changes.items():
        setattr(a, k, v)
    return a


def tables(*rows):
    return b.matrix_table(rows)


BAD_TABLES = [tables((990, 4, 4, 1.0)), tables((-1, 4, 4, 1.0)), tables((0, 0, 4, 1.0)), tables((0, 4, 4, 1.0), (15, 2, 2, 1.0)), tables((0, 4, 4, float("nan"))),
              tables((0, 1 << 40, 1 << 40, 1.0)), tables((1 << 60, 4, 4, 1.0))]


@pytest.mark.parametrize("changes,code", [
    (dict(M=0), -1), (dict(d=0), -1), (dict(d=1 << 30), -1), (dict(storage=3), -1), (dict(x=NONE), -1), (dict(x_next=NONE), -1), (dict(gradient=NONE), -1),
    (dict(momentum=NONE), -1), (dict(momentum_next=NONE), -1), (dict(peers=None), -1), (dict(weights=None), -1), (dict(lr=float("nan")), -1),
    (dict(mu=float("inf")), -1), (dict(decay=float("nan")), -1), (dict(steps=0), -1), (dict(x_next=view(0, 1000, 1000)), -1), (dict(x_next=view(2, 1000, 1000)), -1),
    (dict(x_next=view(1, 1000, 999)), -1), (dict(momentum_next=view(1, 1000, 1000)), -1), (dict(momentum_next=b.View(BASE + (3 << 36) + 4, 1000, 1000)), -1),
    (dict(n_matrices=-1), -1), (dict(n_matrices=257), -1), (dict(matrices=None), -1), (dict(workspace=None), -1), (dict(workspace_bytes=256), -3)]
    + [(dict(matrices=C.addressof(t), n_matrices=len(t)), -1) for t in BAD_TABLES])
def test_step_refuses(changes, code):
    assert code_of(b.lib().netmax_orthogonalised_step, step(**changes)) == code


def test_null_structs_and_sizes_are_refused():
    L = b.lib()
    for call in (L.netmax_layer_forward, L.netmax_layer_backward, L.netmax_orthogonalise, L.netmax_orthogonalised_step):
        assert call(None) == -1
    assert L.netmax_round_orthogonalised(None, None) == -1
    assert L.netmax_workspace_status(None, 0, None) == -1
    assert L.netmax_layer_workspace_size(3, 4, 5, 6, 0, None) == -1
    assert L.netmax_orthogonalise_workspace_size(3, 4, 5, 0, None) == -1
    with pytest.raises(b.NetmaxError):
        b.netmax_orthogonalised_step_workspace_size(3, 10, [(0, 4, 4, 1.0)])


def test_workspace_sizes_hold_what_the_kernels_use():
    """Two fp16 planes of every fp32 operand, rows padded to 16 bytes; iterates twice, with their Gram matrices."""
    assert b.netmax_layer_workspace_size(2, 10, 9, 7, "f32") >= 2 * 4 * (10 * 16 + 7 * 16 + 10 * 8)
    assert b.netmax_layer_workspace_size(2, 10, 9, 7, "bf16") >= 2 * 2 * (10 * 16 + 7 * 16 + 10 * 8)
    assert b.netmax_orthogonalise_workspace_size(5, 11, 13, "f32") >= 5 * (2 * 4 * 11 * 16 + 2 * 4 * 11 * 16)
    table = [(0, 211, 213, 1.0), (44943, 213, 211, 1.0)]    # (matrices that one CTA holds need none)
    assert b.netmax_orthogonalised_step_workspace_size(5, 89886, table, "f32") >= 2 * 5 * (2 * 4 * 211 * 216 + 2 * 4 * 211 * 216)


@pytest.mark.parametrize("struct,name", [(b.View, "netmax_view"), (b.Layer, "netmax_layer"), (b.Orthogonal, "netmax_orthogonal"), (b.Matrix, "netmax_matrix"),
                                         (b.Step, "netmax_step"), (b.Update, "netmax_update")])
def test_structs_match_the_header(struct, name, tmp_path):
    fields = [f for f, _ in struct._fields_]
    src = tmp_path / "layout.c"
    lines = ["#include <stddef.h>", "#include <stdio.h>", f'#include "{os.path.join(ROOT, "include", "netmax.h")}"', "int main(void) {",
             f'  printf("%zu\\n", sizeof({name}));'] + [f'  printf("%zu\\n", offsetof({name}, {f}));' for f in fields] + ["  return 0;", "}"]
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-o", str(exe), str(src)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [C.sizeof(struct)] + [getattr(struct, f).offset for f in fields]
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "netmax.h")).read(), flags=re.S)
    body = re.search(r"typedef struct " + name + r" \{(.*?)\} " + name + ";", header, flags=re.S).group(1)
    assert re.findall(r"\b([A-Za-z_0-9]+)\s*(?:,|;)", body) == fields


def test_views_into_the_same_replicas():
    """Gradients of a layer's weight and bias lie in the same rows of one plane: that is no overlap; one element too many is."""
    import torch
    d = 300
    for offset, code in ((128, -4), (127, -1), (284, -4), (285, -1)):
        if code == -4 and torch.cuda.is_available():
            continue
        a = layer(dweight=view(8, 8, d), dbias=b.View(BASE + (8 << 36) + 4 * offset, 16, d))
        assert code_of(b.lib().netmax_layer_backward, a) == code, offset
        a = layer(dbias=view(8, 16, d), dweight=b.View(BASE + (8 << 36) + 4 * (d - offset), 8, d))
        assert code_of(b.lib().netmax_layer_backward, a) == code, offset
