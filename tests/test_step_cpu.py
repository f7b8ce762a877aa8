"""The loss over a table of classes and orthogonalised updates without a GPU: refusals, which come before any HIP call, the argument blocks' layout, and the
tests' own plain forms against what defines them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2206_08869_amd as iodf
import step_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E_ARG = -1


@pytest.fixture(scope="module")
def lib():
    return iodf.load_library()


@pytest.fixture(scope="module")
def buf():
    raw = (ctypes.c_byte * 8192)()
    return raw, (ctypes.addressof(raw) + 63) // 64 * 64


def loss_args(at, **more):
    a = iodf.ClassLossArgs(rows=4, classes=6, cols=8, type=1, u_stride=8, w_stride=8, du_stride=8, dw_stride=8)
    for name in ("u", "w", "target", "loss", "lse", "dloss", "dlse", "du", "dw"):
        setattr(a, name, at)
    for name, v in more.items():
        setattr(a, name, v)
    return a


NUMBERS = (ctypes.c_float * 48)(*ref.QUINTIC * 16)


def orth_args(at, **more):
    a = iodf.OrthArgs(count=2, in_batch=64, out_batch=64, in_stride=8, out_stride=8, rows=8, cols=8, in_type=0, out_type=1, steps=5, eps=1e-7,
                      coefficients=ctypes.addressof(NUMBERS), in_=at, out=at)
    for name, v in more.items():
        setattr(a, name, v)
    return a


def muon_args(at, **more):
    lists = (ctypes.c_void_p * 64)(*[at] * 64)
    a = iodf.MuonArgs(count=2, weight_stride=8, grad_stride=8, rows=8, cols=8, weight_type=1, grad_type=0, steps=5, nesterov=1, eps=1e-7, rate=0.1, beta=0.9,
                      scale=1.0, coefficients=ctypes.addressof(NUMBERS), weights=ctypes.addressof(lists), grads=ctypes.addressof(lists),
                      momenta=ctypes.addressof(lists))
    a.keep = lists
    for name, v in more.items():
        setattr(a, name, v)
    return a


def test_argument_blocks_have_the_header_s_layout(tmp_path):
    kinds = (("iodf_class_loss", iodf.ClassLossArgs), ("iodf_orth", iodf.OrthArgs), ("iodf_muon", iodf.MuonArgs))
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "iodf.h"', 'int main(void) {']
    for name, kind in kinds:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, field.rstrip("_")) for field, _ in kind._fields_]
    lines.append('printf("%d\\n%d\\n", IODF_ORTH_MOST, IODF_MUON_MOST);')
    (tmp_path / "o.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "o.c"), "-o", str(tmp_path / "o")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "o")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, kind in kinds:
        want.append(ctypes.sizeof(kind))
        want += [getattr(kind, field).offset for field, _ in kind._fields_]
    assert got == want + [iodf.IODF_ORTH_MOST, iodf.IODF_MUON_MOST]


BOTH = [dict(rows=-1), dict(rows=(1 << 24) + 1), dict(classes=0), dict(classes=(1 << 20) + 1), dict(cols=0), dict(cols=65537), dict(type=3), dict(type=-1),
        dict(rows=1 << 24, cols=1025), dict(classes=1 << 20, cols=16385), dict(rows=1 << 20, classes=(1 << 18) + 1), dict(u=None), dict(w=None),
        dict(target=None), dict(lse=None), dict(u_stride=7), dict(w_stride=7)]


@pytest.mark.parametrize("what", BOTH + [dict(loss=None)])
def test_class_loss_refuses(lib, buf, what):
    assert lib.iodf_class_loss_forward(loss_args(buf[1], **what), buf[1], 1 << 50, None) == E_ARG


@pytest.mark.parametrize("what", BOTH + [dict(du_stride=7), dict(dw_stride=7)])
def test_class_loss_backward_refuses(lib, buf, what):
    assert lib.iodf_class_loss_backward(loss_args(buf[1], **what), buf[1], 1 << 50, None) == E_ARG


@pytest.mark.parametrize("off", ["u", "w", "target", "loss", "lse", "dloss", "dlse", "du", "dw"])
def test_class_loss_refuses_addresses_between_elements(lib, buf, off):
    a = loss_args(buf[1])
    setattr(a, off, getattr(a, off) + 1)
    call = lib.iodf_class_loss_forward if off == "loss" else lib.iodf_class_loss_backward
    assert call(a, buf[1], 1 << 50, None) == E_ARG


@pytest.mark.parametrize("what", [dict(count=-1), dict(count=4097), dict(rows=0), dict(cols=0), dict(rows=65537), dict(rows=16385, cols=16385), dict(in_type=3),
                                  dict(out_type=-1), dict(steps=0), dict(steps=17), dict(eps=0.0), dict(eps=float("nan")), dict(coefficients=None), dict(in_=None),
                                  dict(out=None), dict(in_stride=7), dict(out_stride=7), dict(in_batch=0), dict(out_batch=63), dict(count=4096, rows=1024, cols=1025)])
def test_orthogonalise_refuses(lib, buf, what):
    assert lib.iodf_orthogonalise(orth_args(buf[1], **what), buf[1], 1 << 50, None) == E_ARG


@pytest.mark.parametrize("what", [dict(count=-1), dict(count=65), dict(rows=0), dict(cols=65537), dict(weight_type=5), dict(grad_type=-1), dict(steps=0),
                                  dict(eps=-1.0), dict(rate=float("nan")), dict(beta=float("inf")), dict(decay=float("nan")), dict(scale=float("inf")),
                                  dict(coefficients=None), dict(weights=None), dict(grads=None), dict(momenta=None), dict(weight_stride=7), dict(grad_stride=7)])
def test_muon_step_refuses(lib, buf, what):
    assert lib.iodf_muon_step(muon_args(buf[1], **what), buf[1], 1 << 50, None) == E_ARG


def test_muon_step_refuses_tensors_that_are_not_there(lib, buf):
    for name in ("weights", "grads", "momenta"):
        for bad in (None, buf[1] + 1):
            lists = (ctypes.c_void_p * 2)(buf[1], bad)
            assert lib.iodf_muon_step(muon_args(buf[1], **{name: ctypes.addressof(lists)}), buf[1], 1 << 50, None) == E_ARG


@pytest.mark.parametrize("numbers", [(float("nan"), 0, 0), (1.0, float("inf"), 0.0), (100.0, 0.0, 0.0), (0.0, 5000.0, 0.0)])
def test_polynomials_that_let_numbers_grow_are_refused(lib, buf, numbers):
    bad = (ctypes.c_float * 15)(*numbers * 5)
    assert lib.iodf_orthogonalise(orth_args(buf[1], coefficients=ctypes.addressof(bad)), buf[1], 1 << 50, None) == E_ARG
    assert lib.iodf_muon_step(muon_args(buf[1], coefficients=ctypes.addressof(bad)), buf[1], 1 << 50, None) == E_ARG


def test_workspaces_are_checked(lib, buf):
    n = ctypes.c_int64(0)
    a, o, m = loss_args(buf[1]), orth_args(buf[1]), muon_args(buf[1])
    for query, call in ((lambda: lib.iodf_class_loss_workspace(a, 0, n), lambda *w: lib.iodf_class_loss_forward(a, *w, None)),
                        (lambda: lib.iodf_class_loss_workspace(a, 1, n), lambda *w: lib.iodf_class_loss_backward(a, *w, None)),
                        (lambda: lib.iodf_orthogonalise_workspace(o, n), lambda *w: lib.iodf_orthogonalise(o, *w, None)),
                        (lambda: lib.iodf_muon_workspace(m, n), lambda *w: lib.iodf_muon_step(m, *w, None))):
        assert query() == 0 and n.value > 0
        assert call(buf[1], n.value - 1) == E_ARG and call(None, n.value) == E_ARG and call(buf[1] + 8, n.value) == E_ARG
    assert lib.iodf_class_loss_workspace(a, 0, None) == E_ARG and lib.iodf_class_loss_workspace(None, 0, n) == E_ARG
    assert lib.iodf_orthogonalise_workspace(None, n) == E_ARG and lib.iodf_muon_workspace(m, None) == E_ARG


def test_nothing_to_do_is_done(lib, buf):
    assert lib.iodf_class_loss_forward(loss_args(None, rows=0), None, 0, None) == 0
    assert lib.iodf_class_loss_backward(loss_args(None, rows=0), None, 0, None) == 0
    assert lib.iodf_orthogonalise(orth_args(None, count=0), None, 0, None) == 0
    assert lib.iodf_muon_step(muon_args(None, count=0), None, 0, None) == 0
    for call in (lib.iodf_class_loss_forward, lib.iodf_class_loss_backward, lib.iodf_orthogonalise, lib.iodf_muon_step):
        assert call(None, None, 0, None) == E_ARG


def test_a_table_s_gradient_takes_a_bounded_workspace(lib, buf):
    """2^17 rows and 2^17 classes have 2^34 logits: what is kept of them at a time stays at 512 MB, and two parts of a row's sums."""
    n = ctypes.c_int64(0)
    a = loss_args(1 << 20, rows=1 << 17, classes=1 << 17, cols=64, u_stride=64, w_stride=64)
    assert lib.iodf_class_loss_workspace(a, 1, n) == 0
    assert n.value <= (512 << 20) + 64 * (1 << 17) * 64 * 4
    assert lib.iodf_class_loss_workspace(a, 0, n) == 0
    assert n.value <= (1 << 17) * (4 + 2 * 4 * (1 << 17) // 128)


def test_tensors_off_the_gpu_are_refused():
    import torch
    x, y, t = torch.zeros(4, 32), torch.zeros(9, 32), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: iodf.class_loss(x, y, t), lambda: iodf.class_loss_backward(x, y, t, t, t), lambda: iodf.classified(x, y, t), lambda: iodf.orthogonalise(x),
                 lambda: iodf.orthogonalise(np.zeros((4, 4))), lambda: iodf.orthogonalise(torch.zeros(2, 3, 4)), lambda: iodf.muon_step(x, x, x, 0.1),
                 lambda: iodf.muon_step([x], [x, x], [x], 0.1), lambda: iodf.muon_step(None, x, x, 0.1)):
        with pytest.raises(ValueError):
            call()


def test_coefficients_are_checked():
    from paper_2206_08869_amd import step
    assert list(step._polynomials(2, (1.5, -0.5, 0))) == [1.5, -0.5, 0.0] * 2
    assert list(step._polynomials(2, [[1.5, -0.5, 0], (2, 3, 4)])) == [1.5, -0.5, 0, 2, 3, 4]
    for steps, numbers in ((0, (1, 2, 3)), (17, (1, 2, 3)), (2.0, (1, 2, 3)), (2, (1, 2)), (2, ((1, 2, 3),)), (2, ((1, 2), (3, 4))), (1, "abc"), (1, None), (1, ())):
        with pytest.raises(ValueError):
            step._polynomials(steps, numbers)


def test_plain_form_s_loss_is_the_likelihood():
    rng = np.random.default_rng(1)
    u, w, target = rng.standard_normal((5, 4)), rng.standard_normal((7, 4)), np.array([0, 6, 3, 3, 1])
    p = np.exp(u @ w.T)
    loss, lse, _ = ref.loss(u, w, target)
    assert np.allclose(loss, -np.log(p[np.arange(5), target] / p.sum(1))) and np.allclose(lse, np.log(p.sum(1)))


def test_plain_form_s_steps_keep_singular_vectors():
    """The steps against the polynomial of singular values, out of a decomposition."""
    rng = np.random.default_rng(2)
    for shape in ((9, 14), (14, 9)):
        g = rng.standard_normal(shape)
        a, s, b = np.linalg.svd(g, full_matrices=False)
        s = s / np.linalg.norm(s)
        for _ in range(5):
            s = s * (3.4445 - 4.7750 * s ** 2 + 2.0315 * s ** 4)
        assert np.allclose(ref.orthogonalise(g, eps=0.0)[0], a * s @ b, atol=1e-12)
