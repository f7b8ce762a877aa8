"""Scratch of the loss over a table of classes and of orthogonalised updates, which the library answers without a GPU: bounded however many and large the tensors."""
import ctypes

import pytest

import paper_2206_08869_amd as iodf
from test_step_cpu import buf, lib, loss_args, muon_args, orth_args  # noqa: F401

GB = 1 << 30


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("rows,cols,most", [(8192, 8192, 2 * GB), (8192, 16384, 3 * GB), (2048, 512, 2 * GB), (64, 65536, 2 * GB), (4100, 4096, 2 * GB), (100, 100, 2 * GB)])
def test_updates_of_long_lists_take_a_bounded_workspace(lib, buf, rows, cols, most, kind):  # noqa: F811
    n, one = ctypes.c_int64(0), ctypes.c_int64(0)
    a = dict(rows=rows, cols=cols, weight_type=kind, weight_stride=cols, grad_stride=cols)
    assert lib.iodf_muon_workspace(muon_args(buf[1], count=64, **a), n) == 0
    assert 0 < n.value <= most
    assert lib.iodf_muon_workspace(muon_args(buf[1], count=1, **a), one) == 0 and one.value <= n.value
    o = orth_args(buf[1], count=32, rows=rows, cols=cols, out_type=kind, in_stride=cols, out_stride=cols, in_batch=rows * cols, out_batch=rows * cols)
    assert lib.iodf_orthogonalise_workspace(o, n) == 0 and 0 < n.value <= most


@pytest.mark.parametrize("rows,classes", [(1 << 20, 14), (1 << 24, 2), (1 << 24, 1), (300, 5), (1 << 17, 60)])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_gradients_over_a_few_classes_take_what_they_read(lib, buf, rows, classes, kind):  # noqa: F811
    """64 classes, which is what a product reads along its sum, in all parts, beside the copy of 16 columns as 64 of them; not 256 classes."""
    n = ctypes.c_int64(0)
    a = loss_args(1 << 20, rows=rows, classes=classes, cols=16, type=kind, u_stride=16, w_stride=16, du_stride=16, dw_stride=16)
    assert lib.iodf_class_loss_workspace(a, 1, n) == 0
    parts_of_g, parts_of_u, up = (3, 3, rows + 63) if kind == 0 else (2, 1, rows + 63)
    assert n.value <= up * 64 * 2 * (parts_of_g + parts_of_u) + (16 << 20)
