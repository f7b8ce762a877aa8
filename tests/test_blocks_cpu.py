"""The training operators' boundary without a GPU: refusals, which come before any HIP call, the argument blocks' layout, and the
tests' own plain forms against what defines them."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import blocks_ref as ref
import paper_2206_08869_amd as iodf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E_ARG = -1


@pytest.fixture(scope="module")
def lib():
    return iodf.load_library()


@pytest.fixture(scope="module")
def buf():
    raw = (ctypes.c_byte * 8192)()
    at = (ctypes.addressof(raw) + 63) // 64 * 64
    return raw, at


def join_args(at, **more):
    a = iodf.JoinArgs(rows=2, gate_rows=2, cols=32, stream_type=0, block_type=0, eps=1e-6)
    for name in ("alpha", "gate", "w_post", "w_pre", "in_stream", "in_block", "out_stream", "out_block", "xq", "xe", "nq", "ne", "inv_pre",
                 "inv_post", "dalpha", "dgate", "dw_post", "dw_pre"):
        setattr(a, name, at)
    a.in_stream = at + 1024
    for name in ("in_stream_stride", "in_block_stride", "out_stream_stride", "out_block_stride"):
        setattr(a, name, 32)
    for name, v in more.items():
        setattr(a, name, v)
    return a


def test_argument_blocks_have_the_header_s_layout(tmp_path):
    """Every member's offset, as the C compiler lays the header's structs out."""
    kinds = (("iodf_join", iodf.JoinArgs), ("iodf_glu", iodf.GluArgs), ("iodf_wgrad", iodf.WgradArgs))
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "iodf.h"', 'int main(void) {']
    for name, kind in kinds:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, field) for field, _ in kind._fields_]
    (tmp_path / "o.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "o.c"), "-o", str(tmp_path / "o")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "o")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, kind in kinds:
        want.append(ctypes.sizeof(kind))
        want += [getattr(kind, field).offset for field, _ in kind._fields_]
    assert got == want


@pytest.mark.parametrize("what", [
    dict(rows=-1), dict(rows=(1 << 30) + 1), dict(cols=0), dict(cols=16385), dict(stream_type=3), dict(block_type=-1),
    dict(stream_type=1, block_type=2), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(gate_rows=0),
    dict(in_stream=None), dict(in_block=None), dict(out_stream=None), dict(out_block=None), dict(in_stream_stride=31),
    dict(out_block_stride=31), dict(xq=None), dict(xe=None), dict(ne=None), dict(inv_pre=None), dict(inv_post=None)])
def test_join_forward_refuses(lib, buf, what):
    assert lib.iodf_join_forward(join_args(buf[1], **what), None) == E_ARG


@pytest.mark.parametrize("off", ["in_stream", "in_block", "nq", "xq", "alpha", "gate", "w_post", "w_pre", "inv_pre", "inv_post"])
def test_join_forward_refuses_addresses_between_elements(lib, buf, off):
    a = join_args(buf[1])
    setattr(a, off, getattr(a, off) + 1)
    assert lib.iodf_join_forward(a, None) == E_ARG


def test_join_forward_in_place_takes_one_stride(lib, buf):
    assert lib.iodf_join_forward(join_args(buf[1], in_stream=buf[1], out_stream_stride=40), None) == E_ARG


@pytest.mark.parametrize("what", [dict(dalpha=None), dict(dgate=None), dict(dw_post=None), dict(dw_pre=None), dict(alpha=None), dict(gate=None),
                                  dict(nq=None), dict(inv_pre=None), dict(out_block=None), dict(in_block=None), dict(gate_rows=0)])
def test_join_backward_refuses(lib, buf, what):
    a = join_args(buf[1], **what)
    assert lib.iodf_join_backward(a, buf[1], 1 << 40, None) == E_ARG


def test_workspaces_are_checked(lib, buf):
    a, n = join_args(buf[1]), ctypes.c_int64(0)
    assert lib.iodf_join_workspace(a, n) == 0 and n.value > 0
    assert lib.iodf_join_backward(a, buf[1], n.value - 1, None) == E_ARG
    assert lib.iodf_join_backward(a, None, n.value, None) == E_ARG
    assert lib.iodf_join_backward(a, buf[1] + 8, n.value, None) == E_ARG
    assert lib.iodf_join_workspace(a, None) == E_ARG and lib.iodf_join_workspace(None, n) == E_ARG
    w = iodf.WgradArgs(rows=1 << 16, cols=64, out=64, dy_type=1, dy=buf[1], dy_stride=64, q=buf[1], e=buf[1], dw=buf[1], dw_stride=64)
    assert lib.iodf_weight_grad_workspace(w, n) == 0 and n.value > 0
    assert lib.iodf_weight_grad(w, buf[1], n.value - 1, None) == E_ARG
    assert lib.iodf_weight_grad(w, None, n.value, None) == E_ARG
    assert lib.iodf_weight_grad_workspace(w, None) == E_ARG and lib.iodf_weight_grad_workspace(None, n) == E_ARG


@pytest.mark.parametrize("what", [dict(rows=-1), dict(cols=0), dict(cols=65537), dict(out=0), dict(out=65537), dict(dy_type=5), dict(dy=None),
                                  dict(q=None), dict(e=None), dict(dw=None), dict(dy_stride=63), dict(dw_stride=63)])
def test_weight_grad_refuses(lib, buf, what):
    w = iodf.WgradArgs(rows=4, cols=64, out=64, dy_type=1, dy=buf[1], dy_stride=64, q=buf[1], e=buf[1], dw=buf[1], dw_stride=64)
    for name, v in what.items():
        setattr(w, name, v)
    assert lib.iodf_weight_grad(w, buf[1], 1 << 40, None) == E_ARG


@pytest.mark.parametrize("what", [dict(rows=-1), dict(cols=0), dict(cols=65537), dict(type=3), dict(act=3), dict(act=-1), dict(a=None), dict(b=None),
                                  dict(y=None), dict(a_stride=31), dict(ae=None), dict(bq=None)])
def test_glu_forward_refuses(lib, buf, what):
    g = iodf.GluArgs(rows=2, cols=32, type=1, act=1)
    for name in ("a", "b", "y", "dy", "da", "db", "aq", "ae", "bq", "be", "yq", "ye"):
        setattr(g, name, buf[1])
    for name in ("a_stride", "b_stride", "y_stride", "dy_stride", "da_stride", "db_stride"):
        setattr(g, name, 32)
    for name, v in what.items():
        setattr(g, name, v)
    assert lib.iodf_glu_forward(g, None) == E_ARG
    back = {"a": "dy", "b": "da", "y": "db", "a_stride": "dy_stride"}
    for name, v in what.items():
        if name in back:
            setattr(g, back[name], v)
    assert lib.iodf_glu_backward(g, None) == E_ARG


def test_pack_and_unpack_refuse(lib, buf):
    at = buf[1]
    assert lib.iodf_pack(at, 3, 32, 2, 32, None, at, at, None) == E_ARG
    assert lib.iodf_pack(at, 0, 31, 2, 32, None, at, at, None) == E_ARG
    assert lib.iodf_pack(at + 2, 0, 32, 2, 32, None, at, at, None) == E_ARG
    assert lib.iodf_pack(at, 0, 32, 2, 32, None, at + 8, at, None) == E_ARG
    assert lib.iodf_pack(None, 0, 32, 2, 32, None, at, at, None) == E_ARG
    assert lib.iodf_pack(at, 0, 65536, 1 << 30, 65536, None, at, at, None) == E_ARG
    assert lib.iodf_unpack(at, at, 2, 32, at, iodf.IODF_T_F16, 32, None) == E_ARG
    assert lib.iodf_unpack(None, at, 2, 32, at, 0, 32, None) == E_ARG
    assert lib.iodf_pack(None, 0, 32, 0, 32, None, None, None, None) == 0   # no rows: nothing to do
    assert lib.iodf_unpack(None, None, 0, 32, None, 0, 32, None) == 0


def test_null_arguments_are_refused(lib):
    assert lib.iodf_join_forward(None, None) == E_ARG and lib.iodf_join_backward(None, None, 0, None) == E_ARG
    assert lib.iodf_glu_forward(None, None) == E_ARG and lib.iodf_glu_backward(None, None) == E_ARG
    assert lib.iodf_weight_grad(None, None, 0, None) == E_ARG


def test_tensors_off_the_gpu_are_refused():
    import torch
    x = torch.zeros(4, 32)
    codes = iodf.Codes(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 32)
    for call in (lambda: iodf.pack(x), lambda: iodf.unpack(codes), lambda: iodf.join(x, x), lambda: iodf.glu(x, x),
                 lambda: iodf.weight_grad(codes, x), lambda: iodf.unpack((codes.q, codes.e)), lambda: iodf.pack(np.zeros((4, 32)))):
        with pytest.raises(ValueError):
            call()


def test_plain_form_s_codes_hold_what_the_layout_promises():
    """The least power of two with which no code passes 127; half a step of error; the border at 127.5 steps."""
    rng = np.random.default_rng(3)
    v = (rng.standard_normal((64, 96)) * np.exp(3 * rng.standard_normal((64, 1)))).astype(np.float32).astype(np.float64)
    q, e = ref.encode(v)
    assert np.abs(q).max() <= 127 and (np.abs(q.reshape(64, 3, 32)).max(2) >= 64).all()
    step = np.repeat(np.exp2(e.astype(np.float64) - 133), 32, 1)
    assert (np.abs(ref.decode(q, e, 96) - v) <= step / 2).all()
    below, at = np.nextafter(np.float32(127.5), np.float32(0)), 127.5
    assert ref.exponents([below, at, 127.0, 128.0, 0.0, 1e-40, 3.4e38]).tolist() == [133, 134, 133, 134, 16, 16, 254]


def test_plain_form_s_join_gradient_is_its_slope():
    """The plain backward form against differences of the plain forward form, in 64 bits."""
    rng = np.random.default_rng(5)
    rows, cols, eps = 6, 10, 1e-2
    p = dict(h=rng.standard_normal((rows, cols)), f=rng.standard_normal((rows, cols)), alpha=np.array([0.6]), gate=rng.random((3, cols)),
             w_post=rng.standard_normal(cols), w_pre=rng.standard_normal(cols))
    live = np.array([1, 1, 0, 1, 1, 1], bool)
    ch, cu = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))

    def loss(**q):
        r = ref.join(live=live, eps=eps, **q)
        return (ch * r["h"]).sum() + (cu * r["u"]).sum()

    r = ref.join(live=live, eps=eps, **p)
    g = ref.join_backward(r["x"], r["n"], r["inv_pre"], r["inv_post"], ch, cu, p["alpha"], p["gate"], p["w_post"], p["w_pre"], live)
    for name, key in (("h", "dh"), ("f", "df"), ("alpha", "dalpha"), ("gate", "dgate"), ("w_post", "dw_post"), ("w_pre", "dw_pre")):
        for at in np.ndindex(p[name].shape):
            up, down = np.array(p[name]), np.array(p[name])
            up[at] += 1e-5
            down[at] -= 1e-5
            slope = (loss(**dict(p, **{name: up})) - loss(**dict(p, **{name: down}))) / 2e-5
            assert abs(slope - g[key][at]) < 1e-7, (name, at)


@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
def test_plain_form_s_activation_slope(kind):
    a = np.linspace(-8, 8, 401) + 1e-3
    d = (ref.act(a + 1e-6, kind)[0] - ref.act(a - 1e-6, kind)[0]) / 2e-6
    assert np.abs(d - ref.act(a, kind)[1]).max() < 1e-8


def test_more_than_a_launch_can_count_is_refused(lib, buf):
    n = ctypes.c_int64(0)
    a = join_args(buf[1], rows=1 << 24, gate_rows=8)  # 2^21 shared gates: the most that the backward pass takes
    assert lib.iodf_join_workspace(a, n) == 0
    a.gate_rows = 7
    assert lib.iodf_join_workspace(a, n) == E_ARG
    a.gate_rows = 1
    assert lib.iodf_join_workspace(a, n) == 0
    assert lib.iodf_pack(buf[1], 1, 65536, (1 << 18) + 1, 65536, None, buf[1], buf[1], None) == E_ARG
