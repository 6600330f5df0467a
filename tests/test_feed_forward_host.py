"""Host side of the products, the norms between blocks and the table's rows, without a GPU:
structures against the header, and the refusals that need no device."""
import ctypes
import os
import re

import pytest

from paper_2207_10731_gb300 import binding, build, sequence

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, UNSUPPORTED, OK = binding.PSS_ERR_INVALID_ARG, binding.PSS_ERR_UNSUPPORTED, binding.PSS_OK


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def layout(name):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pss.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", src).group(1)
    at, got = 0, []
    for kind, names in re.findall(r"((?:const )?\w+\*?)\s+([^;]+);", body):
        size = 4 if kind in ("int32_t", "float") else 8
        for field in names.split(","):
            at = (at + size - 1) // size * size
            got.append((field.strip(), at, size))
            at += size
    return got, (at + 7) // 8 * 8


@pytest.mark.parametrize("name,form", [("pss_linear_forward_args", "_FORWARD"),
                                       ("pss_linear_backward_args", "_BACKWARD")])
def test_structures_match_the_header(name, form):
    fields, size = layout(name)
    packed = getattr(sequence, form)
    assert packed.size == size
    values = list(range(1, len(fields) + 1))
    raw = packed.pack(*values)
    for (field, at, width), value in zip(fields, values):
        assert int.from_bytes(raw[at:at + width], "little") == value, field


def test_activations_match_the_header():
    src = open(os.path.join(ROOT, "include", "pss.h")).read()
    for name, value in sequence._ACTIVATIONS.items():
        assert re.search(rf"PSS_ACT_{(name or 'none').upper()} = {value}\b", src)


def forward_args(lib, at, **over):
    v = dict(tokens=4, n=8, m=16, x=at, xs=8, w=at, wi=16, wo=1, b=at, r=0, rs=16, y=at, ys=16, z=0, zs=16,
             type=1, y_type=1, act=0, reserved=0)
    v.update(over)
    where = sequence._packed(sequence._FORWARD, *v.values())
    return lib.pss_linear_forward(where, at, 1 << 30, None, None), lib.pss_linear_forward_workspace(where)


def test_products_refuse_before_any_device_work(lib):
    host = (ctypes.c_float * 256)()
    at = ctypes.addressof(host)
    for over in (dict(tokens=-1), dict(n=0), dict(m=0), dict(tokens=2 ** 31), dict(type=0), dict(type=3),
                 dict(y_type=2), dict(act=4), dict(act=-1), dict(xs=7), dict(wi=15), dict(wi=16, wo=2),
                 dict(wi=1, wo=7)):
        assert forward_args(lib, at, **over) == (BAD, 0), over
    assert forward_args(lib, at)[0] == BAD                    # host memory
    assert forward_args(lib, at, tokens=0) == (OK, 0)
    # off the grid of 16 bytes: room for copies
    _, on = forward_args(lib, at // 16 * 16, x=at // 16 * 16, w=at // 16 * 16)
    _, off = forward_args(lib, at // 16 * 16, x=at // 16 * 16 + 2, w=at // 16 * 16 + 2)
    assert off >= on + 512
    assert lib.pss_linear_forward(None, None, 0, None, None) == BAD
    assert lib.pss_linear_backward(None, None, 0, None, None) == BAD
    assert lib.pss_linear_forward_workspace(None) == lib.pss_linear_backward_workspace(None) == 0

    def backward(**over):
        v = dict(tokens=4, n=8, m=16, g=at, gs=16, x=at, xs=8, w=at, wi=16, wo=1, z=at, zs=16, dx=at, dxs=8,
                 dw=at, dwi=16, dwo=1, db=at, type=1, grad_type=1, dw_type=0, act=2)
        v.update(over)
        return lib.pss_linear_backward(sequence._packed(sequence._BACKWARD, *v.values()), at, 1 << 30,
                                       None, None)
    for over in ({}, dict(tokens=-1), dict(gs=15), dict(xs=7), dict(zs=15), dict(dxs=7), dict(wi=4), dict(dwi=4),
                 dict(grad_type=2), dict(dw_type=2), dict(act=9), dict(type=0), dict(tokens=0)):
        assert backward(**over) == BAD, over
    assert backward(tokens=0, dw=0, db=0) == OK


def test_norms_refuse_before_any_device_work(lib):
    def forward(type=1, stream=0, xs=8, rs=8, gates=0, gs=8, rows=4, cols=8, scale=1.0, eps=1e-5, ts=8):
        return lib.pss_residual_norm_forward(None, type, xs, None, stream, rs, None, gates, gs, None, None, rows,
                                             cols, scale, eps, None, ts, None, 8, None, None, None)
    assert forward(type=3) == forward(stream=2) == forward(xs=7) == forward(rs=7) == forward(gates=3) == \
        forward(gates=2, gs=7) == forward(gates=1, gs=0) == forward(rows=-1) == forward(cols=0) == \
        forward(scale=float("inf")) == forward(eps=-1.0) == forward(eps=float("nan")) == forward(ts=7) == BAD
    assert forward() == BAD and forward(rows=0) == OK
    assert forward(cols=16385, xs=16385, rs=16385, ts=16385) == UNSUPPORTED
    assert lib.pss_residual_norm_workspace(0, 8) == lib.pss_residual_norm_workspace(4, 16385) == 0


def test_tables_refuse_before_any_device_work(lib):
    host = (ctypes.c_float * 64)()
    at = ctypes.addressof(host)

    def forward(type=0, ws=8, rows=4, cols=8, tokens=3, scale=1.0, to=0, os=8, weight=at, status=None):
        return lib.pss_embedding_forward(weight, type, ws, rows, cols, at, tokens, scale, at, to, os, status, None)
    assert forward(type=3) == forward(to=-1) == forward(ws=7) == forward(os=7) == forward(rows=-1) == \
        forward(tokens=-1) == forward(scale=float("nan")) == forward(rows=2 ** 31) == BAD
    assert forward() == forward(status=at) == BAD             # host memory
    assert forward(cols=2 ** 20 + 1, ws=2 ** 21, os=2 ** 21) == UNSUPPORTED
    assert forward(tokens=0) == forward(cols=0) == OK
    assert lib.pss_embedding_workspace(0, 4, 8) == lib.pss_embedding_workspace(4, 0, 8) == 0
    assert lib.pss_embedding_workspace(100000, 4, 8) > lib.pss_embedding_workspace(100, 4, 8) > 0
    rc = lib.pss_embedding_backward(at, 0, 8, at, 3, 1.0, 4, 8, at, 0, 8, at, 1 << 20, None, None)
    assert rc == BAD
    assert lib.pss_embedding_backward(None, 0, 8, None, 0, 1.0, 0, 8, None, 0, 8, None, 0, None, None) == OK
