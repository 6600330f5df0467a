"""The sequence operators' host side, without a GPU: sources, structures and the
refusals that need no device."""
import ctypes
import os
import re

import pytest

from paper_2207_10731_gb300 import binding, build, sequence

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SEQ = os.path.join(ROOT, "paper_2207_10731_gb300", "csrc", "seq")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_every_kernel_waits_for_its_predecessor_first():
    found = 0
    for f in sorted(os.listdir(SEQ)):
        src = open(os.path.join(SEQ, f)).read()
        for m in re.finditer(r"__global__", src):
            j, depth, opened = m.end(), 0, False
            while not (src[j] == "{" and depth == 0 and opened):
                depth += {"(": 1, ")": -1}.get(src[j], 0)
                opened = opened or src[j] == "("
                j += 1
            found += 1
            assert src[j + 1:].lstrip().startswith("pdl_prologue();"), f
    assert found >= 8


def test_structures_match_the_header():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "pss.h")).read(), flags=re.S)
    sizes = {"int64_t": 8, "const int64_t*": 8, "int32_t": 4, "float": 4, "void*": 8}

    def layout(name):
        body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", src).group(1)
        at, got = 0, []
        for kind, names in re.findall(r"((?:const )?\w+\*?)\s+([^;]+);", body):
            for _ in names.split(","):
                at = (at + sizes[kind] - 1) // sizes[kind] * sizes[kind]
                got.append((at, sizes[kind]))
                at += sizes[kind]
        return got, (at + 7) // 8 * 8
    fields, size = layout("pss_attention_shape")
    assert size == sequence._SHAPE.size == 64
    assert fields == [(8 * i, 8) for i in range(5)] + [(40 + 4 * i, 4) for i in range(5)]
    fields, size = layout("pss_rows")
    assert size == sequence._ROWS.size == 24 and fields == [(0, 8), (8, 8), (16, 8)]
    # each tensor of a call has its place in the buffer
    assert sequence._structs((1, 0, 0, 2, 3, 4, 4, 64, 1, 0.5), (16, 8, 8), (32, 8, 8))[1:] == \
        [sequence._local.buffer[1] + 64, sequence._local.buffer[1] + 88]


def test_refusals_before_any_device_work(lib):
    bad, unsupported = binding.PSS_ERR_INVALID_ARG, binding.PSS_ERR_UNSUPPORTED

    def norm(x_type=0, rows=4, cols=8, eps=1e-5, xs=8, ys=8):
        return lib.pss_layer_norm_forward(None, x_type, xs, None, None, rows, cols, eps, None, 0, ys,
                                          None, None, None)
    assert norm(x_type=3) == norm(rows=-1) == norm(cols=0) == norm(eps=-1.0) == norm(xs=7) == \
        norm(ys=7) == norm(eps=float("nan")) == bad
    assert norm() == bad                      # null pointers
    assert norm(cols=16385, xs=16385, ys=16385) == unsupported
    assert norm(rows=0) == binding.PSS_OK
    host = (ctypes.c_float * 64)()
    at = ctypes.addressof(host)
    assert lib.pss_layer_norm_forward(at, 0, 8, at, at, 4, 8, 1e-5, at, 0, 8, at, at, None) == bad
    assert lib.pss_layer_norm_workspace(0, 8) == lib.pss_layer_norm_workspace(4, 16385) == 0

    def drop(p=0.5, rows=4, cols=8, xs=8, kind=0):
        return lib.pss_dropout(at, xs, None, 0, rows, cols, p, 0, 0, kind, at, 8, None)
    assert drop(p=-0.1) == drop(p=1.1) == drop(p=float("nan")) == drop(rows=-1) == drop(xs=7) == \
        drop(kind=9) == bad
    assert drop() == bad                      # host memory
    assert drop(rows=0) == drop(cols=0) == binding.PSS_OK

    def attention(**over):
        s = dict(sequences=1, q=at, k=at, q_tokens=4, k_tokens=4, heads=4, kv_heads=2, dim=64,
                 causal=1, scale=0.125)
        s.update(over)
        where = sequence._structs(tuple(s.values()), *[(at, 256, 64)] * 4)
        return lib.pss_attention_forward(*where, at, at, 1 << 20, None, None), \
            lib.pss_attention_workspace(where[0], 0)
    for over in (dict(sequences=-1), dict(q_tokens=-1), dict(k_tokens=2 ** 31), dict(heads=3),
                 dict(kv_heads=0), dict(heads=258), dict(dim=60), dict(dim=136), dict(dim=0),
                 dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf"))):
        assert attention(**over) == (bad, 0), over
    rc, size = attention()
    assert rc == bad and size > 0             # host memory
    assert lib.pss_attention_forward(*[None] * 7, 0, None, None) == bad
    assert lib.pss_attention_backward(*[None] * 11, 0, None, None) == bad


def test_a_register_split_is_checked_before_its_kernel_is_launched():
    # a warpgroup that asks for more registers than the launch brought waits for ever
    kernels = {f: open(os.path.join(SEQ, f)).read() for f in os.listdir(SEQ)}
    users = {f for f, src in kernels.items() if "set_registers<C::" in src}
    assert users == {"attention_forward.cu"}
    src = kernels["attention_forward.cu"]
    assert not re.search(r"set_registers<\d", src)
    more, less = map(int, re.search(r"kMore = (\d+), kLess = (\d+)", src).groups())
    # the launch's registers are a whole number a thread, and at most what 384 threads can have
    assert (2 * more + less) % 3 == 0 and (2 * more + less) // 3 <= 65536 // 384 // 8 * 8
    assert "allow_smem(k, C::kSmem, &ready, C::kLaunch)" in src
    assert "built.numRegs < least_registers" in kernels["attention_tma.h"]
