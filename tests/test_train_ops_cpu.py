"""The operators of a training step (include/hwr_ops.h) without a device: the argument
structures' layout against the C compiler's, what the binding packs, NULL contexts."""
import ctypes as C
import os
import struct
import subprocess

import pytest

from paper_2608_14575_amd import hwr, routed

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ["hwr_linear_args", "hwr_linear_grad_args", "hwr_log_probs_args", "hwr_log_probs_grad_args",
           "hwr_adamw_tensor", "hwr_adamw_config", "hwr_adamw_args"]


def test_layout_matches_header(tmp_path):
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "hwr_ops.h"', "int main(void) {"]
    for s in STRUCTS:
        src.append(f'printf("{s} sizeof %zu\\n", sizeof({s}));')
        src += [f'printf("{s} {f} %zu\\n", offsetof({s}, {f}));' for f, _ in getattr(hwr, s)._fields_]
    src.append("return 0; }")
    c, exe = tmp_path / "layout.c", tmp_path / "layout"
    c.write_text("\n".join(src))
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'include')}", str(c), "-o", str(exe)])
    for line in subprocess.check_output([str(exe)], text=True).splitlines():
        s, f, v = line.split()
        cls = getattr(hwr, s)
        assert int(v) == (C.sizeof(cls) if f == "sizeof" else getattr(cls, f).offset), line


def test_null_contexts():
    lib = hwr.load()
    for fn, args in (("hwr_log_probs", "hwr_log_probs_args"), ("hwr_log_probs_grad", "hwr_log_probs_grad_args")):
        assert getattr(lib, fn)(None, C.byref(getattr(hwr, args)())) == hwr.HWR_ERR_INVALID_ARG
        assert "ops is NULL" in hwr.hwr_ops_last_error(None)
    out = C.c_void_p(7)
    for call in (lambda: lib.hwr_adamw_init(None, C.byref(hwr.hwr_adamw_config()), C.byref(out)),
                 lambda: lib.hwr_adamw_step(None, None, C.byref(hwr.hwr_adamw_args()))):
        assert call() == hwr.HWR_ERR_INVALID_ARG
        assert "ops is NULL" in hwr.hwr_ops_last_error(None)
    hwr.hwr_adamw_free(None)


def test_packed_arguments_are_the_structures():
    for name in ("hwr_log_probs_args", "hwr_log_probs_grad_args", "hwr_adamw_args"):
        cls = getattr(hwr, name)
        call = routed._Args(hwr.load().hwr_log_probs, cls)        # (any function: without a context it reads nothing)
        values = [0.5 if t in (C.c_float, C.c_double) else (i + 3) << (8 if t is C.c_int32 else 40) for i, (_, t) in enumerate(cls._fields_)]
        assert call(None, *values) == hwr.HWR_ERR_INVALID_ARG          # (no context: nothing is read)
        a = cls.from_buffer(call._block)
        assert [getattr(a, f) for f, _ in cls._fields_] == values
        if cls._fields_[0][1] is not C.c_int32:
            continue
        with pytest.raises(hwr.HwrError) as e:
            call(None, 2 ** 31, *values[1:])
        assert e.value.status == hwr.HWR_ERR_INVALID_ARG
    assert struct.calcsize("@i") == C.sizeof(C.c_int32)
