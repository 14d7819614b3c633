"""hwr_ops.h without a device: the argument structures' layout against the C
compiler's, NULL contexts, and the binding's checks of torch tensors."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2608_14575_amd import hwr, routed

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = ["hwr_groups", "hwr_matmul_args", "hwr_matmul_grad_args", "hwr_adapter_args", "hwr_adapter_grad_args"]


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


def test_null_arguments():
    lib = hwr.load()
    g = hwr.hwr_groups()
    assert lib.hwr_ops_init(0, None, None) == hwr.HWR_ERR_INVALID_ARG
    assert "out is NULL" in hwr.hwr_ops_last_error(None)
    assert lib.hwr_ops_reserve(None, 1) == hwr.HWR_ERR_INVALID_ARG
    assert lib.hwr_group_rows(None, 0, None, None, 0, 1, None, None) == hwr.HWR_ERR_INVALID_ARG
    for fn, args in (("hwr_grouped_matmul", "hwr_matmul_args"), ("hwr_grouped_matmul_grad", "hwr_matmul_grad_args"),
                     ("hwr_adapter_matmul", "hwr_adapter_args"), ("hwr_adapter_matmul_grad", "hwr_adapter_grad_args")):
        assert getattr(lib, fn)(None, C.byref(g), C.byref(getattr(hwr, args)())) == hwr.HWR_ERR_INVALID_ARG
        assert "ops is NULL" in hwr.hwr_ops_last_error(None)
    hwr.hwr_ops_free(None)


def test_no_device_is_a_clean_error():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    with pytest.raises(hwr.HwrError) as e:
        routed.RoutedOps()
    assert e.value.status == hwr.HWR_ERR_HIP


@pytest.mark.parametrize("name", STRUCTS[1:])
def test_packed_arguments_are_the_structures(name):
    """What a call packs reads back, through the structures, as what it was given; what
    no field can hold is refused."""
    cls = getattr(hwr, name)
    call = routed._Call(hwr.load().hwr_grouped_matmul, cls)
    values = [(i + 3) << (40 if t is not C.c_int32 else 8) for i, (_, t) in enumerate(cls._fields_)]
    assert call(None, 5, 6, 7 << 40, 0, values) == hwr.HWR_ERR_INVALID_ARG     # (no context: nothing is read)
    g = hwr.hwr_groups.from_buffer(call._block)
    assert (g.n, g.n_groups, g.offsets, g.order) == (5, 6, 7 << 40, None)
    a = cls.from_buffer(call._block, C.sizeof(hwr.hwr_groups))
    assert [getattr(a, f) for f, _ in cls._fields_] == values
    for n, bad in ((2 ** 31, values), (-2 ** 31 - 1, values), (5, [2 ** 31] + values[1:])):
        with pytest.raises(hwr.HwrError) as e:
            call(None, n, 6, 1, 0, bad)
        assert e.value.status == hwr.HWR_ERR_INVALID_ARG


def test_an_empty_table_is_refused():
    """An empty tensor has no address, which the library reads as no table."""
    import torch

    class Library:
        def hwr_group_rows(self, *args):
            raise AssertionError(f"reached the library: {args}")

    ops = object.__new__(routed.RoutedOps)
    ops.ctx, ops._lib, ops.device, ops._i32 = None, Library(), -1, torch.int32
    i = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(hwr.HwrError) as e:
        ops.group(i(4), 2, table=i(0), offsets=i(3), order=i(4))
    assert e.value.status == hwr.HWR_ERR_INVALID_ARG and "table" in str(e.value)
    with pytest.raises(AssertionError, match="reached"):
        ops.group(i(4), 2, table=i(1), offsets=i(3), order=i(4))
