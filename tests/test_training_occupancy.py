"""The rule that parts the backward's products counts the workgroups that a compute unit
holds of each kernel; here they are counted from the built kernels' registers (512 a
SIMD lane, in blocks of eight) and LDS (160 KB)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2607_20652_amd import binding as dpb
from test_kernel_resources import READELF, code_objects


@pytest.fixture(scope="module")
def held(tmp_path_factory):
    """{(kernel, "f32" or "bf16", width): workgroups of four waves on a compute unit}"""
    if not os.path.exists(READELF):
        pytest.skip(f"no {READELF}")
    dpb.load()
    out, tmp = {}, tmp_path_factory.mktemp("co")
    for i, co in enumerate(code_objects(dpb.lib_path)):
        p = tmp / f"{i}.co"
        p.write_bytes(co)
        notes = subprocess.run([READELF, "--notes", str(p)], capture_output=True, text=True, check=True).stdout
        for block in re.split(r"\n\s+- \.(?:agpr_count|args)", notes)[1:]:
            name = re.search(r"attention_(dq|dkv)_kernelI(DF16b|f)Li(\d+)E[\w]*\.kd", block)
            if name:
                field = lambda f: int(re.search(rf"\.{f}:\s+(\d+)", block).group(1))  # noqa: E731
                assert field("max_flat_workgroup_size") == 256      # a wave per SIMD
                waves = 512 // (-(-field("vgpr_count") // 8) * 8)
                out[name[1], "f32" if name[2] == "f" else "bf16", int(name[3])] = min(
                    waves, 163840 // field("group_segment_fixed_size"))
    assert len(out) == 16
    return out


def counted(bf16, width):
    """What the rule goes by: 256 tiles that are as many compute units' first workgroups, long enough for any
    number of parts, have that many parts.  (A function of the library's own, not of its C ABI.)"""
    fn = dpb.load()._ZN3dpb15attention_partsEiiiiiibbPiS0_
    fn.restype, fn.argtypes = None, [ctypes.c_int] * 6 + [ctypes.c_bool] * 2 + [ctypes.POINTER(ctypes.c_int)] * 2
    q, k, unused = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    fn(256, 128, 128 * 64, 1, 1, width, False, bf16, ctypes.byref(q), ctypes.byref(unused))
    fn(256, 128 * 64, 128, 1, 1, width, False, bf16, ctypes.byref(unused), ctypes.byref(k))
    return {"dq": q.value, "dkv": k.value}


@pytest.mark.parametrize("width", [32, 64, 96, 128])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_the_rule_counts_what_a_compute_unit_holds(held, kind, width):
    want = counted(kind == "bf16", width)
    for kernel in ("dq", "dkv"):
        has = held[kernel, kind, width]
        if (kernel, kind, width) == ("dq", "bf16", 32):
            assert has == 4 and want[kernel] == 3       # counted like width 64
        else:
            assert has == want[kernel], (kernel, has, want[kernel])
