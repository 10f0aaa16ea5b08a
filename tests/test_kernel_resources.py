"""Registers of built kernels, from the metadata of the library's own code objects."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2509_23241_amd import build

READELF = shutil.which("llvm-readelf") or "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _kernels(tmp_path):
    """{mangled name: {field: value}} of all kernels in the library."""
    data = open(build.lib_path(), "rb").read()
    out, at = {}, data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + len(MAGIC))
        pos = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, pos)
            name = data[pos + 24: pos + 24 + length]
            pos += 24 + length
            if b"gfx950" in name and size:
                obj = tmp_path / "object"
                obj.write_bytes(data[at + offset: at + offset + size])
                notes = subprocess.run([READELF, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
                for part in re.split(r"\n  - \.a", notes)[1:]:
                    fields = dict(re.findall(r"\.(\w+): +(\S+)", part))
                    out[fields["symbol"].removesuffix(".kd")] = fields
        at = data.find(MAGIC, at + 1)
    return out


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_windowed_attention_dq_keeps_its_registers(tmp_path):
    """No scratch memory, and heads of up to 64 values in bf16 at three waves a SIMD (512 registers in units of 8)."""
    kernels = {k: v for k, v in _kernels(tmp_path).items() if "local_dq_kernel" in k}
    assert len(kernels) >= 14
    for name, k in kernels.items():
        assert int(k["vgpr_spill_count"]) == 0 and int(k["private_segment_fixed_size"]) == 0, (name, k)
        if "IfLi128" not in name:
            assert int(k["vgpr_count"]) <= (168 if "ItLi64" in name else 256), (name, k["vgpr_count"])


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_windowed_attention_dkv_workgroups_on_a_cu(tmp_path):
    """What the launch is cut up for: two workgroups of four waves on a CU, one of fp32 heads above 64 (512 registers a SIMD)."""
    kernels = {k: v for k, v in _kernels(tmp_path).items() if "local_dkv_kernel" in k}
    assert len(kernels) >= 14
    for name, k in kernels.items():
        assert 512 // int(k["vgpr_count"]) >= 2 or "IfLi128" in name, (name, k["vgpr_count"])
        assert 512 // int(k["vgpr_count"]) == 1 or "IfLi128" not in name, (name, k["vgpr_count"])
