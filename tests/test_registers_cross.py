"""Registers and private memory of the cross attention's and the rotary kernels
(and the float32 attention's, which shares their loop), read from the library
built here (CPU only): what their launch bounds rely on, and that nothing in a key
loop lives in memory."""
import os
import re
import struct
import subprocess

import pytest

from test_registers import MAGIC, READELF, ROOT


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Kernel name (mangled) -> its metadata's numbers."""
    if READELF is None:
        pytest.skip("no llvm-readelf")
    from paper_2607_15650_amd import _lib
    _lib.lib()                                            # raises if it is not built
    data = open(os.path.join(ROOT, "paper_2607_15650_amd", "libditango.so"), "rb").read()
    out, at, d = {}, data.find(MAGIC), tmp_path_factory.mktemp("co")
    while at >= 0:
        n, pos = struct.unpack_from("<Q", data, at + len(MAGIC))[0], at + len(MAGIC) + 8
        for _ in range(n):
            off, size, ln = struct.unpack_from("<QQQ", data, pos)
            triple = data[pos + 24:pos + 24 + ln].decode()
            pos += 24 + ln
            if "gfx950" in triple and size:
                f = d / f"{at}.elf"
                f.write_bytes(data[at + off:at + off + size])
                text = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
                for block in re.split(r"- \.agpr_count:", text)[1:]:
                    name = re.search(r"\.name:\s+(\S+)", block).group(1)
                    out[name] = {k: int(x) for k, x in re.findall(r"\.(\w+):\s+(\d+)\n", block)}
        at = data.find(MAGIC, at + 1)
    if not out:
        pytest.skip("the library's code objects are not in a plain bundle")
    return out


# name of the kernel, instances, most vector registers (512 / the waves of a SIMD)
@pytest.mark.parametrize("name,count,most", [
    (r"cross_kernelI", 4, 256),                           # two workgroups of a wave per SIMD
    (r"cross_few_kernelI", 4, 256),
    (r"cross_resident_kernelI.*Li128ELi12E", 3, 168),     # three waves
    (r"cross_resident_kernelI.*Li64ELi16E", 3, 128),      # four
    (r"cross_task_kernelI", 2, 512),                      # one
    (r"cross_join_kernelI", 4, 128),
    (r"cross_(list|pack)_kernel", 2, 64),
    (r"rotary_kernelI", 72, 128),
])
def test_registers(kernels, name, count, most):
    found = {n: k for n, k in kernels.items() if re.search(name, n)}
    assert len(found) == count, sorted(found)
    for n, k in found.items():
        assert k["vgpr_count"] <= most, (n, k["vgpr_count"])
        assert k["private_segment_fixed_size"] == 0 and k["vgpr_spill_count"] == 0, n


def test_float32_forms(kernels):
    """The 256-row form over listed keys keeps a few words in memory from its start
    to its end; none of the others does."""
    found = {n: k for n, k in kernels.items() if re.search(r"(cross|attn)_f32_kernelI", n)}
    assert len(found) == 15
    for n, k in found.items():
        listed = "Li128ELi8ELi1E" in n and "ListedRows" in n
        assert k["private_segment_fixed_size"] <= (32 if listed else 0), (n, k["private_segment_fixed_size"])
