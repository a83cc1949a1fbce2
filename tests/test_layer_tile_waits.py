"""The tiled products wait for their own loads into LDS before the epilogue
reuses the buffers.  Checked in the intermediate code of each shape of tile,
where only the waits that the source asks for exist: those that the compiler adds
come later and are its own choice."""
import re
import subprocess

import pytest

from paper_2403_16125_amd import build

SHAPES = {"256": "256, 256, 2, 4, 2", "128": "128, 128, 2, 2, 2", "128 deep": "128, 128, 2, 2, 4", "64": "64, 64, 2, 2, 4"}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{shape: body of its kernel}"""
    at = tmp_path_factory.mktemp("tiles")
    src = '#include "arena_gemm.h"\nnamespace arena {\nnamespace mm {\n'
    for shape in SHAPES.values():
        src += f"template __global__ void gemm_kernel<Tile<Bf16, {shape}, false, false, kPlain>>(const GemmArgs);\n"
    (at / "tiles.hip").write_text(src + "}\n}\n")
    flags = [f for f in build.FLAGS if f != "-shared"]
    subprocess.run([build.HIPCC, *flags, "--offload-device-only", "-emit-llvm", "-S", "-o", str(at / "tiles.ll"),
                    str(at / "tiles.hip")], check=True, capture_output=True)
    text = (at / "tiles.ll").read_text()
    out = {}
    for m in re.finditer(r"^define [^\n]*amdgpu_kernel void @(\w+)\(.*?^\}", text, flags=re.S | re.M):
        for name, shape in SHAPES.items():
            if "".join(f"Li{v}E" for v in shape.split(", ")) in m[1]:
                out[name] = m[0]
    return out


def vector_loads(immediate):
    """How many loads a wait leaves in flight."""
    return (immediate & 15) | (immediate >> 14 & 3) << 4


@pytest.mark.parametrize("shape", SHAPES)
def test_loads_have_landed_before_the_epilogue(kernels, shape):
    events = re.findall(r"@llvm\.amdgcn\.(global\.load\.lds|s\.barrier|s\.waitcnt)[\w.]*\(([^\n]*)\)", kernels[shape])
    kinds = [k for k, _ in events]
    assert kinds.count("global.load.lds") > 8 and kinds.count("s.barrier") >= 3
    # the last barrier is the epilogue's; no load starts between the wait and it
    before = len(kinds) - 1 - kinds[::-1].index("s.barrier") - 1
    assert kinds[before] == "s.waitcnt", f"{kinds[before]} before the epilogue's barrier"
    assert vector_loads(int(re.search(r"i32 (\d+)", events[before][1])[1])) == 0
    assert "global.load.lds" not in kinds[before:]
