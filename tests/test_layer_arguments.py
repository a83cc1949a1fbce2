"""What the dense products' kernels are handed holds their own fields only: more of them
come before the first load of a short product."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_dense_products_arguments_stay_small(tmp_path):
    """264 bytes of own fields; with those of the groups and of a loss among them, 352, a
    product of 512 x 512 took 4 % longer."""
    src, exe = tmp_path / "size.cpp", str(tmp_path / "size")
    src.write_text('#include <cstdio>\n#include "arena_layer_internal.h"\n'
                   'int main() { printf("%zu", sizeof(arena::mm::GemmArgs)); }\n')
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2403_16125_amd", "csrc"), "-I",
                    os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"), str(src), "-o", exe], check=True)
    assert int(subprocess.run([exe], capture_output=True, text=True, check=True).stdout) <= 264
