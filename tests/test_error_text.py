"""Error texts of the C ABI take no memory: an entry point that refuses its
arguments when none is left still returns a status, where an exception would pass
through a C caller."""
import os
import subprocess

import pytest

from paper_2403_16125_amd import arena

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include "arena.h"
#include "arena_layer.h"
static bool none_left = false;
void* operator new(size_t n)
{
    if (none_left) throw std::bad_alloc();
    if (void* p = malloc(n ? n : 1)) return p;
    throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }
int main()
{
    arena_ctx* c = nullptr;
    if (arena_create(0, &c) != ARENA_OK) return 2;
    none_left = true;
    int bad = 0;
    try {
        int64_t n = 0;
        arena_ffn_desc f;
        memset(&f, 0, sizeof(f));
        f.dtype = 77;
        bad |= arena_norm_forward(c, nullptr, nullptr) != ARENA_ERR_INVALID_ARG || !*arena_last_error(c);
        bad |= arena_ffn_forward_workspace(c, &f, &n) != ARENA_ERR_INVALID_ARG || !strstr(arena_last_error(c), "77");
        bad |= arena_orthogonal_update(c, nullptr, nullptr) != ARENA_ERR_INVALID_ARG;
        bad |= arena_bind_jobs(c, nullptr) != ARENA_ERR_INVALID_ARG || !*arena_last_error(c);
    } catch (...) {
        return 3;
    }
    none_left = false;
    arena_destroy(c);
    return bad;
}
"""


def test_refusals_without_memory(tmp_path):
    arena.load()
    (tmp_path / "t.cpp").write_text(PROGRAM)
    lib = arena.library_path()
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.cpp"), lib, "-o",
                    str(tmp_path / "t"), f"-Wl,-rpath,{os.path.dirname(lib)}", "-Wl,--allow-shlib-undefined"], check=True)
    done = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr)
