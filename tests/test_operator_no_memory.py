"""A refusal where the host has no memory left is still a status: no exception may leave a C entry point.  A small program replaces the
allocation functions of the process by ones that fail once they are told to."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "tad.h"
static bool none = false;
void *operator new(std::size_t n) { if (none) throw std::bad_alloc(); return std::malloc(n ? n : 1); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
int main()
{
    char buf[256];
    tad_rows good{buf, 16, TAD_F32, 0}, bad{buf, 3, TAD_F32, 0}, odd{buf + 1, 16, TAD_F32, 0}, far{buf, int64_t(1) << 40, TAD_F32, 0};
    tad_packed q{reinterpret_cast<uint8_t *>(buf) + 1, reinterpret_cast<uint8_t *>(buf), 16, 4}, p{reinterpret_cast<uint8_t *>(16), reinterpret_cast<uint8_t *>(16), 1 << 24, 1 << 20};
    float f[4];
    for (int turn = 0; turn < 2; ++turn) {
        none = turn == 1;
        const int s[] = {
            tad_pack8(nullptr, 3, 4, &p, nullptr), tad_pack8(&bad, 3, 4, &p, nullptr), tad_pack8(&odd, 3, 4, &p, nullptr), tad_pack8(&good, 3, 4, &q, nullptr),
            tad_pack8(&good, -3, 4, &p, nullptr), tad_pack8(&far, int64_t(1) << 31, 4, &p, nullptr), tad_pack8(&far, (int64_t(1) << 31) - 1, (1 << 24) - 1, &p, nullptr),
            tad_unpack8(&q, 3, 4, &good, nullptr), tad_repack8(&q, 3, 4, &p, nullptr),
            tad_layernorm_forward(&good, 3, 4, nullptr, nullptr, -1.f, &good, f, f, nullptr, nullptr),
            tad_layernorm_backward(&good, nullptr, nullptr, 3, 4, nullptr, f, f, &good, nullptr, nullptr, nullptr, 0, nullptr),
            tad_layernorm_backward(&good, &good, nullptr, 3, 4, nullptr, f, f, &good, &good, nullptr, nullptr, 0, nullptr),
            tad_embed_forward(buf, 16, 3, &good, 3, 4, 1.f, &good, nullptr), tad_embed_backward(buf, 32, 3, &good, 3, 4, 1.f, &good, 0, nullptr, 0, nullptr),
            tad_matmul8(&p, &p, 3, int64_t(1) << 31, 4, &good, nullptr, 0, nullptr), tad_matmul8(nullptr, &p, 3, 3, 4, &good, nullptr, 0, nullptr)};
        none = false;
        for (int v : s) std::printf("%d ", v);
        std::printf("\n");
    }
    std::printf("%s\n", tad_pack8(nullptr, 3, 4, &p, nullptr) == TAD_ERR_INVALID_ARG && tad_last_error()[0] ? "text" : "no text");
    return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="needs a compiler")
def test_refusals_without_memory(tmp_path):
    (tmp_path / "a.cpp").write_text(SOURCE)
    lib = os.path.join(ROOT, "paper_1711_01348_b200")
    subprocess.check_call(["g++", "-std=c++17", "-rdynamic", "-I", os.path.join(ROOT, "include"), str(tmp_path / "a.cpp"), "-o", str(tmp_path / "a"), os.path.join(lib, "libtad.so"),
                           "-Wl,-rpath," + lib, "-L/usr/local/cuda/lib64", "-Wl,-rpath,/usr/local/cuda/lib64"])
    r = subprocess.run([str(tmp_path / "a")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    with_memory, without, text = r.stdout.splitlines()
    assert with_memory == without and "0" not in with_memory.split() and text == "text"
