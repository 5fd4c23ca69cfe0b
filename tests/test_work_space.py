"""The context's work space (work_space.h, plain C++) on a host that records what it is asked for."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HEAD = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "work_space.h"
using namespace malib;
struct Host {
    std::set<void*> live;
    std::vector<void*> kept;
    std::vector<int64_t> sizes;
    int fail_allocate = 0, fail_keep = 0, fail_clear = 0, captured = 0, cleared = 0;
    int may_grow() { return captured ? -4 : 0; }
    int allocate(void** p, int64_t bytes) {
        if (fail_allocate) return fail_allocate;
        *p = std::malloc(16);
        live.insert(*p);
        sizes.push_back(bytes);
        return 0;
    }
    int clear(void* p, int64_t bytes) {
        if (fail_clear) return fail_clear;
        cleared += live.count(p) && bytes == 1000;
        return 0;
    }
    int keep(void* p) {
        if (fail_keep) return fail_keep;
        kept.push_back(p);
        return 0;
    }
    void release(void* p) { live.erase(p); std::free(p); }
};
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
"""


def run(tmp_path, body):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(HEAD + "int main() {\n" + body + "\nreturn 0; }\n")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2106_07551_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_outgrown_blocks_are_kept(tmp_path):
    """A block's address stays good when a larger call replaces it; nothing is freed."""
    run(tmp_path, r"""
    Host h;
    double* p = nullptr;
    int64_t cap = 0;
    std::vector<double*> seen;
    for (int64_t need : {5, 60, 65, 64, 1000, 100000, 3}) {
        CHECK(grow(h, p, cap, need) == 0 && cap >= need);
        if (seen.empty() || seen.back() != p) seen.push_back(p);
        for (double* q : seen) CHECK(h.live.count(q));
    }
    CHECK(seen.size() == 4 && h.kept.size() == 3);
    for (int i = 0; i < 3; ++i) CHECK(h.kept[i] == seen[i]);
    int64_t before = 0;
    for (size_t i = 0; i + 1 < h.sizes.size(); ++i) before += h.sizes[i];
    CHECK(before < h.sizes.back() && h.sizes.back() == cap * 8);
    """)


def test_a_failure_leaves_the_block(tmp_path):
    run(tmp_path, r"""
    Host h;
    int* p = nullptr;
    int64_t cap = 0;
    h.fail_allocate = -2;
    CHECK(grow(h, p, cap, 10) == -2 && !p && cap == 0);
    h.fail_allocate = 0;
    CHECK(grow(h, p, cap, 10) == 0);
    int* const q = p;
    const int64_t had = cap;
    h.fail_allocate = -2;
    CHECK(grow(h, p, cap, 1000) == -2 && p == q && cap == had);
    h.fail_allocate = 0;
    h.fail_keep = -2;
    CHECK(grow(h, p, cap, 1000) == -2 && p == q && cap == had && h.live.size() == 1);
    h.fail_keep = 0;
    CHECK(grow(h, p, cap, 1000) == 0 && p != q && h.live.count(q));
    """)


def test_nothing_grows_during_a_capture(tmp_path):
    """A block taken during a capture would belong to the graph."""
    run(tmp_path, r"""
    Host h;
    int* p = nullptr;
    int64_t cap = 0;
    h.captured = 1;
    CHECK(grow(h, p, cap, 10) == -4 && !p && cap == 0 && h.sizes.empty());
    h.captured = 0;
    CHECK(grow(h, p, cap, 100) == 0);
    int* const q = p;
    const int64_t had = cap;
    h.captured = 1;
    CHECK(grow(h, p, cap, had) == 0 && p == q);
    CHECK(grow(h, p, cap, had + 1) == -4 && p == q && cap == had && h.sizes.size() == 1 && h.kept.empty());
    """)


def test_a_block_that_was_not_cleared_is_not_used(tmp_path):
    """The counters of a context start as zeros, also after a first call that could not write them."""
    run(tmp_path, r"""
    Host h;
    char* p = nullptr;
    h.captured = 1;
    CHECK(take_cleared(h, p, 1000) == -4 && !p);
    h.captured = 0;
    h.fail_clear = -3;
    CHECK(take_cleared(h, p, 1000) == -3 && !p && h.live.empty());
    h.fail_clear = 0;
    CHECK(take_cleared(h, p, 1000) == 0 && p && h.cleared == 1 && h.live.size() == 1);
    char* const q = p;
    CHECK(take_cleared(h, p, 1000) == 0 && p == q && h.cleared == 1);
    """)
