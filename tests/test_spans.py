"""Which buffers of a call may lie over which (spans.h, plain C++)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BODY = r"""
#include <cstdio>
#include "spans.h"
using namespace malib;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
    alignas(16) static char m[1000];
    // side by side, one inside another, one byte in common, none at all
    CHECK(apart(Span(m, 10), Span(m + 10, 5)) && apart(Span(m + 10, 5), Span(m, 10)));
    CHECK(!apart(Span(m, 100), Span(m + 10, 5)) && !apart(Span(m + 10, 5), Span(m, 100)));
    CHECK(!apart(Span(m, 11), Span(m + 10, 5)) && !apart(Span(m, 10), Span(m, 10)));
    CHECK(apart(Span(nullptr, 10), Span(nullptr, 10)) && apart(Span(m, 0), Span(m, 10)) && apart(Span(m, 10), Span(m + 5, 0)));
    // an output over another one, or over the second input
    const Span in[] = {{m, 100}, {m + 300, 50}};
    { const Span out[] = {{m + 100, 20}, {nullptr, 20}, {m + 120, 20}}; CHECK(all_apart(out, in)); }
    { const Span out[] = {{m + 100, 20}, {nullptr, 20}, {m + 119, 20}}; CHECK(!all_apart(out, in)); }
    { const Span out[] = {{m + 100, 20}, {m + 349, 1}}; CHECK(!all_apart(out, in)); }
    { const Span out[] = {{m + 99, 20}}; CHECK(!all_apart(out, in)); }
    // rows: the last one ends with its entries, not with its stride; one row that all share; the largest calls
    CHECK(row_bytes(3, 10, 7, 2) == 54 && row_bytes(5, 0, 7, 4) == 28 && row_bytes(1, 7, 7, 4) == 28 && row_bytes(0, 7, 7, 4) == 0);
    const int64_t n = 1ll << 40, ld = INT64_MAX / 4 / n;
    CHECK(row_bytes(n, ld, 1 << 24, 4) > (1ull << 62) && row_bytes(n, ld, 1 << 24, 4) < (1ull << 63) + (1ull << 27));
    CHECK(!apart(Span(m, row_bytes(n, ld, 1 << 24, 4)), Span(m + 500, 1)));
    return 0;
}
"""


def test_spans(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(BODY)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2106_07551_gb300", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
