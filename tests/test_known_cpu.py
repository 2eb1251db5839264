"""csrc/known.h, which keeps what the library asks the runtime once: a query that
fails is reported and asked again, an answer (zero too) is kept."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "known.h"

struct Key {
    int a, b;
    bool operator==(const Key &o) const { return a == o.a && b == o.b; }
};

int main() {
    isam::Known<Key, 2> known;
    int asked = 0, status = 3, answer = 7;
    const auto get = [&](int a, int b, int *n) {
        return known.get(Key{a, b}, n, [&](int *v) {
            ++asked;
            if (status == 0) *v = answer;
            return status;
        });
    };
    int n = -1;
    if (get(1, 1, &n) != 3 || asked != 1) return 1;               // the failure reaches the caller
    status = 0;
    if (get(1, 1, &n) != 0 || asked != 2 || n != 7) return 2;     // and is not kept
    status = 3, answer = 9, n = -1;
    if (get(1, 1, &n) != 0 || asked != 2 || n != 7) return 3;     // the answer is
    status = 0, answer = 0;
    if (get(1, 2, &n) != 0 || asked != 3 || n != 0) return 4;     // another key; none is an answer
    answer = 5;
    if (get(1, 2, &n) != 0 || asked != 3 || n != 0) return 5;
    for (int i = 0; i < 2; ++i)                                   // no room: asked each time
        if (get(2, 2, &n) != 0 || asked != 4 + i || n != 5) return 6;
    return 0;
}
"""


def test_failed_queries_are_not_kept(tmp_path):
    src, exe = tmp_path / "known.cpp", tmp_path / "known"
    src.write_text(PROGRAM)
    cc = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I",
                         os.path.join(ROOT, "paper_1810_09958_gb300", "csrc"), str(src), "-o", str(exe), "-lpthread"],
                        capture_output=True, text=True, timeout=120)
    assert cc.returncode == 0, cc.stderr
    assert subprocess.run([str(exe)], timeout=30).returncode == 0
