"""Parts of a staged row that warps have to themselves: a warp stages its part of the next row, at any place behind a 16-byte boundary,
while others read theirs of this one.  The arithmetic of the kernels' header, compiled as plain C++; no GPU is needed."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_18183_b200", "csrc")

SOURCE = r"""
#include <cstdio>
#include <initializer_list>
#include "row_parts.cuh"
using hbsjd::Part;

template <int G, int WARPS>
int check(int n) {
    int at = 0;
    for (int P = 0; P < hbsjd::PHASES; ++P) {
        // one after another, all groups, all entries; those in whole are the row's
        int next = 0, entries = 0;
        for (int w = 0; w < WARPS; ++w) {
            const Part<G, WARPS> p(P, n, w);
            if (p.j0 != next || p.j1 < p.j0 || (p.j1 > p.j0 && p.j0 % 2)) return 1;
            next = p.j1;
            if (p.last() > p.first()) entries += p.last() - p.first();
            if (p.inner() < p.j0 || p.outer() > p.j1 || (p.outer() > p.inner() && (p.inner() * G < P || p.outer() * G > P + n))) return 2;
            if (p.last() - p.first() - (p.outer() - p.inner()) * G >= 2 * G) return 3;
        }
        if (next != (P + n + G - 1) / G || entries != n) return 4;
        // what a warp writes of a row at Q is none of what another reads of the one at P
        for (int Q = 0; Q < hbsjd::PHASES; ++Q)
            for (int a = 0; a < WARPS; ++a)
                for (int b = 0; b < WARPS; ++b) {
                    const Part<G, WARPS> x(Q, n, a), y(P, n, b);
                    const int lo = x.j0 > y.j0 ? x.j0 : y.j0, hi = x.j1 < y.j1 ? x.j1 : y.j1;
                    if (a != b && lo < hi) return 5;
                }
        at = next;
    }
    return at < 0;
}

template <int G>
int all(int n) {
    int r = check<G, 1>(n);
    r = r ? r : check<G, 2>(n);
    r = r ? r : check<G, 4>(n);
    r = r ? r : check<G, 8>(n);
    return r ? r : check<G, 16>(n);
}

int main() {
    for (int n = 1; n <= 20000; n += n < 1300 ? 1 : 37) {
        const int r = all<4>(n) ? all<4>(n) : all<8>(n);
        if (r) {
            std::printf("%d entries: %d\n", n, r);
            return 1;
        }
    }
    for (int n : {6450, 6464, 9467, 9472, 16384})
        if (all<4>(n) || all<8>(n)) {
            std::printf("%d entries\n", n);
            return 1;
        }
    return 0;
}
"""


def test_parts_of_rows_at_any_place(tmp_path):
    source, program = tmp_path / "parts.cpp", tmp_path / "parts"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_the_kernels_deal_rows_by_that_header():
    text = open(os.path.join(CSRC, "logit_rows.cuh")).read()
    assert '#include "row_parts.cuh"' in text and "struct Part" not in text


@pytest.mark.gpu
@pytest.mark.parametrize("ds,dt,V", [("bf16", "bf16", 18939), ("bf16", "fp32", 12914), ("fp32", "bf16", 12911), ("fp32", "fp32", 8189), ("bf16", "bf16", 2041),
                                     ("fp32", "fp32", 1023)])
def test_rows_whose_places_change_the_number_of_groups(ds, dt, V):
    """Many rows a CTA at an odd stride, where the groups of one place end at a multiple of what the warps take and those of another
    do not: every entry of every gradient."""
    import torch
    from paper_2608_18183_b200 import binding
    from tests.test_gpu_logits import _compare, _distill_ref, _distill_topk_ref, _rows
    rows, k = 3000000 // V + 900, 40
    s, t = _rows(1, rows, V, 3.0, ds, 1 - V % 2, 1), _rows(2, rows, V, 2.0, dt, 1 - V % 2 + 2, 3)
    w = torch.ones(rows, device="cuda")
    lists = binding.hbsjd_topk_logits(t, k)
    for _ in range(3):
        full = binding.hbsjd_distill(s, t, w)
        listed = binding.hbsjd_distill_topk(s, *lists, w, 1.0, 0.5, 0.5)
        for r in range(0, rows, 300):
            at = slice(r, r + 300)
            _compare(full[0][at], full[1][at], _distill_ref(s[at], t[at], w[at], 1.0, 0.5, 0.5), ds)
            _compare(listed[0][at], listed[1][at], _distill_topk_ref(s[at], *(x[at] for x in lists), w[at], 1.0, 0.5, 0.5), ds)
