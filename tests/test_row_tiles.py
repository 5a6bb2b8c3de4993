"""Rows that one CTA takes tile by tile: a warp fetches its part of the next tile (behind the last one, of the next row's first) while others
read theirs of this one, so no warp's part of one tile may reach into another warp's of any other.  The arithmetic on the CPU, with the
kernels' own rules of splitting and dealing; results on the GPU where the last tile has fewer groups than the others."""
import os
import subprocess

import pytest

from paper_2608_18183_b200 import binding

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_18183_b200", "csrc")

SOURCE = r"""
#include <cstdio>
#include "row_parts.cuh"

template <int G, int WARPS>
int check(int V, int tiles, int slice) {
    if ((tiles - 1) * slice >= V) return 1;  // every tile has entries
    const int kinds[2] = {0, tiles - 1};     // all but the last are alike
    for (int i : kinds)
        for (int P = 0; P < G; ++P) {
            const int n = V - i * slice < slice ? V - i * slice : slice;
            int next = 0, entries = 0;
            for (int w = 0; w < WARPS; ++w) {
                const auto p = hbsjd::tile_part<G, WARPS>(P, V, slice, i, w);
                if (p.n != n || p.j0 != next || p.j1 < p.j0) return 2;
                next = p.j1;
                if (p.last() > p.first()) entries += p.last() - p.first();
            }
            if (next != (P + n + G - 1) / G || entries != n) return 3;
            if (next * G > slice + 16) return 4;  // the place that a CTA has
            // a row's first tile is staged as a slice of its own
            for (int w = 0; w < WARPS; ++w) {
                const hbsjd::Part<G, WARPS> whole(P, slice, w);
                const auto p = hbsjd::tile_part<G, WARPS>(P, V, slice, 0, w);
                if (whole.j0 != p.j0 || whole.j1 != p.j1) return 5;
            }
            for (int k : kinds)
                for (int Q = 0; Q < G; ++Q)
                    for (int a = 0; a < WARPS; ++a) {
                        const auto x = hbsjd::tile_part<G, WARPS>(P, V, slice, i, a);
                        for (int b = 0; b < WARPS; ++b) {
                            const auto y = hbsjd::tile_part<G, WARPS>(Q, V, slice, k, b);
                            if (a != b && (x.j0 > y.j0 ? x.j0 : y.j0) < (x.j1 < y.j1 ? x.j1 : y.j1)) return 6;
                        }
                    }
        }
    return 0;
}

template <int G>
int all(int bytes) {
    int tiled = 0;
    for (int V = 1; V <= 131072; V += V < 130000 ? 3 : 1) {
        const hbsjd::RowSplit s = hbsjd::split_row(1 << 20, V, bytes, 148, hbsjd::SHARED_SM, true);
        if (s.ctas == 1) continue;
        ++tiled;
        const int r4 = check<G, 4>(V, s.ctas, s.slice), r8 = check<G, 8>(V, s.ctas, s.slice);
        if (r4 || r8) {
            std::printf("%d entries of %d bytes in %d tiles of %d: %d, %d\n", V, bytes, s.ctas, s.slice, r4, r8);
            return 1;
        }
    }
    return tiled < 10000;
}

int main() { return all<4>(4) || all<8>(2); }
"""


def test_warps_keep_to_their_parts_from_tile_to_tile(tmp_path):
    source, program = tmp_path / "tiles.cpp", tmp_path / "tiles"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_tiles_are_dealt_by_that_rule_alone():
    text = open(os.path.join(CSRC, "token_kernels.cu")).read()
    body = text[text.index("tile < a.tiles"):]
    body = body[:body.index("next.more = false")]
    assert body.count("tile_part<G, WARPS>(") == 2 and "Part<G, WARPS> " not in body


LONG = [(65537, "fp32"), (49409, "fp32"), (32001, "fp32"), (128257, "fp32"), (65537, "bf16"), (49409, "bf16")]


@pytest.mark.gpu
@pytest.mark.parametrize("V,dtype", LONG)
def test_log_probabilities_of_rows_whose_last_tile_is_shorter(V, dtype):
    """More rows than SMs, every row against 64 bits, and the same bits each time."""
    import torch
    from tests.test_gpu_logits import _gen, _rows
    from tests.token_reference import HALF, Rows, near, sampled
    rows = 1000
    x = _rows(V, rows, V, 3.0, dtype, 0, 1)
    t = sampled(x, 1.0, _gen(V))
    t[::29] = -1
    t[1::31] = V - 1
    first = binding.hbsjd_token_logprobs(x, t)
    alone = binding.hbsjd_token_logprobs(x, t, want_entropy=False)[0]
    for at in range(0, rows, 100):
        s = slice(at, at + 100)
        r = Rows(x[s], t[s], 1.0)
        for logp in (first[0], alone):
            near(logp[s], torch.where(r.live, r.l, 0.0), torch.where(r.live, r.dl, 0.0), HALF["fp32"])
        near(first[1][s], torch.where(r.live, r.H, 0.0), r.dH, HALF["fp32"])
    for _ in range(10):
        again = binding.hbsjd_token_logprobs(x, t)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
        assert torch.equal(binding.hbsjd_token_logprobs(x, t, want_entropy=False)[0], alone)


@pytest.mark.gpu
@pytest.mark.parametrize("V,dtype", LONG)
def test_preference_loss_of_rows_whose_last_tile_is_shorter(V, dtype):
    import torch
    from tests.test_gpu_logits import _gen, _rows
    from tests.test_gpu_preference import _check
    from tests.token_reference import Rows, sampled
    lengths = [61, 100, 3, 49, 70, 40]
    rows = sum(lengths)
    x = _rows(V + 1, rows, V, 3.0, dtype, 0, 1)
    t = sampled(x, 1.0, _gen(V))
    ref = (Rows(x, t, 1.0).l + 0.3 * torch.randn(rows, generator=_gen(2), device="cuda")).float()
    _check(x, t, lengths, dtype, ref)
    offsets = torch.tensor([0] + lengths, device="cuda").cumsum(0).int()
    first = binding.hbsjd_preference_loss(x, t, offsets, ref)
    for _ in range(10):
        again = binding.hbsjd_preference_loss(x, t, offsets, ref)
        assert all(torch.equal(a, b) for a, b in zip(again, first))
