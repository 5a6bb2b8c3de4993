"""hbsjd_clip_gradients against its definition in 64 bits.

The norm is a sum of up to 64 products a thread in fp32 (off by at most 64 half steps, 32 of the root), joined in 64 bits.  The factor is
rounded once, and each product once."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _gen

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _make(sizes, kinds, seed=1, scale=1.0, align=1, shift=0):
    """Views of one buffer a type; `align` and `shift` in elements."""
    import torch
    T = {"fp32": torch.float32, "bf16": torch.bfloat16}
    out, at = [], {"fp32": shift, "bf16": shift}
    room = {k: torch.full((shift + sum(n + align for n in sizes) + 16,), 77.0, device="cuda", dtype=T[k]) for k in T}
    for i, n in enumerate(sizes):
        k = kinds[i % len(kinds)]
        v = room[k][at[k]:at[k] + n]
        v.copy_(torch.randn(n, generator=_gen(seed + i), device="cuda") * scale)
        out.append(v)
        at[k] += -(-n // align) * align
    return out, room


def _norm(gradients, kind):
    import torch
    flat = torch.cat([g.double().reshape(-1) for g in gradients])
    if not flat.numel():
        return 0.0
    return float(flat.norm() if kind == "2" else flat.abs().max())


def _check(gradients, limit, kind="2", outs=None):
    import torch
    norm = _norm(gradients, kind)
    before = [g.double() for g in gradients]
    got = binding.hbsjd_clip_gradients(gradients, limit, kind, outs)
    if norm > 3.4028236e38:  # (beyond fp32, which the norm is given in: it is infinite, and nothing is scaled)
        assert got.shape == () and float(got) == float("inf")
        f = 1.0
    else:
        assert got.shape == () and abs(float(got) - norm) <= 34 * STEP * norm
        f = min(1.0, limit / (norm + 1e-6))
    for x, b, y in zip(gradients, before, gradients if outs is None else outs):
        half = 2.0 ** -8 if x.dtype == torch.bfloat16 else STEP
        off = (y.double() - b * f).abs() - (35 * STEP + half) * (b * f).abs() - 1.5e-45 * (x.dtype == torch.float32) - 1e-40 * (x.dtype == torch.bfloat16)
        assert off.numel() == 0 or float(off.max()) <= 0
        if f == 1.0 or outs is not None:
            assert torch.equal(x.double(), b)
        if f == 1.0:
            assert torch.equal(y, x)
    return got


SIZES = [[1], [0, 1], [7, 1, 3, 0, 64, 1000], [32768, 16384, 16383, 32769, 5], [1000003, 17, 65536 * 3 + 1]]


@pytest.mark.parametrize("kinds", [["fp32"], ["bf16"], ["fp32", "bf16"]])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("align,shift", [(1, 0), (1, 3), (64, 0)])
def test_norms_and_scaling(sizes, kinds, align, shift):
    import torch
    for kind in ("2", "max"):
        for part in (0.3, 2.0):
            g, room = _make(sizes, kinds, 1, 1.0, align, shift)
            norm = _norm(g, kind)
            _check(g, norm * part, kind)
            g, room = _make(sizes, kinds, 1, 1.0, align, shift)
            o, oroom = _make(sizes, kinds, 50, 1.0, align, shift + 1)   # another place behind 16 bytes
            _check(g, norm * part, kind, o)
            o, oroom = _make(sizes, kinds, 50, 1.0, align, shift)
            kept = {k: v.clone() for k, v in oroom.items()}
            _check(g, norm * part, kind, o)
            for y in o:                                                  # nothing else is written
                y.fill_(0)
            for k, v in oroom.items():
                inside = v != kept[k]
                assert int(inside.sum()) <= sum(y.numel() for y in o)
                assert bool((v[kept[k] == 77.0] == 77.0).all())


@pytest.mark.parametrize("count", [127, 128, 129, 1024, 1025, 2500])
def test_many_arrays(count):
    sizes = [(i * 37) % 211 for i in range(count)]
    g, _ = _make(sizes, ["fp32", "bf16", "fp32"], 3)
    _check(g, 0.4 * _norm(g, "2"))
    g, _ = _make(sizes, ["fp32"], 3)
    _check(g, 0.4 * _norm(g, "max"), "max")


def test_a_model_s_gradients():
    import torch
    g = [torch.randn(s, generator=_gen(i), device="cuda") * 10.0 ** (i % 5 - 3) for i, s in enumerate(
        [(5000, 333), (999, 333), (333,), (333, 333), (2001, 333), (333, 1000)] * 4)]
    _check(g, 1.0)
    _check([x.bfloat16() for x in g], 1e9)


def test_dense_in_any_order_and_what_is_not():
    import torch
    a = torch.randn(40, 60, generator=_gen(1), device="cuda")
    b = torch.randn(4, 5, 6, generator=_gen(2), device="cuda").permute(2, 0, 1)
    norm = _norm([a, b], "2")
    want = [x * (0.5 * norm / (norm + 1e-6)) for x in (a, b)]
    binding.hbsjd_clip_gradients([a.t(), b], 0.5 * norm)
    torch.testing.assert_close(a, want[0], rtol=1e-5, atol=0)
    torch.testing.assert_close(b, want[1], rtol=1e-5, atol=0)
    for bad in ([a[:, ::2]], [a.expand(2, 40, 60)], [a, a], [a, a[3]], [a[:10], a[9:]], [a.half()], [a.cpu()], [a, b.cpu()], [], [None], [a, 3],
                [a.long()]):
        with pytest.raises(binding.HbsjdError) as e:
            binding.hbsjd_clip_gradients(bad, 1.0)
        assert e.value.code == -1
    for out in ([torch.empty_like(a)], [torch.empty(60, 40, device="cuda"), b], [a, torch.empty_like(b)], [torch.empty_like(a).bfloat16(), torch.empty_like(b)],
                [a[1:], torch.empty_like(b)], [torch.empty(60, 40, device="cuda").t(), torch.empty_like(b)]):
        with pytest.raises(binding.HbsjdError):
            binding.hbsjd_clip_gradients([a, b], 1.0, out=out)
    for limit in (-1.0, float("nan")):
        with pytest.raises(binding.HbsjdError):
            binding.hbsjd_clip_gradients([a], limit)
    with pytest.raises(binding.HbsjdError):
        binding.hbsjd_clip_gradients([a], 1.0, norm="1")


@pytest.mark.parametrize("kinds", [["fp32"], ["bf16"]])
def test_gradients_near_the_type_s_ends(kinds):
    """Squares that overflow or vanish in 32 bits do not in the sum."""
    for scale in (1e37, 1e20, 1e-20, 1e-30, 1e-37):
        g, _ = _make([100, 70000, 3], kinds, 5, scale)
        _check(g, float("inf"))
        _check(g, float("inf"), "max")
        if scale > 1:
            _check(g, scale)
    # one large among small ones, and zeros
    g, _ = _make([70000, 50000], kinds, 5, 1e-25)
    g[1].zero_()
    _check(g, float("inf"))
    g[1][777] = 1e19
    _check(g, float("inf"))
    g[0].zero_()
    g[1].zero_()
    _check(g, 1.0)
    _check(g, 0.0)


def test_limits_of_zero_and_without_end():
    import torch
    g, _ = _make([1000, 33], ["fp32"], 7)
    kept = [x.clone() for x in g]
    _check(g, float("inf"))
    assert all(torch.equal(a, b) for a, b in zip(g, kept))
    _check(g, 0.0)
    assert not any(bool(x.any()) for x in g)


@pytest.mark.parametrize("kind", ["2", "max"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_norm_that_is_no_number_scales_nothing(kind, value):
    import math
    import torch
    for dtype in ("fp32", "bf16"):
        g, _ = _make([50000, 33, 40], [dtype], 7)
        g[1][5] = value
        kept = [x.clone() for x in g]
        got = float(binding.hbsjd_clip_gradients(g, 0.5, kind))
        assert math.isnan(got) if math.isnan(value) else got == math.inf
        out = [torch.zeros_like(x) for x in g]
        binding.hbsjd_clip_gradients(g, 0.5, kind, out)
        for a, b, c in zip(g, kept, out):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(c.view(torch.uint8), b.view(torch.uint8))


def test_streams_graphs_and_autograd():
    import torch
    g, _ = _make([70000, 100, 5000], ["fp32", "bf16"], 9)
    kept = [x.clone() for x in g]
    want = binding.hbsjd_clip_gradients(g, 1.0)
    done = [x.clone() for x in g]
    restore = lambda: [x.copy_(y) for x, y in zip(g, kept)]
    restore()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.hbsjd_clip_gradients(g, 1.0, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(g, done))
    restore()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.hbsjd_clip_gradients(g, 1.0)
    for _ in range(3):
        restore()
        graph.replay()
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(g, done))
    before = [x._version for x in g]
    binding.hbsjd_clip_gradients(g)
    assert [x._version for x in g] == before
    binding.hbsjd_clip_gradients(g, 1.0)
    assert all(x._version > b for x, b in zip(g, before))


def test_an_array_beyond_32_bits():
    import torch
    n = 2 ** 31 + 12345
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[-1], x[0], x[2 ** 31 + 1] = 3.0, 4.0, 12.0
    y = torch.full((77,), 0.0, device="cuda")
    norm = binding.hbsjd_clip_gradients([y, x], 1.3)
    assert float(norm) == 13.0
    assert [float(x[i]) for i in (-1, 0, 2 ** 31 + 1)] == [float(torch.tensor(v * 0.1 / (1 + 1e-6 / 13)).bfloat16()) for v in (3.0, 4.0, 12.0)]
    assert int(torch.count_nonzero(x)) == 3
