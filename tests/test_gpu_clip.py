"""GPU parity of the gradient norm and clipping through the C ABI, against the
fp64 oracle.

Tolerances: squares of fp32 are summed in fp32 over a few dozen elements and
in more bits beyond: 64 roundings of 2^-24 bound the norm's relative error by 2e-6
(half of it, in fact: the root).  A clipped element is one product with a
coefficient rounded to fp32: three roundings on top of the norm's error; one
more of 2^-9 for bf16.  A product below the normal range of either type has its
spacing there, 2^-149 for fp32 and 2^-133 for bf16."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2606_19528_gb300 import lora
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

NAN = float("nan")


def run(pairs, max_norm, coef=True):
    arr = lora.make_grads(pairs)
    norm, cf = torch.full((3,), NAN, device="cuda"), torch.full((3,), NAN, device="cuda")
    n = lora.lora_clip_workspace_size(arr)
    ws = torch.full((n + 256,), 0x7f, dtype=torch.uint8, device="cuda")
    lora.lora_clip_grads(arr, max_norm, norm[1:], cf[1:] if coef else None, ws, n)
    torch.cuda.synchronize()
    assert (ws[n:] == 0x7f).all()
    assert torch.isnan(norm[0]) and torch.isnan(norm[2]) and torch.isnan(cf[0]) and torch.isnan(cf[2])
    return float(norm[1]), float(cf[1])


def tensors(seed, sizes, dtypes=(torch.float32,), std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(std * torch.randn(n, generator=g, device="cuda")).to(dtypes[i % len(dtypes)])
            for i, n in enumerate(sizes)]


def check(grads, outs, max_norm, in_place=False):
    """outs: same-shaped destinations; in_place: they are the grads."""
    src = [G.host_f64(g) for g in grads]
    want_norm, want_coef, want = oracle.clip_grads(src, max_norm)
    norm, coef = run(list(zip(grads, outs)), max_norm)
    assert norm == pytest.approx(want_norm, rel=2e-6)
    assert coef == pytest.approx(want_coef, rel=2e-6)
    for g, o, w in zip(grads, outs, want):
        if o is not None:
            tol, step = (3e-6, 2.0 ** -149) if o.dtype == torch.float32 else (2.0 ** -8, 2.0 ** -133)
            assert (np.abs(G.host_f64(o) - w) <= tol * np.abs(w) + step).all()
    return coef


SIZES = [[1], [3], [1, 1, 1], [8191, 8192, 8193], [100000], [49152, 16384, 49152, 4096], [5, 70001, 12, 333, 8192 * 3]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("frac", [0.3, 2.0])
def test_clip(sizes, dtypes, frac):
    grads = tensors(len(sizes), sizes, dtypes, 0.01)
    outs = [torch.full_like(g, NAN) for g in grads]
    limit = frac * 0.01 * math.sqrt(sum(sizes)) + (10.0 if frac > 1 else 0.0)
    coef = check(grads, outs, limit)
    if frac > 1:
        assert coef == 1.0 and all(torch.equal(g, o) for g, o in zip(grads, outs))
    same = [g.clone() for g in grads]
    assert check(same, same, limit) == coef
    assert all(torch.equal(a, b) for a, b in zip(same, outs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 2, 7, 9, 255, 8190, 8200, 30001])
def test_unaligned_slices(dtype, n):
    """Every offset of source and destination from a 16-byte boundary; the neighbours stay."""
    for a in range(0, 9 if dtype == torch.bfloat16 else 5):
        for b in {a, 0, 1, 3}:
            src = tensors(a, [n + 16], (dtype,))[0]
            dst = torch.full((n + 16,), 9.0, dtype=dtype, device="cuda")
            check([src[a:a + n]], [dst[b:b + n]], 0.25)
            assert (dst[:b] == 9).all() and (dst[b + n:] == 9).all()
            keep = src.clone()
            check([src[a:a + n]], [src[a:a + n]], 0.25)
            assert torch.equal(src[:a], keep[:a]) and torch.equal(src[a + n:], keep[a + n:])


def test_norm_alone_and_tensors_that_are_only_counted():
    grads = tensors(1, [1000, 33, 4096])
    keep = [g.clone() for g in grads]
    out = torch.full_like(grads[1], NAN)
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    norm, coef = run([(grads[0], None), (grads[1], out), (grads[2], None)], 2.0)
    assert norm == pytest.approx(want, rel=2e-6) and coef == pytest.approx(2.0 / want, rel=2e-6)
    assert torch.allclose(out, grads[1] * coef, rtol=1e-6, atol=0)
    norm, coef = run([(g, g) for g in grads], math.inf)
    assert norm == pytest.approx(want, rel=2e-6) and coef == 1.0
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    arr = lora.make_grads([(g, None) for g in grads])
    only = torch.empty(1, device="cuda")
    ws = G.workspace(lora.lora_clip_workspace_size(arr))
    lora.lora_clip_grads(arr, 1.0, only, None, ws, ws.numel())
    assert float(only) == norm


def test_empty_and_zero_tensors():
    empty = torch.empty(0, device="cuda")
    assert run([(empty, empty)], 1.0) == (0.0, 1.0)
    z = torch.zeros(10, device="cuda")
    assert run([(z, z), (empty, None)], 0.0) == (0.0, 1.0)
    g = torch.ones(10, device="cuda")
    norm, coef = run([(empty, empty), (g, g), (empty, None)], 0.0)
    assert norm == pytest.approx(math.sqrt(10)) and coef == 0.0 and (g == 0).all()


@pytest.mark.parametrize("std", [1e-30, 1e-22, 1e-12, 1e12, 1e25, 1e36])
def test_whole_range_of_fp32(std):
    """Squares that fp32 cannot hold, alone and beside ordinary values."""
    grads = tensors(2, [5000, 123], std=std)
    outs = [torch.empty_like(g) for g in grads]
    check(grads, outs, 0.5 * std * math.sqrt(5123))
    mixed = grads + tensors(3, [777])
    check(mixed, [torch.empty_like(g) for g in mixed], 1e-3)


@pytest.mark.parametrize("bits", [1, 0x8000, 0x7FFFFF])
def test_subnormals_alone(bits):
    """Elements of one bit pattern each; the norm is a subnormal or a little above: one spacing, and the root's rounding."""
    n = 4999
    g = torch.full((n,), bits, dtype=torch.int32, device="cuda").view(torch.float32)
    out = torch.empty_like(g)
    norm, coef = run([(g, out)], 1.0)
    assert abs(norm - bits * 2.0**-149 * math.sqrt(n)) <= 2.0**-149 + 1e-6 * norm
    assert coef == 1.0 and torch.equal(out.view(torch.int32), g.view(torch.int32))


def test_large_values_in_one_place():
    """One element whose square overflows among small ones of the same thread's."""
    g = torch.full((30000,), 1e-3, device="cuda")
    g[12345] = 3e30
    check([g], [torch.empty_like(g)], 1.0)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), NAN])
def test_not_finite(bad):
    grads = tensors(4, [9000, 50])
    grads[0][8500] = bad
    outs = [torch.zeros_like(g) for g in grads]
    norm, coef = run(list(zip(grads, outs)), 0.1)
    assert not math.isfinite(norm) and coef == 1.0
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(grads, outs))


@pytest.mark.parametrize("count", [999, 1000, 1001, 2500])
def test_more_tensors_than_one_launch_takes(count):
    sizes = [1 + (7 * i) % 40 for i in range(count)]
    grads = tensors(count, sizes)
    outs = [torch.full_like(g, NAN) for g in grads]
    check(grads, outs, 3.0)


def test_same_bits_every_time_and_on_another_stream():
    grads = tensors(5, [300001, 77, 49152])
    outs = [torch.empty_like(g) for g in grads]
    first = run(list(zip(grads, outs)), 1.0)
    keep = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for o in outs:
                o.zero_()
            assert run(list(zip(grads, outs)), 1.0) == first
        assert all(torch.equal(a, b) for a, b in zip(keep, outs))


def test_follows_the_gradients_in_stream_order():
    """The clip right behind the kernels that write the gradients, several times over: no stale norm."""
    g = torch.ones(100000, device="cuda")
    norms = torch.empty(20, device="cuda")
    arr = lora.make_grads([(g, g)])
    ws = G.workspace(lora.lora_clip_workspace_size(arr))
    for i in range(20):
        g.fill_(float(i + 1))
        lora.lora_clip_grads(arr, 1.0, norms[i:], None, ws, ws.numel())
    torch.cuda.synchronize()
    want = torch.arange(1, 21, device="cuda") * math.sqrt(100000)
    assert torch.allclose(norms, want, rtol=2e-6)
    assert torch.allclose(g, torch.full_like(g, 1 / math.sqrt(100000)), rtol=4e-6)


def test_tensor_past_two_to_the_31_elements():
    n = (1 << 31) + 77
    g = torch.full((n,), 2.0, dtype=torch.bfloat16, device="cuda")
    norm, coef = run([(g, g)], math.sqrt(n))
    assert norm == pytest.approx(2.0 * math.sqrt(n), rel=2e-6) and coef == pytest.approx(0.5, rel=2e-6)
    assert (g[:100] == 1).all() and (g[-100:] == 1).all() and float(g[::4096].float().sum()) == g[::4096].numel()


@pytest.mark.parametrize("n", [300001, 3000001])
def test_large_calls_follow_the_gradients_in_stream_order(n):
    """Above the size of one launch, right behind the kernels that write the gradients, with the workspace of the
    call before: each call's norm, coefficient and clipped tensor are those of its own gradients."""
    g = torch.empty(n, device="cuda")
    norms, coefs, outs = torch.empty(20, device="cuda"), torch.empty(20, device="cuda"), torch.empty(20, n, device="cuda")
    arrs = [lora.make_grads([(g, out)]) for out in outs]
    ws = G.workspace(lora.lora_clip_workspace_size(arrs[0]))
    for i, arr in enumerate(arrs):
        g.fill_(float(2 ** (i % 5) * (i + 1)))
        lora.lora_clip_grads(arr, 1.0, norms[i:], coefs[i:], ws, ws.numel())
    torch.cuda.synchronize()
    want = torch.tensor([2 ** (i % 5) * (i + 1) for i in range(20)], device="cuda").double() * math.sqrt(n)
    assert torch.allclose(norms.double(), want, rtol=2e-6, atol=0) and torch.allclose(coefs.double(), 1 / want, rtol=2e-6, atol=0)
    assert ((outs.double() * math.sqrt(n) - 1).abs() <= 3e-6).all()


def test_pieces_past_one_launch_table():
    """2^40 elements listed (one tensor of 2^31, counted 513 times) and a small tensor behind them, which begins a
    second table: its norm is not the call's."""
    n = 1 << 31
    big = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    small = torch.arange(1.0, 101.0, device="cuda")
    out = torch.full_like(small, NAN)
    norm, coef = run([(big, None)] * 513 + [(small, out)], 0.5)
    want = math.sqrt(513 * n * 2.0 ** -20 + float((small.double() ** 2).sum()))
    assert norm == pytest.approx(want, rel=2e-6) and coef == pytest.approx(0.5 / want, rel=2e-6)
    assert ((out.double() - small.double() * 0.5 / want).abs() <= 3e-6 * small.double()).all()


# The two launches that calls of more than 256 pieces of 1024 elements take: the cases above again beside a counted
# tensor of 300000 elements, and calls on both sides of that number.
MANY = 300000


def check_beside_many(grads, outs, max_norm, std=1.0):
    """As check(), with MANY elements of standard deviation std that are counted and not written."""
    many = tensors(MANY, [MANY], std=std)[0]
    keep = many.clone()
    want_norm, want_coef, want = oracle.clip_grads([G.host_f64(g) for g in grads + [many]], max_norm)
    norm, coef = run(list(zip(grads, outs)) + [(many, None)], max_norm)
    assert norm == pytest.approx(want_norm, rel=2e-6)
    assert coef == pytest.approx(want_coef, rel=2e-6)
    for o, w in zip(outs, want):
        tol, step = (3e-6, 2.0 ** -149) if o.dtype == torch.float32 else (2.0 ** -8, 2.0 ** -133)
        assert (np.abs(G.host_f64(o) - w) <= tol * np.abs(w) + step).all()
    assert torch.equal(many, keep)
    return coef


@pytest.mark.parametrize("sizes", SIZES + [[262144], [262145], [256 * 1024 - 1, 2]])
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("frac", [0.3, 2.0])
def test_many_elements(sizes, dtypes, frac):
    grads = tensors(len(sizes), sizes, dtypes, 0.01)
    outs = [torch.full_like(g, NAN) for g in grads]
    limit = frac * 0.01 * math.sqrt(sum(sizes) + MANY)
    coef = check_beside_many(grads, outs, limit, 0.01)
    assert (coef == 1.0) == (frac > 1)
    if frac > 1:
        assert all(torch.equal(g, o) for g, o in zip(grads, outs))
    same = [g.clone() for g in grads]
    assert check_beside_many(same, same, limit, 0.01) == coef
    assert all(torch.equal(a, b) for a, b in zip(same, outs))


@pytest.mark.parametrize("pieces", [255, 256, 257, 304, 305])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_both_sides_of_one_launch(pieces, dtype):
    """Calls of so many pieces: whole outputs, from sources and into destinations that lie off 16 bytes."""
    n = pieces * 1024
    for a, b in ((0, 0), (1, 0), (0, 3), (1, 1)):
        src = tensors(pieces + a, [n + 8], (dtype,))[0]
        dst = torch.full((n + 8,), 9.0, dtype=dtype, device="cuda")
        check([src[a:a + n]], [dst[b:b + n]], 0.25)
        assert (dst[:b] == 9).all() and (dst[b + n:] == 9).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 9, 255, 8190, 30001])
def test_unaligned_slices_beside_many(dtype, n):
    for a in range(0, 9 if dtype == torch.bfloat16 else 5):
        for b in {a, 0, 3}:
            src = tensors(a, [n + 16], (dtype,))[0]
            dst = torch.full((n + 16,), 9.0, dtype=dtype, device="cuda")
            check_beside_many([src[a:a + n]], [dst[b:b + n]], 0.25)
            assert (dst[:b] == 9).all() and (dst[b + n:] == 9).all()
            keep = src.clone()
            check_beside_many([src[a:a + n]], [src[a:a + n]], 0.25)
            assert torch.equal(src[:a], keep[:a]) and torch.equal(src[a + n:], keep[a + n:])


@pytest.mark.parametrize("std", [1e-30, 1e-22, 1e-12, 1e12, 1e25, 1e35])
def test_whole_range_of_fp32_beside_many(std):
    """As test_whole_range_of_fp32; several pieces of a warp are taken again."""
    grads = tensors(2, [50000, 123], std=std)
    check_beside_many(grads, [torch.empty_like(g) for g in grads], 0.5 * std * math.sqrt(50123 + MANY), std)
    mixed = grads + tensors(3, [777])
    check_beside_many(mixed, [torch.empty_like(g) for g in mixed], 1e-3, std)


@pytest.mark.parametrize("bits", [1, 0x8000, 0x7FFFFF])
def test_subnormals_among_many_zeros(bits):
    """As test_subnormals_alone, with MANY zeros behind them."""
    n = 4999
    g = torch.full((n,), bits, dtype=torch.int32, device="cuda").view(torch.float32)
    out, zeros = torch.empty_like(g), torch.zeros(MANY, device="cuda")
    norm, coef = run([(g, out), (zeros, None)], 1.0)
    assert abs(norm - bits * 2.0**-149 * math.sqrt(n)) <= 2.0**-149 + 1e-6 * norm
    assert coef == 1.0 and torch.equal(out.view(torch.int32), g.view(torch.int32))


@pytest.mark.parametrize("at", [0, 12345, 299999])
def test_large_value_in_one_place_of_many(at):
    g = torch.full((MANY,), 1e-3, device="cuda")
    g[at] = 3e30
    check([g], [torch.empty_like(g)], 1.0)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), NAN])
def test_not_finite_among_many(bad):
    grads = tensors(4, [MANY, 50, 3])
    grads[0][285000] = bad
    outs = [torch.zeros_like(g) for g in grads]
    norm, coef = run(list(zip(grads, outs)), 0.1)
    assert not math.isfinite(norm) and coef == 1.0
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(grads, outs))


def test_norm_alone_of_many():
    grads = tensors(1, [MANY, 33, 4096, 70001])
    keep = [g.clone() for g in grads]
    out = torch.full_like(grads[1], NAN)
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    norm, coef = run([(grads[0], None), (grads[1], out), (grads[2], None), (grads[3], None)], 2.0)
    assert norm == pytest.approx(want, rel=2e-6) and coef == pytest.approx(2.0 / want, rel=2e-6)
    assert torch.allclose(out, grads[1] * coef, rtol=1e-6, atol=0)
    assert run([(g, g) for g in grads], math.inf) == (norm, 1.0)
    assert run([(g, None) for g in grads], math.inf) == (norm, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))


def test_norm_past_fp32():
    """A norm of 4e39 is written as infinity; the coefficient is still max_norm over it."""
    for n in (100, MANY):
        g = torch.full((n,), 3e38, device="cuda")
        out = torch.empty_like(g)
        norm, coef = run([(g, out)], 1e10)
        assert norm == math.inf and coef == pytest.approx(1e10 / (3e38 * math.sqrt(n)), rel=2e-6, abs=0)
        assert torch.allclose(out.double(), torch.full((1,), 1e10 / math.sqrt(n), device="cuda").double(), rtol=3e-6, atol=0)


@pytest.mark.parametrize("sizes", [[5000, 77], [MANY, 77, 40001]])
def test_in_a_graph(sizes):
    """Captured once, replayed on other gradients in place."""
    grads = tensors(6, sizes)
    outs = [torch.empty_like(g) for g in grads]
    arr = lora.make_grads(list(zip(grads, outs)))
    norm, coef = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = G.workspace(lora.lora_clip_workspace_size(arr))
    lora.lora_clip_grads(arr, 1.0, norm, coef, ws, ws.numel())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lora.lora_clip_grads(arr, 1.0, norm, coef, ws, ws.numel())
    for seed in (7, 8):
        for g, new in zip(grads, tensors(seed, sizes, std=float(seed))):
            g.copy_(new)
        lora.lora_clip_grads(arr, 1.0, norm, coef, ws, ws.numel())
        torch.cuda.synchronize()
        want = [v.clone() for v in [norm, coef] + outs]
        for v in [norm, coef] + outs:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [norm, coef] + outs)) and float(norm) > 0
