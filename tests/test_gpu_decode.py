"""GPU parity of the few-token forward with 4-bit weights through the C ABI,
against the fp64 oracle on the same codes, parameters and bf16 inputs.

Tolerance, per element: y is rounded to bf16 once (at most 2^-9 |y|, and
2^-8 |y| leaves room for the tie of a value that fp32 sums move across it),
and fp32 sums of K products in blocks of 16 err by less than 2^-20 of the sum
of the products' magnitudes.  Exact where the arithmetic is exact."""
import numpy as np
import pytest
import torch

import oracle
from paper_2606_19528_gb300 import lora, synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

GUARD = 24


def bits(a):
    return synth.to_bf16_bits(np.asarray(a, np.float64))


class Proj:
    """Inputs of one projection on the device, y between guards, its oracle."""

    def __init__(self, seed, T, K, N, r, s=1.5, x=None):
        g = np.random.default_rng(seed)
        self.T, self.K, self.N, self.r, self.s = T, K, N, r, s
        self.x_bits = bits(g.standard_normal((T, K))) if x is None else x
        codes = g.integers(0, 256, (N, K // 2), dtype=np.uint8)
        sd = K ** -0.5
        sc = g.uniform(0.2, 0.45, (N, K // 64)) * sd * g.choice([1, 1, -1], (N, K // 64))
        params = bits(np.stack([sc, -7.0 * sc + 0.3 * sd * g.standard_normal(sc.shape)], axis=-1))
        self.fill(codes, params, bits(g.uniform(-sd, sd, (r, K))), bits(0.05 * g.standard_normal((N, r))))

    def fill(self, codes, params, A, B):
        sb = synth.bf16_bits_to_f64(params)
        W = synth.bf16_bits_to_f64(synth.to_bf16_bits(oracle.dequant_q4(codes, sb[..., 0], sb[..., 1])))
        x = synth.bf16_bits_to_f64(self.x_bits)
        A64, B64 = synth.bf16_bits_to_f64(A), synth.bf16_bits_to_f64(B)
        su = self.s * (x @ A64.T)
        self.want = x @ W.T + su @ B64.T
        self.size = np.abs(x) @ np.abs(W).T + np.abs(self.s) * (np.abs(x) @ np.abs(A64).T) @ np.abs(B64).T
        self.x = G.dev_bf16(self.x_bits)
        self.codes, self.params = torch.from_numpy(codes).cuda(), G.dev_bf16(params)
        self.A, self.B = (G.dev_bf16(A), G.dev_bf16(B)) if self.r else (None, None)
        self.out = torch.full((GUARD + self.T * self.N + GUARD,), 77.0, dtype=torch.bfloat16, device="cuda")
        self.y = self.out[GUARD:GUARD + self.T * self.N].view(self.T, self.N)

    def proj(self, **kw):
        args = dict(x=self.x, A=self.A, B=self.B, y=self.y, Wq=lora.make_q4(self.codes, self.params))
        args.update(kw)
        return lora.make_proj(lora.make_shape(self.T, self.K, self.N, self.r, self.s), **args)

    def check(self):
        got = G.host_f64(self.y)
        bad = np.abs(got - self.want) > 2.0 ** -8 * np.abs(self.want) + 2.0 ** -20 * self.size
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], self.want[bad][:4])
        assert (self.out[:GUARD] == 77).all() and (self.out[GUARD + self.T * self.N:] == 77).all()


def run(ps, stream=None):
    projs = lora.make_projs([p.proj() for p in ps])
    n = lora.lora_decode_workspace_size(projs)
    ws = torch.full((n + 256,), 0x7f, dtype=torch.uint8, device="cuda")  # NaN-like contents: it needs no clearing
    lora.lora_decode_q4(projs, ws, n, stream)
    torch.cuda.synchronize()
    assert (ws[n:] == 0x7f).all()
    assert lora.lora_read_status() == lora.LORA_OK


@pytest.mark.parametrize("T", range(1, 17))
def test_every_token_count(T):
    p = Proj(T, T, 192, 40, 8)
    run([p])
    p.check()


@pytest.mark.parametrize("K,N", [(64, 1), (64, 16), (128, 17), (192, 15), (320, 33), (1024, 129), (1088, 7),
                                 (4160, 250), (8192, 3), (256, 4099), (12288, 31)])
@pytest.mark.parametrize("T", [1, 3, 8, 11])
def test_sizes(K, N, T):
    p = Proj(K + N, T, K, N, 16)
    run([p])
    p.check()


@pytest.mark.parametrize("r", [0, 1, 2, 3, 7, 8, 13, 16, 24, 33, 64, 127, 128])
@pytest.mark.parametrize("T", [1, 9, 16])
def test_ranks(r, T):
    p = Proj(100 + r, T, 512, 100, r)
    run([p])
    p.check()


def test_layer_projections_together():
    """Different widths, depths, ranks (also none) and token counts in one call."""
    shapes = [(1, 3072, 1024, 16), (1, 3072, 256, 0), (5, 2048, 515, 64), (16, 64, 48, 3), (2, 2112, 77, 0)]
    ps = [Proj(200 + i, *s) for i, s in enumerate(shapes)]
    run(ps)
    for p in ps:
        p.check()


def test_sixty_four_projections():
    x = Proj(0, 2, 128, 8, 0).x_bits
    ps = [Proj(300 + i, 2, 128, 5 + i, i % 4, x=x) for i in range(64)]
    run(ps)
    for p in ps:
        p.check()


def test_no_adapter_takes_no_workspace():
    p = Proj(7, 3, 256, 50, 0)
    projs = lora.make_projs([p.proj()])
    assert lora.lora_decode_workspace_size(projs) == 0
    lora.lora_decode_q4(projs, None, 0)
    torch.cuda.synchronize()
    p.check()


def test_exact_integers():
    """Codes minus 8 as weights, small integers everywhere: every sum is exact in fp32 and fits bf16."""
    g = np.random.default_rng(3)
    T, K, N, r = 7, 64, 24, 4
    p = Proj(1, T, K, N, r, s=2.0, x=bits(g.integers(-1, 2, (T, K)) * (g.random((T, K)) < 0.2)))
    params = bits(np.tile([1.0, -8.0], (N, 1, 1)))
    A = bits(g.integers(-1, 2, (r, K)) * (g.random((r, K)) < 0.1))
    p.fill(g.integers(0, 256, (N, K // 2), dtype=np.uint8), params, A, bits(g.integers(-1, 2, (N, r))))
    run([p])
    assert np.abs(p.want).max() <= 256
    assert np.array_equal(G.host_f64(p.y), p.want)


def test_same_weights_as_the_training_forward():
    """One-hot activations read the weight out: bit for bit what lora_linear_fwd_q4 multiplies."""
    T, K, N = 8, 256, 64
    x = np.zeros((T, K))
    x[np.arange(T), 31 * np.arange(T) + 5] = 1.0
    p = Proj(11, T, K, N, 0, x=bits(x))
    run([p])
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    st = lora.make_shape(T, K, N, 0, p.s)
    ws = G.workspace(lora.lora_workspace_size(st, lora.LORA_FWD))
    lora.lora_linear_fwd_q4(st, p.x, lora.make_q4(p.codes, p.params), None, None, y, None, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(p.y, y)


def test_infinite_and_nan_activations_stay_in_their_token():
    p = Proj(13, 4, 256, 40, 8)
    p.x[1, 3] = float("inf")
    p.x[2, 200] = float("nan")
    run([p])
    got = G.host_f64(p.y)
    assert not np.isfinite(got[1]).any() and np.isnan(got[2]).all()
    for t in (0, 3):
        assert (np.abs(got[t] - p.want[t]) <= 2.0 ** -8 * np.abs(p.want[t]) + 2.0 ** -20 * p.size[t]).all()


def test_same_bits_every_time_and_on_another_stream():
    ps = [Proj(17, 5, 2048, 300, 16), Proj(18, 5, 2048, 90, 0)]
    run(ps)
    first = [p.y.clone() for p in ps]
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for p in ps:
                p.y.fill_(float("nan"))
            projs = lora.make_projs([p.proj() for p in ps])
            ws = G.workspace(lora.lora_decode_workspace_size(projs))
            lora.lora_decode_q4(projs, ws, ws.numel())
        torch.cuda.synchronize()
        assert all(torch.equal(p.y, f) for p, f in zip(ps, first))


@pytest.mark.parametrize("T,K,N", [(16, 3072, 30000), (16, 1024, 20001), (8, 3072, 30000), (9, 320, 50000),
                                   (16, 6144, 6000), (3, 11008, 2048), (16, 12288, 1000), (16, 4416, 40001),
                                   (13, 64, 200003), (16, 8192, 3000), (9, 16448, 1000), (16, 8192, 9000)])
def test_many_tiles_come_out_the_same_in_every_call(T, K, N):
    """Every SM takes many tiles through its rings, with little room for them beside 16 tokens: 100 calls, bit for
    bit, and against the product in fp32."""
    g = torch.Generator(device="cuda").manual_seed(K + N)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    sd = K ** -0.5
    s = torch.empty(N, K // 64, device="cuda").uniform_(0.2, 0.45, generator=g) * sd
    params = torch.stack([s, -7.5 * s], dim=-1).to(torch.bfloat16).contiguous()
    x = torch.randn(T, K, generator=g, device="cuda").to(torch.bfloat16)
    words = codes.view(torch.int32)[:, :, None, None]
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device="cuda", dtype=torch.int32)
    q = ((words >> shift) & 15).float().view(N, K // 64, 64)
    W = (params[:, :, :1].float() * q + params[:, :, 1:].float()).to(torch.bfloat16).float().view(N, K)
    y = torch.full((T, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    projs = lora.make_projs([lora.make_proj(lora.make_shape(T, K, N, 0, 1.0), x=x, y=y,
                                            Wq=lora.make_q4(codes, params))])
    lora.lora_decode_q4(projs, None, 0)
    first, bad = y.clone(), 0
    for _ in range(100):
        y.zero_()
        lora.lora_decode_q4(projs, None, 0)
        bad += (y != first).sum()
    assert int(bad) == 0
    want = x.float() @ W.T
    size = x.float().abs() @ W.abs().T  # the bound of the module's head, twice the sums' part for the fp32 product
    assert ((first.float() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all()


def test_chain_of_calls_in_a_graph():
    """y of one call is x of the next, captured and replayed with other inputs in place."""
    K = 256
    a, c = Proj(21, 3, K, K, 16), Proj(22, 3, K, 128, 8)
    both = [lora.make_projs([a.proj()]), lora.make_projs([c.proj(x=a.y)])]
    ws = [G.workspace(lora.lora_decode_workspace_size(p)) for p in both]

    def step():
        for p, w in zip(both, ws):
            lora.lora_decode_q4(p, w, w.numel())

    a.out[GUARD:GUARD + 3 * K] = 0
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x2 = torch.randn(3, K, device="cuda").to(torch.bfloat16)
    a.x.copy_(x2)
    step()
    torch.cuda.synchronize()
    want = c.y.clone()
    c.y.zero_()
    a.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.y, want) and not torch.equal(want, torch.zeros_like(want))


@pytest.mark.parametrize("T,K,shapes", [
    (16, 1024, [(40001, 16), (30000, 0), (129, 128), (2500, 13)]), (1, 4160, [(90001, 64)]), (9, 192, [(150000, 1), (7, 3)]),
    (12, 8192, [(20011, 128), (20000, 0)]),
    # tiles whose columns are shared out
    (16, 8192, [(3000, 16)]), (16, 8192, [(8191, 7)]), (11, 8256, [(5000, 24), (1000, 0)]), (16, 16448, [(1000, 13)]),
    (13, 16384, [(130, 128)]), (16, 12288, [(2200, 0)])])
def test_many_rows_with_adapters(T, K, shapes):
    """Projections of tens of thousands of rows that share an activation, with adapters of any rank or none: the
    launch for many rows, against fp32 products (the bound of the module's head, twice the sums' part)."""
    g = torch.Generator(device="cuda").manual_seed(K + T)
    sd = K ** -0.5
    x = torch.randn(T, K, generator=g, device="cuda").to(torch.bfloat16)
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device="cuda", dtype=torch.int32)
    projs, check = [], []
    for N, r in shapes:
        codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        s = torch.empty(N, K // 64, device="cuda").uniform_(0.2, 0.45, generator=g) * sd
        params = torch.stack([s, -7.5 * s], dim=-1).to(torch.bfloat16).contiguous()
        A = (torch.randn(r, K, generator=g, device="cuda") * sd).to(torch.bfloat16) if r else None
        B = (torch.randn(N, r, generator=g, device="cuda") * 0.1).to(torch.bfloat16) if r else None
        out = torch.full((GUARD + T * N + GUARD,), 77.0, dtype=torch.bfloat16, device="cuda")
        projs.append(lora.make_proj(lora.make_shape(T, K, N, r, 2.0), x=x, A=A, B=B, y=out[GUARD:],
                                    Wq=lora.make_q4(codes, params)))
        check.append((N, codes, params, A, B, out))
    projs = lora.make_projs(projs)
    ws = G.workspace(lora.lora_decode_workspace_size(projs))
    for _ in range(3):
        lora.lora_decode_q4(projs, ws, ws.numel())
    torch.cuda.synchronize()
    assert lora.lora_read_status() == lora.LORA_OK
    for N, codes, params, A, B, out in check:
        q = ((codes.view(torch.int32)[:, :, None, None] >> shift) & 15).float().view(N, K // 64, 64)
        W = (params[:, :, :1].float() * q + params[:, :, 1:].float()).to(torch.bfloat16).float().view(N, K)
        want, size = x.float() @ W.T, x.float().abs() @ W.abs().T
        if A is not None:
            want = want + 2.0 * (x.float() @ A.float().T) @ B.float().T
            size = size + 2.0 * (x.float().abs() @ A.float().abs().T) @ B.float().abs().T
        y = out[GUARD:GUARD + T * N].view(T, N).float()
        assert ((y - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all()
        assert (out[:GUARD] == 77).all() and (out[GUARD + T * N:] == 77).all()


def test_codes_past_two_to_the_32_bytes():
    """2^20 rows of 8704 columns: 4.6 GB of codes; the last rows against the oracle."""
    T, K, N, last = 2, 8704, 1 << 20, 40
    p = Proj(31, T, K, last, 4)
    codes = torch.zeros(N, K // 2, dtype=torch.uint8, device="cuda")
    params = torch.zeros(N, K // 64, 2, dtype=torch.bfloat16, device="cuda")
    B = torch.zeros(N, 4, dtype=torch.bfloat16, device="cuda")
    codes[-last:], params[-last:], B[-last:] = p.codes, p.params, p.B
    y = torch.full((T, N), 5.0, dtype=torch.bfloat16, device="cuda")
    projs = lora.make_projs([lora.make_proj(lora.make_shape(T, K, N, 4, p.s), x=p.x, A=p.A, B=B, y=y,
                                            Wq=lora.make_q4(codes, params))])
    ws = G.workspace(lora.lora_decode_workspace_size(projs))
    lora.lora_decode_q4(projs, ws, ws.numel())
    torch.cuda.synchronize()
    assert (y[:, :-last] == 0).all()
    p.y.copy_(y[:, -last:])
    p.check()


class Fp32:
    """A projection of any size, its y between guards, against fp32 products (the bound of the module's head, twice the
    sums' part)."""

    def __init__(self, g, T, K, N, r, x, s=2.0, w_scale=1.0):
        self.T, self.K, self.N, self.r, self.s, self.x = T, K, N, r, s, x
        sd = K ** -0.5 * w_scale
        sc = torch.empty(N, K // 64, device="cuda").uniform_(0.2, 0.45, generator=g) * sd
        self.codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        self.params = torch.stack([sc, -7.5 * sc], dim=-1).to(torch.bfloat16).contiguous()
        self.A = (torch.randn(r, K, generator=g, device="cuda") * sd).to(torch.bfloat16) if r else None
        self.B = (torch.randn(N, r, generator=g, device="cuda") * 0.1).to(torch.bfloat16) if r else None
        self.out = torch.full((GUARD + T * N + GUARD,), 77.0, dtype=torch.bfloat16, device="cuda")

    def proj(self):
        return lora.make_proj(lora.make_shape(self.T, self.K, self.N, self.r, self.s), x=self.x, A=self.A, B=self.B,
                              y=self.out[GUARD:], Wq=lora.make_q4(self.codes, self.params))

    def y(self):
        return self.out[GUARD:GUARD + self.T * self.N].view(self.T, self.N)

    def weight(self):
        shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device="cuda", dtype=torch.int32)
        q = ((self.codes.view(torch.int32)[:, :, None, None] >> shift) & 15).float().view(self.N, self.K // 64, 64)
        p = self.params.float()
        return (p[:, :, :1] * q + p[:, :, 1:]).to(torch.bfloat16).float().view(self.N, self.K)

    def check(self):
        x, W = self.x.float(), self.weight()
        want, size = x @ W.T, x.abs() @ W.abs().T
        if self.r:
            A, B = self.A.float(), self.B.float()
            want = want + self.s * (x @ A.T) @ B.T
            size = size + abs(self.s) * (x.abs() @ A.abs().T) @ B.abs().T
        y = self.y().float()
        assert ((y - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all()
        assert (self.out[:GUARD] == 77).all() and (self.out[GUARD + self.T * self.N:] == 77).all()


@pytest.mark.parametrize("shapes", [
    # (T, K, N, r, activation): two launches for many rows on activations of their own, narrow projections between them
    [(2, 512, 100, 3, 0), (16, 3072, 30000, 0, 1), (5, 2048, 515, 64, 2), (9, 8192, 3000, 16, 3), (16, 3072, 20000, 13, 1),
     (1, 64, 48, 16, 4), (16, 3072, 40, 0, 5)],
    [(9, 3072, 30000, 16, 0), (16, 8192, 9000, 8, 1), (16, 4160, 257, 128, 2)],
    # without adapters, no launch goes before
    [(16, 3072, 30000, 0, 0), (3, 512, 1000, 0, 1), (9, 8192, 9000, 0, 2), (16, 1024, 40001, 0, 3)],
    # wide ones alone, the second with the only adapter
    [(16, 3072, 30000, 0, 0), (12, 3072, 30000, 64, 1)],
])
def test_kinds_of_launches_together(shapes):
    """Calls whose projections take several launches after su's, listed in any order, on inputs that change from call to
    call, nothing waiting between; the workspace holds NaN before the first."""
    g = torch.Generator(device="cuda").manual_seed(len(shapes))
    xs = {}
    for T, K, N, r, i in shapes:
        xs.setdefault(i, torch.zeros(T, K, dtype=torch.bfloat16, device="cuda"))
    ps = [Fp32(g, T, K, N, r, xs[i]) for T, K, N, r, i in shapes]
    projs = lora.make_projs([p.proj() for p in ps])
    n = lora.lora_decode_workspace_size(projs)
    ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")
    last = None
    for seed in range(4):
        new = [torch.randn(x.shape, generator=g, device="cuda").to(torch.bfloat16) for x in xs.values()]
        for x, v in zip(xs.values(), new):
            x.copy_(v)
        for p in ps:
            p.out[GUARD:-GUARD] = float("nan")
        for _ in range(3):
            lora.lora_decode_q4(projs, ws, n)
        for p in ps:
            p.check()
        now = [p.y().clone() for p in ps]
        lora.lora_decode_q4(projs, ws, n)
        assert all(torch.equal(a, p.y()) for a, p in zip(now, ps))
        assert last is None or not any(torch.equal(a, b) for a, b in zip(last, now))
        last = now
    assert (ws[n:] == 0xff).all() and lora.lora_read_status() == lora.LORA_OK


@pytest.mark.parametrize("T,K,sizes", [(16, 3072, [(4000, 0)] * 9), (9, 2048, [(3000 + 129 * i, 4 * (i % 3)) for i in range(20)]),
                                       (16, 1024, [(1000 + i, 16) for i in range(64)])])
def test_many_rows_of_more_than_eight_projections(T, K, sizes):
    """The launch for many rows with the larger of its tables."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, K, generator=g, device="cuda").to(torch.bfloat16)
    ps = [Fp32(g, T, K, N, r, x) for N, r in sizes]
    projs = lora.make_projs([p.proj() for p in ps])
    n = lora.lora_decode_workspace_size(projs)
    ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        lora.lora_decode_q4(projs, ws, n)
    for p in ps:
        p.check()
    assert (ws[n:] == 0xff).all() and lora.lora_read_status() == lora.LORA_OK


@pytest.mark.parametrize("T", [1, 5, 8])
def test_one_launch_with_and_without_adapters(T):
    """Ranks 16, 0, 3 and 0 in the launch that computes su itself."""
    ps = [Proj(400 + i, T, 512, N, r) for i, (N, r) in enumerate([(300, 16), (90, 0), (17, 3), (33, 0)])]
    run(ps)
    for p in ps:
        p.check()


@pytest.mark.parametrize("K,N", [(256, 64), (2048, 40000)])
def test_small_weights_are_those_of_the_training_forward(K, N):
    """Weights down to 2^-86, where both launches' scaled form still holds every bit: one-hot activations read them
    out."""
    T = 16
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    x[torch.arange(T, device="cuda"), 13 * torch.arange(T, device="cuda") + 5] = 1.0
    p = Fp32(g, T, K, N, 0, x)
    # s from 2^-86 to 2^-84 and b = -8 s: |s q + b| is 0 or at least |s|
    s = torch.exp2(torch.randint(-86, -84, (N, K // 64), generator=g, device="cuda").float())
    s = s * (1 + torch.randint(0, 128, s.shape, generator=g, device="cuda") / 128.0)
    p.params.copy_(torch.stack([s, -8 * s], dim=-1).to(torch.bfloat16))
    lora.lora_decode_q4([p.proj()], None, 0)
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    st = lora.make_shape(T, K, N, 0, 1.0)
    ws = G.workspace(lora.lora_workspace_size(st, lora.LORA_FWD))
    lora.lora_linear_fwd_q4(st, x, lora.make_q4(p.codes, p.params), None, None, y, None, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(p.y(), y) and float(y.abs().max()) < 2.0 ** -80
    assert torch.equal(y.float(), x.float() @ p.weight().T)
