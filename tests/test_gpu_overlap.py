"""Calls in a row on one stream, nothing waiting between them: launches overlap the ones before (programmatic dependent
launch), so that each call has to read what the call before it wrote, and not what lay there earlier.  Every result is
compared bit for bit with the same call on its own, in buffers of its own."""
import pytest
import torch

from paper_2606_19528_gb300 import lora
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def rand(g, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=g, device="cuda")).to(torch.bfloat16)


@pytest.mark.parametrize("V,d,k", [(700, 128, 16), (9000, 64, 24), (33000, 64, 16)])
def test_table_then_cross_entropy(V, d, k):
    """The table of an embedding that changes, and the loss over it."""
    g = torch.Generator(device="cuda").manual_seed(V)
    T, rounds = 96, 6
    Es, hs = [rand(g, V, d) for _ in range(rounds)], [rand(g, T, d) for _ in range(rounds)]
    ys = [torch.randint(0, V, (T,), generator=g, device="cuda").int() for _ in range(rounds)]
    mask = (torch.rand(T, generator=g, device="cuda") < 0.6).to(torch.uint8)
    E, h, y = torch.empty_like(Es[0]), torch.empty_like(hs[0]), torch.empty_like(ys[0])
    table_ws = G.workspace(lora.lora_topk_workspace_size(V, d, k))

    def buffers():
        return (torch.zeros(V, k, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"),
                torch.zeros(T, device="cuda"), torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"))

    def call(E, h, y, out, table_ws, ce_ws):
        table, loss, per, dh = out
        lora.lora_topk_table(E, V, d, k, table, table_ws, table_ws.numel())
        a = lora.make_ce_args(T, d, V, h, E, y, loss, mask=mask, topk=table, ld_topk=k, k=k, token_loss=per, dh=dh)
        ce_ws = ce_ws if ce_ws is not None else G.workspace(lora.lora_ce_workspace_size(a))
        lora.lora_ce_fwd_bwd(a, ce_ws, ce_ws.numel())
        return ce_ws

    want = []
    for i in range(rounds):
        out = buffers()
        call(Es[i], hs[i], ys[i], out, G.workspace(table_ws.numel()), None)
        torch.cuda.synchronize()
        want.append(out)
    out, got, ce_ws = buffers(), [], None
    for i in range(rounds):
        E.copy_(Es[i])
        h.copy_(hs[i])
        y.copy_(ys[i])
        ce_ws = call(E, h, y, out, table_ws, ce_ws)
        got.append([o.clone() for o in out])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T,r", [(128, 8), (1024, 16), (256, 7)])
def test_training_steps_with_new_adapters(T, r):
    g = torch.Generator(device="cuda").manual_seed(T)
    K = N = 512
    rounds = 6
    x, W, dy = rand(g, T, K), rand(g, N, K, std=K ** -0.5), rand(g, T, N)
    As, Bs = [rand(g, r, K, std=K ** -0.5) for _ in range(rounds)], [rand(g, N, r, std=0.1) for _ in range(rounds)]
    A, B = torch.empty_like(As[0]), torch.empty_like(Bs[0])

    def buffers():
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        return dict(y=torch.zeros(T, N, **bf16), su=torch.zeros(T, r, **bf16), dx=torch.zeros(T, K, **bf16),
                    dA=torch.zeros(r, K, device="cuda"), dB=torch.zeros(N, r, device="cuda"))

    def call(A, B, out, ws):
        projs = [lora.make_proj(lora.make_shape(T, K, N, r, 2.0), x=x, W=W, A=A, B=B, dy=dy, **out)]
        if ws is None:
            ws = G.workspace(lora.lora_stack_workspace_size(projs, lora.LORA_FWD_BWD))
        lora.lora_stack_step(projs, lora.LORA_FWD_BWD, ws, ws.numel())
        return ws

    want = []
    for i in range(rounds):
        out = buffers()
        call(As[i], Bs[i], out, None)
        torch.cuda.synchronize()
        want.append(out)
    out, got, ws = buffers(), [], None
    for i in range(rounds):
        A.copy_(As[i])
        B.copy_(Bs[i])
        ws = call(A, B, out, ws)
        got.append({k: v.clone() for k, v in out.items()})
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[k], b[k]) for k in b)


class Decode:
    """A projection with 4-bit weights for T tokens."""

    def __init__(self, g, T, K, N, r, x=None):
        self.T, self.K, self.N, self.r = T, K, N, r
        s = torch.empty(N, K // 64, device="cuda").uniform_(0.2, 0.45, generator=g) * K ** -0.5
        self.params = torch.stack([s, -7.5 * s], dim=-1).to(torch.bfloat16).contiguous()
        self.codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        self.A = rand(g, r, K, std=K ** -0.5) if r else None
        self.B = rand(g, N, r, std=0.1) if r else None
        self.x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda") if x is None else x
        self.y = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")

    def projs(self, x=None, y=None):
        return lora.make_projs([lora.make_proj(lora.make_shape(self.T, self.K, self.N, self.r, 2.0),
                                               x=self.x if x is None else x, A=self.A, B=self.B,
                                               y=self.y if y is None else y, Wq=lora.make_q4(self.codes, self.params))])


@pytest.mark.parametrize("T,K,N,r", [(1, 256, 256, 8), (5, 512, 512, 0), (3, 512, 512, 32), (16, 1024, 1024, 0),
                                     (16, 3072, 30000, 0), (9, 3072, 30000, 16)])
def test_decode_of_what_the_call_before_wrote(T, K, N, r):
    """Three projections in a row, each of the last one's output; without adapters and as one launch the blocks' first
    loads come right behind the wait."""
    g = torch.Generator(device="cuda").manual_seed(T + K + N)
    first = Decode(g, T, K, K, r)
    second = Decode(g, T, K, K, r, first.y)
    third = Decode(g, T, K, N, r, second.y)
    chain = (first, second, third)
    calls = [p.projs() for p in chain]
    n = max(lora.lora_decode_workspace_size(c) for c in calls)
    ws = G.workspace(n)
    xs = [rand(g, T, K) for _ in range(8)]
    want = []
    for x in xs:
        outs = []
        for p in chain:
            y = torch.zeros_like(p.y)
            lora.lora_decode_q4(p.projs(x, y), G.workspace(n), max(n, 256))
            torch.cuda.synchronize()
            outs.append(y)
            x = y
        want.append(outs)
    got = []
    for x in xs:
        first.x.copy_(x)
        for c in calls:
            lora.lora_decode_q4(c, ws, ws.numel())
        got.append([p.y.clone() for p in chain])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b)) and not torch.equal(a[-1], torch.zeros_like(a[-1]))
