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
