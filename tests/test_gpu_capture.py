"""Captured calls keep their memory: eager calls that need larger workspaces on the captured stream, and tensors that then take the old
ones' places, neither change what a replay gives nor are changed by it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _work(L, t):
    """Calls that all need a workspace: K split in the thin, tile and large forms, sums over tokens, factors."""
    y, z = L.loract_linear(t["x"], t["w"], lora_t=t["lt"], lora_b=t["lb"], act="gelu", save_preact=True)
    thin = L.loract_linear(t["x"][:4], t["w"])
    f = L.loract_linear(t["xf"], t["wf"])
    dp, db, d_b = L.loract_linear_backward(y, z, lora_t=t["lt"], act="gelu")
    heads = y.view(300, 4, 64)
    dq, _, dg, _ = L.loract_qknorm_rope_backward(heads, None, t["gamma"], None, t["table"], heads, None)
    u, v = L.loract_compress(t["x"], 16, seed=3)
    return y, z, thin, f, dp, db, d_b, dq, dg, u, v, L.loract_lora_grad(u, v, dp, t["lb"])


def test_replays_after_the_streams_workspace_has_grown():
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(4)
    rand = lambda *s, dtype=torch.bfloat16: (torch.randn(*s, generator=gen) * 0.1).to(dtype).cuda()
    t = dict(x=rand(300, 4096), w=rand(256, 4096), lt=rand(300, 8), lb=rand(8, 256), xf=rand(300, 2048, dtype=torch.float32),
             wf=rand(40, 2048, dtype=torch.float32), gamma=torch.ones(64, device="cuda"), table=L.loract_rope_table(300, 64))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [v.clone() for v in _work(L, t)]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = _work(L, t)
    big, wide = rand(1000, 8192), rand(512, 8192)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        large = L.loract_linear(big, wide)                       # grows the stream's workspace
        fill = [torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 20, 1 << 21, 1 << 22, 1 << 23) for _ in range(4)]
    side.synchronize()
    for _ in range(4):
        for v in got:
            v.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):                            # beside the replay, which runs on another stream
            again = L.loract_linear(big, wide)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(bool((f == 0x5A).all()) for f in fill)
        assert torch.equal(large, again)
