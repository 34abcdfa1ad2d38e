"""Outputs beside, between and in place of a call's inputs give what separate ones give; outputs that other inputs lie in are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _rand(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m", [1, 5, 300])
def test_linear_between_the_columns_of_one_matrix(m, dtype):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(m)
    x, w, res = _rand(gen, m, 96, dtype=dtype), _rand(gen, 96, 96, dtype=dtype), _rand(gen, m, 96, dtype=dtype)
    want = L.loract_linear(x, w, residual=res, act="silu")
    big = torch.empty((m, 3 * 96), dtype=dtype, device="cuda")
    a, b, c = big[:, :96], big[:, 96:192], big[:, 192:]
    a.copy_(x), b.copy_(res)
    assert torch.equal(L.loract_linear(a, w, residual=b, act="silu", out=c), want)
    assert torch.equal(L.loract_linear(a, w, residual=b, act="silu", out=b), want)
    assert torch.equal(a, x) and torch.equal(c, want)
    b.copy_(res)
    shifted = big[:, 48:144]
    for out in ([a, shifted] if m > 1 else [a]):
        with pytest.raises(L.LoractError):
            L.loract_linear(a, w, residual=b, act="silu", out=out)
    with pytest.raises(L.LoractError):
        L.loract_linear(a, w, residual=b, out=w[:m] if m <= 96 else a)
    assert torch.equal(a, x) and torch.equal(b, res)


@pytest.mark.parametrize("act,r", [("none", 0), ("gelu", 8), ("silu", 48)])
def test_backward_in_place_of_either_input(act, r):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(3)
    dy, z, t = _rand(gen, 200, 136), _rand(gen, 200, 136), _rand(gen, 200, r) if r else None
    call = lambda d, zz, out=None: L.loract_linear_backward(d, zz, lora_t=t, act=act, p_drop=0.1, seed=2, out=out)
    want = call(dy, z)
    for which in (0, 1):
        d, zz = dy.clone(), z.clone()
        if act == "none" and which:
            continue
        got = call(d, zz, (d, zz)[which])
        assert all(a is b or torch.equal(a, b) for a, b in zip(want, got))
    both = torch.cat([dy, z])
    with pytest.raises(L.LoractError):
        call(both[:200], both[200:], both[1:201])


@pytest.mark.parametrize("d,heads", [(64, 3), (50, 2)])
def test_heads_of_queries_and_keys_in_turn(d, heads):
    """A projection packed head by head: q, k and v of a head lie side by side, and all heads of q between those of k."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(d)
    packed = _rand(gen, 40, heads, 3, d)
    q, k = packed[:, :, 0], packed[:, :, 1]
    table, gamma = L.loract_rope_table(40, d), torch.ones(d, device="cuda")
    want = L.loract_qknorm_rope_forward(q.clone(), k.clone(), gamma, gamma, table)
    v = packed[:, :, 2].clone()
    got = L.loract_qknorm_rope_forward(q, k, gamma, gamma, table, out=(q, k))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(packed[:, :, 2], v)
    dq, dk = _rand(gen, 40, heads, d), _rand(gen, 40, heads, d)
    grads = L.loract_qknorm_rope_backward(want[0], want[1], gamma, gamma, table, dq, dk)
    back = L.loract_qknorm_rope_backward(want[0], want[1], gamma, gamma, table, dq, dk, out=(q, k))
    assert all(torch.equal(a, b) for a, b in zip(grads, back)) and torch.equal(packed[:, :, 2], v)
    for out in ((k, q), (q, q), (q, packed[:, :, 0])):
        with pytest.raises(L.LoractError):
            L.loract_qknorm_rope_forward(q, k, gamma, gamma, table, out=out)
    flat = torch.zeros(40 * heads * d + 8, dtype=torch.bfloat16, device="cuda")
    meeting = flat.as_strided((40, heads, d), (d, d, 1))
    with pytest.raises(L.LoractError):
        L.loract_qknorm_rope_forward(q, None, gamma, None, table, out=(meeting, None))
