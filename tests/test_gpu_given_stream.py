"""Calls on a given stream: what they allocate comes from that stream's pool, since
memory that the current stream let go may still be in use there."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu


def pool_of(t):
    """The stream whose pool a tensor's memory belongs to."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


def given_stream():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert side.cuda_stream != torch.cuda.current_stream().cuda_stream
    return side


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("plen", [0, 50, 3000])
def test_cached_steps(device, quant, plen):
    mk = lambda: Problem(torch.bfloat16, quant, 3, 2, 64, plen, 40, plen + 30, 0, [1, 2, 33])
    a, b = mk(), mk()
    want = a.run()
    side = given_stream()
    got = b.run(stream=side)
    side.synchronize()
    assert pool_of(got) == side.cuda_stream
    assert torch.equal(got, want) and torch.equal(a.lse, b.lse) and torch.equal(a.len_out, b.len_out)


@pytest.mark.parametrize("given", ["nothing", "k", "v"])
def test_load(device, given):
    p = Problem(torch.bfloat16, True, 3, 2, 64, 0, 40, 30, 0, [1, 2, 33])
    want = pa.pi_attn_cache_load(*p.own, *p.own_exp, 25)
    side = given_stream()
    mine = {} if given == "nothing" else {given: torch.empty_like(want[0])}
    got = pa.pi_attn_cache_load(*p.own, *p.own_exp, 25, stream=side, **mine)
    side.synchronize()
    for x, y, name in zip(got, want, "kv"):
        assert x is mine[name] if name in mine else pool_of(x) == side.cuda_stream
        assert torch.equal(x.nan_to_num(9), y.nan_to_num(9))


def same(call, n_out):
    """call(stream=None) and on a given stream: the same bits, the latter's from the stream's pool."""
    want = call()
    side = given_stream()
    got = call(stream=side)
    side.synchronize()
    want, got = (x if isinstance(x, tuple) else (x,) for x in (want, got))
    assert len(got) == len(want) == n_out
    for x, y in zip(got, want):
        assert pool_of(x) == side.cuda_stream
        assert torch.equal(x, y)


def test_full_sequence_calls(device):
    B, H, N, D, k, pi = 1, 2, 200, 64, 40, 50
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    q, kk, v, dout = (rnd(B, H, N, D) for _ in range(4))
    gate = torch.rand(H, generator=g, device="cuda")
    u, w2 = rnd(B, N, 32), rnd(H, 32)
    same(lambda **kw: pa.pi_attn_index_set(30, 4, 7, **kw), 1)
    same(lambda **kw: pa.pi_attn_forward(q, kk, v, gate, k, pi, return_lse=True, **kw), 2)
    same(lambda **kw: pa.pi_attn_forward_gated(q, kk, v, u, w2, None, k, pi, return_lse=True, **kw), 3)
    out, lse = pa.pi_attn_forward(q, kk, v, gate, k, pi, return_lse=True)
    for d in (dout, dout.transpose(1, 2).contiguous().transpose(1, 2)):   # the latter is copied first
        same(lambda **kw: pa.pi_attn_backward(q, kk, v, gate, k, pi, out, lse, d, **kw), 4)
    same(lambda **kw: pa.pi_attn_forward_shard(q[:, :, 80:], kk, v, gate, k, pi, N, 80, 0, return_lse=True, **kw), 2)
    same(lambda **kw: pa.pi_attn_backward_shard_q(q, kk, v, gate, k, pi, N, 0, 0, out, lse, dout, **kw), 3)
    rt = pa.pi_attn_backward_shard_q(q, kk, v, gate, k, pi, N, 0, 0, out, lse, dout)[2]
    same(lambda **kw: pa.pi_attn_backward_shard_kv(q, kk, v, gate, k, pi, N, 0, 0, lse, rt, dout, **kw), 2)


def test_decode_step(device):
    S, H, D, cap = 3, 2, 64, 50
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(S, H, D, generator=g, device="cuda")
    kc, vc = (torch.randn(S, H, cap, D, generator=g, device="cuda") for _ in range(2))
    lens = torch.tensor([0, 20, 49], dtype=torch.int32, device="cuda")
    gate = torch.zeros(H, device="cuda")
    same(lambda **kw: pa.pi_attn_decode_step(lens, x, x, x, kc, vc, gate, 10, 15, **kw), 1)
