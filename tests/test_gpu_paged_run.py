"""The operators in the order in which a program uses them: a prompt by chunks through a paged cache, then tokens one by one,
against one pass over the whole sequence; and a training step through the rotation."""
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.paged_ref import Cache, frequencies

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def prompt(S, H, N, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(S, H, N, D, generator=g).to(dtype).cuda() for _ in range(3)]


@pytest.mark.parametrize("D,page,kw,pi", [(64, 16, 100, 150), (128, 7, 1000, 0), (128, 64, 33, 64)])
def test_chunked_prompt_then_tokens(device, D, page, kw, pi):
    """bf16: chunks of a prompt, each turned, stored and attended over what the cache holds; then decode steps that turn their own
    rows.  The same rows enter the attention as in one pass over the whole sequence."""
    S, H, N, chunk, first = 2, 4, 300, 96, 240
    q, k, v = prompt(S, H, N, D, BF, 1)
    gate = torch.linspace(-1, 1, H, device="cuda")
    freq = frequencies(D // 2).cuda()
    qt, kt = pa.pi_attn_rotate(q, k, None, freq)
    whole = pa.pi_attn_forward(qt, kt, v, gate, kw, pi)
    cache = Cache(S, H, D, page, -(-N // page), BF, False, 2)
    outs = []
    for lo in range(0, first, chunk):
        n = min(chunk, first - lo)
        part = slice(lo, lo + n)
        start = torch.full((S,), lo, dtype=torch.int32, device="cuda")
        pos = torch.arange(lo, lo + n, dtype=torch.int32, device="cuda")
        qc, _ = pa.pi_attn_rotate(q[:, :, part], None, pos, freq)
        pa.pi_attn_paged_store(k[:, :, part], v[:, :, part], cache.k, cache.v, cache.table, start, freq=freq)
        kc, vc = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, lo + n)
        outs.append(pa.pi_attn_forward_shard(qc, kc, vc, gate, kw, pi, N, lo, 0))
        assert torch.equal(kc, kt[:, :, :lo + n])
    assert torch.equal(torch.cat(outs, 2), whole[:, :, :first])
    lens, nxt = torch.full((S,), first, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    for t in range(first, N):
        out = pa.pi_attn_decode_step_paged(lens, *(x[:, :, t].contiguous() for x in (q, k, v)), cache.k, cache.v, cache.table, gate, kw,
                                           pi, freq=freq, len_out=nxt)
        lens, nxt = nxt, lens
        # values up to 5: the pass's bf16 weights and queries, and both outputs' rounding
        assert (out.float() - whole[:, :, t].float()).abs().max() <= 2e-2
    kc, vc = pa.pi_attn_paged_load(cache.k, cache.v, cache.table, N)
    assert torch.equal(kc, kt) and torch.equal(vc, v) and lens.tolist() == [N, N]


def test_captured_run(device):
    """Rotation, store, load and a split step in a graph, replayed with new data and eager calls between: as the eager run."""
    S, H, Hk, D, n = 2, 8, 2, 64, 1500
    g = torch.Generator().manual_seed(9)
    freq = frequencies(32).cuda()
    gate = torch.zeros(H, device="cuda")
    k, v = (torch.empty(S, Hk, n, D, dtype=BF, device="cuda") for _ in range(2))
    q1, k1, v1 = (torch.empty(S, h, D, dtype=BF, device="cuda") for h in (H, Hk, Hk))
    count = torch.tensor([n, 900], dtype=torch.int32, device="cuda")
    cache = Cache(S, Hk, D, 16, 100, BF, False, 2)

    def one():
        kt, _ = pa.pi_attn_rotate(k, None, None, freq)
        pa.pi_attn_paged_store(kt, v, cache.k, cache.v, cache.table, count=count)
        out = pa.pi_attn_decode_step_paged(count, q1, k1, v1, cache.k, cache.v, cache.table, gate, 1400, 1450, freq=freq)
        return (kt, out, *pa.pi_attn_paged_load(cache.k, cache.v, cache.table, n + 1, count=count + 1))

    def fill():
        for x in (k, v, q1, k1, v1):
            x.copy_(torch.randn(x.shape, generator=g))

    fill()
    one()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = one()
    for _ in range(3):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        got_now = [x.clone() for x in got]
        for a, b in zip(got_now, one()):
            assert torch.equal(a, b)


def test_streaming_with_pages_given_back(device):
    """A window that moves on: pages behind it are given to the sequence's next positions, and nothing changes."""
    H, D, page, kw = 3, 64, 8, 30
    N = 200
    q, k, v = prompt(1, H, N, D, F, 3)
    gate = torch.zeros(H, device="cuda")
    long = Cache(1, H, D, page, N // page, F, False, 4)
    short = Cache(1, H, D, page, N // page, F, False, 4)
    free = list(range(6))          # six pages hold a window of 30 rows and the new one
    short.k, short.v = short.k[:6].contiguous(), short.v[:6].contiguous()
    short.table.fill_(-1)
    for t in range(N):
        if t % page == 0:
            old = (t - kw) // page - 1   # wholly behind the window
            if old >= 0 and int(short.table[0, old]) >= 0:
                free.append(int(short.table[0, old]))
                short.table[0, old] = -1
            short.table[0, t // page] = free.pop(0)
        n = torch.tensor([t], dtype=torch.int32, device="cuda")
        a, b = (pa.pi_attn_decode_step_paged(n, *(x[:, :, t].contiguous() for x in (q, k, v)), c.k, c.v, c.table, gate, kw, 0)
                for c in (long, short))
        assert torch.equal(a, b), t


def test_training_step_through_the_rotation(device):
    """Gradients of the attention of turned queries and keys, with respect to the unturned ones, against autograd in 64 bits."""
    B, H, N, D, kw, pi = 1, 2, 40, 64, 12, 20
    q, k, v = prompt(B, H, N, D, F, 5)
    g = torch.Generator().manual_seed(6)
    w = torch.randn(B, H, N, D, generator=g).cuda()
    gate = torch.tensor([0.3, -0.7], device="cuda")
    sections, freq = (12, 10, 10), frequencies(32).cuda()
    pos = torch.randint(0, 500, (3, B, N), generator=g, dtype=torch.int32).cuda()
    qt, kt = pa.pi_attn_rotate(q, k, pos, freq, sections)
    out, lse = pa.pi_attn_forward(qt, kt, v, gate, kw, pi, return_lse=True)
    dq, dk, dv, dg = pa.pi_attn_backward(qt, kt, v, gate, kw, pi, out, lse, w)
    dq, dk = pa.pi_attn_rotate_backward(dq, dk, pos, freq, sections)

    leaves = [x.cpu().double().requires_grad_() for x in (q, k, v)]
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(sections))
    angle = (pos.cpu().double()[axis] * freq.cpu().double()[:, None, None]).permute(1, 2, 0)[:, None]
    z = torch.polar(torch.ones_like(angle), angle)

    def turn(x):
        y = torch.complex(x[..., :32], x[..., 32:]) * z
        return torch.cat([y.real, y.imag], -1)

    scores = turn(leaves[0]) @ turn(leaves[1]).transpose(2, 3) / 8.0
    t, j = torch.arange(N)[:, None], torch.arange(N)[None]
    a = 1e-4 + (1 - 2e-4) * torch.sigmoid(gate.cpu().double())[None, :, None, None]
    prior = torch.where(t - j == pi, torch.log(1 - a), torch.log(a))
    seen = ((j <= t) & (t - j <= kw)) | (t - j == pi)
    p = torch.softmax(torch.where(seen, scores + prior, float("-inf")), -1)
    (p @ leaves[2] * w.cpu().double()).sum().backward()
    for got, leaf in zip((dq, dk, dv), leaves):
        # float32 sums of up to 64 products and 40 rows, turned twice: 2^-24 * (64 + 40) of the largest gradient, times ten
        # for the cancellation in the softmax's derivative
        assert (got.cpu().double() - leaf.grad).abs().max() <= 2.0 ** -24 * 104 * 10 * leaf.grad.abs().max()
