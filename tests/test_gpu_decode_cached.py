"""The decode step over quantised caches and the one behind a shared prefix,
against the definition in 64 bits over the rows as they are stored."""
import numpy as np
import pytest
import torch

import paper_2511_10696_amd as pa
from tests.cached_ref import E4M3, Step, f64, quantise, value_of

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


class Problem:
    """S sequences of lens[s] own rows (cap at most) behind plen shared ones, every row that no window holds poisoned."""

    def __init__(self, dtype, quant, S, H, D, plen, cap, k, pi, lens, clamp=0.0, per_seq=False, seed=1, spare=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.quant, self.S, self.H, self.D = dtype, quant, S, H, D
        self.plen, self.cap, self.k, self.pi, self.clamp = plen, cap, k, pi, clamp
        rnd = lambda *s: (torch.randn(s, generator=g, device="cuda") * 1.5).to(dtype)
        self.q, self.kn, self.vn = rnd(S, H, D), rnd(S, H, D), rnd(S, H, D)
        self.gate = torch.rand((S, H) if per_seq else (H,), generator=g, device="cuda") * 2 - 1
        self.lens_np = np.array(lens, np.int32)
        self.lens = torch.tensor(self.lens_np, device="cuda")
        own, shared = [rnd(S, H, cap, D) for _ in range(2)], [rnd(H, plen + spare, D) for _ in range(2)]
        used = np.zeros(plen, bool)
        for s, n in enumerate(self.lens_np):
            for x in own:
                seen = np.zeros(cap, bool)
                if 0 <= n < cap:
                    t = plen + n
                    at = list(range(max(0, t - k), t)) + ([t - pi] if pi > k and t >= pi else [])
                    seen[[j - plen for j in at if j >= plen]] = True
                    used[[j for j in at if j < plen]] = True
                x[s][:, torch.tensor(~seen, device="cuda")] = float("nan")
        for x in shared:
            x[:, plen:] = float("nan")
            x[:, :plen][:, torch.tensor(~used, device="cuda")] = float("nan")
        if quant:
            self.own, self.own_exp = zip(*(self.cached(x) for x in own))
            self.long, self.long_exp = zip(*(self.cached(x) for x in shared))
            self.shared_exp = [x[:, :plen] for x in self.long_exp]
        else:
            self.own, self.long, self.own_exp, self.shared_exp = own, shared, [None] * 2, [None] * 2
        self.shared = [x[:, :plen] for x in self.long]

    @staticmethod
    def cached(x):
        y = x[None] if x.dim() == 3 else x
        c = torch.empty(y.shape, dtype=E4M3, device="cuda")
        e = torch.empty(y.shape[:3], dtype=torch.uint8, device="cuda")
        pa.pi_attn_cache_store(y, y, c, c.clone(), e, e.clone())
        return (c[0], e[0]) if x.dim() == 3 else (c, e)

    def run(self, lse=True, **kw):
        self.lse = torch.full((self.S, self.H), 5.0, device="cuda") if lse else None
        self.len_out = torch.empty_like(self.lens)
        kw = dict(logit_clamp=self.clamp, lse=self.lse, len_out=self.len_out, **kw)
        if self.plen == 0 and self.quant:
            return pa.pi_attn_decode_step_e4m3(self.lens, self.q, self.kn, self.vn, *self.own, *self.own_exp, self.gate,
                                               self.k, self.pi, **kw)
        return pa.pi_attn_decode_step_prefix(
            self.lens, self.q, self.kn, self.vn, *self.shared, *self.own, self.gate, self.k, self.pi,
            k_prefix_exp=self.shared_exp[0], v_prefix_exp=self.shared_exp[1], k_exp=self.own_exp[0],
            v_exp=self.own_exp[1], **kw)

    def expected(self):
        """Of the state before the step."""
        rows = []
        shared = [value_of(c, e) if self.quant else f64(c) for c, e in zip(self.shared, self.shared_exp)]
        own = [value_of(c, e) if self.quant else f64(c) for c, e in zip(self.own, self.own_exp)]
        self.new = []
        for x in (self.kn, self.vn):
            codes, byte = quantise(x)
            self.new.append(np.ldexp(codes, byte.astype(np.int64)[..., None] - 127) if self.quant else f64(x))
        for s, n in enumerate(self.lens_np):
            ok = 0 <= n < self.cap
            rows.append([np.concatenate([a, b[s][:, :n], c[s][:, None]], 1) for a, b, c in zip(shared, own, self.new)]
                        if ok else None)
        return Step(self.q, self.gate, self.k, self.pi, self.clamp, rows, self.dtype, self.plen)

    def check(self, **kw):
        want = self.expected()
        before = [x.view(torch.uint8).clone() for x in (*self.own, *self.shared) ]
        out = self.run(**kw)
        torch.cuda.synchronize()
        want.check(out, self.lse)
        lens = [n + (1 if 0 <= n < self.cap else 0) for n in self.lens_np.tolist()]
        assert self.len_out.tolist() == lens
        # the new rows are there, and nothing else has changed
        for i, (c, e) in enumerate(zip(self.own, self.own_exp)):
            for s, n in enumerate(self.lens_np.tolist()):
                if not 0 <= n < self.cap:
                    assert torch.equal(c.view(torch.uint8)[s], before[i][s])
                    continue
                got = value_of(c[s, :, n], e[s, :, n]) if self.quant else f64(c[s, :, n])
                assert np.array_equal(got, self.new[i][s])
                rest = torch.arange(self.cap, device="cuda") != n
                assert torch.equal(c.view(torch.uint8)[s][:, rest], before[i][s][:, rest])
        for x, b in zip(self.shared, before[2:]):
            assert torch.equal(x.view(torch.uint8), b)
        return out


def edges(k, cap):
    """Lengths around the window's, empty and invalid ones among them."""
    return [0, 1, min(max(k - 1, 2), cap - 1), min(k, cap - 1), min(k + 1, cap - 1), cap - 1, cap, -1]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k", [0, 1, 4, 31, 33, 130, 520])
@pytest.mark.parametrize("pi,clamp", [(0, 0.0), (1, 3.0), (70, 0.0)])   # no partner, next to the window, further
def test_e4m3(device, dtype, D, k, pi, clamp):
    cap = k + 80
    Problem(dtype, True, 8, 3, D, 0, cap, k, k + pi if pi else 0, edges(k, cap), clamp, per_seq=bool(pi)).check()


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("k", [4096, 9000])
def test_e4m3_long_windows_split(device, dtype, D, k):
    """Few (s, h) with long windows: over several work-groups; lengths that leave most of them without rows."""
    p = Problem(dtype, True, 4, 2, D, 0, k + 30, k, k + 9, [k + 29, 5, 0, k + 30])
    assert pa.pi_attn_decode_workspace(dtype, 4, 2, D, 0, k + 30, k) > 0
    p.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 8, 17, 33, 40, 65, 130])   # each side of the groups of queries
@pytest.mark.parametrize("plen,k,pi", [(200, 1000, 0), (333, 150, 190), (64, 63, 64), (1, 1, 2)])
def test_prefix(device, dtype, quant, D, S, plen, k, pi):
    cap = 60
    lens = (edges(k, cap) * (S // 8 + 1))[:S] if S > 1 else [7]
    Problem(dtype, quant, S, 3, D, plen, cap, k, pi, lens, per_seq=S > 20).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("k,pi,clamp", [(40, 41, 2.5), (40, 700, 0.0), (2000, 0, 2.5), (0, 300, 0.0), (0, 0, 0.0)])
def test_prefix_windows(device, dtype, quant, k, pi, clamp):
    """Windows that end in the prefix, leave it, never reach it; partners in it and behind it."""
    lens = [0, 1, 2, 39, 40, 41, 42, 200, 299, 300, 301]
    Problem(dtype, quant, len(lens), 2, 64, 500, 320, k, pi, lens, clamp).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S", [3, 70])
def test_prefix_of_many_chunks(device, dtype, quant, S):
    """A long prefix of few heads, with windows that begin in the middle of chunks; own windows are split too."""
    k = 5000
    lens = [(i * 397) % 4600 for i in range(S)]
    Problem(dtype, quant, S, 1, 128, 4500, 4610, k, 7000, lens).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
def test_no_prefix_rows(device, dtype, quant):
    """plen = 0: the own rows alone; with caches in the working type as pi_attn_decode_step."""
    p = Problem(dtype, quant, 8, 2, 64, 0, 90, 40, 60, edges(40, 90))
    if quant:
        empty = torch.empty((2, 0, 64), dtype=E4M3, device="cuda")
        e = torch.empty((2, 0), dtype=torch.uint8, device="cuda")
        a = pa.pi_attn_decode_step_prefix(p.lens, p.q, p.kn, p.vn, empty, empty, *[x.clone() for x in p.own], p.gate, 40,
                                          60, k_prefix_exp=e, v_prefix_exp=e, k_exp=p.own_exp[0].clone(),
                                          v_exp=p.own_exp[1].clone())
        assert torch.equal(a.nan_to_num(9), p.run().nan_to_num(9))
        return
    p.check()
    again = pa.pi_attn_decode_step(p.lens, p.q, p.kn, p.vn, *p.own, p.gate, 40, 60)
    got = p.run()
    assert np.allclose(f64(got), f64(again), rtol=2.0 ** -7, atol=1e-5, equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S,D,H", [(5, 64, 2), (50, 64, 2), (20, 128, 80), (50, 128, 40), (100, 128, 20), (140, 64, 20)])
def test_masked_rows_that_are_not_finite(device, dtype, quant, S, D, H):
    """A prefix row with NaN and infinities in the windows of some sequences only: those get NaN, the others their values."""
    plen, k, cap = 300, 200, 150
    lens = [(i * 29) % cap for i in range(S)]
    p = Problem(dtype, quant, S, H, D, plen, cap, k, 0, lens)
    bad = 170   # met by the sequences with plen + n - k <= 170, n <= 70
    clean = p.expected()
    for x in p.shared:
        if quant:
            x.view(torch.uint8)[:, bad, 7] = 0x7f
            x.view(torch.uint8)[:, bad, 9] = 0xff
        else:
            x[:, bad, 7], x[:, bad, 9] = float("nan"), float("inf")
    out = p.run()
    hit = torch.tensor([n <= bad - plen + k for n in lens], device="cuda")
    assert bool(hit.any()) and not bool(hit.all())
    assert bool(torch.isnan(out[hit]).any(-1).all()) and bool(torch.isnan(p.lse[hit]).all())
    clean.out[hit.cpu().numpy()] = np.nan
    clean.lse[hit.cpu().numpy()] = np.nan
    keep = ~hit.cpu().numpy()
    assert np.all(np.abs(f64(out)[keep] - clean.out[keep]) <= clean.out_tol[keep])
    assert np.all(np.abs(f64(p.lse)[keep] - clean.lse[keep]) <= clean.lse_tol[keep])


@pytest.mark.parametrize("quant", [False, True])
def test_value_rows_that_are_not_finite(device, quant):
    """Infinite or NaN values of one dim of a masked row, the keys finite: only that dim of the sequences that meet it."""
    plen, k, cap, S, bad = 300, 200, 150, 9, 170
    lens = [(i * 29) % cap for i in range(S)]
    p = Problem(torch.bfloat16, quant, S, 2, 128, plen, cap, k, 0, lens)
    want = p.expected()
    v = p.shared[1]
    if quant:
        v.view(torch.uint8)[:, bad, 77] = 0x7f
    else:
        v[:, bad, 77] = float("inf")
    out = f64(p.run())
    for s, n in enumerate(lens):
        if n <= bad - plen + k:
            assert not np.isfinite(out[s, :, 77]).any()
            out[s, :, 77] = want.out[s, :, 77]
    assert np.all(np.abs(out - want.out) <= want.out_tol)
    assert np.all(np.abs(f64(p.lse) - want.lse) <= want.lse_tol)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("plen", [400, 4000])
def test_one_row_dominates(device, quant, plen):
    """A prefix row with nearly all of the weight: its value row, to the output's rounding."""
    p = Problem(torch.bfloat16, quant, 20, 2, 64, plen, 30, 5000, 0, [i % 30 for i in range(20)])
    q = p.q.float()
    key = torch.where(q[:1] > 0, 40.0, -40.0)
    p.q.copy_(torch.sign(q[:1]).expand_as(q))   # every sequence asks for the same row
    rows = p.shared[0]
    if quant:
        c, e = Problem.cached(key.view(1, 2, 1, 64).to(torch.bfloat16))
        rows.view(torch.uint8)[:, 123] = c.view(torch.uint8)[0, :, 0]
        p.shared_exp[0][:, 123] = e[0, :, 0]
    else:
        rows[:, 123] = key[0].to(torch.bfloat16)
    value = value_of(p.shared[1][:, 123], p.shared_exp[1][:, 123]) if quant else f64(p.shared[1][:, 123])
    out = f64(p.run())
    assert np.all(np.abs(out - value) <= 2.0 ** -8 * np.abs(value) + 1e-12)


@pytest.mark.parametrize("quant", [False, True])
def test_workspace_streams_and_graphs(device, quant):
    """The caller's workspace, whatever it holds; another stream; steps captured two to a graph and replayed with the
    caches growing, against eager steps: the same bits."""
    S, H, D, plen, cap, k, pi = 6, 4, 128, 700, 64, 650, 690
    mk = lambda: Problem(torch.bfloat16, quant, S, H, D, plen, cap, k, pi, [0, 3, 9, 20, 31, 5], seed=5)
    a, b = mk(), mk()
    for x in (a, b):   # rows that later steps meet
        for t in (*x.own, *x.long):
            y = torch.randn(t.shape, generator=torch.Generator(device="cuda").manual_seed(t.numel()), device="cuda")
            t.view(torch.uint8).copy_(y.to(t.dtype).view(torch.uint8))
        if quant:
            for t in (*x.own_exp, *x.long_exp):
                t.fill_(127)
    need = pa.pi_attn_decode_workspace(torch.bfloat16, S, H, D, plen, cap, k)
    work = torch.full((need + 5,), float("nan"), device="cuda")
    eager = []
    for _ in range(6):
        eager.append(a.run().clone())
        a.lens.copy_(a.len_out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = b.run(work=work)
    side.synchronize()
    assert torch.equal(first, eager[0])
    other = torch.empty_like(b.lens)
    outs = [torch.empty_like(first) for _ in range(2)]

    def step(src, dst, out):
        b.lens, keep = src, b.lens
        b.len_out = dst
        args = dict(len_out=dst, out=out, work=work)
        pa.pi_attn_decode_step_prefix(src, b.q, b.kn, b.vn, *b.shared, *b.own, b.gate, k, pi,
                                      k_prefix_exp=b.shared_exp[0], v_prefix_exp=b.shared_exp[1], k_exp=b.own_exp[0],
                                      v_exp=b.own_exp[1], **args)
        b.lens = keep

    torch.cuda.synchronize()
    lens = b.lens
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(lens, other, outs[0])
        step(other, lens, outs[1])
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], eager[2 * i]) and torch.equal(outs[1], eager[2 * i + 1])


def test_from_prompt_to_steps(device):
    """As a server runs them: a prompt in two chunks (the second one attends the first as it was stored), its cache as the
    prefix of several answers, steps behind it; against the steps of as many full caches."""
    H, D, k, pi, n1, n2, S, steps = 4, 128, 300, 350, 256, 201, 5, 3
    g = torch.Generator(device="cuda").manual_seed(41)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)
    gate = torch.rand(H, generator=g, device="cuda") * 2 - 1
    cap = 600
    kc, vc = (torch.zeros((1, H, cap, D), device="cuda").to(E4M3) for _ in range(2))
    ke, ve = (torch.zeros((1, H, cap), dtype=torch.uint8, device="cuda") for _ in range(2))
    q1, k1, v1, q2, k2, v2 = (rnd(1, H, n, D) for n in (n1, n1, n1, n2, n2, n2))
    pa.pi_attn_forward(q1, k1, v1, gate, k, pi)
    pa.pi_attn_cache_store(k1, v1, kc, vc, ke, ve)
    pa.pi_attn_cache_store(k2, v2, kc, vc, ke, ve, torch.tensor([n1], dtype=torch.int32, device="cuda"))
    lk, lv = pa.pi_attn_cache_load(kc, vc, ke, ve, n1 + n2)
    chunk = pa.pi_attn_forward_shard(q2, lk, lv, gate, k, pi, n1 + n2, n1, 0)
    q = torch.cat([torch.zeros_like(q1), q2], 2)
    whole = pa.pi_attn_forward(q, lk, lv, gate, k, pi)
    assert torch.equal(chunk, whole[:, :, n1:])
    plen, own = n1 + n2, 8
    kp, vp, kpe, vpe = kc[0, :, :plen], vc[0, :, :plen], ke[0, :, :plen], ve[0, :, :plen]
    oc = [torch.zeros((S, H, own, D), device="cuda").to(E4M3) for _ in range(2)]
    oe = [torch.zeros((S, H, own), dtype=torch.uint8, device="cuda") for _ in range(2)]
    fc = [x.expand(S, -1, -1, -1).contiguous() for x in (kc.view(torch.uint8), vc.view(torch.uint8))]
    fc = [x.view(E4M3) for x in fc]
    fe = [x.expand(S, -1, -1).contiguous() for x in (ke, ve)]
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    for i in range(steps):
        qn, kn, vn = rnd(S, H, D), rnd(S, H, D), rnd(S, H, D)
        a = pa.pi_attn_decode_step_prefix(lens, qn, kn, vn, kp, vp, *oc, gate, k, pi, k_prefix_exp=kpe, v_prefix_exp=vpe,
                                          k_exp=oe[0], v_exp=oe[1])
        b = pa.pi_attn_decode_step_e4m3(lens + plen, qn, kn, vn, *fc, *fe, gate, k, pi)
        lens = lens + 1
        # both within their bounds: half a step of bf16 each and, of the prefix' weights, another; values up to 5
        assert float((a.float() - b.float()).abs().max()) <= 3 * 2.0 ** -8 * 5
        for x, y in ((oc[0], fc[0]), (oc[1], fc[1])):
            assert torch.equal(x.view(torch.uint8)[:, :, :i + 1], y.view(torch.uint8)[:, :, plen:plen + i + 1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("S,H,D", [(20, 40, 64), (40, 40, 64), (60, 40, 128), (70, 30, 64), (140, 16, 64), (33, 40, 128), (130, 16, 128)])
def test_prefix_in_chunks(device, dtype, quant, S, H, D):
    """Prefixes that are taken in chunks: every number of groups of queries, a window in the middle of a tile, some windows
    that end before the last tile."""
    plen, cap, k, pi = 700, 40, 600, 640
    lens = [(7 * s) % cap for s in range(S)]
    p = Problem(dtype, quant, S, H, D, plen, cap, k, pi, lens, clamp=6.0 if S % 20 else 0.0)
    assert pa.pi_attn_decode_workspace(dtype, S, H, D, plen, cap, k) > 0
    p.check()


def test_windows_that_have_left_the_prefix(device):
    """Lengths past the window: no row of the prefix but the partners, whose chunks have nothing to do."""
    S, H, k = 40, 40, 300
    Problem(torch.bfloat16, True, S, H, 64, 2000, 700, k, 900, [350 + 8 * s for s in range(S)]).check()


@pytest.mark.parametrize("quant", [False, True])
def test_same_bits_by_the_python_marshalling(device, quant):
    """A given stream takes the Python marshalling: the same kernels, the same bits, with its own workspace."""
    mk = lambda: Problem(torch.bfloat16, quant, 33, 40, 128, 700, 40, 600, 640, [s for s in range(33)])
    a, b = mk(), mk()
    x = a.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = b.run(stream=side)
    side.synchronize()
    assert torch.equal(x, y) and torch.equal(a.lse, b.lse) and torch.equal(a.len_out, b.len_out)


def test_workspace_of_a_given_stream(device, monkeypatch):
    """Its memory comes from the pool of the stream that the step runs on: what another stream let go may still be in use
    there."""
    p = Problem(torch.bfloat16, True, 33, 40, 128, 700, 40, 600, 640, [s for s in range(33)])
    side, empty, streams = torch.cuda.Stream(), torch.empty, []

    def note(*a, **kw):
        streams.append(torch.cuda.current_stream())
        return empty(*a, **kw)

    side.wait_stream(torch.cuda.current_stream())
    monkeypatch.setattr(torch, "empty", note)
    p.run(stream=side)
    monkeypatch.undo()
    assert streams == [side]
    side.synchronize()


def test_integers_beyond_32_bits(device):
    """Refused, where their lowest 32 bits would be a valid window, period or count."""
    p = Problem(torch.bfloat16, True, 2, 3, 64, 50, 20, 30, 0, [1, 2])
    before = [x.view(torch.uint8).clone() for x in p.own]
    big = 1 << 32
    for k, pi in ((big + 30, 0), (30, big)):
        with pytest.raises(ValueError, match="32 bits"):
            pa.pi_attn_decode_step_prefix(p.lens, p.q, p.kn, p.vn, *p.shared, *p.own, p.gate, k, pi,
                                          k_prefix_exp=p.shared_exp[0], v_prefix_exp=p.shared_exp[1], k_exp=p.own_exp[0],
                                          v_exp=p.own_exp[1])
        with pytest.raises(ValueError, match="32 bits"):
            pa.pi_attn_decode_step_e4m3(p.lens, p.q, p.kn, p.vn, *p.own, *p.own_exp, p.gate, k, pi)
    with pytest.raises(ValueError, match="32 bits"):
        pa.pi_attn_cache_load(*p.own, *p.own_exp, big + 3)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y.view(torch.uint8)) for x, y in zip(before, p.own))


def test_refusals(device):
    """What the binding refuses, each with one thing wrong."""
    S, H, D, plen, cap = 2, 3, 64, 50, 20
    p = Problem(torch.bfloat16, True, S, H, D, plen, cap, 30, 0, [1, 2])
    before = [x.view(torch.uint8).clone() for x in p.own]

    def step(**kw):
        a = dict(len_in=p.lens, q=p.q, kn=p.kn, vn=p.vn, kp=p.shared[0], vp=p.shared[1], kc=p.own[0], vc=p.own[1],
                 gate=p.gate, kpe=p.shared_exp[0], vpe=p.shared_exp[1], ke=p.own_exp[0], ve=p.own_exp[1], k=30, pi=0, more={})
        a.update(kw)
        return pa.pi_attn_decode_step_prefix(a["len_in"], a["q"], a["kn"], a["vn"], a["kp"], a["vp"], a["kc"], a["vc"],
                                             a["gate"], a["k"], a["pi"], k_prefix_exp=a["kpe"], v_prefix_exp=a["vpe"],
                                             k_exp=a["ke"], v_exp=a["ve"], **a["more"])

    plain = torch.zeros(S, H, cap, D, device="cuda", dtype=torch.bfloat16)
    for kw, error in [
        (dict(ke=None), ValueError), (dict(vpe=None), ValueError), (dict(kpe=p.shared_exp[0].contiguous()), ValueError),
        (dict(kp=p.shared[0][:, :, ::2]), ValueError), (dict(kp=p.shared[0].contiguous()), ValueError),
        (dict(kp=p.shared[0][:2]), ValueError), (dict(kc=plain, vc=plain), ValueError), (dict(len_in=p.lens.long()), ValueError),
        (dict(q=p.q.half()), ValueError), (dict(kn=p.kn.float()), ValueError), (dict(gate=p.gate.double()), TypeError),
        (dict(gate=torch.zeros(H + 1, device="cuda")), ValueError), (dict(k=-1), pa.PiAttnError), (dict(pi=-1), pa.PiAttnError),
        (dict(more=dict(scale=0.0)), pa.PiAttnError), (dict(more=dict(logit_clamp=float("nan"))), pa.PiAttnError),
        (dict(more=dict(len_out=p.lens)), pa.PiAttnError), (dict(more=dict(out=p.q.float())), ValueError),
        (dict(more=dict(lse=torch.zeros(S, device="cuda"))), ValueError), (dict(more=dict(work=torch.zeros(9))), RuntimeError),
        (dict(ke=p.own_exp[0].int()), ValueError), (dict(kc=p.own[0].transpose(0, 1)), ValueError),
    ]:
        with pytest.raises(error):
            step(**kw)
    k = torch.zeros(S, H, 5, D, device="cuda")
    for args, error in [((k, k.half()), ValueError), ((k.half(), k.half()), TypeError), ((k[:, :, :, :32], k[:, :, :, :32]), ValueError),
                        ((k[:1], k[:1]), ValueError), ((k, k.transpose(0, 1).contiguous().transpose(0, 1)), ValueError)]:
        with pytest.raises(error):
            pa.pi_attn_cache_store(*args, *p.own, *p.own_exp)
    with pytest.raises(ValueError):
        pa.pi_attn_cache_store(k, k, *p.own, *p.own_exp, start=p.lens.long())
    with pytest.raises(ValueError):
        pa.pi_attn_cache_load(*p.own, *p.own_exp, -1)
    with pytest.raises(ValueError):
        pa.pi_attn_cache_load(*p.own, *p.own_exp, 4, k=k[:, :, :4], v=k[:, :, :4].transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(pa.PiAttnError):   # rows that lie on one another
        one = torch.zeros(1, 1, 1, D, device="cuda").expand(S, H, 5, D)
        pa.pi_attn_cache_load(*p.own, *p.own_exp, 5, k=one, v=one.clone().as_strided(one.shape, one.stride()))
    with pytest.raises(TypeError):
        pa.pi_attn_cache_load(*p.own, *p.own_exp, 4, dtype=torch.float16)
    torch.cuda.synchronize()
    for x, y in zip(p.own, before):
        assert torch.equal(x.view(torch.uint8), y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("what", ["key", "value"])
@pytest.mark.parametrize("S,D", [(5, 64), (5, 128), (20, 64), (40, 128), (70, 64), (140, 128)])
def test_not_finite_in_chunks(device, dtype, quant, what, S, D):
    """The same where the prefix is taken in chunks: rows with NaN and infinities that only some windows hold; the other
    sequences of the work-group keep their values."""
    plen, cap, H, bad = (3000, 150, 2, 150) if D == 64 else (1600, 150, 2, 150)
    k = plen - 100
    lens = [(s * 29) % cap for s in range(S)]
    p = Problem(dtype, quant, S, H, D, plen, cap, k, 0, lens)
    assert pa.pi_attn_decode_workspace(dtype, S, H, D, plen, cap, k) > 0
    want = p.expected()
    x = p.shared[what == "value"]
    for row, dim in ((bad, 33), (bad + 1, 33), (bad - 40, 5)):
        if quant:
            x.view(torch.uint8)[:, row, dim] = 0x7f if row == bad else 0xff
        else:
            x[:, row, dim] = float("nan") if row == bad else float("-inf")
    out, lse = f64(p.run()), f64(p.lse)
    for s, n in enumerate(lens):
        lo = plen + n - k
        if what == "key" and lo <= bad:   # the NaN logit, or one that is infinite of either sign
            assert np.isnan(out[s]).all() and np.isnan(lse[s]).all()
            continue
        if what == "value":
            for dim, rows in ((33, (bad, bad + 1)), (5, (bad - 40,))):
                if lo <= max(rows):
                    assert not np.isfinite(out[s, :, dim]).any()
                    out[s, :, dim] = want.out[s, :, dim]
        if what == "key" and lo <= bad + 1:
            continue
        assert np.all(np.abs(out[s] - want.out[s]) <= want.out_tol[s]), s
        assert np.all(np.abs(lse[s] - want.lse[s]) <= want.lse_tol[s]), s


def test_scale_past_the_largest_float(device):
    """A value row whose scale byte makes its codes infinite, in windows of some sequences: the others keep their values."""
    S, D, H, plen, cap, bad = 40, 128, 2, 1600, 150, 150
    k = plen - 100
    lens = [(s * 29) % cap for s in range(S)]
    p = Problem(torch.bfloat16, True, S, H, D, plen, cap, k, 0, lens)
    want = p.expected()
    p.shared[1].view(torch.uint8)[:, bad] = 0x7e   # 448 * 2^(254 - 127)
    p.shared_exp[1][:, bad] = 254
    out = f64(p.run())
    for s, n in enumerate(lens):
        if plen + n - k <= bad:
            assert not np.isfinite(out[s]).any()
        else:
            assert np.all(np.abs(out[s] - want.out[s]) <= want.out_tol[s]), s
