"""The launches that full batches and long prefixes take, sampled sequences against
the definition: reads past the caches, wavefronts by the launch, every shape of
work-group over the prefix."""
import numpy as np
import pytest
import torch

from tests.cached_ref import Step, f64, quantise, value_of
from tests.test_gpu_decode_cached import Problem

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def check_some(p, seqs):
    """One step, of which the sequences `seqs` are compared."""
    new = []
    for x in (p.kn, p.vn):
        codes, byte = quantise(x)
        new.append(np.ldexp(codes, byte.astype(np.int64)[..., None] - 127) if p.quant else f64(x))
    shared = [value_of(c, e) if p.quant else f64(c) for c, e in zip(p.shared, p.shared_exp)]
    rows = []
    for s in seqs:
        n = int(p.lens_np[s])
        own = [value_of(c[s, :, :n], e[s, :, :n]) if p.quant else f64(c[s, :, :n]) for c, e in zip(p.own, p.own_exp)]
        rows.append([np.concatenate([a, b, c[s][:, None]], 1) for a, b, c in zip(shared, own, new)])
    want = Step(p.q[seqs], p.gate, p.k, p.pi, p.clamp, rows, p.dtype, p.plen)
    out = p.run()
    want.check(out[seqs], p.lse[seqs])
    assert bool(torch.isfinite(out).all()) and torch.equal(p.len_out, p.lens + 1)
    for table, exp, x in zip(p.own, p.own_exp, new):
        for s in seqs:
            n = int(p.lens_np[s])
            got = value_of(table[s, :, n], exp[s, :, n]) if p.quant else f64(table[s, :, n])
            assert np.array_equal(got, x[s])


def sampled(S, m):
    return sorted({0, S - 1, *np.random.default_rng(S).integers(0, S, m).tolist()})


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [9, 20, 33, 60, 100, 130, 200])
@pytest.mark.parametrize("clamp", [0.0, 6.0])
def test_prefix_past_the_caches(device, dtype, quant, D, S, clamp):
    """14 MB of prefix rows and more, windows that begin in the middle of tiles and a last tile that is not whole."""
    es = 1 if quant else 4 if dtype == torch.float32 else 2
    H = 10
    k = (14 << 20) // (2 * H * D * es)
    plen, cap = k + 77, 45
    assert 2 * H * k * D * es > 12 << 20
    p = Problem(dtype, quant, S, H, D, plen, cap, k, k + 50, [(7 * s) % cap for s in range(S)], clamp)
    check_some(p, sampled(S, 2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k", [0, 12, 100, 520])
def test_full_batches(device, dtype, quant, D, k):
    """2048 (s, h) without a prefix."""
    S, H, cap = 64, 32, k + 40
    p = Problem(dtype, quant, S, H, D, 0, cap, k, k + 20, [cap - 1 - s % 35 for s in range(S)], clamp=5.0 if k == 12 else 0.0)
    check_some(p, sampled(S, 4))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("plen", [20, 1700])   # read by each sequence, in chunks
@pytest.mark.parametrize("cap", [9, 50, 300, 700])
def test_full_batches_behind_a_prefix(device, dtype, quant, D, plen, cap):
    S, H = 64, 32
    p = Problem(dtype, quant, S, H, D, plen, cap, plen + cap, 0, [cap - 1 - s % min(cap, 40) for s in range(S)])
    check_some(p, sampled(S, 2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("cap", [50, 200, 900])
def test_small_batches_behind_a_prefix(device, dtype, quant, cap):
    """Below 2048 (s, h): four wavefronts, eight from 33 loads of own rows on."""
    p = Problem(dtype, quant, 12, 16, 128, 2000, cap, 1900 + cap, 0, [cap - 1 - s for s in range(12)])
    check_some(p, sampled(12, 3))
