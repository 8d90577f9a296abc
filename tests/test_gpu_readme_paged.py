"""The README's example of rotary positions, shared key heads and pages runs as it is printed, and its results are those of the
formula in float32."""
import os
import re

import pytest
import torch

import paper_2511_10696_amd as pa
from tests.conftest import ROOT

pytestmark = pytest.mark.gpu


def test_example(device):
    with open(os.path.join(ROOT, "README.md")) as f:
        code, = (x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "pi_attn_paged_store" in x)
    B, H, Hk, N, D, window, period, theta = 2, 4, 2, 150, 128, 40, 64, 1e4
    g = torch.Generator().manual_seed(1)

    def rand(*shape):
        return torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()

    n_pages = 8
    names = dict(pa=pa, torch=torch, B=B, H=H, Hk=Hk, N=N, D=D, window=window, period=period, theta=theta, n_pages=n_pages,
                 q=rand(B, H, N, D), k=rand(B, Hk, N, D), v=rand(B, N, Hk, D).transpose(1, 2), dout=rand(B, H, N, D),
                 gate=torch.linspace(-1, 1, H, device="cuda"), pos=torch.randint(0, 99, (3, B, N), generator=g, dtype=torch.int32).cuda(),
                 table=torch.randperm(n_pages, generator=g, dtype=torch.int32).view(B, n_pages // B).cuda(),
                 start=torch.zeros(B, dtype=torch.int32, device="cuda"), lengths=torch.full((B,), N, dtype=torch.int32, device="cuda"),
                 q_new=rand(B, H, D), k_new=rand(B, Hk, D), v_new=rand(B, Hk, D),
                 pos_new=torch.randint(0, 99, (3, B), generator=g, dtype=torch.int32).cuda(),
                 new_lengths=torch.zeros(B, dtype=torch.int32, device="cuda"))
    r = dict(names)
    # the store takes v in k's layout
    r["v"] = names["v"].contiguous()
    exec(code, r)
    assert r["new_lengths"].tolist() == [N + 1] * B

    # the same on the whole sequence with the new row, in float64 on the CPU
    f = {x: names[x].cpu().double() for x in ("q", "k", "v", "q_new", "k_new", "v_new", "dout", "gate")}
    for x in ("q", "k", "v"):
        f[x].requires_grad_()
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(r["sections"]))
    freq = r["freq"].cpu().double()

    def turn(x, pos):
        z = torch.polar(torch.ones(()).double(), pos.cpu().double()[axis].movedim(0, -1) * freq)
        y = torch.complex(x[..., :D // 2], x[..., D // 2:]) * z[:, None]
        return torch.cat([y.real, y.imag], -1)

    alpha = 1e-4 + (1 - 2e-4) * torch.sigmoid(f["gate"])[None, :, None, None]

    def attend(q, k, v, t):
        """Rows t [n] of a sequence."""
        j = torch.arange(k.shape[2])[None]
        t = t[:, None]
        prior = torch.where(t - j == period, torch.log(1 - alpha), torch.log(alpha))
        seen = ((j <= t) & (t - j <= window)) | (t - j == period)
        s = q @ k.repeat_interleave(H // Hk, 1).transpose(2, 3) / D ** 0.5 + prior
        return torch.softmax(torch.where(seen, s, float("-inf")), -1) @ v.repeat_interleave(H // Hk, 1)

    kt = turn(f["k"], names["pos"])
    out = attend(turn(f["q"], names["pos"]), kt, f["v"], torch.arange(N))
    # bf16 rows, weights and results: a few half steps (2^-8) of values up to 4
    assert (r["out"].cpu().double() - out).abs().max() <= 6 * 2.0 ** -8 * 4
    (out * f["dout"]).sum().backward()
    for x, got in (("q", r["dq"]), ("k", r["dk"]), ("v", r["dv"])):
        assert (got.cpu().double() - f[x].grad).abs().max() <= 6 * 2.0 ** -8 * f[x].grad.abs().max(), x
    new = [turn(f["q_new"][:, :, None], names["pos_new"][..., None]), turn(f["k_new"][:, :, None], names["pos_new"][..., None])]
    want = attend(new[0], torch.cat([kt, new[1]], 2), torch.cat([f["v"], f["v_new"][:, :, None]], 2), torch.tensor([N]))[:, :, 0]
    # keys rounded to bf16 once turned: logits off by 2^-8 of at most 4, and the result's rounding
    assert (r["out_new"].cpu().double() - want).abs().max() <= 6 * 2.0 ** -8 * 4
