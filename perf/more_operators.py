"""Measured cases of rotary positions and of the paged KV cache.

Each case is one kind of pass:
  rotate  pi_attn_rotate: queries and keys turned by their positions, on one axis or on time, height and width
  back    pi_attn_rotate_backward: the gradients of both, as pi_attn_backward gives them
  store   pi_attn_paged_store: rows of keys and values into a paged cache, the keys turned on the way
  load    pi_attn_paged_load: rows of a paged cache in sequence, as the attention of a prompt's next chunk takes them
  decode  pi_attn_decode_step_paged: a decode step over a paged cache

Rotation: element i < P and element i + D/2 of a row are a pair, turned by the angle pos_a * freq_i, where a is the axis of
pair i: the first pairs belong to axis 0, the next ones to axis 1, and so on.  Pairs from P on stay as they are.

A paged cache holds pages [pages][heads][page][D]; position j of sequence s lies in page table[s][j // page], row j % page.  A
table entry that names no page has no rows.  Quantised pages hold e4m3 codes and a byte b for each row: element d is
code_d * 2^(b - 127), where e = b - 127 is the least integer from -126 on with max |x| <= 448 * 2^e.

With own = False, run() computes the same in elementary torch operations.
"""
import math

import torch

own = False

GATE_EPS = 1e-4
E4M3 = torch.float8_e4m3fn


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


# ---- the cases -----------------------------------------------------------------
def _turn(name, kind, dtype, B, H, Hk, N, D, **more):
    """rotate, back: B sequences of N positions, H query and Hk key heads; rot pairs of a row are turned."""
    c = {"name": name, "kind": kind, "dtype": dtype, "B": B, "H": H, "Hk": Hk, "N": N, "D": D, "rot": D // 2, "axes": 1,
         "far": 0, "theta": 1e4, "layout": "bhnd", "to": dtype}
    c.update(more)
    return c


def _rows(name, kind, dtype, S, Hk, D, n, page, **more):
    """store, load: n rows a sequence behind `behind` others, in pages of page rows."""
    c = {"name": name, "kind": kind, "dtype": dtype, "S": S, "Hk": Hk, "D": D, "n": n, "page": page, "behind": 0,
         "e4m3": False, "rot": 0, "axes": 1, "theta": 1e4, "layout": "shnd", "ragged": False}
    c.update(more)
    return c


def _step(name, dtype, S, H, Hk, D, k, pi, page, lo, hi, **more):
    """decode: sequences of lo to hi rows; where `evict`, the pages before the window are gone for every second one."""
    c = {"name": name, "kind": "decode", "dtype": dtype, "S": S, "H": H, "Hk": Hk, "D": D, "k": k, "pi": pi, "page": page,
         "lo": lo, "hi": hi, "e4m3": False, "rot": 0, "axes": 1, "theta": 1e4, "clamp": 0.0, "evict": False}
    c.update(more)
    return c


def listed():
    return [
        # A layer of a small float32 model: launch latency.
        _turn("rotate_tiny_f32", "rotate", "f32", 1, 2, 2, 33, 64),
        # Prompts with images: positions in time, height and width, q and k as views of the projection's [B][N][H][D] output,
        # shared key heads, a quarter of each row left as it is.
        _turn("rotate_video", "rotate", "bf16", 4, 16, 4, 4000, 128, rot=48, axes=3, layout="bnhd", theta=1e6),
        # A training step of a float32 model with images, odd length.
        _turn("back_video_f32", "back", "f32", 2, 8, 8, 1001, 64, axes=3),
        # A training step of one long sequence; far positions, the float32 gradients of the attention to bf16.
        _turn("back_32k", "back", "f32", 1, 32, 32, 32768, 128, far=200000, theta=1e6, to="bf16"),
        # A batch's new tokens enter the cache of a model whose attention runs elsewhere: latency.
        _rows("store_tokens", "store", "bf16", 64, 8, 128, 1, 16, behind=700, rot=64, ragged=True),
        # Prompts of different lengths, keys turned on the way, views of the projection's [S][n][H][D] output.
        _rows("store_prompts", "store", "bf16", 8, 16, 128, 6000, 64, rot=64, layout="snhd", ragged=True),
        # What was cached of a short prompt, for its next chunk: float32, small odd pages.
        _rows("load_f32", "load", "f32", 3, 4, 64, 301, 5, ragged=True),
        # The same of long prompts in e4m3.
        _rows("load_e4m3", "load", "bf16", 4, 8, 128, 16000, 64, e4m3=True, ragged=True),
        # A decode step of one user.
        _step("decode_1", "bf16", 1, 32, 32, 128, 512, 1024, 16, 1500, 1500, rot=64),
        # A few sequences of odd lengths from empty on, float32, three heads to a key head, small odd pages, the paper's logit
        # clamp, and pages that the window has left behind given back.
        _step("decode_odd_f32", "f32", 7, 12, 4, 64, 100, 101, 5, 0, 332, rot=32, clamp=20.0, evict=True),
        # A full batch of chats with shared key heads, dense in all that they hold.
        _step("decode_64", "bf16", 64, 32, 8, 128, 8192, 0, 64, 2000, 8191, rot=64),
        # Two long documents in e4m3, eight heads to a key head.
        _step("decode_long_e4m3", "bf16", 2, 16, 2, 128, 131072, 0, 128, 100000, 131071, e4m3=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "back", "store", "load", "decode", "decode", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D, Hk, G = rng.choice([64, 128]), rng.choice([1, 2, 5, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
    axes, theta = rng.choice([1, 1, 3]), rng.choice([1e4, 1e6])
    rot = rng.choice([D // 2, D // 2, 3 * D // 8, D // 4 + 1])
    page = rng.choice([16, 32, 64, 128, 1 + rng.randrange(40)])
    if kind in ("rotate", "back"):
        N = _log(rng, 1, 16384)
        B = _log(rng, 1, max(1, min(64, 64 * 16384 * 64 // (N * (G + 1) * Hk * D))))
        c = _turn("", kind, "f32" if kind == "back" else dtype, B, G * Hk, Hk, N, D, rot=rot, axes=axes, theta=theta,
                  far=rng.choice([0, 0, _log(rng, 100, 1000000)]), layout=rng.choice(["bhnd", "bnhd"]), to=dtype)
    elif kind in ("store", "load"):
        n, behind = _log(rng, 1, 16384), rng.choice([0, _log(rng, 1, 2000)])
        S = _log(rng, 1, max(1, min(64, 64 * 16384 * 64 // ((n + behind) * Hk * D))))
        e4m3 = rng.random() < 0.4
        c = _rows("", kind, dtype, S, Hk, D, n, page, behind=behind, e4m3=e4m3, theta=theta, axes=axes,
                  rot=0 if e4m3 or kind == "load" else rot, layout=rng.choice(["shnd", "snhd"]), ragged=rng.random() < 0.5)
    else:
        hi = _log(rng, 1, 32768)
        k = rng.choice([hi + 1, hi + 1, _log(rng, 1, 2048), _log(rng, 1, 2048)])
        pi = rng.choice([0, k + 1, 2 * k, k + 1 + rng.randrange(2 * k)])
        S = _log(rng, 1, max(1, min(64, 32768 * 128 * 8 // ((hi + page) * Hk * D))))
        e4m3 = rng.random() < 0.3
        c = _step("", dtype, S, G * Hk, Hk, D, k, pi, page, rng.choice([0, hi // 2, hi]), hi, e4m3=e4m3, theta=theta,
                  rot=0 if e4m3 else rng.choice([0, rot]), axes=axes, clamp=rng.choice([0.0, 0.0, 20.0]),
                  evict=rng.random() < 0.5)
    del c["name"]
    return c


def _sections(c):
    """How many pairs each axis has."""
    side = 3 * c["rot"] // 8
    return (c["rot"],) if c["axes"] == 1 else (c["rot"] - 2 * side, side, side)


# ---- rows as quantised pages hold them --------------------------------------------
def _quantise(x):
    """Codes (float8) and scale bytes of the rows of x: the scale by the largest finite element."""
    x = x.float()
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)                              # amax = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -126).clamp(min=-126)
    y = torch.where(torch.isfinite(x), torch.ldexp(x, -e[..., None]), math.nan)
    return y.to(E4M3), (e + 127).to(torch.uint8)


def _values(codes, byte):
    return torch.ldexp(codes.float(), byte.to(torch.int32)[..., None] - 127)


# ---- inputs ---------------------------------------------------------------------
def _spread(g, S, lo, hi):
    """S whole numbers, evenly from lo to hi, in the seed's order: the same sum for every seed."""
    v = torch.tensor([lo + (hi - lo) * i // max(1, S - 1) for i in range(S)], dtype=torch.int32)
    return v[torch.randperm(S, generator=g)].cuda()


def _freq(c):
    i = torch.arange(c["rot"], dtype=torch.float64)
    return (c["theta"] ** (-i / c["rot"])).float().cuda()


def _grid(first, n):
    """Positions [3, n] in time, height and width: text, then frames of 12 by 20 patches, one after the other."""
    i = torch.arange(n, dtype=torch.int32)
    text = n // 4
    j = (i - text).clamp(min=0)
    t = torch.where(i < text, i, text + j // 240)
    h = torch.where(i < text, i, text + j // 20 % 12)
    w = torch.where(i < text, i, text + j % 20)
    return torch.stack([t, h, w]) + first


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) * 7919 + 29)
    dt, D = _dtype(c["dtype"]), c["D"]

    def rows(*shape):
        """Keys or values: a few dims larger than the others, as trained projections give them, and rows of unlike size."""
        x = torch.randn(*shape, D, generator=g, device="cuda", dtype=dt)
        dims = torch.where(torch.rand(D, generator=g, device="cuda") < 0.05, 3.0, 1.0)
        size = 0.5 + torch.rand(*shape, 1, generator=g, device="cuda")
        return x.mul_(dims.to(dt)).mul_(size.to(dt))

    s = {"freq": _freq(c) if c["rot"] else None, "sections": _sections(c) if c["rot"] else None}
    if c["kind"] in ("rotate", "back"):
        B, N = c["B"], c["N"]
        for x, H in (("q", c["H"]), ("k", c["Hk"])):
            shape = (B, N, H) if c["layout"] == "bnhd" else (B, H, N)
            y = rows(*shape)
            s[x] = y.transpose(1, 2) if c["layout"] == "bnhd" else y
        # the sequences of a batch start at positions of their own
        first = torch.randint(c["far"], c["far"] + 50, (B,), generator=cpu, dtype=torch.int32)
        pos = [torch.arange(N, dtype=torch.int32)[None] + f if c["axes"] == 1 else _grid(f, N) for f in first]
        s["pos"] = torch.stack(pos, 1).cuda()                                                       # [axes, B, N]
        return s
    S, Hk, page = c["S"], c["Hk"], c["page"]
    end = c["hi"] + 1 if c["kind"] == "decode" else c["behind"] + c["n"]    # rows that a sequence may come to hold
    need = -(-end // page)
    pages = S * need + 3
    for x in ("k", "v"):
        if c["kind"] == "store":
            if c["e4m3"]:
                s[x + "p"] = torch.zeros(pages, Hk, page, D, device="cuda").to(E4M3)
                s[x + "e"] = torch.full((pages, Hk, page), 127, device="cuda", dtype=torch.uint8)
            else:
                s[x + "p"], s[x + "e"] = torch.zeros(pages, Hk, page, D, device="cuda", dtype=dt), None
        else:
            y = rows(pages, Hk, page)
            s[x + "p"], s[x + "e"] = _quantise(y) if c["e4m3"] else (y, None)
    table = torch.randperm(pages, generator=cpu, dtype=torch.int32)[:S * need].view(S, need)
    if c["kind"] == "decode":
        H = c["H"]
        s["q"] = torch.randn(S, H, D, generator=g, device="cuda", dtype=dt)
        s["k"], s["v"] = rows(S, Hk), rows(S, Hk)
        s["gate"] = torch.rand((H,), generator=g, device="cuda") * 2 - 1
        s["len_in"] = _spread(cpu, S, c["lo"], c["hi"])
        s["len_out"] = torch.zeros_like(s["len_in"])
        s["lse"] = torch.zeros(S, H, device="cuda")
        if c["axes"] == 3:
            # a sequence with images has fewer steps in time than rows
            s["pos"] = torch.stack([s["len_in"] // 2 + 7, s["len_in"] // 2 + 3, s["len_in"] // 2 + 5])
        else:
            s["pos"] = None
        if c["evict"]:
            t = s["len_in"].cpu()[:, None]
            gone = (torch.arange(need)[None] + 1) * page <= t - c["k"]
            gone[::2] = False
            table[gone] = -1
        s["table"] = table.cuda()
        return s
    n = c["n"]
    if c["kind"] == "store":
        shape = (S, n, Hk) if c["layout"] == "snhd" else (S, Hk, n)
        s["k"], s["v"] = (rows(*shape) for _ in range(2))
        if c["layout"] == "snhd":
            s["k"], s["v"] = s["k"].transpose(1, 2), s["v"].transpose(1, 2)
        s["pos"] = torch.stack([_grid(7 * i, n) for i in range(S)], 1).cuda() if c["axes"] == 3 else None
    else:
        shape = (S, n, Hk, D) if c["layout"] == "snhd" else (S, Hk, n, D)
        s["out"] = [torch.empty(shape, dtype=dt, device="cuda") for _ in range(2)]
        if c["layout"] == "snhd":
            s["out"] = [x.transpose(1, 2) for x in s["out"]]
    s["count"] = _spread(cpu, S, (n + 1) // 2, n) if c["ragged"] else None
    s["start"] = _spread(cpu, S, c["behind"] // 2, c["behind"]) if c["behind"] else None
    s["table"] = table.cuda()
    return s


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# ---- the plain forms --------------------------------------------------------------
def _angles(c, s, pos):
    """cos and sin [..., rot] at pos [axes, ...]: the angles in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_sections(c), device="cuda"))
    a = pos.double().movedim(0, -1)[..., axis] * s["freq"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _turned(c, x, cos, sin):
    """Rows x [..., D] turned, in float32."""
    P, half = c["rot"], c["D"] // 2
    x = x.float()
    a, b = x[..., :P], x[..., half:half + P]
    return torch.cat([a * cos - b * sin, x[..., P:half], a * sin + b * cos, x[..., half + P:]], -1)


def _placed(c, s):
    """For rows [S, n]: their positions, pages, rows of the page, and which of them are there."""
    i = torch.arange(c["n"], device="cuda")[None]
    at = i + (s["start"][:, None] if s["start"] is not None else torch.zeros(c["S"], 1, dtype=torch.int32, device="cuda"))
    there = at < s["table"].shape[1] * c["page"]
    if s["count"] is not None:
        there = there & (i < s["count"][:, None])
    p = at.clamp(max=s["table"].shape[1] * c["page"] - 1)
    return at, torch.gather(s["table"], 1, p // c["page"]).long(), p % c["page"], there


def _put(pages, exps, page, row, x):
    """Rows x [m, Hk, D] into rows `row` of pages `page`."""
    if exps is None:
        pages[page, :, row] = x.to(pages.dtype)
    else:
        q, e = _quantise(x)
        # float8 has no indexed write of its own: as bytes
        pages.view(torch.uint8)[page, :, row] = q.view(torch.uint8)
        exps[page, :, row] = e


def _get(pages, exps, page, row):
    """Rows `row` of pages `page`, [..., Hk, D] in float32."""
    if exps is None:
        return pages[page, :, row].float()
    return _values(pages.view(torch.uint8)[page, :, row].view(E4M3), exps[page, :, row])


def _store(c, s):
    at, page, row, there = _placed(c, s)
    k = s["k"].transpose(1, 2)                                                            # [S, n, Hk, D]
    if c["rot"]:
        pos = s["pos"] if s["pos"] is not None else at[None].expand(c["axes"], -1, -1)
        cos, sin = _angles(c, s, pos)
        k = _turned(c, k, cos[:, :, None], sin[:, :, None])
    for x, y in (("k", k), ("v", s["v"].transpose(1, 2))):
        _put(s[x + "p"], s[x + "e"], page[there], row[there], y[there])


def _load(c, s):
    at, page, row, there = _placed(c, s)
    for x, out in zip("kv", s["out"]):
        y = _get(s[x + "p"], s[x + "e"], page, row)
        out.copy_(torch.where(there[..., None, None], y, 0.0).transpose(1, 2))


def _decode(c, s):
    S, H, Hk, D, k, pi, page = (c[x] for x in ("S", "H", "Hk", "D", "k", "pi", "page"))
    t = s["len_in"].long()
    seq = torch.arange(S, device="cuda")
    q, kn = s["q"].float(), s["k"].float()
    if c["rot"]:
        pos = s["pos"] if s["pos"] is not None else t[None].expand(c["axes"], -1)
        cos, sin = (x[:, None] for x in _angles(c, s, pos))
        q, kn = _turned(c, q, cos, sin), _turned(c, kn, cos, sin)
    q = q.view(S, Hk, H // Hk, D)
    a = GATE_EPS + (1 - 2 * GATE_EPS) / (1 + torch.exp(-s["gate"]))
    bias = [torch.log(x).view(1, Hk, H // Hk, 1) for x in (a, 1 - a)]
    new = s["table"][seq, t // page].long()
    for x, y in (("k", kn), ("v", s["v"])):
        _put(s[x + "p"], s[x + "e"], new, t % page, y)

    def rows(at):
        """Keys and values [S, Hk, n, D] at positions [S, n], and which are there."""
        j = at.clamp(min=0)
        p = torch.gather(s["table"], 1, j // page).long()
        kv = [_get(s[x + "p"], s[x + "e"], p.clamp(min=0), j % page).transpose(1, 2) for x in "kv"]
        return kv, ((at >= 0) & (p >= 0))[:, None, None]

    def logits(kk, there, b):
        d = torch.matmul(q, kk.transpose(2, 3).contiguous()) / math.sqrt(D) + b
        d = d.clamp(-c["clamp"], c["clamp"]) if c["clamp"] > 0 else d
        return torch.where(there, d, -math.inf)

    w = min(k, c["hi"]) + 1
    (kk, vv), there = rows(t[:, None] - torch.arange(w, device="cuda"))
    d = logits(kk, there, bias[0])
    if pi > k:
        (kk, pv), there = rows((t - pi)[:, None])
        d = torch.cat([d, logits(kk, there, bias[1])], -1)
        vv = torch.cat([vv, pv], 2)
    m = d.amax(-1, keepdim=True)
    p = torch.exp(d - m)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, vv.contiguous()) / total
    return out.view(S, H, D).to(s["q"].dtype), (m + torch.log(total)).view(S, H), s["len_in"] + 1


def run(state):
    c, s = state["case"], state
    if own:
        import paper_2511_10696_amd as pa
    if c["kind"] == "rotate":
        if own:
            q, k = pa.pi_attn_rotate(s["q"], s["k"], s["pos"], s["freq"], s["sections"])
        else:
            cos, sin = (x[:, None] for x in _angles(c, s, s["pos"]))
            q, k = (_turned(c, s[x], cos, sin).to(s[x].dtype) for x in "qk")
        return {"q": q, "k": k}
    if c["kind"] == "back":
        to = _dtype(c["to"])
        if own:
            dq, dk = pa.pi_attn_rotate_backward(s["q"], s["k"], s["pos"], s["freq"], s["sections"], dtype=to)
        else:
            cos, sin = (x[:, None] for x in _angles(c, s, s["pos"]))
            dq, dk = (_turned(c, s[x], cos, -sin).to(to) for x in "qk")
        return {"dq": dq, "dk": dk}
    if c["kind"] == "store":
        if own:
            pa.pi_attn_paged_store(s["k"], s["v"], s["kp"], s["vp"], s["table"], s["start"], s["count"], k_exp=s["ke"],
                                   v_exp=s["ve"], freq=s["freq"], pos=s["pos"] if c["rot"] else None,
                                   sections=s["sections"])
        else:
            _store(c, s)
        r = {"k": s["kp"], "v": s["vp"]}
    elif c["kind"] == "load":
        k, v = s["out"]
        if own:
            pa.pi_attn_paged_load(s["kp"], s["vp"], s["table"], c["n"], s["start"], s["count"], k_exp=s["ke"],
                                  v_exp=s["ve"], k=k, v=v)
        else:
            _load(c, s)
        return {"k": k, "v": v}
    else:
        lse, length = s["lse"], s["len_out"]
        if own:
            out = pa.pi_attn_decode_step_paged(
                s["len_in"], s["q"], s["k"], s["v"], s["kp"], s["vp"], s["table"], s["gate"], c["k"], c["pi"],
                k_exp=s["ke"], v_exp=s["ve"], freq=s["freq"], pos=s["pos"] if c["rot"] else None,
                sections=s["sections"], logit_clamp=c["clamp"], len_out=length, lse=lse)
        else:
            out, lse, length = _decode(c, s)
        r = {"out": out, "lse": lse, "len": length, "k": s["kp"], "v": s["vp"]}
    if s["ke"] is not None:
        r["k_exp"], r["v_exp"] = s["ke"], s["ve"]
    return r


# ---- what a pass cannot do without --------------------------------------------------
def work(case):
    c = case
    es, D = (4 if c["dtype"] == "f32" else 2), c["D"]
    if c["kind"] in ("rotate", "back"):
        rows = c["B"] * c["N"] * (c["H"] + c["Hk"])
        by = rows * D * (es + (4 if c["to"] == "f32" else 2)) + 4 * c["axes"] * c["B"] * c["N"]
        return {"bytes": by, "flops": rows * 6 * c["rot"]}
    S, Hk, page = c["S"], c["Hk"], c["page"]
    row = D + 1 if c["e4m3"] else D * es
    if c["kind"] in ("store", "load"):
        n = c["n"]
        held = sum((n + 1) // 2 + (n - (n + 1) // 2) * i // max(1, S - 1) for i in range(S)) if c["ragged"] else S * n
        # absent rows are written too by a load, as zeros
        wide = held if c["kind"] == "store" else S * n
        by = 2 * Hk * (held * row + wide * D * es) + 4 * -(-held // page)
        if c["rot"] and c["axes"] == 3:
            by += 12 * held
        return {"bytes": by, "flops": held * Hk * (6 * c["rot"] + (4 * D if c["e4m3"] else 0))}
    seen = 0
    for i in range(S):
        t = c["lo"] + (c["hi"] - c["lo"]) * i // max(1, S - 1)
        # the new row among them; a partner in a page that was given back is not there for every second sequence
        seen += min(t, c["k"]) + 1 + (1 if c["pi"] > c["k"] and t >= c["pi"] and not (c["evict"] and i % 2) else 0)
    H = c["H"]
    # cached rows, the new ones read and stored, queries, outputs and their lse, the table
    by = 2 * Hk * (seen - S) * row + 2 * S * Hk * (D * es + row) + S * H * (2 * D * es + 4) + 4 * -(-seen // page)
    return {"bytes": by, "flops": 4 * D * H * seen}


# ---- the same in 64 bits ---------------------------------------------------------------
def _stored64(x):
    """The row's codes and bytes by the definition: the least e from -126 on with amax <= 448 * 2^e, halves to even."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -140) / 448)) - 1
    while bool((short := amax > 448 * torch.exp2(e)).any()):
        e = e + short
    e = e.clamp(min=-126)
    y = x * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, (e[..., 0] + 127).to(torch.uint8)


def _turned64(c, x, pos, sign=1.0):
    """Rows x [..., D] turned by pos [axes, ...] as complex numbers, pair by pair of each axis."""
    x, half, first = x.double(), c["D"] // 2, 0
    z = torch.complex(x[..., :half], x[..., half:])
    freq = _freq(c).double()
    for a, n in enumerate(_sections(c)):
        angle = sign * pos[a].double()[..., None] * freq[first:first + n]
        z[..., first:first + n] *= torch.polar(torch.ones_like(angle), angle)
        first += n
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] in ("rotate", "back"):
        sign, names = (1.0, ("q", "k")) if c["kind"] == "rotate" else (-1.0, ("dq", "dk"))
        return {n: _turned64(c, s[x], s["pos"][:, :, None], sign) for n, x in zip(names, "qk")}
    S, Hk, page, D = c["S"], c["Hk"], c["page"], c["D"]
    codes = {x: s[x + "p"].double() for x in "kv"}
    byte = {x: s[x + "e"] for x in "kv"}
    table = s["table"].long()

    def value(x, i, at):
        """Rows `at` of sequence i, [Hk, len(at), D]"""
        y = codes[x][table[i][at // page], :, at % page]
        if byte[x] is not None:
            y = y * torch.exp2(byte[x][table[i][at // page], :, at % page].double() - 127)[..., None]
        return y.transpose(0, 1)

    def enter(x, i, at, y):
        """Rows y [Hk, len(at), D] at positions `at` of sequence i"""
        y = y.transpose(0, 1).double()
        if byte[x] is not None:
            y, e = _stored64(y)
            byte[x][table[i][at // page], :, at % page] = e
        codes[x][table[i][at // page], :, at % page] = y

    def pages():
        r = {"k": codes["k"], "v": codes["v"]}
        if c["e4m3"]:
            r["k_exp"], r["v_exp"] = byte["k"], byte["v"]
        return r

    if c["kind"] in ("store", "load"):
        counts = s["count"].tolist() if s["count"] is not None else [c["n"]] * S
        starts = s["start"].tolist() if s["start"] is not None else [0] * S
        r = {x: torch.zeros(S, Hk, c["n"], D, dtype=torch.float64, device="cuda") for x in "kv"} if c["kind"] == "load" else 0
        for i, (m, first) in enumerate(zip(counts, starts)):
            at = first + torch.arange(m, device="cuda")
            if c["kind"] == "load":
                for x in "kv":
                    r[x][i, :, :m] = value(x, i, at)
                continue
            k = s["k"][i, :, :m]
            if c["rot"]:
                pos = s["pos"][:, i, :m] if s["pos"] is not None else at[None]
                k = _turned64(c, k, (pos if c["axes"] == len(pos) else pos.expand(c["axes"], -1))[:, None])
            enter("k", i, at, k)
            enter("v", i, at, s["v"][i, :, :m])
        return r if c["kind"] == "load" else pages()
    H, k, pi, clamp = c["H"], c["k"], c["pi"], c["clamp"]
    alpha = (GATE_EPS + (1 - 2 * GATE_EPS) * torch.sigmoid(s["gate"].double())).view(Hk, H // Hk, 1)
    out = torch.empty(S, H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(S, H, dtype=torch.float64, device="cuda")
    for i, t in enumerate(s["len_in"].tolist()):
        q, kn = s["q"][i].double(), s["k"][i].double()
        if c["rot"]:
            pos = s["pos"][:, i] if s["pos"] is not None else torch.full((c["axes"],), t, device="cuda")
            q, kn = (_turned64(c, x, pos[:, None]) for x in (q, kn))
        now = torch.tensor([t], device="cuda")
        enter("k", i, now, (kn if byte["k"] is not None else kn.to(_dtype(c["dtype"])))[:, None])
        enter("v", i, now, s["v"][i][:, None])
        at = torch.arange(max(0, t - k), t + 1, device="cuda")
        bias = [torch.log(alpha).expand(-1, -1, len(at))]
        if pi > k and t >= pi:
            at = torch.cat([at, torch.tensor([t - pi], device="cuda")])
            bias.append(torch.log(1 - alpha))
        there = table[i][at // page] >= 0
        kk, vv = (value(x, i, at[there]) for x in "kv")
        d = torch.matmul(q.view(Hk, H // Hk, D), kk.transpose(1, 2)) / math.sqrt(D) + torch.cat(bias, -1)[..., there]
        d = d.clamp(-clamp, clamp) if clamp > 0 else d
        total = torch.logsumexp(d, -1)
        lse[i] = total.view(H)
        out[i] = torch.matmul(torch.exp(d - total[..., None]), vv).view(H, D)
    return {"out": out, "lse": lse, "len": s["len_in"] + 1, **pages()}
