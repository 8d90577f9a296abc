"""Measured cases of the quantised KV cache and of the decode step over a shared prefix.

Each case is one kind of pass:
  store   pi_attn_cache_store: rows of keys and values written into an e4m3 cache
  load    pi_attn_cache_load: rows read back in the working type
  chunk   a chunk of a prompt stored, then the whole prompt so far read back for the chunk's attention
  decode  pi_attn_decode_step_e4m3: a decode step over e4m3 caches
  prefix  pi_attn_decode_step_prefix: a decode step of a batch that shares a prompt

A stored row is D e4m3 codes and a byte b: element d is code_d * 2^(b - 127), where e = b - 127 is the least integer from -126
on with max |x| <= 448 * 2^e.  Caches are returned as their codes (a float8 type) and those bytes.

With own = False, run() computes the same in elementary torch operations.
"""
import math

import torch

own = False

GATE_EPS = 1e-4
E4M3 = torch.float8_e4m3fn


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


# ---- the cases -----------------------------------------------------------------
def _rows(name, kind, dtype, S, H, D, n, cap, **more):
    """store, load, chunk: n rows a sequence of caches of cap rows."""
    c = {"name": name, "kind": kind, "dtype": dtype, "S": S, "H": H, "D": D, "n": n, "cap": cap, "layout": "shnd",
         "ragged": False}
    c.update(more)
    return c


def _step(name, kind, dtype, S, H, D, k, pi, cap, lo, hi, **more):
    """decode, prefix: sequences of lo to hi rows in their own caches of cap rows, after plen shared ones."""
    c = {"name": name, "kind": kind, "dtype": dtype, "S": S, "H": H, "D": D, "k": k, "pi": pi, "cap": cap, "lo": lo,
         "hi": hi, "plen": 0, "e4m3": kind == "decode", "clamp": 0.0}
    c.update(more)
    return c


def listed():
    return [
        # A short prompt of a small float32 model enters its cache: launch latency.
        _rows("store_tiny_f32", "store", "f32", 1, 4, 64, 33, 64),
        # A batch of prompts of different lengths, k and v as views of the projection's [S][n][H][D] output.
        _rows("store_batch", "store", "bf16", 8, 16, 64, 1500, 2048, layout="snhd", ragged=True),
        # The longest prompt.
        _rows("store_32k", "store", "bf16", 1, 32, 128, 32768, 32768),
        # The third chunk of a few prompts: stored, and everything so far read back for its attention.
        _rows("chunk_f32", "chunk", "f32", 3, 8, 128, 500, 2000, ragged=True),
        # The rows of a batch that is moved on to a card without e4m3 caches.
        _rows("load_batch", "load", "bf16", 16, 32, 128, 2000, 2048, layout="snhd", ragged=True),
        # A decode step of one user.
        _step("decode_1", "decode", "bf16", 1, 32, 128, 512, 1024, 2048, 1500, 1500),
        # A few sequences of odd lengths, from empty on, in float32, with the paper's logit clamp.
        _step("decode_odd_f32", "decode", "f32", 7, 12, 64, 100, 101, 333, 0, 332, clamp=20.0),
        # A full batch.
        _step("decode_64", "decode", "bf16", 64, 32, 128, 512, 1024, 1160, 1024, 1159),
        # Four answers to one short prompt, the first tokens.
        _step("prefix_short", "prefix", "bf16", 4, 16, 64, 128, 256, 100, 0, 50, plen=1000),
        # A batch behind a common instruction, dense in the last 2000 rows, float32.
        _step("prefix_f32", "prefix", "f32", 16, 8, 64, 2000, 4096, 300, 0, 299, plen=5000),
        # Long document, a few questions: dense attention over all of it.
        _step("prefix_64k", "prefix", "bf16", 24, 16, 128, 70000, 0, 400, 0, 399, plen=65536),
        # The same in e4m3 for a full batch.
        _step("prefix_e4m3_32k", "prefix", "bf16", 64, 32, 128, 40000, 0, 256, 0, 255, plen=32768, e4m3=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "load", "chunk", "decode", "decode", "prefix", "prefix", "prefix"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D, H = rng.choice([64, 128]), rng.choice([2, 8, 12, 16, 32])
    if kind in ("store", "load", "chunk"):
        n = _log(rng, 1, 8192)
        chunk = kind == "chunk"
        S = _log(rng, 1, max(1, min(64, 32 * 32768 * (16 if chunk else 64) // (n * H * D))))
        c = _rows("", kind, dtype, S, H, D, n, 3 * n + rng.randrange(9) if chunk else n + rng.randrange(1, 200),
                  layout=rng.choice(["shnd", "snhd"]), ragged=rng.random() < 0.5)
    elif kind == "decode":
        k = _log(rng, 1, 2048)
        pi = rng.choice([0, k + 1, 2 * k, k + 1 + rng.randrange(2 * k)])
        cap = pi + _log(rng, 2, 600) + k
        S = _log(rng, 1, max(1, min(64, 64 * 32 * 1160 * 128 // (cap * H * D))))
        c = _step("", kind, dtype, S, H, D, k, pi, cap, rng.choice([0, cap // 2]), cap - 1,
                  clamp=rng.choice([0.0, 0.0, 20.0]))
    else:
        plen = _log(rng, 20, 32768)
        k = rng.choice([plen + 1000, _log(rng, 16, plen), _log(rng, 16, plen)])
        pi = rng.choice([0, k + 1, k + 1 + rng.randrange(plen)])
        S, cap = _log(rng, 1, 64), _log(rng, 8, 400)
        c = _step("", kind, dtype, S, min(H, 16) if dtype == "f32" else H, D, k, pi, cap, 0, cap - 1, plen=plen,
                  e4m3=rng.random() < 0.5, clamp=rng.choice([0.0, 0.0, 20.0]))
    del c["name"]
    return c


# ---- rows as they are stored ------------------------------------------------------
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


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 23)
    cpu = torch.Generator()
    cpu.manual_seed(int(seed) * 7919 + 23)
    dt = _dtype(c)
    S, H, D, cap = c["S"], c["H"], c["D"], c["cap"]

    def rows(*shape):
        """Keys or values: a few dims larger than the others, as trained projections give them, and rows of unlike size."""
        x = torch.randn(*shape, D, generator=g, device="cuda", dtype=dt)
        dims = torch.where(torch.rand(D, generator=g, device="cuda") < 0.05, 3.0, 1.0)
        size = 0.5 + torch.rand(*shape, 1, generator=g, device="cuda")
        return x.mul_(dims.to(dt)).mul_(size.to(dt))

    def cached(*shape):
        """Rows as they lie in a cache: (codes, bytes) or (rows, None)."""
        x = rows(*shape)
        return _quantise(x) if c.get("e4m3", True) else (x, None)

    s = {}
    if c["kind"] in ("store", "load", "chunk"):
        n = c["n"]
        if c["kind"] != "load":
            shape = (S, n, H) if c["layout"] == "snhd" else (S, H, n)
            s["k"], s["v"] = (rows(*shape) for _ in range(2))
            if c["layout"] == "snhd":
                s["k"], s["v"] = s["k"].transpose(1, 2), s["v"].transpose(1, 2)
        for name in ("k", "v"):
            if c["kind"] == "store":
                s[name + "c"] = torch.zeros(S, H, cap, D, device="cuda").to(E4M3)
                s[name + "e"] = torch.full((S, H, cap), 127, device="cuda", dtype=torch.uint8)
            else:
                s[name + "c"], s[name + "e"] = cached(S, H, cap)
        s["count"] = _spread(cpu, S, (n + 1) // 2, n) if c["ragged"] else None
        # a chunk goes behind two others; otherwise the rows lie at the front of the caches
        s["start"] = torch.full((S,), 2 * n, dtype=torch.int32, device="cuda") if c["kind"] == "chunk" else None
        if c["kind"] == "chunk":
            s["upto"] = (s["count"] if c["ragged"] else torch.full((S,), n, dtype=torch.int32, device="cuda")) + 2 * n
        else:
            s["upto"] = s["count"]
        if c["kind"] != "store":
            # the attention's input: a padded batch in the projection's layout, or one row run a head
            m = 3 * n if c["kind"] == "chunk" else n
            shape = (S, m, H, D) if c["layout"] == "snhd" else (S, H, m, D)
            s["out"] = [torch.empty(shape, dtype=dt, device="cuda") for _ in range(2)]
            if c["layout"] == "snhd":
                s["out"] = [x.transpose(1, 2) for x in s["out"]]
        return s
    s["q"] = torch.randn(S, H, D, generator=g, device="cuda", dtype=dt)
    s["k"], s["v"] = rows(S, H), rows(S, H)
    for name in ("k", "v"):
        s[name + "c"], s[name + "e"] = cached(S, H, cap)
        if c["kind"] == "prefix":
            s[name + "p"], s[name + "pe"] = cached(H, c["plen"])
    s["gate"] = torch.rand((H,), generator=g, device="cuda") * 2 - 1
    s["len_in"] = _spread(cpu, S, c["lo"], c["hi"])
    s["len_out"] = torch.zeros_like(s["len_in"])
    s["lse"] = torch.zeros(S, H, device="cuda")
    return s


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# ---- the plain forms --------------------------------------------------------------
def _placed(c, start, count, n):
    """Cache rows [S, n] of rows i < n, and which of them are there."""
    i = torch.arange(n, device="cuda")[None]
    at = i + (start[:, None] if start is not None else torch.zeros(c["S"], 1, dtype=torch.int32, device="cuda"))
    there = (at >= 0) & (at < c["cap"])
    if count is not None:
        there = there & (i < count[:, None])
    return at.clamp(0, c["cap"] - 1), there


def _store(c, x, start, count, codes, byte):
    at, there = _placed(c, start, count, x.shape[2])
    q, e = _quantise(x)
    s, i = there.nonzero(as_tuple=True)
    # float8 has no indexed write of its own: as bytes
    codes.view(torch.uint8)[s, :, at[s, i]] = q.view(torch.uint8)[s, :, i]
    byte[s, :, at[s, i]] = e[s, :, i]


def _load(c, codes, byte, n, start, count, out):
    at, there = _placed(c, start, count, n)
    s = torch.arange(c["S"], device="cuda")[:, None]
    x = _values(codes.view(torch.uint8)[s, :, at].view(E4M3), byte[s, :, at])    # [S, n, H, D]
    return out.copy_(torch.where(there[..., None, None], x, 0.0).transpose(1, 2))


def _priors(gate, clamp):
    a = GATE_EPS + (1 - 2 * GATE_EPS) / (1 + torch.exp(-gate))
    return torch.log(a)[None], torch.log(1 - a)[None]                                 # [1, H]


def _logits(q, rows, bias, c):
    """[S, H, n] of q [S, H, D] with rows [S, H, n, D]."""
    d = torch.matmul(rows, q[..., None])[..., 0] / math.sqrt(c["D"]) + bias[..., None]
    return d.clamp(-c["clamp"], c["clamp"]) if c["clamp"] > 0 else d


def _decode(c, s):
    quant = c["kind"] == "decode" or c["e4m3"]
    plen, cap, k, pi = c["plen"], c["cap"], c["k"], c["pi"]
    n = s["len_in"].long()
    t = plen + n
    seq = torch.arange(c["S"], device="cuda")
    q = s["q"].float()
    lw, lp = _priors(s["gate"], c["clamp"])
    # the new row, as stored
    for x in ("k", "v"):
        if quant:
            codes, byte = _quantise(s[x])
            s[x + "c"].view(torch.uint8)[seq, :, n] = codes.view(torch.uint8)
            s[x + "e"][seq, :, n] = byte
        else:
            s[x + "c"][seq, :, n] = s[x]

    def own_rows(x, at):
        if quant:
            return _values(s[x + "c"].view(torch.uint8)[seq[:, None], :, at].view(E4M3), s[x + "e"][seq[:, None], :, at])
        return s[x + "c"][seq[:, None], :, at].float()

    def prefix_rows(x, at):
        """[H, ..., D]"""
        if quant:
            return _values(s[x + "p"].view(torch.uint8)[:, at].view(E4M3), s[x + "pe"][:, at])
        return s[x + "p"][:, at].float()

    # own window rows, the new one among them
    w = min(k, cap - 1) + 1
    at = n[:, None] - torch.arange(w, device="cuda")
    at_in = at.clamp(min=0)
    kk, vv = (own_rows(x, at_in).transpose(1, 2) for x in ("k", "v"))              # [S, H, w, D]
    logits = [torch.where((at >= 0)[:, None], _logits(q, kk, lw, c), -math.inf)]
    if pi > k:
        at = t - pi
        pk, pv = (own_rows(x, (at - plen).clamp(min=0)[:, None])[:, 0] for x in ("k", "v"))   # [S, H, D]
        if plen:
            there = (at < plen)[:, None, None]
            pk, pv = (torch.where(there, prefix_rows(x, at.clamp(0, plen - 1)).transpose(0, 1), y)
                      for x, y in (("k", pk), ("v", pv)))
        logits.append(torch.where((at >= 0)[:, None, None], _logits(q, pk[:, :, None], lp, c), -math.inf))
    near = min(k, plen)
    if near:
        j = torch.arange(plen - near, plen, device="cuda")
        ck, cv = (prefix_rows(x, j) for x in ("k", "v"))                                # [H, near, D]
        d = torch.matmul(q.transpose(0, 1), ck.transpose(1, 2)).transpose(0, 1) / math.sqrt(c["D"]) + lw[..., None]
        d = d.clamp(-c["clamp"], c["clamp"]) if c["clamp"] > 0 else d
        logits.append(torch.where((j >= (t - k)[:, None])[:, None], d, -math.inf))
    logits = torch.cat(logits, -1)
    m = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - m)
    total = p.sum(-1, keepdim=True)
    out = (p[..., :w, None] * vv).sum(2)
    if pi > k:
        out += p[..., w:w + 1] * pv
    if near:
        out += torch.matmul(p[..., -near:].transpose(0, 1).contiguous(), cv).transpose(0, 1)
    return (out / total).to(s["q"].dtype), (m + torch.log(total))[..., 0], s["len_in"] + 1


def run(state):
    c, s = state["case"], state
    if own:
        import paper_2511_10696_amd as pa
    if c["kind"] in ("store", "load", "chunk"):
        if c["kind"] != "load":
            if own:
                pa.pi_attn_cache_store(s["k"], s["v"], s["kc"], s["vc"], s["ke"], s["ve"], s["start"], s["count"])
            else:
                _store(c, s["k"], s["start"], s["count"], s["kc"], s["ke"])
                _store(c, s["v"], s["start"], s["count"], s["vc"], s["ve"])
        if c["kind"] == "store":
            return {"k": s["kc"], "v": s["vc"], "k_exp": s["ke"], "v_exp": s["ve"]}
        k, v = s["out"]
        n = k.shape[2]
        if own:
            k, v = pa.pi_attn_cache_load(s["kc"], s["vc"], s["ke"], s["ve"], n, None, s["upto"], k=k, v=v)
        else:
            k, v = _load(c, s["kc"], s["ke"], n, None, s["upto"], k), _load(c, s["vc"], s["ve"], n, None, s["upto"], v)
        return {"k": k, "v": v}
    lse, length = s["lse"], s["len_out"]
    if not own:
        out, lse, length = _decode(c, s)
    elif c["kind"] == "decode":
        out = pa.pi_attn_decode_step_e4m3(s["len_in"], s["q"], s["k"], s["v"], s["kc"], s["vc"], s["ke"], s["ve"],
                                          s["gate"], c["k"], c["pi"], logit_clamp=c["clamp"], len_out=length, lse=lse)
    else:
        out = pa.pi_attn_decode_step_prefix(s["len_in"], s["q"], s["k"], s["v"], s["kp"], s["vp"], s["kc"], s["vc"],
                                            s["gate"], c["k"], c["pi"], k_prefix_exp=s["kpe"], v_prefix_exp=s["vpe"],
                                            k_exp=s["ke"], v_exp=s["ve"], logit_clamp=c["clamp"], len_out=length,
                                            lse=lse)
    r = {"out": out, "lse": lse, "len": length, "k": s["kc"], "v": s["vc"]}
    if s["ke"] is not None:
        r["k_exp"], r["v_exp"] = s["ke"], s["ve"]
    return r


# ---- what a pass cannot do without --------------------------------------------------
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    S, H, D = c["S"], c["H"], c["D"]
    if c["kind"] in ("store", "load", "chunk"):
        n = c["n"]
        stored = sum((n + 1) // 2 + (n - (n + 1) // 2) * i // max(1, S - 1) for i in range(S)) if c["ragged"] else S * n
        wide, narrow = 2 * H * D * es, 2 * H * (D + 1)    # K and V of one position, in the working type and stored
        by = 0
        if c["kind"] != "load":
            by += stored * (wide + narrow)
        if c["kind"] != "store":
            before = 2 * n * S if c["kind"] == "chunk" else 0
            # absent rows are written too, as zeros
            by += (before if c["kind"] == "chunk" else stored) * narrow + (before + S * n) * wide
        return {"bytes": by, "flops": stored * 2 * H * D * 2}
    row = D + 1 if c["kind"] == "decode" or c["e4m3"] else D * es
    mine = shared = pairs = 0
    plen, k, pi = c["plen"], c["k"], c["pi"]
    for i in range(S):
        n = c["lo"] + (c["hi"] - c["lo"]) * i // max(1, S - 1)
        t = plen + n
        lo = max(0, t - k)
        partner = 1 if pi > k and t >= pi else 0
        mine += t - max(lo, plen) + partner
        shared = max(shared, plen - lo)
        pairs += t - lo + 1 + partner
    # cached rows, the shared ones once; q, k and v, the rows stored, the output and its lse
    by = 2 * H * (mine + shared) * row + S * H * (3 * D * es + 2 * row + D * es + 4)
    return {"bytes": by, "flops": 4 * D * H * pairs}


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


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    S, H, D, cap = c["S"], c["H"], c["D"], c["cap"]
    codes = {x: s[x + "c"].double() for x in ("k", "v")}
    byte = {x: s[x + "e"] for x in ("k", "v")}

    def value(x, i, at):
        """Rows at of sequence i's cache, all heads: [H, len(at), D]"""
        y = codes[x][i][:, at]
        return y if byte[x] is None else y * torch.exp2(byte[x][i][:, at].double() - 127)[..., None]

    if c["kind"] in ("store", "load", "chunk"):
        n = c["n"]
        counts = s["count"].tolist() if c["ragged"] else [n] * S
        if c["kind"] != "load":
            first = 2 * n if c["kind"] == "chunk" else 0
            for x in ("k", "v"):
                for i, m in enumerate(counts):
                    m = min(m, cap - first)
                    y, e = _stored64(s[x][i][:, :m])
                    codes[x][i][:, first:first + m], byte[x][i][:, first:first + m] = y, e
        if c["kind"] == "store":
            return {"k": codes["k"], "v": codes["v"], "k_exp": byte["k"], "v_exp": byte["v"]}
        before = 2 * n if c["kind"] == "chunk" else 0
        r = {x: torch.zeros(S, H, before + n, D, dtype=torch.float64, device="cuda") for x in ("k", "v")}
        for x in ("k", "v"):
            for i, m in enumerate(counts):
                r[x][i, :, :before + m] = value(x, i, torch.arange(before + m, device="cuda"))
        return r
    quant = byte["k"] is not None
    plen, k, pi, clamp = c["plen"], c["k"], c["pi"], c["clamp"]
    shared = {}
    if plen:
        for x in ("k", "v"):
            shared[x] = s[x + "p"].double()
            if quant:
                shared[x] *= torch.exp2(s[x + "pe"].double() - 127)[..., None]
    alpha = GATE_EPS + (1 - 2 * GATE_EPS) * torch.sigmoid(s["gate"].double())
    out = torch.empty(S, H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(S, H, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["len_in"].tolist()):
        for x in ("k", "v"):
            if quant:
                codes[x][i][:, n], byte[x][i][:, n] = _stored64(s[x][i])
            else:
                codes[x][i][:, n] = s[x][i].double()
        t = plen + n
        lo = max(0, t - k)
        kk, vv = ([value(x, i, torch.arange(max(lo - plen, 0), n + 1, device="cuda"))] for x in ("k", "v"))
        if lo < plen:
            kk, vv = kk + [shared["k"][:, lo:]], vv + [shared["v"][:, lo:]]
        bias = [torch.log(alpha)[:, None].expand(H, t - lo + 1)]
        if pi > k and t >= pi:
            j = t - pi
            for x, y in (("k", kk), ("v", vv)):
                y.append(shared[x][:, j:j + 1] if j < plen else value(x, i, torch.tensor([j - plen], device="cuda")))
            bias.append(torch.log(1 - alpha)[:, None])
        kk, vv = torch.cat(kk, 1), torch.cat(vv, 1)
        d = (kk * s["q"][i].double()[:, None]).sum(-1) / math.sqrt(D) + torch.cat(bias, 1)
        d = d.clamp(-clamp, clamp) if clamp > 0 else d
        lse[i] = torch.logsumexp(d, -1)
        out[i] = (torch.exp(d - lse[i][:, None])[..., None] * vv).sum(1)
    r = {"out": out, "lse": lse, "len": s["len_in"] + 1, "k": codes["k"], "v": codes["v"]}
    if quant:
        r["k_exp"], r["v_exp"] = byte["k"], byte["v"]
    return r
