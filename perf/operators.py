"""The 4-bit cache, the attention over it and the int4 projections, for timing.

Each case is one call (or, for the cache's store, the write and the read) as a program makes it: `listed()`
gives the cases, `draw()` more of the same ranges, `prepare()` what the program holds before the call, `run()`
one pass, `work()` the bytes and operations it cannot do without, and `exact()` the same outputs in 64 bits.
With `own` false `run` computes the plain forms from elementary torch operations; with `own` true it calls the
package.

Kinds of case:
  store   keys and values of new tokens quantised into the cache, then read back (the values the cache holds)
  attend  attention of `n` tokens per sequence over the 4-bit cache, the tokens at its end
  matvec  y = add + W h for a few tokens, W in int4 with a scale per 128 columns, h = x or its RMS norm
"""
import math
import random

import torch

own = False

GROUP = 64         # dims that share a scale and a base in the cache
WGROUP = 128       # columns that share a scale in an int4 matrix
EPS = 1e-6
SIGMA = 0.02       # weights are N(0, 0.02)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # The key and value of one decode token written at the end of a 4096-position cache: the smallest call.
        {"name": "store_token", "kind": "store", "B": 1, "n": 1, "L": 4096, "ragged": False, "empty": False,
         "kv": 4, "d": 128, "dtype": "f32"},
        # A decode batch: 16 sequences of different lengths, one token each.
        {"name": "store_batch16", "kind": "store", "B": 16, "n": 1, "L": 4096, "ragged": True, "empty": False,
         "kv": 8, "d": 128, "dtype": "bf16"},
        # Prompt chunks of four sequences, odd lengths (they start and end inside a block of the cache).
        {"name": "store_chunks", "kind": "store", "B": 4, "n": 2047, "L": 6001, "ragged": True, "empty": False,
         "kv": 8, "d": 128, "dtype": "bf16"},
        # Attention of one decode token at the end of a 4096-position context (the headline workload's heads).
        {"name": "attend_token", "kind": "attend", "B": 1, "n": 1, "L": 4096, "ragged": False, "empty": False,
         "heads": 32, "kv": 4, "d": 128, "window": 0, "dtype": "f32"},
        # One token at the end of a long document: the cache's bandwidth.
        {"name": "attend_long", "kind": "attend", "B": 1, "n": 1, "L": 131071, "ragged": False, "empty": False,
         "heads": 64, "kv": 8, "d": 128, "window": 0, "dtype": "bf16"},
        # A serving batch: 16 sequences of different lengths, one of them without any position.
        {"name": "attend_batch16", "kind": "attend", "B": 16, "n": 1, "L": 16384, "ragged": True, "empty": True,
         "heads": 32, "kv": 8, "d": 128, "window": 0, "dtype": "bf16"},
        # Several tokens per sequence to be checked at once, seven query heads per key head, a sliding window.
        {"name": "attend_few", "kind": "attend", "B": 5, "n": 4, "L": 3001, "ragged": True, "empty": False,
         "heads": 14, "kv": 2, "d": 64, "window": 1024, "dtype": "f32"},
        # A prompt chunk at the end of a context of 8192: the matrix-core side.
        {"name": "attend_chunk", "kind": "attend", "B": 1, "n": 2048, "L": 8192, "ragged": False, "empty": False,
         "heads": 32, "kv": 4, "d": 128, "window": 0, "dtype": "bf16"},
        # Short prompts of odd lengths, nothing cached before them for some.
        {"name": "attend_prompts", "kind": "attend", "B": 6, "n": 389, "L": 701, "ragged": True, "empty": False,
         "heads": 16, "kv": 4, "d": 64, "window": 0, "dtype": "bf16"},
        # The fused q/k/v projection of one decode token with its pre-norm (hidden size 2048, 32 + 2 x 4 heads).
        {"name": "matvec_token", "kind": "matvec", "T": 1, "N": 5120, "K": 2048, "norm": True, "add": False},
        # The output projection of 16 tokens, added to the residual.
        {"name": "matvec_batch16", "kind": "matvec", "T": 16, "N": 2048, "K": 4096, "norm": False, "add": True},
        # A vocabulary-sized projection of an odd number of tokens, rows that fill no tile.
        {"name": "matvec_vocabulary", "kind": "matvec", "T": 3, "N": 131071, "K": 2048, "norm": True, "add": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "attend", "matvec", "matvec"])
    if kind == "matvec":
        K = WGROUP * _log(rng, 1, 64)
        return {"kind": kind, "T": rng.choice([1, 1, 2, 16, rng.randint(1, 16)]),
                "N": _log(rng, 1, min(131071, 131071 * 2048 // K)), "K": K, "norm": rng.random() < 0.5,
                "add": rng.random() < 0.5}
    d = rng.choice([64, 64, 128, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 4, 8])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "store":
        B = _log(rng, 1, 16)
        n = rng.choice([1, _log(rng, 1, 2047 * 4 // B)])
        return {"kind": kind, "B": B, "n": n, "L": n + _log(rng, 1, 4096), "ragged": rng.random() < 0.6,
                "empty": rng.random() < 0.2, "kv": kv, "d": d if n * B <= 4096 else min(d, 128), "dtype": dtype}
    mode = rng.choice(["token", "token", "few", "chunk"])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    if mode == "token":
        B, n = _log(rng, 1, 16), 1
        L = _log(rng, 1, min(131071, 131071 * 8 * 128 // (B * kv * d)))
    elif mode == "few":
        B, n = _log(rng, 1, 8), rng.randint(2, 16)
        L = _log(rng, 2, 16384)
    else:
        B, n = _log(rng, 1, 4), _log(rng, 24, 2048)
        L = n + _log(rng, 1, 6144)
        # no dearer than 2048 tokens of 32 heads of 128 over 8192 positions
        kv, group = min(kv, 4), min(group, 8)
        n = max(1, min(n, 2048 * 8192 * 32 * 128 // (B * L * kv * group * d)))
    return {"kind": kind, "B": B, "n": n, "L": L, "ragged": rng.random() < 0.6, "empty": rng.random() < 0.2,
            "heads": kv * group, "kv": kv, "d": d,
            "window": rng.choice([0, 0, _log(rng, 1, 4096)]), "dtype": dtype}


def _lengths(case):
    """(new tokens, cache length with them) of each sequence: fixed by the case, whatever the seed."""
    rng = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    B, n, L = case["B"], case["n"], case["L"]
    ns, ls = [], []
    for b in range(B):
        nb = rng.randint(max(1, n // 4), n) if case["ragged"] and b else n
        lb = rng.randint(max(nb, L // 4), max(nb, L)) if case["ragged"] and b != 1 else max(nb, L)
        ns.append(nb)
        ls.append(lb)
    if case["empty"]:
        ls[-1] = ns[-1] // 2  # fewer positions than tokens: the first tokens are padding
    return ns, ls


# ------------------------------------------------------------------------------------------------ inputs ---
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale)


def _keys_values(rows, kv, d, dtype, g):
    """Keys with a few strong channels and an offset per channel, values with neither."""
    gain = torch.exp(_normal((kv, d), g, 0.5))
    shift = _normal((kv, d), g, 0.3)
    k = torch.empty((rows, kv, d), dtype=DT[dtype], device="cuda")
    v = torch.empty_like(k)
    for i in range(0, rows, 16384):  # a piece at a time: the 32-bit draws are larger than what is kept
        m = min(16384, rows - i)
        k[i:i + m] = _normal((m, kv, d), g).mul_(gain).add_(shift)
        v[i:i + m] = _normal((m, kv, d), g, 0.5)
    return k, v


def _inputs(case, seed):
    """Every tensor of a case, made from the seed alone."""
    g = _gen(seed)
    c = case
    if c["kind"] == "matvec":
        T, N, K = c["T"], c["N"], c["K"]
        w = _normal((N, K // WGROUP, WGROUP), g, SIGMA)
        s = (w.abs().amax(-1) / 7.0).to(torch.bfloat16)
        q = torch.round(w.div_(s.float().unsqueeze(-1))).clamp_(-8, 7).to(torch.int8).view(N, K // 2, 2)
        nib = ((q[..., 0] & 15) | (q[..., 1] << 4)).view(torch.uint8)
        return {"x": _normal((T, K), g), "w": torch.cat([nib.reshape(-1), s.view(-1).view(torch.uint8)]),
                "add": _normal((T, N), g) if c["add"] else None}
    ns, ls = _lengths(c)
    r = {"ns": ns, "ls": ls, "T": sum(ns),
         "kv_len": torch.tensor(ls, dtype=torch.int32, device="cuda"),
         "q_start": torch.tensor([sum(ns[:b]) for b in range(len(ns) + 1)], dtype=torch.int32, device="cuda")}
    if c["kind"] == "store":
        r["k"], r["v"] = _keys_values(r["T"], c["kv"], c["d"], c["dtype"], g)
        return r
    # the context that the cache holds, in the rows' order: sequence by sequence
    r["k"], r["v"] = _keys_values(sum(ls), c["kv"], c["d"], "bf16", g)
    q = _normal((r["T"], c["heads"], c["d"]), g)
    r["q"] = (q / torch.sqrt((q * q).mean(-1, keepdim=True) + EPS)).to(DT[c["dtype"]])
    return r


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = c = case
    if c["kind"] == "matvec":
        s["y"] = torch.empty((c["T"], c["N"]), device="cuda")
    elif own:
        import paper_2605_29135_amd as moe
        moe.moe_init(torch.cuda.current_device())
        max_pos = -(-max(max(s["ls"]), 1) // 32) * 32
        s["cache"] = moe.kv4_cache(c["B"], c["kv"], c["d"], max_pos)
        if c["kind"] == "store":
            s["out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        else:
            start = torch.tensor([sum(s["ls"][:b]) for b in range(c["B"] + 1)], dtype=torch.int32, device="cuda")
            if sum(s["ls"]):
                moe.moe_kv4_append(s["k"], s["v"], s["cache"], s["kv_len"], q_start=start)
            s["out"] = torch.empty_like(s["q"])
            n = moe.moe_kv4_attention_workspace_bytes(s["T"], c["B"], c["heads"], c["kv"], c["d"], c["n"], max_pos)
            s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
            del s["k"], s["v"]
    elif c["kind"] == "attend":
        s["k"], s["v"] = _pack(s["k"]), _pack(s["v"])
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------- plain forms ---
def _quantise(x):
    """Codes 0..15, scale and base of each group of 64: x [..., d] -> [..., d/64, 64], [..., d/64, 1] twice."""
    x = x.float().unflatten(-1, (-1, GROUP))
    base = x.amin(-1, keepdim=True).to(torch.bfloat16).float()
    scale = ((x.amax(-1, keepdim=True) - base) * (1.0 / 15.0)).to(torch.bfloat16).float()
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    t = (x - base).double()  # rounded to 32 bits, then divided in 64: quotients next to a half
    u = torch.where(scale > 0, torch.round(t / scale.double()), torch.zeros_like(t)).clamp_(0, 15)
    return u.float(), scale, base


def _pack(x):
    """The plain cache: two codes a byte, and scales and bases in bf16."""
    out = []
    for i in range(0, max(x.shape[0], 1), 16384):
        u, s, m = _quantise(x[i:i + 16384])
        u = u.to(torch.uint8)
        out.append((u[..., 0::2] | (u[..., 1::2] << 4), s.to(torch.bfloat16), m.to(torch.bfloat16)))
    return tuple(torch.cat(t) for t in zip(*out))


def _unpack(p, lo, hi):
    """Values [kv, hi - lo, d] of rows lo..hi of a plain cache."""
    b, s, m = (t[lo:hi] for t in p)
    u = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()
    return (u * s.float() + m.float()).flatten(-2).transpose(0, 1).contiguous()


def _attend(s):
    c = s["case"]
    G, d, window = c["heads"] // c["kv"], c["d"], c["window"]
    out = torch.zeros_like(s["q"])
    t0 = r0 = 0
    for n, L in zip(s["ns"], s["ls"]):
        if L:
            first = max(0, L - n - window + 1) if window else 0
            K, V = _unpack(s["k"], r0 + first, r0 + L), _unpack(s["v"], r0 + first, r0 + L)
            q = s["q"][t0:t0 + n].float().view(n, c["kv"], G, d).permute(1, 0, 2, 3).reshape(c["kv"], n * G, d)
            z = torch.bmm(q, K.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(c["kv"], n, G, L - first)
            at = torch.arange(L - n, L, device="cuda").view(n, 1, 1)
            p = torch.arange(first, L, device="cuda")
            hidden = p > at
            if window:
                hidden |= p <= at - window
            z.masked_fill_(hidden, -math.inf)
            z = torch.exp_(z.sub_(z.amax(-1, keepdim=True).clamp_(min=-3e38)))
            total = z.sum(-1).view(c["kv"], n * G, 1)
            o = torch.bmm(z.view(c["kv"], n * G, L - first), V) / torch.where(total > 0, total, 1.0)
            out[t0:t0 + n] = o.view(c["kv"], n, G, d).permute(1, 0, 2, 3).reshape(n, c["heads"], d).to(out.dtype)
        t0 += n
        r0 += L
    return out


def _store(s):
    out = []
    for x in (s["k"], s["v"]):
        u, sc, m = _quantise(x)
        y = (u * sc + m).flatten(-2).to(x.dtype)
        t0 = 0
        for n, L in zip(s["ns"], s["ls"]):
            if L < n:
                y[t0:t0 + n - L] = 0
            t0 += n
        out.append(y)
    return tuple(out)


def _matvec(s):
    c = s["case"]
    N, K = c["N"], c["K"]
    b = s["w"][:N * K // 2]
    u = torch.stack([b & 15, b >> 4], -1).float().view(N, K // WGROUP, WGROUP)
    u = torch.where(u > 7, u - 16, u)
    scale = s["w"][N * K // 2:].view(torch.bfloat16).float().view(N, K // WGROUP, 1)
    x = s["x"]
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    y = x @ (u * scale).view(N, K).T
    return y + s["add"] if s["add"] is not None else y


def run(s):
    c = s["case"]
    if not own:
        return {"store": _store, "attend": _attend, "matvec": _matvec}[c["kind"]](s)
    import paper_2605_29135_amd as moe
    if c["kind"] == "store":
        moe.moe_kv4_append(s["k"], s["v"], s["cache"], s["kv_len"], q_start=s["q_start"])
        return moe.moe_kv4_read(s["cache"], s["kv_len"], s["T"], q_start=s["q_start"], k_out=s["out"][0],
                                v_out=s["out"][1])
    if c["kind"] == "attend":
        return moe.moe_kv4_attention(s["q"], s["cache"], s["kv_len"], q_start=s["q_start"], max_q=c["n"],
                                     window=c["window"], out=s["out"], workspace=s["ws"])
    return moe.moe_matvec_int4(s["x"], s["w"], c["N"], y=s["y"], add=s["add"], rmsnorm=c["norm"])


# -------------------------------------------------------------------------------------------------- work ---
def work(case):
    c = case
    if c["kind"] == "matvec":
        T, N, K = c["T"], c["N"], c["K"]
        return {"bytes": N * K // 2 + N * K // 64 + 4 * T * K + 4 * T * N * (2 if c["add"] else 1),
                "flops": 2 * T * N * K}
    ns, ls = _lengths(c)
    d, kv, size = c["d"], c["kv"], 4 if c["dtype"] == "f32" else 2
    held = kv * (d + d // 8)  # bytes of one position, keys and values
    if c["kind"] == "store":
        kept = sum(min(n, L) for n, L in zip(ns, ls))
        return {"bytes": kept * (2 * kv * d * size + 2 * held) + sum(ns) * 2 * kv * d * size,
                "flops": kept * 2 * kv * d * 8}
    seen = pairs = 0
    for n, L in zip(ns, ls):
        w = c["window"] or L + 1
        seen += L - max(0, L - n - w + 1)
        pairs += sum(min(p + 1, w) for p in range(max(0, L - n), L))
    return {"bytes": 2 * sum(ns) * c["heads"] * d * size + seen * held, "flops": 4 * d * c["heads"] * pairs}


# ------------------------------------------------------------------------------------------------- exact ---
def _held(x):
    """The values the cache holds for the vectors x, in 64 bits."""
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for g in range(x.shape[-1] // GROUP):
        v = x[..., g * GROUP:(g + 1) * GROUP].to(torch.float32)
        lo = torch.min(v, -1, keepdim=True).values.bfloat16().float()
        step = ((torch.max(v, -1, keepdim=True).values - lo) * torch.tensor(1 / 15, device=x.device)).bfloat16()
        step = step.double() * (step.double() >= 2.0 ** -126)
        codes = ((v - lo).double() / step.clamp(min=2.0 ** -126)).round().clamp(0, 15) * (step > 0)
        y[..., g * GROUP:(g + 1) * GROUP] = codes * step + lo.double()
    return y


def exact(case, seed):
    c = case
    s = _inputs(case, seed)
    f8 = torch.float64
    if c["kind"] == "matvec":
        N, K = c["N"], c["K"]
        x = s["x"].to(f8)
        if c["norm"]:
            x = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS)
        y = torch.empty((c["T"], N), dtype=f8, device="cuda")
        scale = s["w"][N * K // 2:].view(torch.bfloat16).view(N, -1).to(f8)
        for i in range(0, N, 8192):
            m = min(8192, N - i)
            b = s["w"][i * K // 2:(i + m) * K // 2].view(m, K // 2)
            w = torch.empty((m, K), dtype=f8, device="cuda")
            w[:, 0::2] = ((b.to(torch.int16) & 15) + 8) % 16 - 8
            w[:, 1::2] = ((b.to(torch.int16) >> 4) + 8) % 16 - 8
            y[:, i:i + m] = x @ (w * scale[i:i + m].repeat_interleave(WGROUP, 1)).T
        return y if s["add"] is None else y + s["add"].to(f8)
    if c["kind"] == "store":
        out = []
        for x in (s["k"], s["v"]):
            y = _held(x)
            t = 0
            for n, L in zip(s["ns"], s["ls"]):
                y[t:t + max(0, n - L)] = 0
                t += n
            out.append(y)
        return tuple(out)
    G, d = c["heads"] // c["kv"], c["d"]
    out = torch.zeros(s["q"].shape, dtype=f8, device="cuda")
    t = r = 0
    for n, L in zip(s["ns"], s["ls"]):
        for h in range(c["kv"] if L else 0):
            K, V = _held(s["k"][r:r + L, h]), _held(s["v"][r:r + L, h])
            p = torch.arange(L, device="cuda")
            for i in range(max(0, n - L), n, 256):  # the rows that see something
                j = min(n, i + 256)
                at = torch.arange(L - n + i, L - n + j, device="cuda").unsqueeze(1)
                see = (p <= at) & (p > at - (c["window"] or L + 1))
                q = s["q"][t + i:t + j, h * G:(h + 1) * G].to(f8)
                z = (q.reshape(-1, d) @ K.T).view(j - i, G, L) / math.sqrt(d)
                w = torch.softmax(torch.where(see.unsqueeze(1), z, torch.tensor(-math.inf, dtype=f8, device="cuda")), -1)
                out[t + i:t + j, h * G:(h + 1) * G] = (w.view(-1, L) @ V).view(j - i, G, d)
        t += n
        r += L
    return out
