"""The paged key/value cache: its tables, its store and the attention over it, for timing.

Each case is one call (for a tree of drafted tokens, its masks and the attention) as a program makes it: `listed()`
gives the cases, `draw()` more of the same ranges, `prepare()` what the program holds before the call, `run()`
one pass, `work()` the bytes and operations it cannot do without, and `exact()` the same outputs in 64 bits.
With `own` false `run` computes the plain forms from elementary torch operations; with `own` true it calls the
package.

Kinds of case:
  tables  pages for the new tokens of a batch, and their rows, positions and slots, from the requests' lengths
  append  keys and values of new tokens written to their slots
  attend  attention of `n` tokens per sequence over the cache, the tokens at its end; with a window the first
          `sinks` positions stay visible, and no page is held for what no token sees
  tree    the same for `n` drafted tokens of a tree each, with the masks made from the tokens' parents
"""
import math
import random

import torch

own = False

EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BF16 = torch.bfloat16


def listed():
    return [
        # One decode step of a serving batch: a token each, a new page for few of them.  The smallest call.
        {"name": "tables_step", "kind": "tables", "B": 256, "n": 1, "L": 16384, "page": 16},
        # Prompts of odd lengths admitted together, some of them with a cached beginning.
        {"name": "tables_prompts", "kind": "tables", "B": 61, "n": 2047, "L": 32768, "page": 64},
        # The keys and values of a decode step of 64 sequences, as a projection in 32 bits leaves them.
        {"name": "append_step", "kind": "append", "T": 64, "run": 1, "pad": 0, "kv": 8, "d": 128, "page": 16,
         "dtype": "f32"},
        # A prompt chunk, rows of padding behind it.
        {"name": "append_prompts", "kind": "append", "T": 16384, "run": 2047, "pad": 131, "kv": 8, "d": 128, "page": 64,
         "dtype": "bf16"},
        # Attention of one decode token at the end of a 4096-position context (the headline workload's heads).
        {"name": "attend_token", "kind": "attend", "B": 1, "n": 1, "L": 4096, "ragged": False, "empty": False,
         "heads": 32, "kv": 4, "d": 128, "page": 16, "window": 0, "sinks": 0, "dtype": "f32"},
        # A serving batch of different lengths, one of its sequences without any position: the cache's bandwidth.
        {"name": "attend_batch32", "kind": "attend", "B": 32, "n": 1, "L": 16384, "ragged": True, "empty": True,
         "heads": 32, "kv": 8, "d": 128, "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # Many long documents in a layer with a window: what lies between the first tokens and it is held no more.
        {"name": "attend_window", "kind": "attend", "B": 128, "n": 1, "L": 131071, "ragged": True, "empty": False,
         "heads": 64, "kv": 8, "d": 64, "page": 32, "window": 1024, "sinks": 4, "dtype": "bf16"},
        # A prompt chunk at the end of a context of 8192: the matrix-core side.
        {"name": "attend_chunk", "kind": "attend", "B": 1, "n": 2048, "L": 8192, "ragged": False, "empty": False,
         "heads": 32, "kv": 4, "d": 128, "page": 64, "window": 0, "sinks": 0, "dtype": "bf16"},
        # Prompts of odd lengths in a layer with an odd window.
        {"name": "attend_prompts", "kind": "attend", "B": 6, "n": 1789, "L": 5001, "ragged": True, "empty": False,
         "heads": 16, "kv": 4, "d": 64, "page": 16, "window": 1000, "sinks": 5, "dtype": "bf16"},
        # One user's drafted tokens to be verified behind a context of 8192.
        {"name": "tree_one", "kind": "tree", "B": 1, "n": 60, "L": 8252, "ragged": False, "empty": False,
         "heads": 32, "kv": 8, "d": 128, "page": 16, "window": 0, "sinks": 0, "dtype": "bf16"},
        # Small trees of a batch, in a layer with a window.
        {"name": "tree_batch16", "kind": "tree", "B": 16, "n": 25, "L": 16384, "ragged": True, "empty": False,
         "heads": 32, "kv": 4, "d": 128, "page": 32, "window": 4096, "sinks": 4, "dtype": "bf16"},
        # Wide trees of two short sequences, in 32 bits, heads of 256.
        {"name": "tree_wide", "kind": "tree", "B": 2, "n": 250, "L": 701, "ragged": True, "empty": False,
         "heads": 4, "kv": 2, "d": 256, "page": 16, "window": 0, "sinks": 0, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["tables", "append", "attend", "attend", "attend", "tree", "tree"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "tables":
        B = _log(rng, 1, 2048)
        n = rng.choice([1, _log(rng, 1, min(2047, 131072 // B))])
        return {"kind": kind, "B": B, "n": n, "L": n + _log(rng, 1, min(131071, (1 << 19) * page // B)), "page": page}
    d = rng.choice([64, 64, 128, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 4, 8])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "append":
        step = rng.random() < 0.4  # a token of each sequence, or prompts
        T = _log(rng, 1, 256 if step else 16384 * 8 * 64 // (kv * d))
        return {"kind": kind, "T": T, "run": 1 if step else _log(rng, 64, 4096), "pad": rng.choice([0, _log(rng, 1, T)]),
                "kv": kv, "d": d, "page": page, "dtype": dtype}
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    window = rng.choice([0, 0, _log(rng, 256 if kind == "tree" else 1, 8192)])
    sinks = rng.choice([0, 1, 4, 4, _log(rng, 1, 100)]) if window else 0
    mode = "tree" if kind == "tree" else rng.choice(["token", "token", "few", "chunk"])
    most = 16384 * 8 * 128 * 16  # positions x heads x dims that are held and read
    if mode == "token":
        B, n = _log(rng, 1, 128), 1
        L = _log(rng, 1, 131071)
        if window:
            B = max(1, min(B, most // ((window + sinks + 2 * page) * kv * d)))
        else:
            L = max(1, min(L, most // (B * kv * d)))
    elif mode == "few":
        B, n, kv = _log(rng, 1, 8), rng.randint(2, 16), min(kv, 4)
        L = n + _log(rng, 1, 16384)
    elif mode == "tree":
        B, n = _log(rng, 1, 16), _log(rng, 2, 256)
        L = n + _log(rng, 1, 8192)
        n = max(2, min(n, 1750 * 8192 * 32 * 128 // (B * L * kv * group * d * (16 if dtype == "f32" else 1))))
    else:
        dtype = "bf16"
        B, n = _log(rng, 1, 4), _log(rng, 24, 2048)
        L = n + _log(rng, 1, 6144)
        # no dearer than 2048 tokens of 32 heads of 128 over 8192 positions
        kv, group = min(kv, 4), min(group, 8)
        n = max(1, min(n, 1750 * 8192 * 32 * 128 // (B * L * kv * group * d)))
    return {"kind": kind, "B": B, "n": n, "L": L, "ragged": rng.random() < 0.6, "empty": rng.random() < 0.2,
            "heads": kv * group, "kv": kv, "d": d, "page": page, "window": window, "sinks": sinks, "dtype": dtype}


def _rng(case):
    """What a case fixes whatever the seed: its lengths, and its trees' shapes."""
    return random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """(new tokens, cache length with them) of each sequence."""
    rng = _rng(case)
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


def _requests(case):
    """tables: (positions held, new tokens) of each sequence; some bring no token in this step."""
    rng = _rng(case)
    held, new = [], []
    for b in range(case["B"]):
        n = case["n"] if b == 0 else 0 if rng.random() < 0.05 else rng.randint(1, case["n"])
        new.append(n)
        held.append(0 if case["n"] > 1 and rng.random() < 0.5 else rng.randint(0, case["L"] - n))
    return held, new


def _parents(case, ns):
    """tree: the parent of each drafted token among its sequence's, -1 for a child of the last cached one.  A few
    tokens at each step, each below one of the last step's."""
    rng = _rng(case)
    out = []
    for n in ns:
        par, last = [], [-1]
        while len(par) < n:
            width = min(n - len(par), rng.randint(1, max(2, n // 4)))
            par += sorted(rng.choice(last) for _ in range(width))
            last = list(range(len(par) - width, len(par)))
        out += par
    return out


def _seen(case, n, L):
    """Positions that some token of a sequence sees: [0, first part's end) and [second part's start, L)."""
    first = max(0, L - n - case["window"] + 1) if case["window"] else 0
    return min(case["sinks"], first), first


# ------------------------------------------------------------------------------------------------ inputs ---
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, g, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(ns):
    out = [0]
    for n in ns:
        out.append(out[-1] + n)
    return out


def _keys_values(shape, g, dtype=BF16):
    """Keys with a few strong channels and an offset per channel, values with neither: shape [rows, kv, page, d]."""
    gain = torch.exp(_normal((shape[1], 1, shape[3]), g, 0.5))
    shift = _normal((shape[1], 1, shape[3]), g, 0.3)
    k = torch.empty(shape, dtype=dtype, device="cuda")
    v = torch.empty_like(k)
    step = max(1, (1 << 24) // (shape[1] * shape[2] * shape[3]))
    for i in range(0, shape[0], step):  # a piece at a time: the 32-bit draws are larger than what is kept
        m = min(step, shape[0] - i)
        k[i:i + m] = _normal((m, *shape[1:]), g).mul_(gain).add_(shift)
        v[i:i + m] = _normal((m, *shape[1:]), g, 0.5)
    return k, v


def _inputs(case, seed):
    """Every tensor of a case, made from the seed alone."""
    g = _gen(seed)
    c, page = case, case["page"]
    if c["kind"] == "tables":
        held, new = _requests(c)
        width = -(-c["L"] // page)
        owned = [-(-h // page) for h in held]
        need = sum(-(-(h + n) // page) - o for h, n, o in zip(held, new, owned))
        total = sum(owned) + need + 64
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        table = torch.full((c["B"], width), -1, dtype=torch.int32, device="cuda")
        at = torch.arange(width, device="cuda")
        mine = at < _ints(owned).unsqueeze(1)
        table[mine] = order[:sum(owned)]
        return {"held": _ints(held), "new": _ints(new), "table": table, "free": order[sum(owned):].contiguous(),
                "first": _ints([0]), "T": sum(new), "total": total}
    if c["kind"] == "append":
        T, kv, d = c["T"], c["kv"], c["d"]
        real = T - min(c["pad"], T - 1)
        n_pages = -(-real // page) + (-(-real // c["run"])) + 3
        # runs of `run` tokens, each from some position inside a page of its own
        pages = torch.randperm(n_pages, generator=g, device="cuda").tolist()
        rng = _rng(c)
        slots, t = [], 0
        while t < real:
            m = min(c["run"], real - t)
            offset = rng.randint(0, page - m) if m < page else 0
            for i in range(0, m, page):
                p = pages.pop()
                slots += [p * page + offset + j for j in range(min(page, m - i))]
            t += m
        k, v = _keys_values((T, kv, 1, d), g, DT[c["dtype"]])
        kc, vc = _keys_values((n_pages, kv, page, d), g)
        return {"k": k.view(T, kv, d), "v": v.view(T, kv, d), "kc": kc, "vc": vc, "slots": _ints(slots + [-1] * (T - real))}
    ns, ls = _lengths(c)
    r = {"ns": ns, "ls": ls, "T": sum(ns), "kv_len": _ints(ls), "q_start": _ints(_starts(ns))}
    parts = [_seen(c, n, L) for n, L in zip(ns, ls)]
    held = [[*range(-(-sink // page)), *range(max(first // page, -(-sink // page)), -(-L // page))]
            for (sink, first), L in zip(parts, ls)]
    n_pages = sum(map(len, held)) + 2
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    width = max(1, max(-(-L // page) for L in ls))
    r["table"] = torch.full((c["B"], width), -1, dtype=torch.int32, device="cuda")
    flat = torch.tensor([b * width + p for b, ps in enumerate(held) for p in ps], dtype=torch.int64, device="cuda")
    r["table"].view(-1)[flat] = order[:flat.numel()]
    r["kc"], r["vc"] = _keys_values((n_pages, c["kv"], page, c["d"]), g)
    q = _normal((r["T"], c["heads"], c["d"]), g)
    r["q"] = (q / torch.sqrt((q * q).mean(-1, keepdim=True) + EPS)).to(DT[c["dtype"]])
    if c["kind"] == "tree":
        r["parents"] = _ints(_parents(c, ns))
    return r


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = c = case
    if c["kind"] == "tables":
        s["out"] = {"kv_len": torch.empty_like(s["held"]), "q_start": torch.empty(c["B"] + 1, dtype=torch.int32, device="cuda"),
                    "positions": torch.empty(s["T"], dtype=torch.int32, device="cuda"),
                    "slots": torch.empty(s["T"], dtype=torch.int32, device="cuda"),
                    "free_next": torch.empty(1, dtype=torch.int32, device="cuda")}
    elif c["kind"] in ("attend", "tree"):
        s["out"] = torch.empty_like(s["q"])
        if c["kind"] == "tree":
            s["masks"] = torch.empty((s["T"], -(-c["n"] // 64)), dtype=torch.int64, device="cuda")
            s["positions"] = torch.empty(s["T"], dtype=torch.int32, device="cuda")
    if own:
        import paper_2605_29135_amd as moe
        moe.moe_init(torch.cuda.current_device())
        if c["kind"] in ("attend", "tree"):
            s["max_kv"] = max(max(s["ls"]), 1)
            n = moe.moe_paged_attention_workspace_bytes(s["T"], c["B"], c["heads"], c["kv"], c["d"], c["n"], s["max_kv"])
            s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------- plain forms ---
def _tables(s):
    page, table, o = s["case"]["page"], s["table"], s["out"]
    held, new = s["held"].long(), s["new"].long()
    dev = held.device
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), torch.cumsum(new, 0)])
    have = (held + page - 1) // page
    need = (held + new + page - 1) // page - have
    before = torch.cumsum(need, 0) - need + s["first"].long()
    # the pages: column have + i of a sequence's row, i < need
    at = torch.arange(table.shape[1], device=dev) - have.unsqueeze(1)
    fresh = (at >= 0) & (at < need.unsqueeze(1))
    table[fresh] = s["free"][(before.unsqueeze(1) + at)[fresh]]
    # the tokens
    t = torch.arange(s["T"], device=dev)
    seq = torch.repeat_interleave(torch.arange(held.numel(), device=dev), new, output_size=s["T"])
    pos = t - starts[seq] + held[seq]
    o["kv_len"].copy_(held + new)
    o["q_start"].copy_(starts)
    o["positions"].copy_(pos)
    o["slots"].copy_(table[seq, pos // page].long() * page + pos % page)
    o["free_next"].copy_(s["first"] + need.sum())
    return o["kv_len"], o["q_start"], o["positions"], o["slots"], o["free_next"], table


def _append(s):
    page, slots = s["case"]["page"], s["slots"].long()
    keep = slots >= 0
    p, off = slots[keep] // page, slots[keep] % page
    s["kc"][p, :, off] = s["k"][keep].to(BF16)
    s["vc"][p, :, off] = s["v"][keep].to(BF16)
    return s["kc"], s["vc"]


def _masks(s):
    """Each drafted token's row of bits (itself and the tokens above it), and its position."""
    masks, positions = s["masks"], s["positions"]
    dev, words = masks.device, masks.shape[1]
    weight = torch.ones(64, dtype=torch.int64, device=dev) << torch.arange(64, device=dev)
    t0 = 0
    for n, L in zip(s["ns"], s["ls"]):
        par = s["parents"][t0:t0 + n].long()
        see = torch.eye(n, dtype=torch.float32, device=dev)
        link = torch.zeros((n, n + 1), dtype=torch.float32, device=dev)
        link[torch.arange(n, device=dev), torch.where(par < 0, n, par)] = 1
        link = link[:, :n].contiguous()  # (a child of the cache has no other token above it)
        hops = 1
        while hops < n:  # what is within `hops` steps above, doubled
            see = ((see + link @ see) > 0).float()
            link = link @ link
            hops *= 2
        bits = torch.zeros((n, words * 64), dtype=torch.int64, device=dev)
        bits[:, :n] = see.long()
        masks[t0:t0 + n] = (bits.view(n, words, 64) * weight).sum(-1)
        positions[t0:t0 + n] = (L - n - 1 + see.sum(-1)).to(torch.int32)
        t0 += n
    return masks, positions


def _attend(s):
    c = s["case"]
    G, d, kv, page, window, sinks = c["heads"] // c["kv"], c["d"], c["kv"], c["page"], c["window"], c["sinks"]
    out, dev = s["out"], s["q"].device
    tree = c["kind"] == "tree"
    if tree:
        masks, positions = _masks(s)
    t0 = 0
    for b, (n, L) in enumerate(zip(s["ns"], s["ls"])):
        sink, first = _seen(c, n, L)
        if L:
            p = torch.cat([torch.arange(sink, device=dev), torch.arange(first, L, device=dev)])
            m, at = p.numel(), s["table"][b].long()[p // page]
            K = s["kc"][at, :, p % page].float().transpose(0, 1).contiguous()
            V = s["vc"][at, :, p % page].float().transpose(0, 1).contiguous()
            q = s["q"][t0:t0 + n].float().view(n, kv, G, d).permute(1, 0, 2, 3).reshape(kv, n * G, d)
            z = torch.bmm(q, K.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(kv, n, G, m)
            row = torch.arange(L - n, L, device=dev)
            own_pos = (positions[t0:t0 + n].long() if tree else row).view(n, 1, 1)
            hidden = p > own_pos
            if window:
                hidden = hidden | ((p <= own_pos - window) & (p >= sinks))
            if tree:
                j = p - (L - n)
                bit = (masks[t0:t0 + n][:, (j.clamp(min=0) // 64)] >> (j % 64)) & 1
                hidden = torch.where(j >= 0, bit.view(n, 1, m) == 0, hidden)
            hidden = hidden | (row < 0).view(n, 1, 1)
            z.masked_fill_(hidden, -math.inf)
            z = torch.exp_(z.sub_(z.amax(-1, keepdim=True).clamp_(min=-3e38)))
            total = z.sum(-1).view(kv, n * G, 1)
            o = torch.bmm(z.view(kv, n * G, m), V) / torch.where(total > 0, total, 1.0)
            out[t0:t0 + n] = o.view(kv, n, G, d).permute(1, 0, 2, 3).reshape(n, c["heads"], d).to(out.dtype)
        else:
            out[t0:t0 + n] = 0
        t0 += n
    return (out, masks, positions) if tree else out


def run(s):
    c = s["case"]
    if not own:
        return {"tables": _tables, "append": _append, "attend": _attend, "tree": _attend}[c["kind"]](s)
    import paper_2605_29135_amd as moe
    if c["kind"] == "tables":
        o = s["out"]
        moe.moe_page_tables(s["held"], s["new"], s["free"], s["table"], c["page"], s["total"], s["T"], free_first=s["first"],
                            kv_len_out=o["kv_len"], q_start=o["q_start"], positions=o["positions"], slots=o["slots"],
                            free_next=o["free_next"])
        return o["kv_len"], o["q_start"], o["positions"], o["slots"], o["free_next"], s["table"]
    if c["kind"] == "append":
        moe.moe_paged_append(s["k"], s["v"], s["kc"], s["vc"], s["slots"])
        return s["kc"], s["vc"]
    tree = None
    if c["kind"] == "tree":
        tree, _ = moe.moe_tree_masks(s["parents"], q_start=s["q_start"], max_q=c["n"], kv_len=s["kv_len"],
                                     masks=s["masks"], positions=s["positions"])
    out = moe.moe_paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["kv_len"], q_start=s["q_start"], max_q=c["n"],
                                  max_kv=s["max_kv"], window=c["window"], sinks=c["sinks"], tree=tree, out=s["out"],
                                  workspace=s["ws"])
    return (out, tree, s["positions"]) if c["kind"] == "tree" else out


# -------------------------------------------------------------------------------------------------- work ---
def work(case):
    c, page = case, case["page"]
    if c["kind"] == "tables":
        held, new = _requests(c)
        fresh = sum(-(-(h + n) // page) - -(-h // page) for h, n in zip(held, new))
        # lengths in and out, starts, positions, slots, the pages taken and those that tokens continue
        return {"bytes": 4 * (4 * c["B"] + 2 * sum(new) + 2 * fresh + sum(1 for h, n in zip(held, new) if n and h % page) + 3),
                "flops": 4 * sum(new) + 8 * c["B"]}
    if c["kind"] == "append":
        kept, size = c["T"] - min(c["pad"], c["T"] - 1), 4 if c["dtype"] == "f32" else 2
        return {"bytes": kept * 2 * c["kv"] * c["d"] * (size + 2) + 4 * c["T"], "flops": kept * 2 * c["kv"] * c["d"]}
    ns, ls = _lengths(c)
    d, kv, size = c["d"], c["kv"], 4 if c["dtype"] == "f32" else 2
    tree = c["kind"] == "tree"
    par, t0 = _parents(c, ns) if tree else [], 0
    seen = pairs = 0
    for n, L in zip(ns, ls):
        sink, first = _seen(c, n, L)
        seen += sink + L - first
        w, depth = c["window"] or L + 1, []
        for i in range(n):
            if tree:
                depth.append(0 if par[t0 + i] < 0 else depth[par[t0 + i]] + 1)
            at = L - n + (depth[i] if tree else i)  # the token's position
            if L - n + i < 0:
                continue
            lo = max(0, at - w + 1)
            cached = max(0, L - n)
            if tree:
                pairs += min(min(c["sinks"], lo), cached) + max(0, cached - lo) + min(depth[i] + 1, L)
            else:
                pairs += min(c["sinks"], lo) + at + 1 - lo
        t0 += n
    extra = sum(ns) * (8 * -(-c["n"] // 64) + 8) if tree else 0
    return {"bytes": 2 * sum(ns) * c["heads"] * d * size + seen * 4 * kv * d + extra, "flops": 4 * d * c["heads"] * pairs}


# ------------------------------------------------------------------------------------------------- exact ---
def _exact_tables(s, c):
    page, T = c["page"], s["T"]
    table = s["table"].cpu().tolist()
    free, k = s["free"].tolist(), s["first"].item()
    lens, starts, positions, slots = [], [0], [], []
    for row, h, n in zip(table, s["held"].tolist(), s["new"].tolist()):
        for col in range(-(-h // page), -(-(h + n) // page)):
            row[col] = free[k]
            k += 1
        positions += range(h, h + n)
        slots += [row[p // page] * page + p % page for p in range(h, h + n)]
        lens.append(h + n)
        starts.append(starts[-1] + n)
    return _ints(lens), _ints(starts), _ints(positions), _ints(slots), _ints([k]), _ints(table)


def exact(case, seed):
    c = case
    s = _inputs(case, seed)
    f8, page = torch.float64, case["page"]
    if c["kind"] == "tables":
        return _exact_tables(s, c)
    if c["kind"] == "append":
        out = []
        for x, cache in ((s["k"], s["kc"]), (s["v"], s["vc"])):
            y = cache.to(f8).transpose(1, 2).contiguous()  # [page, position, head, dim]
            keep = torch.nonzero(s["slots"] >= 0).flatten()
            y.view(-1, c["kv"], c["d"]).index_copy_(0, s["slots"][keep].long(), x[keep].to(f8))
            out.append(y.transpose(1, 2).contiguous())
        return tuple(out)
    G, d, tree = c["heads"] // c["kv"], c["d"], c["kind"] == "tree"
    out = torch.zeros(s["q"].shape, dtype=f8, device="cuda")
    words = -(-c["n"] // 64)
    masks, positions = [], []
    par = s["parents"].tolist() if tree else None
    t = 0
    for b, (n, L) in enumerate(zip(s["ns"], s["ls"])):
        lines = []
        for i in range(n if tree else 0):  # a token's line is its parent's and itself
            lines.append((lines[par[t + i]] if par[t + i] >= 0 else 0) | 1 << i)
            positions.append(L - n - 1 + bin(lines[i]).count("1"))
            for w in range(words):
                m = lines[i] >> 64 * w & (1 << 64) - 1
                masks.append(m - (1 << 64) if m >> 63 else m)
        sink, first = _seen(c, n, L)
        p = torch.tensor([*range(sink), *range(first, L)], device="cuda")
        rows = s["table"][b, p // page].long() * c["kv"] * page + p % page if L else p
        if tree and L:
            draft = torch.tensor([[line >> j & 1 for j in range(n)] for line in lines], dtype=torch.bool, device="cuda")
        for h in range(c["kv"] if L else 0):
            K, V = (x.view(-1, d)[rows + h * page].to(f8) for x in (s["kc"], s["vc"]))
            for i in range(max(0, n - L), n, 256):  # the rows that see something
                j = min(n, i + 256)
                at = torch.arange(L - n + i, L - n + j, device="cuda").unsqueeze(1)
                if tree:
                    at = torch.tensor(positions[t + i:t + j], device="cuda").unsqueeze(1)
                see = (p <= at) & ((p > at - (c["window"] or L + 1)) | (p < c["sinks"]))
                if tree:
                    drafted = p >= L - n
                    see[:, drafted] = draft[i:j, n - int(drafted.sum()):]
                q = s["q"][t + i:t + j, h * G:(h + 1) * G].to(f8)
                z = (q.reshape(-1, d) @ K.T).view(j - i, G, -1) / math.sqrt(d)
                w = torch.softmax(torch.where(see.unsqueeze(1), z, torch.tensor(-math.inf, dtype=f8, device="cuda")), -1)
                out[t + i:t + j, h * G:(h + 1) * G] = torch.nan_to_num(w.view((j - i) * G, -1) @ V).view(j - i, G, d)
        t += n
    if not tree:
        return out
    return out, torch.tensor(masks, dtype=torch.int64, device="cuda").view(-1, words), _ints(positions)
