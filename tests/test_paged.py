"""The paged key/value cache, its tables, the attention over it with windows, first positions and drafted trees, against
plain 64-bit implementations."""
import math
import random

import pytest
import torch

import paper_2605_29135_amd as moe

F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
OK_PTR = 1 << 20  # an aligned address that no refused call touches


def refused(name, *args):
    code = getattr(moe.lib(), name)(*args)
    assert code == -1, (name, args, code)
    assert moe.lib().moe_last_error()


def ints(v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


def starts(ns):
    out = [0]
    for n in ns:
        out.append(out[-1] + n)
    return out


def flags(code=None):
    """The device's sticky error, which has to be `code` (None: no error); cleared."""
    if code is None:
        return moe.moe_sync_check()
    with pytest.raises(moe.MoeError) as e:
        moe.moe_sync_check()
    assert e.value.code == code


RANGE, BUDGET = -2, -4


# ------------------------------------------------------------------------------------------ plain forms ---
def plain_tables(lens, new, free, first, table, page, T):
    """(table, lengths, starts, positions, slots, next) by the definition, pages one by one."""
    table = [list(r) for r in table]
    out_len, q_start, positions, slots = [], [0], [], []
    for row, h, n in zip(table, lens, new):
        n = min(n, T - len(positions))
        for col in range(-(-h // page), -(-(h + n) // page)):
            row[col] = free[first] if first < len(free) else -1
            first += 1
        for p in range(h, h + n):
            positions.append(p)
            slots.append(row[p // page] * page + p % page if row[p // page] >= 0 else -1)
        out_len.append(h + n)
        q_start.append(len(positions))
    pad = [-1] * (T - len(positions))
    return table, out_len, q_start, positions + pad, slots + pad, min(first, len(free))


def line(parents, i):
    """A drafted token and those above it, as bits."""
    bits = 0
    while i >= 0:
        bits |= 1 << i
        i = parents[i]
    return bits


def as_words(bits, words):
    w = [(bits >> 64 * k) & (2 ** 64 - 1) for k in range(words)]
    return [x - 2 ** 64 if x >> 63 else x for x in w]


def sees(n, L, window, sinks, bits=None):
    """Which of L positions each of a sequence's n tokens sees: bool [n, L]."""
    p = torch.arange(L)
    out = torch.zeros((n, L), dtype=torch.bool)
    for i in range(n):
        row = L - n + i
        if row < 0:
            continue
        at = row if bits is None else L - n - 1 + max(1, bin(bits[i] & ((1 << n) - 1)).count("1"))
        near = (p > at - window) | (p < sinks) if window else torch.ones(L, dtype=torch.bool)
        out[i] = near & (p <= at)
        if bits is not None:
            for j in range(max(0, n - L), n):
                out[i, L - n + j] = bool(bits[i] >> j & 1)
    return out


def attend(q, ks, vs, visible, G, scale, f32):
    """Plain attention of q (per sequence [n, heads, d], float64) over per-sequence vectors [L, kv, d], and the two parts
    of its error bound: `amount` (sum of P |V|), and `shift`, how far a score can be off, in natural units.  With T terms
    of a query's elements a score is the sum of T d / 32 matrix products of 32, each with four roundings of 2^-24 of what
    has been added up; its way to the exponent has two more, of the score."""
    outs, amounts, shifts = [], [], []
    for x, K, V, see in zip(q, ks, vs, visible):
        n, heads, d = x.shape
        out = torch.zeros_like(x)
        amount, shift = torch.zeros_like(x), torch.zeros((n, heads, 1), dtype=F64)
        steps = (3 if f32 else 1) * d / 32 * 4 + 4
        for h in range(heads // G if K.shape[0] else 0):
            cols = slice(h * G, (h + 1) * G)
            z = (x[:, cols] @ K[:, h].T) * scale
            zz = torch.where(see.unsqueeze(1), z, torch.tensor(-math.inf, dtype=F64))
            w = torch.where(see.any(1).view(n, 1, 1), torch.softmax(zz, -1), torch.zeros_like(z))
            w = torch.nan_to_num(w)
            out[:, cols], amount[:, cols] = w @ V[:, h], w @ V[:, h].abs()
            e = x[:, cols].abs() @ K[:, h].abs().T * abs(scale) * steps * 2.0 ** -24 + z.abs() * 2.0 ** -22
            shift[:, cols] = torch.where(see.unsqueeze(1), e, torch.zeros_like(e)).amax(-1, keepdim=True)
        outs.append(out), amounts.append(amount), shifts.append(shift)
    return torch.cat(outs), torch.cat(amounts), torch.cat(shifts)


def tolerance(ref, amount, shift, dtype, L):
    """Errors e of the scores change a probability by e, and the sum of them by at most as much again; exponentials 2^-22;
    sums over L positions: a lane adds up at most L / 8 of them, then the joins (64 at most), 2^-24 each, in the sum and in
    the output; a probability is rounded to three bf16 terms (2^-24), or to one at least (2^-8, calls of many rows)."""
    term = 2.0 ** -24 if dtype is F32 else 2.0 ** -8
    return amount * (2 * shift + 2.0 ** -21 + 2 * (L / 8 + 64) * 2.0 ** -24 + term) + ref.abs() * torch.finfo(dtype).eps / 2 + 1e-30


def relative_rms(out, ref):
    return float((out.cpu().double() - ref).square().mean().sqrt() / ref.square().mean().sqrt())


# Largest relative rms error over values of one size and scores of a few units.  fp32: scores of up to 16 in log2 units, each
# within 2^-23 with both signs, and the exponential's last place; about 4e-7.  bf16: the output's rounding, 2^-8 at most and
# evenly spread (2^-8 / sqrt 3 of the lowest value of a binade, 1.66e-3 over all), and for calls of many rows one such
# rounding of the probabilities beside it: 2.35e-3 together.
RMS = {F32: 1e-6, BF16: 2.6e-3}


# --------------------------------------------------------------------------------------- a cache to test on ---
class Cache:
    """Pools whose unseen places hold NaN, and tables whose unneeded entries are no pages."""

    def __init__(self, ls, n_kv, d, page, gen, extra=3, interleaved=False, spare=0, amplitude=1.0):
        self.page, self.ls, self.n_kv, self.d = page, ls, n_kv, d
        need = [-(-L // page) for L in ls]
        n_pages = sum(need) + extra
        order = torch.randperm(n_pages, generator=gen).tolist()
        width = max(1, max(need)) + spare
        self.table = [[order.pop() for _ in range(m)] + [-7] * (width - m) for m in need]
        if interleaved:
            both = torch.full((n_pages, 2, n_kv, page, d), math.nan, dtype=BF16, device="cuda")
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = moe.paged_cache(n_pages, n_kv, page, d)
            self.k.fill_(math.nan), self.v.fill_(math.nan)
        self.ks = [(torch.randn((L, n_kv, d), generator=gen) * amplitude).to(BF16) for L in ls]
        self.vs = [torch.randn((L, n_kv, d), generator=gen).to(BF16) for L in ls]

    def slots(self, b, lo, hi):
        return [self.table[b][p // self.page] * self.page + p % self.page for p in range(lo, hi)]

    def put(self, seen=None):
        """Writes the vectors of the positions that some token sees (`seen`: bool [L] per sequence; None: all)."""
        slots, ks, vs = [], [], []
        for b, L in enumerate(self.ls):
            keep = torch.ones(L, dtype=torch.bool) if seen is None else seen[b]
            slots += [s for s, x in zip(self.slots(b, 0, L), keep.tolist()) if x]
            ks.append(self.ks[b][keep]), vs.append(self.vs[b][keep])
        moe.moe_paged_append(torch.cat(ks).cuda(), torch.cat(vs).cuda(), self.k, self.v, ints(slots))
        if seen is not None:  # pages that no token sees are not there
            for b, L in enumerate(self.ls):
                for c in range(-(-L // self.page)):
                    if not seen[b][c * self.page:(c + 1) * self.page].any():
                        self.table[b][c] = -1 - c
        return self

    @property
    def dev_table(self):
        return ints(self.table)


def random_tree(n, rng, wide):
    return [rng.randint(-1, i - 1) if wide else max(-1, i - 1 - rng.randint(0, 2)) for i in range(n)]


def run_case(d, n_kv, G, page, ns, ls, window, sinks, tree, dtype, seed=0, scale=None, amplitude=1.0, **kw):
    """(outputs, reference, amount, shift, cache and batch) of one attention."""
    gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
    cache = Cache(ls, n_kv, d, page, gen, amplitude=amplitude)
    parents = [random_tree(n, rng, tree == "wide") for n in ns] if tree else None
    bits = [[line(p, i) for i in range(len(p))] for p in parents] if tree else [None] * len(ns)
    visible = [sees(n, L, window, sinks, b) for n, L, b in zip(ns, ls, bits)]
    cache.put([v.any(0) for v in visible])
    T = sum(ns)
    q = torch.randn((T, n_kv * G, d), generator=gen).to(dtype)
    scale = d ** -0.5 if scale is None else scale
    batch = dict(q_start=ints(starts(ns)), max_q=max(ns))
    masks = None
    if tree:
        flat = [x for p in parents for x in p]
        masks, positions = moe.moe_tree_masks(ints(flat), kv_len=ints(ls), **batch)
        words = -(-max(ns) // 64)
        assert masks.cpu().tolist() == [as_words(x, words) for b in bits for x in b]
        assert positions.cpu().tolist() == [L - n - 1 + bin(x).count("1") for n, L, b in zip(ns, ls, bits) for x in b]
    args = dict(batch, window=window, sinks=sinks, tree=masks, scale=scale, max_kv=max(max(ls), 1))
    out = moe.moe_paged_attention(q.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), **args, **kw)
    qs = [q[a:b].double() for a, b in zip(starts(ns), starts(ns)[1:])]
    ref = attend(qs, [k.double() for k in cache.ks], [v.double() for v in cache.vs], visible, G, scale, dtype is F32)
    return out, *ref, (cache, q, args)


# ------------------------------------------------------------------------------------------------ refusals ---
def test_tables_refusals():
    P = OK_PTR
    good = dict(kv_len=P, n_new=P, n_seq=3, T=8, page=16, n_pages=100, free=P, n_free=10, first=P, table=P, max_pages=8, out=P,
                qs=P, pos=P, slots=P, next=P)
    bads = [dict(kv_len=None), dict(table=None), dict(out=None), dict(qs=None), dict(free=None), dict(n_seq=-1),
            dict(n_seq=65536), dict(T=-1), dict(T=(1 << 30) + 1), dict(page=8), dict(page=48), dict(page=0), dict(page=65536),
            dict(n_pages=0), dict(n_pages=1 << 27), dict(n_free=-1), dict(max_pages=0), dict(max_pages=(1 << 22) + 1),
            dict(slots=P + 2), dict(table=P + 1)]
    for b in bads:
        refused("moe_page_tables", *{**good, **b}.values(), None)


def test_append_refusals():
    P = OK_PTR
    good = dict(k=P, v=P, dtype=0, ks=256, vs=256, T=4, n_kv=4, d=64, slots=P, kp=P, vp=P, kps=4096, vps=4096, n_pages=9, page=16)
    bads = [dict(k=None), dict(v=None), dict(slots=None), dict(kp=None), dict(vp=None), dict(k=P + 8), dict(kp=P + 8),
            dict(dtype=2), dict(dtype=-1), dict(ks=252), dict(vs=258), dict(ks=-256), dict(T=-1), dict(n_kv=0), dict(n_kv=70000),
            dict(d=32), dict(d=96), dict(kps=4088), dict(vps=4100), dict(kps=1 << 31), dict(n_pages=0), dict(page=17),
            dict(slots=P + 2)]
    for b in bads:
        refused("moe_paged_append", *{**good, **b}.values(), None)
    assert moe.lib().moe_paged_append(None, None, 0, 0, 0, 0, 4, 64, None, None, None, 0, 0, 9, 16, None) == 0


def test_tree_refusals():
    P = OK_PTR
    good = dict(par=P, T=9, n_seq=2, qs=P, max_q=8, kv_len=P, masks=P, words=1, pos=P)
    for b in [dict(par=None), dict(masks=None), dict(T=-1), dict(n_seq=-1), dict(n_seq=65536), dict(qs=None), dict(max_q=0),
              dict(max_q=257, words=4), dict(max_q=65), dict(words=0), dict(words=5), dict(masks=P + 4), dict(pos=P + 2)]:
        refused("moe_tree_masks", *{**good, **b}.values(), None)
    assert moe.lib().moe_tree_masks(None, 0, 0, None, 1, None, None, 1, None, None) == 0


def test_attention_refusals():
    P, big = OK_PTR, 1 << 40
    good = dict(q=P, dtype=1, qs=512, kp=P, vp=P, kps=4096, vps=4096, n_pages=300, page=16, table=P, max_pages=256, T=2, n_seq=2,
                heads=8, n_kv=4, d=64, q_start=None, max_q=1, kv_len=P, max_kv=4096, window=0, sinks=0, tree=None, words=0,
                scale=0.125, out=P, os=512, ws=P, wb=big)
    bads = [dict(q=None), dict(out=None), dict(kp=None), dict(vp=None), dict(table=None), dict(kv_len=None), dict(q=P + 2),
            dict(out=P + 8), dict(kp=P + 8), dict(qs=508), dict(os=516), dict(kps=4088), dict(dtype=3), dict(T=3), dict(heads=9),
            dict(heads=0), dict(n_kv=0), dict(d=48), dict(n_pages=0), dict(page=24), dict(max_pages=0), dict(max_kv=0),
            dict(max_kv=4097), dict(max_kv=(1 << 26) + 1), dict(window=-1), dict(window=(1 << 30) + 1), dict(sinks=-1),
            dict(scale=math.inf), dict(scale=math.nan), dict(scale=-4.5e9), dict(ws=None), dict(ws=P + 4), dict(wb=16),
            dict(q_start=P, max_q=0), dict(q_start=P, max_q=1 << 24), dict(tree=P, words=0), dict(tree=P + 4, words=1),
            dict(tree=P, words=1, window=1, q_start=P, max_q=2), dict(table=P + 2),
            dict(T=200, q_start=P, max_q=65, tree=P, words=1)]
    for b in bads:
        refused("moe_paged_attention", *{**good, **b}.values(), None)
    size = moe.moe_paged_attention_workspace_bytes
    assert size(2, 2, 8, 4, 64, 1, 4096) > 0
    assert size(2, 2, 9, 4, 64, 1, 4096) == size(2, 2, 8, 4, 65, 1, 4096) == size(2, 2, 8, 4, 64, 1, 0) == 0
    none = {**good, **dict(q=None, table=None, kv_len=None, out=None, T=0, n_seq=0, ws=None, wb=0)}
    assert moe.lib().moe_paged_attention(*none.values(), None) == 0


def test_binding_refuses_host_tensors_and_shapes():
    k, v = moe.paged_cache(4, 2, 16, 64, device="cpu")
    q = torch.zeros((2, 4, 64))
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    table, lens = torch.zeros((2, 3), dtype=torch.int32), i32(2)
    for call in [lambda: moe.moe_paged_attention(q, k, v, table, lens),  # host tensors
                 lambda: moe.moe_paged_attention(q, k.float(), v, table, lens),
                 lambda: moe.moe_paged_attention(q, k, v[:3], table, lens),
                 lambda: moe.moe_paged_attention(q[:, :, :32], k, v, table, lens),
                 lambda: moe.moe_paged_attention(q, k, v, table[0], lens),
                 lambda: moe.moe_paged_attention(q, k, v, table.long(), lens),
                 lambda: moe.moe_paged_attention(q, k, v, table, lens[:1]),
                 lambda: moe.moe_paged_attention(q, k, v, table, lens, window=-1),
                 lambda: moe.moe_paged_attention(q, k, v, table, lens, sinks=1 << 31),
                 lambda: moe.moe_paged_attention(q, k, v, table, lens, tree=i32((2, 1))),
                 lambda: moe.moe_paged_attention(q, k.transpose(1, 2), v.transpose(1, 2), table, lens),
                 lambda: moe.moe_paged_append(q[:, :2], q[:, :2], k, v, i32(2)),
                 lambda: moe.moe_paged_append(q[:, :3], q[:, :3], k, v, i32(2)),
                 lambda: moe.moe_tree_masks(i32(3), q_start=i32(2)),
                 lambda: moe.moe_tree_masks(i32((3, 1))),
                 lambda: moe.moe_page_tables(lens, None, i32(4), table, 16, 4, 2),
                 lambda: moe.moe_page_tables(lens, None, i32(4), table, 16, 4, 1 << 31)]:
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------------------------------------- tables ---
def requests(n_seq, most, page, seed, width=24):
    rng = random.Random(seed)
    new = [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(n_seq)]
    lens = [rng.choice([0, page, rng.randint(0, width * page - n)]) if width * page - n >= page else 0 for n in new]
    pool = list(range(n_seq * width + 500))
    rng.shuffle(pool)
    table = [[pool.pop() if c < -(-h // page) else -5 for c in range(width)] for h in lens]
    return lens, new, table, pool


@pytest.mark.gpu
@pytest.mark.parametrize("n_seq,most,page", [(1, 1, 16), (1, 300, 16), (5, 40, 32), (63, 200, 16), (300, 1, 64), (300, 50, 16),
                                             (2047, 9, 16), (2049, 3, 16), (5000, 2, 128), (7, 90000, 4096)])
@pytest.mark.parametrize("pad", [0, 5, 2000])
def test_tables_match_the_plain_form(n_seq, most, page, pad):
    lens, new, table, pool = requests(n_seq, most, page, n_seq + most)
    T, first = sum(new) + pad, 3
    want = plain_tables(lens, new, pool, first, table, page, T)
    dev = ints(table)
    got = moe.moe_page_tables(ints(lens), ints(new), ints(pool), dev, page, 1 << 20 if page <= 1024 else 1 << 18, T,
                              free_first=ints([first]))
    flags()
    assert dev.cpu().tolist() == want[0]
    assert [t.cpu().tolist() for t in got] == [*map(list, want[1:5]), [want[5]]]


@pytest.mark.gpu
def test_tables_in_place_and_one_token_each():
    """A step's lengths and first free page in place, over and over, with no positions asked for."""
    page, B = 16, 9
    lens, pool = [15, 16, 17, 0, 31, 32, 33, 1, 47], list(range(200))
    table = [[100 + 5 * b + c if c < -(-h // page) else -1 for c in range(8)] for b, h in enumerate(lens)]
    dev, dl, first, free = ints(table), ints(lens), ints([0]), ints(pool)
    slots, q_start = ints([0] * (B + 2)), ints([0] * (B + 1))
    at = 0
    for _ in range(40):
        want = plain_tables(lens, [1] * B, pool, at, table, page, B + 2)
        moe.moe_page_tables(dl, None, free, dev, page, 4096, B + 2, free_first=first, kv_len_out=dl, q_start=q_start, slots=slots,
                            free_next=first)
        table, lens, at = want[0], want[1], want[5]
        assert dev.cpu().tolist() == table and dl.cpu().tolist() == lens and first.item() == at
        assert slots.cpu().tolist() == want[4] and q_start.cpu().tolist() == want[2]
    flags()


@pytest.mark.gpu
def test_tables_errors():
    page = 16
    blank = [[-1] * 4 for _ in range(3)]

    def call(lens, new, pool, T, first=None, n_pages=1000, table=blank):
        dev = ints(table)
        r = moe.moe_page_tables(ints(lens), None if new is None else ints(new), ints(pool), dev, page, n_pages, T,
                                free_first=None if first is None else ints([first]))
        return [dev.cpu().tolist(), *(t.cpu().tolist() for t in r)]

    # the free pages end: entries and slots are -1 from there on
    got = call([0, 0, 0], [20, 20, 20], [7, 8, 9], 60)
    assert got[0] == [[7, 8, -1, -1], [9, -1, -1, -1], [-1, -1, -1, -1]] and got[5] == [3]
    assert got[4] == [*range(112, 132), *range(144, 160)] + [-1] * 24
    flags(BUDGET)
    got = call([0, 0, 0], [20, 20, 20], [], 60)
    assert got[0] == blank and got[4] == [-1] * 60 and got[5] == [0]
    flags(BUDGET)
    # lengths and counts that do not fit
    full = [[0, 1, 2, 3], [4, -1, -1, -1], [-1] * 4]
    got = call([64, 3, -1], [1, 2, 5], [7, 8], 8, table=full)
    assert got[0] == full and got[1] == [64, 5, 0] and got[2] == [0, 0, 2, 2] and got[3] == [3, 4] + [-1] * 6
    flags(RANGE)
    got = call([65, 3, 0], [0, -2, 1], [7, 8], 8, table=full)
    assert got[1] == [0, 3, 1] and got[2] == [0, 0, 0, 1] and got[0][2] == [7, -1, -1, -1] and got[4] == [112] + [-1] * 7
    flags(RANGE)
    got = call([2**31 - 1, 3, 0], [2**31 - 1] * 3, [7, 8], 8, table=full)
    assert got[1] == [0, 3, 0] and got[2] == [0, 0, 0, 0] and got[4] == [-1] * 8
    flags(RANGE)
    # tokens past the last row are not added
    got = call([0, 0, 0], [10, 20, 20], [7, 8, 9], 17)
    assert got[1] == [10, 7, 0] and got[2] == [0, 10, 17, 17] and got[0] == [[7, -1, -1, -1], [8, -1, -1, -1], [-1] * 4]
    assert got[5] == [2]
    flags(RANGE)
    # pages that are none, in the list and in the table
    got = call([0, 3, 0], [1, 1, 1], [1000, -3], 3, table=[[-1] * 4, [5000, -1, -1, -1], [-1] * 4])
    assert got[0] == [[-1] * 4, [5000, -1, -1, -1], [-1] * 4] and got[4] == [-1] * 3
    flags(RANGE)
    for first in (-1, 3):
        call([0, 0, 0], [0, 0, 0], [7, 8], 0, first=first)
        flags(RANGE)
    # no sequence, no row
    r = moe.moe_page_tables(ints([]), None, ints([]), ints([]).view(0, 4), page, 10, 3)
    assert [t.cpu().tolist() for t in r] == [[], [0], [-1] * 3, [-1] * 3, [0]]
    r = moe.moe_page_tables(ints([5]), ints([0]), ints([]), ints([[1]]), page, 10, 0)
    assert [t.cpu().tolist() for t in r] == [[5], [0, 0], [], [], [0]]
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("wrong", [-1, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("T", [40, 9000])  # (the rows by one launch, and by one of their own)
def test_tables_report_a_page_of_the_table_that_is_missing(T, wrong):
    """A bad entry that a new token continues; one that no new token lies on is nobody's business."""
    page, n_pages, lens, new = 16, 1000, [0, 35, 16, 20], [T - 10, 4, 2, 0]
    blank = [-5] * 600
    for entry in (901, wrong):
        table = [blank, [900, 902, entry] + blank[3:], [903] + blank[1:], [904, wrong] + blank[2:]]
        want = plain_tables(lens, new, list(range(700)), 0, table, page, T)
        slots = [s if s < n_pages * page else -1 for s in want[4]]
        assert slots.count(-1) == (4 if entry == 901 else 8)  # (rows of padding, and the second sequence's)
        dev = ints(table)
        got = moe.moe_page_tables(ints(lens), ints(new), ints(list(range(700))), dev, page, n_pages, T)
        flags(None if entry == 901 else RANGE)
        assert dev.cpu().tolist() == want[0]
        assert [t.cpu().tolist() for t in got] == [*map(list, want[1:4]), slots, [want[5]]]


@pytest.mark.gpu
@pytest.mark.parametrize("n_seq,most,page,width", [(5000, 30, 16, 6), (65535, 3, 32, 2), (2049, 200, 16, 16)])
def test_tables_of_many_sequences_and_rows(n_seq, most, page, width):
    """Rows by a launch of their own, of more sequences than it looks at in one go."""
    lens, new, table, pool = requests(n_seq, most, page, n_seq, width=width)
    T = sum(new) + 3000
    assert T > 3 * 8192
    want = plain_tables(lens, new, pool, 0, table, page, T)
    dev = ints(table)
    got = moe.moe_page_tables(ints(lens), ints(new), ints(pool), dev, page, 1 << 20, T)
    flags()
    assert dev.cpu().tolist() == want[0]
    assert [t.cpu().tolist() for t in got] == [*map(list, want[1:5]), [want[5]]]


@pytest.mark.gpu
def test_tables_after_a_step_without_free_pages():
    """Its own call raises MOE_ERR_BUDGET; tokens that the next one adds to the missing page are not dropped in silence."""
    table = ints([[-5] * 4])
    lens, _, _, slots, _ = moe.moe_page_tables(ints([0]), ints([20]), ints([7]), table, 16, 100, 20)
    assert slots.cpu().tolist() == [*range(112, 128)] + [-1] * 4
    flags(BUDGET)
    lens, _, _, slots, _ = moe.moe_page_tables(lens, ints([14]), ints([8]), table, 16, 100, 14)
    assert slots.cpu().tolist() == [-1] * 12 + [128, 129] and table.cpu().tolist() == [[7, -1, 8, -5]]
    flags(RANGE)


# ------------------------------------------------------------------------------------------------- append ---
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,n_kv,page,T", [(64, 1, 16, 1), (64, 3, 32, 77), (128, 8, 16, 300), (192, 5, 64, 40),
                                           (256, 40, 16, 9), (256, 1, 32768, 3), (64, 8, 128, 4099)])
@pytest.mark.parametrize("layout", ["apart", "interleaved"])
def test_append_writes_the_slots_and_nothing_else(dtype, d, n_kv, page, T, layout):
    gen = torch.Generator().manual_seed(d + T)
    n_pages = -(-T // page) + 3
    if layout == "interleaved":
        both = torch.zeros((n_pages, 2, n_kv, page, d), dtype=BF16, device="cuda")
        kp, vp = both[:, 0], both[:, 1]
    else:
        kp, vp = (x.zero_() for x in moe.paged_cache(n_pages, n_kv, page, d))
    slots = torch.randperm(n_pages * page, generator=gen)[:T].to(torch.int32)
    slots[T // 2] = -1
    if T > 2:
        slots[1], slots[2] = n_pages * page, -2
    # tokens as a projection leaves them: keys and values side by side
    x = torch.randn((T, 2 * n_kv + 1, d), generator=gen).to(dtype).cuda()
    k, v = x[:, :n_kv], x[:, n_kv:2 * n_kv]
    moe.moe_paged_append(k, v, kp, vp, slots.cuda())
    flags(RANGE if T > 2 else None)
    ok = (slots >= 0) & (slots < n_pages * page)
    for src, pool in ((k, kp), (v, vp)):
        want = torch.zeros((n_pages * page, n_kv, d), dtype=BF16)
        want[slots[ok].long()] = src.cpu()[ok].to(BF16)
        assert torch.equal(pool.cpu().transpose(1, 2).reshape(n_pages * page, n_kv, d), want)


@pytest.mark.gpu
def test_append_of_more_tokens_than_a_launch_takes():
    T, n_kv, d, page = (1 << 24) + 100, 17, 64, 16  # one block a token; 36 GB, of which four tokens are stored
    x = torch.empty((T, n_kv, d), dtype=BF16, device="cuda")
    kp, vp = (x.zero_() for x in moe.paged_cache(2, n_kv, page, d))
    slots = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    want = torch.zeros((2 * page, n_kv, d), dtype=BF16, device="cuda")
    for slot, t in ((3, 0), (20, (1 << 22) + 1), (31, T - 100), (7, T - 1)):
        x[t] = want[slot] = torch.randn((n_kv, d), device="cuda").to(BF16)
        slots[t] = slot
    moe.moe_paged_append(x, x, kp, vp, slots)
    flags()
    for pool in (kp, vp):
        assert torch.equal(pool.transpose(1, 2).reshape(2 * page, n_kv, d), want)


@pytest.mark.gpu
def test_append_rounds_to_nearest_even():
    x = torch.tensor([1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8, -1.0 - 2.0 ** -8 - 2.0 ** -20, 3.39e38, math.inf, math.nan, 2.0 ** -130, -0.0])
    k = x.repeat(8).view(1, 1, 64).cuda()
    kp, vp = moe.paged_cache(1, 1, 16, 64)
    moe.moe_paged_append(k, -k, kp, vp, ints([5]))
    for pool, want in ((kp, k), (vp, -k)):
        got = pool[0, 0, 5].cpu().float()
        assert torch.equal(torch.isnan(got), torch.isnan(want.cpu().flatten()))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want.cpu().flatten().to(BF16).float()))


# -------------------------------------------------------------------------------------------------- trees ---
@pytest.mark.gpu
@pytest.mark.parametrize("shape", ["chain", "star", "random", "binary"])
def test_tree_masks_match_the_plain_form(shape):
    rng = random.Random(3)
    ns = [1, 256, 64, 65, 0, 2, 200, 127]
    make = {"chain": lambda i: i - 1, "star": lambda i: -1 if i == 0 else 0, "random": lambda i: rng.randint(-1, i - 1),
            "binary": lambda i: (i - 1) // 2}[shape]
    parents = [[make(i) for i in range(n)] for n in ns]
    ls = [n + 1000 * b for b, n in enumerate(ns)]
    T = sum(ns)
    masks = torch.full((T + 2, 4), 77, dtype=torch.int64, device="cuda")
    positions = torch.full((T + 2,), 77, dtype=torch.int32, device="cuda")
    flat = [p for q in parents for p in q] + [9, 9]
    moe.moe_tree_masks(ints(flat), q_start=ints(starts(ns)), max_q=256, kv_len=ints(ls), masks=masks, positions=positions)
    flags()
    rows = [line(p, i) for p in parents for i in range(len(p))]
    assert masks.cpu().tolist() == [as_words(r, 4) for r in rows] + [[77] * 4] * 2
    at = [L - n - 1 for n, L in zip(ns, ls) for _ in range(n)]
    assert positions.cpu().tolist() == [a + bin(r).count("1") for a, r in zip(at, rows)] + [77, 77]
    # one token each, none cached
    masks, positions = moe.moe_tree_masks(ints([-1] * 5))
    assert masks.cpu().tolist() == [[1]] * 5 and positions.cpu().tolist() == [0] * 5
    flags()


@pytest.mark.gpu
def test_tree_masks_errors():
    qs = ints([0, 3, 6])
    masks, positions = moe.moe_tree_masks(ints([-1, 0, 1, -1, 1, -2]), q_start=qs, max_q=3, kv_len=ints([3, 10]))
    assert masks.cpu().tolist() == [[1], [3], [7], [1], [2], [4]]  # (its own parent, and none: children of the cache)
    assert positions.cpu().tolist() == [0, 1, 2, 7, 7, 7]
    flags(RANGE)
    # a range of tokens that does not fit has none
    masks = torch.full((6, 1), 5, dtype=torch.int64, device="cuda")
    moe.moe_tree_masks(ints([-1, 0, 1, -1, 0, 0]), q_start=ints([0, 4, 6]), max_q=3, masks=masks)
    assert masks.cpu().tolist() == [[5]] * 4 + [[1], [3]]
    flags(RANGE)
    moe.moe_tree_masks(ints([-1, 0]), q_start=ints([0, 7, 2]), max_q=2)
    flags(RANGE)


# ---------------------------------------------------------------------------------------------- attention ---
CASES = [  # (d, n_kv, group, page, tokens, lengths, window, sinks, tree)
    (64, 1, 1, 16, [1], [1], 0, 0, None),
    (128, 2, 4, 16, [1, 1, 1], [1, 33, 700], 0, 0, None),
    (128, 1, 8, 32, [1, 1, 1, 1], [16, 17, 2049, 64], 0, 0, None),
    (64, 3, 5, 64, [1, 1], [31, 1000], 0, 0, None),
    (192, 2, 2, 16, [1, 1], [5, 300], 0, 0, None),
    (256, 1, 16, 128, [1, 1], [257, 90], 0, 0, None),
    (256, 2, 3, 16, [7, 1, 4], [100, 1, 4], 0, 0, None),
    (128, 2, 2, 16, [3, 5], [1, 2], 0, 0, None),               # padding in front
    (64, 2, 8, 16, [0, 4, 1, 0], [50, 0, 3, 0], 0, 0, None),   # no token, no position
    (128, 1, 4, 16, [1, 1, 1, 1], [10, 40, 41, 3000], 8, 0, None),
    (64, 2, 4, 16, [1, 1, 1, 1], [10, 40, 90, 1700], 33, 4, None),
    (64, 1, 2, 32, [1, 1, 1], [200, 500, 97], 32, 33, None),   # first positions past a block, window at its borders
    (128, 2, 4, 16, [5, 9, 2], [400, 1000, 300], 100, 17, None),
    (64, 1, 4, 16, [300], [300], 50, 100, None),               # first positions that the window still holds
    (64, 1, 4, 16, [300], [800], 50, 100, None),
    (128, 1, 2, 64, [70], [70], 1, 1, None),
    (128, 4, 4, 16, [130, 1, 77], [400, 1, 77], 0, 0, None),
    (64, 4, 8, 16, [200, 150], [1000, 150], 0, 0, None),
    (64, 4, 8, 32, [200, 150], [1000, 700], 128, 5, None),
    (192, 2, 8, 16, [130], [520], 0, 0, None),
    (192, 2, 8, 16, [130], [520], 97, 40, None),
    (256, 2, 8, 64, [130, 20], [520, 20], 0, 0, None),
    (256, 2, 8, 16, [130, 20], [520, 300], 65, 1, None),
    (128, 8, 4, 16, [513], [1500], 0, 0, None),
    (128, 2, 4, 16, [10, 1, 30], [300, 1, 30], 0, 0, "deep"),
    (64, 2, 8, 16, [60, 33], [1000, 500], 0, 0, "wide"),
    (128, 1, 8, 32, [60, 17], [1000, 500], 64, 4, "deep"),
    (64, 1, 2, 16, [256, 129], [300, 2000], 300, 0, "deep"),
    (256, 1, 4, 16, [100, 65], [100, 400], 0, 0, "wide"),
    (192, 2, 1, 16, [20], [700], 20, 33, "wide"),
    (128, 4, 8, 16, [200, 64], [900, 1100], 0, 0, "wide"),
    (128, 1, 4, 16, [9, 5], [4, 0], 0, 0, "deep"),             # drafted tokens before position 0
    (128, 2, 8, 16, [20, 3, 14], [2000, 1100, 14], 0, 0, "wide"),  # (more than 32 rows over more than 1024 positions)
    (64, 2, 8, 64, [9, 5], [1500, 1300], 700, 33, None),
    (256, 1, 8, 16, [40, 3], [1500, 1300], 700, 33, None),
    (192, 1, 8, 16, [60, 25], [900, 1300], 0, 0, "deep"),
    (128, 4, 8, 32, [840, 801], [1000, 1640], 0, 0, None),     # (193 to 256 blocks of 256 rows: eight waves a block)
    (128, 4, 8, 32, [840, 840], [1640, 900], 300, 70, None),
    (64, 4, 8, 16, [256, 250, 9, 1, 200, 256, 77], [700, 250, 500, 1, 333, 300, 400], 0, 0, "wide"),
    (64, 8, 4, 16, [1500], [2100], 0, 0, None),
    (256, 4, 4, 16, [130, 90, 70], [1500, 900, 70], 0, 0, None),   # (40: large heads of many rows, more than 256 blocks of 16)
    (192, 4, 4, 32, [120, 20, 140], [700, 300, 1500], 200, 33, None),
    (256, 4, 4, 16, [100, 65, 90], [100, 400, 90], 0, 0, "wide"),
    (192, 4, 8, 16, [60, 25, 64], [900, 1300, 64], 70, 5, "deep"),
    (128, 2, 8, 16, [150, 40], [1500, 1300], 300, 20, None),       # (more than 1024 positions)
    (128, 2, 8, 16, [60, 17], [1500, 1100], 64, 4, "deep"),
    (128, 4, 8, 16, [64, 40, 33, 50, 9], [500, 40, 100, 300, 9], 0, 0, None),  # (320 blocks of 32 rows)
]


def cases(both, bf16):
    """Cases for both types, and ones whose kernels fp32 tensors do not reach."""
    return pytest.mark.parametrize("case,dtype", [(c, t) for c in both for t in (F32, BF16)] + [(c, BF16) for c in bf16])


@pytest.mark.gpu
@cases(range(32), range(32, len(CASES)))
def test_attention_matches_the_plain_form(case, dtype):
    out, ref, amount, shift, (cache, _, _) = run_case(*CASES[case], dtype)
    flags()
    err = (out.cpu().double() - ref).abs()
    tol = tolerance(ref, amount, shift, dtype, max(cache.ls))
    assert out.dtype is dtype and torch.isfinite(out).all()
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))
    if ref.numel() >= 4096:
        assert relative_rms(out, ref) <= RMS[dtype]


# Calls of at most 32 rows (a sequence's tokens times the query heads of a key/value head) take probabilities as two bf16
# terms: rounding to one leaves up to 2^-8 of it, rounding that to another 2^-16.  Over values of one size the error is then
# the output's own rounding: of normal values of any scale 1.66e-3 to 1.67e-3 rms, of 16384 and more sampled to 1 % or so.  One
# term would add as much again from the probabilities, 2.35e-3 together.
FEW_RMS = 1.72e-3
FEW = [  # (d, n_kv, group, page, tokens, lengths, window, sinks, tree)
    (128, 8, 4, 16, [1] * 6, [40, 100, 700, 1500, 3000, 2049], 0, 0, None),
    (128, 8, 8, 32, [4, 3, 4], [500, 700, 4000], 0, 0, None),
    (64, 16, 8, 16, [1] * 3, [200, 900, 5000], 300, 5, None),
    (64, 16, 4, 16, [8, 5, 7], [400, 2500, 1300], 0, 0, "wide"),
    (192, 8, 2, 16, [1, 5, 3], [300, 900, 2000], 0, 0, None),
    (256, 4, 4, 16, [8, 2, 6], [100, 700, 2500], 0, 0, "deep"),
]


def few_tolerance(ref, amount, shift, L):
    return tolerance(ref, amount, shift, F32, L) - ref.abs() * 2.0 ** -24 + amount * 2.0 ** -16 + ref.abs() * torch.finfo(BF16).eps / 2


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(FEW)))
def test_calls_of_few_rows_keep_two_terms_of_a_probability(case):
    out, ref, amount, shift, (cache, _, _) = run_case(*FEW[case], BF16, seed=case)
    flags()
    err = (out.cpu().double() - ref).abs()
    tol = few_tolerance(ref, amount, shift, max(cache.ls))
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))
    assert ref.numel() >= 16384 and relative_rms(out, ref) <= FEW_RMS


def test_the_bounds_tell_one_term_from_two():
    """The plain form with its probabilities as one bf16 term, or two, and the output rounded: only two pass."""
    gen = torch.Generator().manual_seed(4)
    n, L, kv, G, d = 4, 700, 4, 8, 128
    q = torch.randn((n, kv * G, d), generator=gen).to(BF16).double()
    K, V = (torch.randn((L, kv, d), generator=gen).to(BF16).double() for _ in range(2))
    see = sees(n, L, 0, 0)
    ref, amount, shift = attend([q], [K], [V], [see], G, d ** -0.5, False)
    passed = []
    for terms in (1, 2):
        out = torch.zeros_like(ref)
        for h in range(kv):
            z = (q[:, h * G:(h + 1) * G] @ K[:, h].T * d ** -0.5).masked_fill(~see.unsqueeze(1), -math.inf)
            p = torch.exp(z - z.amax(-1, keepdim=True))
            kept, rest = torch.zeros_like(p), p.clone()
            for _ in range(terms):
                t = rest.to(BF16).double()
                kept, rest = kept + t, rest - t
            out[:, h * G:(h + 1) * G] = kept @ V[:, h] / (kept if terms == 1 else p).sum(-1, keepdim=True)
        out = out.to(BF16)
        err = (out.double() - ref).abs()
        passed.append((bool((err <= few_tolerance(ref, amount, shift, L)).all()), relative_rms(out, ref) <= FEW_RMS))
        assert (err <= tolerance(ref, amount, shift, BF16, L)).all()
    assert passed == [(False, False), (True, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("scale,amplitude", [(0.0, 1.0), (-0.3, 1.0), (20.0, 30.0), (1e-30, 1.0), (2.0 ** 32, 1.0), (2.0 ** -20, 2.0 ** 20)])
@cases([1, 12, 17, 27], [37, 40])
def test_attention_scales(case, scale, amplitude, dtype):
    out, ref, amount, shift, (cache, _, _) = run_case(*CASES[case], dtype, scale=scale, amplitude=amplitude)
    err = (out.cpu().double() - ref).abs()
    # (far scores: which of two near ones wins may be undecided, then any mixture of the values is right)
    tol = torch.where(shift < 0.1, tolerance(ref, amount, shift, dtype, max(cache.ls)), torch.tensor(12.0, dtype=F64))
    assert torch.isfinite(out).all() and (err <= tol).all(), float((err / tol).max())
    flags()


@pytest.mark.gpu
@cases([1, 2, 8, 12, 17, 18, 22, 26], [30, 34, 37, 38, 41, 45])
def test_attention_strides_rows_behind_and_loose_bounds(case, dtype):
    """Tokens of a projection's rows, an output inside another, rows behind the last sequence, loose max_q and max_kv."""
    c = CASES[case]
    out, ref, amount, shift, (cache, q, args) = run_case(*c, dtype)
    d, n_kv, G, page, ns = c[:5]
    T, heads = sum(ns), n_kv * G
    wide = torch.full((T + 3, heads + 2 * n_kv, d), math.nan, dtype=dtype, device="cuda")
    wide[:T, :heads] = q.cuda()
    into = torch.full((T + 3, heads + 1, d), 7.0, dtype=dtype, device="cuda")
    both = torch.full((cache.k.shape[0], 3, n_kv, page, d), math.nan, dtype=BF16, device="cuda")
    both[:, 0], both[:, 2] = cache.k, cache.v
    table = torch.cat([cache.dev_table, ints([[-9] * 5] * len(ns))], 1)
    masks = args["tree"]
    if masks is not None:
        masks = torch.cat([masks, torch.full((3, masks.shape[1]), -1, dtype=torch.int64, device="cuda")])
        masks = torch.cat([masks, torch.full_like(masks, -1)], 1)
    loose = dict(args, max_q=min(T + 3, args["window"] or T + 3) if masks is not None else T + 3, max_kv=table.shape[1] * page, tree=masks)
    if masks is not None and loose["max_q"] > 64 * masks.shape[1]:
        loose["max_q"] = 64 * masks.shape[1]
    moe.moe_paged_attention(wide[:, :heads], both[:, 0], both[:, 2], table, ints(c[5]), out=into[:, :heads], **loose)
    flags()
    err = (into[:T, :heads].cpu().double() - ref).abs()
    assert (err <= tolerance(ref, amount, shift, dtype, max(cache.ls))).all()
    assert (into[T:] == 7.0).all() and (into[:, heads:] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@cases([12, 16, 20, 24, 25, 28], [17, 18, 22, 27, 33, 34, 37, 38, 40, 43, 45])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(case, value, dtype):
    """One element of a value, seen by some of the tokens: their outputs of its dim are NaN, all else is what it was."""
    c = CASES[case]
    d, n_kv, G, page, ns, ls, window, sinks = c[:8]
    out, ref, amount, shift, (cache, q, args) = run_case(*c, dtype)
    n, L = ns[0], ls[0]
    p, h, dim = L - n // 2 - 1, n_kv - 1, d - 3
    slot = cache.slots(0, p, p + 1)[0]
    cache.v[slot // page, h, slot % page, dim] = value
    bad = moe.moe_paged_attention(q.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), **args)
    bits = None
    if args["tree"] is not None:
        bits = [sum((int(w) & (2 ** 64 - 1)) << 64 * k for k, w in enumerate(r)) for r in args["tree"][:n].cpu().tolist()]
    see = sees(n, L, window, sinks, bits)[:, p]
    assert see.any() and not see.all()
    hit = torch.zeros(ref.shape, dtype=torch.bool)
    hit[:n, h * G:(h + 1) * G, dim] = see.unsqueeze(1)
    got = bad.cpu()
    assert torch.isnan(got[hit]).all()
    err = (got.double() - ref).abs()[~hit]
    assert (err <= tolerance(ref, amount, shift, dtype, max(ls))[~hit]).all()
    # and a key: all of the rows that see it, no others
    cache.v[slot // page, h, slot % page, dim] = 0.0
    cache.k[slot // page, h, slot % page, dim] = math.nan
    got = moe.moe_paged_attention(q.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), **args).cpu()
    hit = torch.zeros(ref.shape, dtype=torch.bool)
    hit[:n, h * G:(h + 1) * G] = see.view(-1, 1, 1)
    assert torch.isnan(got[hit]).all() and torch.isfinite(got[~hit]).all()
    # a query: its own row
    cache.k[slot // page, h, slot % page, dim] = 0.0
    q2 = q.clone()
    q2[n // 2, 0, 1] = value
    got2 = moe.moe_paged_attention(q2.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), **args).cpu()
    keep = torch.ones(ref.shape[:2], dtype=torch.bool)
    keep[n // 2, 0] = False
    assert not torch.isfinite(got2[~keep]).any() and torch.isfinite(got2[keep]).all()
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 3), (64, 0), (700, 33)])
@pytest.mark.parametrize("d,n_kv,G,ns,ls", [(64, 2, 4, [5, 1, 7], [200, 97, 1300]), (128, 1, 8, [40, 33], [900, 41]),
                                            (256, 1, 8, [48, 3], [1500, 700])])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_of_any_bits(d, n_kv, G, ns, ls, window, sinks, dtype):
    """Drafted tokens that see later ones, not themselves, or none; bits past the sequence's tokens; two words a row more."""
    gen, rng = torch.Generator().manual_seed(d), random.Random(d)
    bits = [[rng.choice((0, rng.getrandbits(n), 1 << rng.randrange(n))) for _ in range(n)] for n in ns]
    visible = [sees(n, L, window, sinks, b) for n, L, b in zip(ns, ls, bits)]
    # (the tokens' own keys and values are there, seen or not)
    cache = Cache(ls, n_kv, d, 16, gen).put([v.any(0) | (torch.arange(L) >= L - n) for v, n, L in zip(visible, ns, ls)])
    q = torch.randn((sum(ns), n_kv * G, d), generator=gen).to(dtype)
    stray = [[x | rng.getrandbits(192 - n) << n for x in b] for n, b in zip(ns, bits)]
    masks = torch.tensor([as_words(x, 3) for b in stray for x in b], dtype=torch.int64).cuda()
    out = moe.moe_paged_attention(q.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), q_start=ints(starts(ns)), max_q=max(ns),
                                  max_kv=max(ls), window=window, sinks=sinks, tree=masks)
    flags()
    qs = [q[a:b].double() for a, b in zip(starts(ns), starts(ns)[1:])]
    ref, amount, shift = attend(qs, [k.double() for k in cache.ks], [v.double() for v in cache.vs], visible, G, d ** -0.5, dtype is F32)
    assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, max(ls))).all()


@pytest.mark.gpu
@cases([2, 10, 17, 25], [18, 34, 37, 38, 40, 45])
def test_a_page_that_is_missing_counts_as_unseen(case, dtype):
    c = CASES[case]
    d, n_kv, G, page, ns, ls, window, sinks, tree = c
    _, _, _, _, (cache, q, args) = run_case(*c, dtype)
    b = len(ls) - 1
    col = max(0, ls[b] - ns[b] - 1) // page  # the page in front of the tokens, or their first
    for wrong in (-1, cache.k.shape[0], 2 ** 31 - 1):
        cache.table[b][col] = wrong
        out = moe.moe_paged_attention(q.cuda(), cache.k, cache.v, cache.dev_table, ints(ls), **args)
        flags(RANGE)
        visible = []
        t = 0
        for i, (n, L) in enumerate(zip(ns, ls)):
            bits = None
            if tree:
                bits = [sum((int(w) & (2 ** 64 - 1)) << 64 * k for k, w in enumerate(r)) for r in args["tree"][t:t + n].cpu().tolist()]
            see = sees(n, L, window, sinks, bits)
            if i == b:
                see[:, col * page:(col + 1) * page] = False
            visible.append(see)
            t += n
        qs = [q[x:y].double() for x, y in zip(starts(ns), starts(ns)[1:])]
        ref, amount, shift = attend(qs, [k.double() for k in cache.ks], [v.double() for v in cache.vs], visible, G, d ** -0.5, dtype is F32)
        assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, max(ls))).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_batches(dtype):
    """Lengths and token ranges that do not fit: such a sequence has no position, or no token; the others are as they were."""
    gen = torch.Generator().manual_seed(5)
    ns, ls = [4, 2, 3], [40, 70, 9]
    cache = Cache(ls, 2, 64, 16, gen).put()
    q = torch.randn((9, 8, 64), generator=gen).to(dtype).cuda()
    call = lambda qs, kl, **kw: moe.moe_paged_attention(q, cache.k, cache.v, cache.dev_table, ints(kl), q_start=ints(qs), max_q=4,
                                                       out=torch.full_like(q, 3.0), **{**dict(max_kv=70), **kw})
    good = call([0, 4, 6, 9], ls)
    flags()
    for kl in ([40, 71, 9], [40, -1, 9], [40, 2 ** 31 - 1, 9]):
        out = call([0, 4, 6, 9], kl)
        flags(RANGE)
        assert (out[4:6] == 0).all() and torch.equal(out[:4], good[:4]) and torch.equal(out[6:], good[6:])
    out = call([0, 4, 3, 9], ls)  # (descending, and then more than max_q)
    flags(RANGE)
    assert torch.equal(out[:4], good[:4]) and (out[4:] == 3.0).all()
    out = call([0, 4, 6, 10], ls)
    flags(RANGE)
    assert torch.equal(out[:6], good[:6]) and (out[6:] == 3.0).all()


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^32 in the pools, one token and a prompt."""
    gen = torch.Generator().manual_seed(8)
    n_kv, d, page = 8, 128, 64
    n_pages = (1 << 32) // (n_kv * d * page) + 40  # 8.6 GB a pool
    k, v = moe.paged_cache(n_pages, n_kv, page, d)
    L, n = 700, 70
    table = [[n_pages - 1 - 3 * c for c in range(11)], [c for c in range(11)]]
    keys, values = (torch.randn((L, n_kv, d), generator=gen).to(BF16) for _ in range(2))
    for row in table:
        moe.moe_paged_append(keys.cuda(), values.cuda(), k, v, ints([row[p // page] * page + p % page for p in range(L)]))
    for m in (1, n):
        q = torch.randn((m, 32, d), generator=gen).to(BF16).cuda()
        outs = [moe.moe_paged_attention(q, k, v, ints([row]), ints([L]), q_start=ints([0, m]), max_q=m, max_kv=L) for row in table]
        assert torch.equal(*outs)
        ref, amount, shift = attend([q.cpu().double()], [keys.double()], [values.double()], [sees(m, L, 0, 0)], 4, d ** -0.5, False)
        assert ((outs[0].cpu().double() - ref).abs() <= tolerance(ref, amount, shift, BF16, L)).all()
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("n,dtype", [(1, F32), (1, BF16), (9, BF16), (200, BF16)])
def test_attention_long_and_split(n, dtype):
    """A long cache, whose positions are split over blocks; with a window only a part of it is."""
    d, n_kv, G, page, L = 128, 2, 4, 64, 20011
    for window, sinks in ((0, 0), (5000, 70)):
        out, ref, amount, shift, _ = run_case(d, n_kv, G, page, [n], [L], window, sinks, None, dtype, seed=n)
        assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, L)).all()
        assert relative_rms(out, ref) <= RMS[dtype]
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("n,n_seq,L", [(1, 1, 1 << 22), (40, 1, 1 << 22), (40, 512, 1 << 21)])  # (many rows: split, and whole)
def test_long_sums_of_large_values(n, n_seq, L):
    """Scores that rise behind the first positions of every piece by 7.9 in log2 units, which many rows do not follow at once:
    probabilities of 2^7.9 with values of 2^100 would add up to 2^128.9 and more.  All values of a dim are one power of two, so
    that is what comes out, rounded: probabilities that follow the maximum are 1, whose sums are whole numbers below 2^24, and
    of the first ones, a 64th of the positions at 2^-7.9 each, all may be lost beside them (2^-13)."""
    d, page = 64, 64
    k, v = moe.paged_cache(L // page, 1, page, d)
    k.fill_(1.0), v.fill_(2.0 ** 100)
    k[::64] = 0.0
    v[..., 1::2] = -2.0 ** 99
    table = torch.arange(L // page, dtype=torch.int32, device="cuda").repeat(n_seq, 1)
    q = torch.ones((n_seq * n, 1, d), dtype=BF16, device="cuda")
    out = moe.moe_paged_attention(q, k, v, table, ints([L] * n_seq), q_start=ints([n * b for b in range(n_seq + 1)]), max_q=n,
                                  scale=5.5 / d)
    flags()
    want = v[0, 0, 0].double().cpu().expand(n_seq * n, 1, d)
    assert ((out.cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -11)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window,sinks,tree", [(0, 0, None), (0, 0, "deep"), (9000, 40, None), (100, 5, None)])
def test_a_ragged_batch_in_equal_shares(window, sinks, tree, dtype):
    """Sequences that share units and units that share sequences, ones without tokens and without positions among them; with
    the short window the same call has few positions and cuts the sequences into pieces."""
    ns, ls = [1, 3, 1, 0, 2, 1, 1, 1, 3], [9001, 3, 0, 500, 15000, 8000, 1, 63, 4999]
    out, ref, amount, shift, _ = run_case(64, 16, 2, 16, ns, ls, window, sinks, tree, dtype)
    flags()
    assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, max(ls))).all()


LONG, HALF, EVEN = ([9001, 3, 0, 500, 15000, 8000, 1, 63, 4999], [5001, 3, 0, 300, 7000, 3500, 1, 63, 2499],
                    [1200, 1100, 1213, 1150, 1190, 1212, 1213, 1170, 1100])


def share_blocks(case, dtype):
    """(tiles of 16 rows of a wave, row blocks, blocks of positions in a share) by the sizes alone, which have to give shares."""
    d, n_kv, G, _, ns, ls, window, sinks, tree = case
    f32, rows = dtype is F32, max(ns) * G
    tiles = 1 if rows <= 16 or d > 128 or (f32 and d > 64) else 2
    blocks = -(-rows // (16 * tiles))
    if not f32 and rows > 32:  # (the kernel for few rows all the same)
        few = blocks * n_kv * len(ns)
        assert d > 128 and few <= 256 and few * max(ls) <= 1 << 18
    fill = 256 if d // 64 * tiles > 2 else 512
    target = fill // (blocks * n_kv)
    assert blocks * n_kv * len(ns) < fill and len(ns) * max(ls) >= 1024 * target
    total = 0
    for n, L in zip(ns, ls):
        first = max(0, L - n - window + 1) // 32 if window else 0
        assert first == 0 or sinks <= 32 * first
        total += max(1, (-(-sinks // 32) if first else 0) + -(-L // 32) - first) if n else 0
    return tiles, blocks, -(-total // target)


@pytest.mark.gpu
@pytest.mark.parametrize("case,tiles,blocks,dtype", [
    ((64, 16, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], LONG, 0, 0, None), 2, 1, BF16),
    ((64, 16, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], LONG, 0, 0, "deep"), 2, 1, F32),
    ((64, 16, 8, 16, [1, 5, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 2, 2, F32),
    ((128, 16, 4, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], LONG, 0, 0, None), 1, 1, BF16),
    ((128, 16, 4, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], LONG, 10000, 40, None), 1, 1, F32),
    ((128, 16, 8, 32, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 2, 1, BF16),
    ((128, 16, 8, 16, [1, 3, 1, 0, 2, 1, 4, 1, 3], HALF, 6000, 40, "deep"), 2, 1, BF16),
    ((128, 16, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 1, 2, F32),
    ((192, 16, 4, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 1, 1, BF16),
    ((192, 8, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, "wide"), 1, 2, F32),
    ((256, 16, 4, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, "deep"), 1, 1, BF16),
    ((256, 8, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 1, 2, BF16),
    ((256, 8, 8, 16, [1, 3, 1, 0, 2, 1, 1, 1, 3], HALF, 0, 0, None), 1, 2, F32),
    ((256, 8, 16, 16, [1, 3, 1, 2, 2, 1, 1, 3, 3], EVEN, 0, 0, None), 1, 3, BF16),
])
def test_equal_shares_of_every_head_size_and_number_of_rows(case, tiles, blocks, dtype):
    """One tile of rows or two, one block of rows or more, of which a sequence of few tokens has fewer."""
    found = share_blocks(case, dtype)
    assert found[:2] == (tiles, blocks) and found[2] >= 32
    out, ref, amount, shift, _ = run_case(*case, dtype)
    flags()
    L = max(case[5])
    few = dtype is BF16 and max(case[4]) * case[2] <= 32
    err, tol = (out.cpu().double() - ref).abs(), few_tolerance(ref, amount, shift, L) if few else tolerance(ref, amount, shift, dtype, L)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.gpu
def test_more_sequences_than_a_wave_has_lanes():
    ns, ls = [1 + b % 3 for b in range(150)], [1 + 37 * b % 411 for b in range(150)]
    ls = [max(n, L) for n, L in zip(ns, ls)]
    for window, sinks in ((0, 0), (60, 3)):
        out, ref, amount, shift, _ = run_case(64, 1, 2, 16, ns, ls, window, sinks, None, BF16)
        assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, BF16, 411)).all()
    flags()


SIZES = ("T", "n_seq", "n_heads", "n_kv", "head_dim", "max_q", "max_kv")


def random_sizes(rng):
    """Sizes of an attention call and of one with the same heads that is no larger in any of them."""
    log = lambda hi: int(hi ** rng.random())
    n_kv, group, d = rng.choice([1, 2, 3, 4, 8, 16, 24]), rng.choice([1, 2, 3, 4, 5, 8, 16]), rng.choice([64, 128, 192, 256])
    n_seq, max_q, max_kv = log(1000), log(4096), log(1 << 20)
    T = n_seq * log(max_q)
    large = (T, n_seq, n_kv * group, n_kv, d, max_q, max_kv)
    small = [rng.randint(1, n) if rng.random() < 0.7 else n for n in (T, n_seq, max_q, max_kv)]
    return large, (small[0], min(small[1], small[0]), n_kv * group, n_kv, d, *small[2:])


def test_a_workspace_serves_smaller_calls_too():
    size, rng = moe.moe_paged_attention_workspace_bytes, random.Random(2)
    for _ in range(20000):
        large, small = random_sizes(rng)
        assert size(*small) <= size(*large), (dict(zip(SIZES, small)), dict(zip(SIZES, large)))


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that pass all checks would run, on addresses that are none")
def test_what_a_call_asks_for_is_within_the_size():
    L, rng, P = moe.lib(), random.Random(3), OK_PTR
    asked = 0
    for _ in range(20000):
        T, n_seq, heads, n_kv, d, max_q, max_kv = random_sizes(rng)[1]
        each = n_kv * 16 * d
        for dtype in (0, 1):
            code = L.moe_paged_attention(P, dtype, heads * d, P, P, each, each, 9, 16, P, 1 << 16, T, n_seq, heads, n_kv, d, P, max_q,
                                         P, max_kv, 0, 0, None, 0, 0.125, P, heads * d, None, 0, None)
            message = L.moe_last_error().decode()
            need = int(message.split("workspace of ")[1].split()[0]) if code == -1 else 0
            assert code == -6 or need > 0, message  # (no device, or no workspace)
            assert need <= moe.moe_paged_attention_workspace_bytes(T, n_seq, heads, n_kv, d, max_q, max_kv)
            asked += need > 0
    assert asked > 2000


@pytest.mark.gpu
def test_one_workspace_for_prompts_and_steps():
    """Sized once by the largest bounds, taken by every smaller call; what lies behind it is left alone."""
    gen = torch.Generator().manual_seed(9)
    n_kv, G, d, page = 8, 4, 128, 16
    lens = [3000, 17, 900, 2100]
    cache = Cache(lens, n_kv, d, page, gen, spare=3).put()
    size = moe.moe_paged_attention_workspace_bytes(32 * 256, 32, n_kv * G, n_kv, d, 256, 16384)
    ws = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    for dtype in (F32, BF16):
        for n in (1, 4, 9, 16, 64):
            for max_kv in (3000, 3050):
                q = torch.randn((4 * n, n_kv * G, d), generator=gen).to(dtype).cuda()
                args = dict(q_start=ints([0, n, 2 * n, 3 * n, 4 * n]), max_q=n, max_kv=max_kv)
                ref = moe.moe_paged_attention(q, cache.k, cache.v, cache.dev_table, ints(lens), **args)
                out = moe.moe_paged_attention(q, cache.k, cache.v, cache.dev_table, ints(lens), workspace=ws[:size], **args)
                assert torch.equal(out, ref)
    assert (ws[size:] == 0x5a).all()
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("d,G,n,n_seq,lo,hi,dtype", [
    (64, 2, 3, 150, 1, 1500, BF16), (128, 4, 1, 300, 1, 2000, F32), (256, 3, 2, 100, 1, 900, BF16),  # pieces of few rows
    (64, 4, 2, 150, 2500, 6000, BF16), (128, 8, 1, 200, 1500, 4000, F32),                            # shares
    (128, 8, 7, 100, 1, 1500, BF16), (64, 16, 5, 130, 1, 1200, BF16),                                # pieces of many rows
])
def test_more_sequences_than_lanes_split(d, G, n, n_seq, lo, hi, dtype):
    rng = random.Random(n_seq)
    ns, ls = [rng.randint(0, n) for _ in range(n_seq)], [rng.randint(lo, hi) for _ in range(n_seq)]
    ns[5], ls[5], ls[70] = n, hi, 0
    for window, sinks in ((0, 0), (400, 33)):
        out, ref, amount, shift, _ = run_case(d, 1, G, 16, ns, ls, window, sinks, None, dtype)
        assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, hi)).all()
    flags()


@pytest.mark.gpu
@pytest.mark.parametrize("case", [(128, 1, 64, 16, [1, 1, 2], [3000, 20, 700], 0, 0, None), (64, 1, 128, 16, [1, 2], [700, 1800], 64, 5, None),
                                  (256, 1, 71, 16, [1, 1], [900, 31], 0, 0, None), (128, 2, 13, 32, [3, 1], [500, 2000], 0, 0, "deep"),
                                  (192, 1, 33, 16, [1], [40], 0, 0, None)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_query_heads_per_key_value_head(case, dtype):
    out, ref, amount, shift, (cache, _, _) = run_case(*case, dtype)
    flags()
    assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, dtype, max(cache.ls))).all()


# -------------------------------------------------------------------------- graphs, streams, together (GPU) ---
def rotate(x, positions):
    """A stand-in for what a model does between projection and cache: something that depends on the position."""
    return x * (1.0 + 0.01 * positions.view(-1, 1, 1).to(x.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_a_batch_served_from_pages_equals_plain_attention(window, sinks):
    """Prompts, decode steps and a drafted tree with its accepted branch, all through tables, append and attention: every
    output against plain attention over each sequence's own history."""
    gen, rng = torch.Generator().manual_seed(31), random.Random(31)
    B, n_kv, G, d, page, width = 4, 2, 4, 64, 16, 20
    kp, vp = moe.paged_cache(200, n_kv, page, d)
    kp.fill_(math.nan), vp.fill_(math.nan)
    free = list(range(200))
    rng.shuffle(free)
    free, first = ints(free), ints([0])
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    lens = ints([0] * B)
    history = [([], []) for _ in range(B)]

    def step(new, tree=None):
        T = sum(new) + 2  # (two rows of padding)
        global_len, q_start, positions, slots, _ = moe.moe_page_tables(
            lens, ints(new), free, table, page, 200, T, free_first=first, kv_len_out=lens, free_next=first)
        masks, bits = None, [None] * B
        if tree:
            flat = [p for t in tree for p in t] + [-1, -1]
            masks, positions = moe.moe_tree_masks(ints(flat), q_start=q_start, max_q=max(new), kv_len=lens)
            bits = [[line(t, i) for i in range(len(t))] for t in tree]
        x = torch.randn((T, (G + 2) * n_kv, d), generator=gen).to(BF16).cuda()
        q, k, v = x[:, :G * n_kv], rotate(x[:, G * n_kv:(G + 1) * n_kv], positions), x[:, (G + 1) * n_kv:]
        moe.moe_paged_append(k, v, kp, vp, slots)
        out = moe.moe_paged_attention(q, kp, vp, table, lens, q_start=q_start, max_q=max(new), window=window, sinks=sinks,
                                      tree=masks, out=torch.full((T, G * n_kv, d), 9.0, dtype=BF16, device="cuda"))
        flags()
        assert (out[-2:] == 9.0).all()
        qs, ks, vs, vis, t = [], [], [], [], 0
        for b, n in enumerate(new):
            history[b][0].extend(k[t:t + n].cpu()), history[b][1].extend(v[t:t + n].cpu())
            L = len(history[b][0])
            qs.append(q[t:t + n].cpu().double())
            for src, dst in ((history[b][0], ks), (history[b][1], vs)):
                dst.append(torch.stack(src).double() if src else torch.zeros((0, n_kv, d), dtype=F64))
            vis.append(sees(n, L, window, sinks, bits[b]))
            t += n
        assert lens.cpu().tolist() == [len(h[0]) for h in history]
        ref, amount, shift = attend(qs, ks, vs, vis, G, d ** -0.5, False)
        assert ((out[:-2].cpu().double() - ref).abs() <= tolerance(ref, amount, shift, BF16, 300)).all()

    step([37, 1, 90, 16])
    step([1, 1, 1, 1])
    step([1, 20, 1, 0])
    for _ in range(4):
        step([1, 1, 1, 1])
        tree = [random_tree(rng.randint(1, 30), rng, True) for _ in range(B)]
        step([len(t) for t in tree], tree)
        # the first branch is accepted as far as it is a run of the tokens, and what was drafted behind it given up; its
        # pages stay in the table, behind the length
        keep = [next((i for i, p in enumerate(t) if p != i - 1), len(t)) for t in tree]
        back = [len(t) - m for t, m in zip(tree, keep)]
        for b in range(B):
            for part in history[b]:
                del part[len(part) - back[b]:]
        lens.sub_(ints(back))


@pytest.mark.gpu
@pytest.mark.parametrize("case,at", [(2, 2), (10, 2), (12, 1), (18, 1), (26, 1), (38, 3)])
def test_parts_of_a_batch_called_by_themselves(case, at):
    """A batch in two calls, each with its part of the lengths, of the starts and of the table, into one output."""
    d, n_kv, G, page, ns, ls = CASES[case][:6]
    _, ref, amount, shift, (cache, q, args) = run_case(*CASES[case], BF16)
    masks, q = args["tree"], q.cuda()
    out = torch.full_like(q, 5.0)
    for lo, hi in ((at, len(ns)), (0, at)):
        q_start, table, lens = args["q_start"][lo:hi + 1], cache.dev_table[lo:hi], ints(ls)[lo:hi]
        if masks is not None:  # (a part's masks lie in the whole batch's rows, too)
            part = torch.full_like(masks, 3 << 40)
            moe.moe_tree_masks(ints([-1] * sum(ns)), q_start=q_start, max_q=max(ns[lo:hi]), kv_len=lens, masks=part)
            first, last = starts(ns)[lo], starts(ns)[hi]
            assert (part[:first] == 3 << 40).all() and (part[last:] == 3 << 40).all() and (part[first:last] != 3 << 40).all()
        before = out.clone()
        moe.moe_paged_attention(q, cache.k, cache.v, table, lens, out=out, **dict(args, q_start=q_start, max_q=max(ns[lo:hi]), max_kv=max(ls[lo:hi])))
        keep = torch.ones(sum(ns), dtype=torch.bool)
        keep[starts(ns)[lo]:starts(ns)[hi]] = False
        assert torch.equal(out[keep.cuda()], before[keep.cuda()])
    flags()
    assert ((out.cpu().double() - ref).abs() <= tolerance(ref, amount, shift, BF16, max(ls))).all()


@pytest.mark.gpu
def test_captured_steps_replay_with_new_lengths():
    """Tables, store, masks and attention of a step captured twice, for one token each and for drafted trees, sharing pools
    and a workspace: replays in turn, with eager work between them, equal the eager calls."""
    gen, rng = torch.Generator().manual_seed(41), random.Random(41)
    B, n_kv, G, d, page, width, n = 3, 2, 4, 128, 16, 200, 12
    heads = n_kv * G

    def fresh():
        k, v = (x.zero_() for x in moe.paged_cache(700, n_kv, page, d))
        lens = [5, 700, 1900]
        table = [[600 - (b * 130 + c) if c < -(-L // page) else -1 for c in range(width)] for b, L in enumerate(lens)]
        g = torch.Generator().manual_seed(42)
        slots = [table[b][p // page] * page + p % page for b, L in enumerate(lens) for p in range(L)]
        x = torch.randn((len(slots), 2 * n_kv, d), generator=g).to(BF16).cuda()
        moe.moe_paged_append(x[:, :n_kv], x[:, n_kv:], k, v, ints(slots))
        return dict(k=k, v=v, table=ints(table), lens=ints(lens), first=ints([0]), free=ints(list(range(100))))

    x1 = torch.randn((B, (G + 2) * n_kv, d), generator=gen).to(BF16).cuda()
    x2 = torch.randn((B * n, (G + 2) * n_kv, d), generator=gen).to(BF16).cuda()
    parents, new = ints([i - 1 for _ in range(B) for i in range(n)]), ints([n] * B)
    size = max(moe.moe_paged_attention_workspace_bytes(B, B, heads, n_kv, d, 1, width * page),
               moe.moe_paged_attention_workspace_bytes(B * n, B, heads, n_kv, d, n, width * page))
    assert size > 0

    def step(s, x, new, parents, out, ws):
        m = 1 if parents is None else n
        _, q_start, _, slots, _ = moe.moe_page_tables(s["lens"], new, s["free"], s["table"], page, 700, B * m,
                                                      free_first=s["first"], kv_len_out=s["lens"], free_next=s["first"])
        masks = None
        if parents is not None:
            masks, _ = moe.moe_tree_masks(parents, q_start=q_start, max_q=n, kv_len=s["lens"])
        moe.moe_paged_append(x[:, heads:heads + n_kv], x[:, heads + n_kv:], s["k"], s["v"], slots)
        moe.moe_paged_attention(x[:, :heads], s["k"], s["v"], s["table"], s["lens"], q_start=q_start, max_q=m, window=1000,
                                sinks=4, tree=masks, out=out, workspace=ws)

    mine, eager = fresh(), fresh()
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out1, out2 = torch.empty((B, heads, d), dtype=BF16, device="cuda"), torch.empty((B * n, heads, d), dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1, stream=side):
        step(mine, x1, None, None, out1, ws)
    with torch.cuda.graph(g2, stream=side):
        step(mine, x2, new, parents, out2, ws)
    for i in range(5):
        for graph, x, nw, par, out in ((g1, x1, None, None, out1), (g2, x2, new, parents, out2)):
            x.copy_(torch.randn(x.shape, generator=gen))
            if par is not None:
                par.copy_(ints([rng.randint(-1, j - 1) for _ in range(B) for j in range(n)]))
            graph.replay()
            ref = torch.empty_like(out)
            step(eager, x, nw, par, ref, torch.empty_like(ws))
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
        for name in ("k", "v", "table", "lens", "first"):
            assert torch.equal(mine[name], eager[name]), name
    flags()


@pytest.mark.gpu
def test_calls_on_another_stream():
    gen = torch.Generator().manual_seed(22)
    x = torch.randn((64, 8, 128), generator=gen).cuda()
    lens, new, free = ints([0]), ints([64]), ints(list(range(8)))

    def all_of_it(stream):
        k, v = moe.paged_cache(8, 2, 16, 128)
        table = ints([[-1] * 6])
        if stream is not None:
            (stream if isinstance(stream, torch.cuda.Stream) else side).wait_stream(torch.cuda.current_stream())
        kl, qs, _, slots, _ = moe.moe_page_tables(lens, new, free, table, 16, 8, 64, stream=stream)
        masks, _ = moe.moe_tree_masks(ints([i - 1 for i in range(64)]) if stream is None else parents, q_start=qs, max_q=64, kv_len=kl, stream=stream)
        moe.moe_paged_append(x[:, 4:6], x[:, 6:], k, v, slots, stream=stream)
        return moe.moe_paged_attention(x[:, :4], k, v, table, kl, q_start=qs, tree=masks, stream=stream)

    side = torch.cuda.Stream()
    parents = ints([i - 1 for i in range(64)])
    ref = all_of_it(None)
    for stream in (side, side.cuda_stream):
        out = all_of_it(stream)
        side.synchronize()
        assert torch.equal(out, ref)
    moe.moe_sync_check(side)


@pytest.mark.gpu
def test_no_tokens_is_a_no_op():
    k, v = moe.paged_cache(4, 2, 16, 64)
    none = torch.empty((0, 2, 64), device="cuda")
    moe.moe_paged_append(none, none, k, v, ints([]))
    out = moe.moe_paged_attention(torch.empty((0, 4, 64), device="cuda"), k, v, ints([[0], [1]]), ints([3, 4]), q_start=ints([0, 0, 0]))
    assert out.shape == (0, 4, 64)
    out = moe.moe_paged_attention(torch.empty((0, 4, 64), device="cuda"), k, v, ints([]).view(0, 2), ints([]))
    assert out.shape == (0, 4, 64)
    assert moe.moe_tree_masks(ints([]), q_start=ints([0, 0]))[0].shape == (0, 1)
    flags()
