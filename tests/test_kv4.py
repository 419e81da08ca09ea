"""The 4-bit key/value cache, the attention over it, int4 matrix-vector products and the block made of them,
against plain 64-bit implementations."""
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

import paper_2605_29135_amd as moe
from paper_2605_29135_amd import binding

F32, BF16 = torch.float32, torch.bfloat16
GROUP = 64
EPS = 1e-6


# ------------------------------------------------------------------------------------- plain 64-bit forms ---
def quantised(x):
    """(codes, scale, base) of each group of 64 of the last dimension, float64 [..., d/64, 64 | 1 | 1], by the
    cache's definition: the base and scale in bf16, x - base and the range in fp32, the quotient exact."""
    x = x.float().unflatten(-1, (-1, GROUP))
    m = x.amin(-1, keepdim=True).to(BF16).float()
    s = ((x.amax(-1, keepdim=True) - m) * torch.tensor(1 / 15, dtype=F32)).to(BF16).float()
    s = torch.where(s >= 2.0 ** -126, s, torch.zeros_like(s))
    bad = ~(torch.isfinite(x).all(-1, keepdim=True) & torch.isfinite(s) & torch.isfinite(m))
    s, m, x = (torch.where(bad, torch.zeros_like(t), t) for t in (s, m, x))
    t = (x - m).double()
    u = torch.where(s > 0, torch.round(t / torch.where(s > 0, s, torch.ones_like(s)).double()), torch.zeros_like(t))
    return u.clamp(0, 15), s.double(), m.double()


def held(x):
    u, s, m = quantised(x)
    return (u * s + m).flatten(-2)


def magnitude(x):
    """What the kernels' exact partial products of a held value can amount to: (16 + u) s + 16 s + |m|."""
    u, s, m = quantised(x)
    return ((32 + u) * s + m.abs()).flatten(-2)


def attend(q, ks, vs, ns, ls, G, window, scale, dtype):
    """Plain attention and its error bound: q [T, heads, d] float64; ks, vs: per sequence [L, n_kv, d] vectors
    before quantisation.  The bound per output is the sum of the roundings on its way:
      scores: queries within 2^-22 of the head's largest element, products in fp32 sums of at most 32 partial
              results (2^-24 each of what they amount to), two roundings on the way to the exponent, and for
              bf16 tensors keys as fp16 (2^-11); an error e of a score changes a probability by e;
      exponentials and the sum: 2^-20 together;
      probabilities and values: two fp16 terms (2^-22) or three fp16 roundings (3 x 2^-11)."""
    keys = 0.0 if dtype is F32 else 2.0 ** -11
    T, heads, d = q.shape
    out = torch.zeros((T, heads, d), dtype=torch.float64)
    amount = torch.zeros((T, heads, d), dtype=torch.float64)  # sum of P x magnitude
    shift = torch.zeros((T, heads, 1), dtype=torch.float64)   # largest error of a score
    t0 = 0
    for n, L, k, v in zip(ns, ls, ks, vs):
        first = max(0, n - L)  # tokens before it are padding
        at = torch.arange(L - n + first, L).view(-1, 1, 1)
        p = torch.arange(L)
        see = (p <= at) & (p > at - (window or L + 1))
        for h in range(heads // G if n > first else 0):
            rows, cols = slice(t0 + first, t0 + n), slice(h * G, (h + 1) * G)
            K, V, mk, mv = held(k[:, h]), held(v[:, h]), magnitude(k[:, h]), magnitude(v[:, h])
            x = q[rows, cols]
            z = x @ K.T * scale
            w = torch.softmax(torch.where(see, z, torch.tensor(-math.inf, dtype=torch.float64)), -1)
            out[rows, cols], amount[rows, cols] = w @ V, w @ mv
            e = x.abs() @ mk.T * 2.0 ** -19 + mk.sum(1) * x.abs().amax(-1, keepdim=True) * 2.0 ** -22 + x.abs() @ K.abs().T * keys
            shift[rows, cols] = torch.where(see, e * abs(scale) + z.abs() * 2.0 ** -22, 0.0).amax(-1, keepdim=True)
        t0 += n
    return out, amount, shift


def attention_tolerance(ref, amount, shift, dtype):
    term = 2.0 ** -22 if dtype is F32 else 3 * 2.0 ** -11
    return amount * (2 * shift + 2.0 ** -20 + term) + ref.abs() * torch.finfo(dtype).eps / 2 + 1e-30


def int4_matrix(N, K, gen, sigma=0.02):
    """(bytes as stored, float64 values) of a random int4-g128 matrix."""
    w = torch.randn((N, K // 128, 128), generator=gen) * sigma
    s = (w.abs().amax(-1, keepdim=True) / 7).to(BF16)
    q = torch.clamp(torch.round(w / s.float()), -8, 7)
    nib = q.to(torch.int32).view(N, K // 2, 2) & 15
    raw = (nib[..., 0] | (nib[..., 1] << 4)).to(torch.uint8).flatten()
    return torch.cat([raw, s.flatten().view(torch.uint8)]), (q.double() * s.double()).view(N, K)


def batch(ns, ls, extra=0):
    starts = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    return (torch.from_numpy(starts).cuda(), torch.tensor(ls, dtype=torch.int32).cuda(), int(starts[-1]) + extra)


def fill(cache, byte=0xFF):
    """What was never written may be anything: scales and bases of NaN."""
    cache.fill_(byte)
    return cache


def put(ks, vs, cache, dtype):
    """Append whole sequences (lists of [L, n_kv, d])."""
    ls = [k.shape[0] for k in ks]
    qs, kl, T = batch(ls, ls)
    if T:
        moe.moe_kv4_append(torch.cat(ks).to(dtype).cuda(), torch.cat(vs).to(dtype).cuda(), cache, kl, q_start=qs)


# ---------------------------------------------------------------------------------------- refusals (CPU) ---
OK_PTR = 1 << 20  # an aligned address that no refused call touches


def refused(name, *args):
    code = getattr(moe.lib(), name)(*args)
    assert code == -1, (name, args, code)
    assert moe.lib().moe_last_error()


def test_cache_bytes():
    assert moe.moe_kv4_cache_bytes(1, 1, 64, 32) == 36 * 64
    assert moe.moe_kv4_cache_bytes(3, 4, 128, 4096) == 3 * 4 * 128 * 36 * 128
    assert moe.moe_kv4_cache_bytes(1024, 64, 256, 1 << 26) == 1024 * 64 * (1 << 21) * 36 * 256  # past 32 bits
    for bad in [(1, 1, 63, 32), (1, 1, 96, 32), (1, 1, 320, 32), (1, 0, 64, 32), (-1, 1, 64, 32), (1, 1, 64, 0),
                (1, 1, 64, 33), (1, 1, 64, (1 << 26) + 32), (65536, 1, 64, 32), (1, 65536, 64, 32)]:
        assert moe.moe_kv4_cache_bytes(*bad) == 0, bad
    with pytest.raises(moe.MoeError):
        moe.kv4_cache(1, 1, 80, 32, device="cpu")
    assert moe.kv4_cache(2, 3, 64, 96, device="cpu").shape == (2, 3, 3, 36 * 64)


def test_append_and_read_refusals():
    big = 1 << 40
    good = dict(k=OK_PTR, v=OK_PTR, dtype=0, ks=256, vs=256, T=4, n_seq=2, n_kv=4, d=64, mp=64, q_start=OK_PTR, max_q=4,
                kv_len=OK_PTR, cache=OK_PTR, bytes=big)
    bads = [dict(k=None), dict(v=None), dict(k=OK_PTR + 8), dict(dtype=2), dict(dtype=-1), dict(ks=255), dict(vs=258),
            dict(ks=252), dict(T=-1), dict(n_seq=-1), dict(n_kv=0), dict(d=32), dict(d=100), dict(mp=48), dict(mp=0),
            dict(q_start=None), dict(max_q=0), dict(max_q=-3), dict(max_q=(1 << 24) + 1), dict(kv_len=None),
            dict(cache=None), dict(cache=OK_PTR + 4), dict(bytes=2 * 4 * 2 * 36 * 64 - 1), dict(n_seq=70000)]
    for b in bads:
        a = {**good, **b}
        refused("moe_kv4_append", a["k"], a["v"], a["dtype"], a["ks"], a["vs"], a["T"], a["n_seq"], a["n_kv"], a["d"],
                a["mp"], a["q_start"], a["max_q"], a["kv_len"], a["cache"], a["bytes"], None)
        if b in (dict(k=None), dict(v=None)):
            continue
        refused("moe_kv4_read", a["cache"], a["bytes"], a["T"], a["n_seq"], a["n_kv"], a["d"], a["mp"], a["q_start"],
                a["max_q"], a["kv_len"], a["k"], a["v"], a["dtype"], a["ks"], a["vs"], None)
    refused("moe_kv4_read", OK_PTR, big, 4, 2, 4, 64, 64, OK_PTR, 4, OK_PTR, None, None, 0, 256, 256, None)
    # nothing to do: no pointer is looked at
    assert moe.lib().moe_kv4_append(None, None, 0, 0, 0, 0, 2, 4, 64, 64, OK_PTR, 0, None, None, 0, None) == 0
    assert moe.lib().moe_kv4_read(None, 0, 0, 0, 4, 64, 64, None, 0, None, None, None, 0, 0, 0, None) == 0


def test_attention_refusals():
    big = 1 << 40
    good = dict(q=OK_PTR, dtype=1, qs=512, cache=OK_PTR, bytes=big, T=2, n_seq=2, heads=8, n_kv=4, d=64, mp=4096,
                q_start=None, max_q=1, kv_len=OK_PTR, window=0, scale=0.125, out=OK_PTR, os=512, ws=OK_PTR, wb=big)
    bads = [dict(q=None), dict(out=None), dict(q=OK_PTR + 2), dict(out=OK_PTR + 8), dict(qs=508), dict(os=516),
            dict(dtype=3), dict(T=3), dict(heads=9), dict(heads=0), dict(n_kv=0), dict(d=48), dict(mp=4097),
            dict(window=-1), dict(window=(1 << 30) + 1), dict(scale=math.inf), dict(scale=math.nan), dict(scale=-4.5e9), dict(cache=None),
            dict(kv_len=None), dict(bytes=100), dict(ws=None), dict(ws=OK_PTR + 4), dict(wb=16),
            dict(q_start=OK_PTR, max_q=0), dict(q_start=OK_PTR, max_q=1 << 24)]
    for b in bads:
        a = {**good, **b}
        refused("moe_kv4_attention", a["q"], a["dtype"], a["qs"], a["cache"], a["bytes"], a["T"], a["n_seq"], a["heads"],
                a["n_kv"], a["d"], a["mp"], a["q_start"], a["max_q"], a["kv_len"], a["window"], a["scale"], a["out"],
                a["os"], a["ws"], a["wb"], None)
    assert moe.moe_kv4_attention_workspace_bytes(2, 2, 8, 4, 64, 1, 4096) > 0
    assert moe.moe_kv4_attention_workspace_bytes(2, 2, 9, 4, 64, 1, 4096) == 0
    assert moe.moe_kv4_attention_workspace_bytes(2, 2, 8, 4, 65, 1, 4096) == 0
    assert moe.lib().moe_kv4_attention(None, 0, 0, None, 0, 0, 0, 8, 4, 64, 32, None, 0, None, 0, 1.0, None, 0, None, 0, None) == 0


def test_matvec_and_block_refusals():
    far = OK_PTR + (1 << 30)
    for a in [(OK_PTR, OK_PTR, 17, 64, 128, None, far, 0), (OK_PTR, OK_PTR, -1, 64, 128, None, far, 0),
              (OK_PTR, OK_PTR, 1, -1, 128, None, far, 0), (OK_PTR, OK_PTR, 1, 64, 64, None, far, 0),
              (OK_PTR, OK_PTR, 1, 64, 0, None, far, 0), (None, OK_PTR, 1, 64, 128, None, far, 0),
              (OK_PTR, None, 1, 64, 128, None, far, 0), (OK_PTR, OK_PTR, 1, 64, 128, None, None, 0),
              (OK_PTR + 4, OK_PTR, 1, 64, 128, None, far, 0), (OK_PTR, OK_PTR + 8, 1, 64, 128, None, far, 0),
              (OK_PTR, OK_PTR, 1, 64, 128, None, far + 2, 0), (OK_PTR, OK_PTR, 1, 64, 128, far + 1, far, 0),
              (OK_PTR, OK_PTR, 1, 64, 128, None, OK_PTR, 0), (OK_PTR, OK_PTR, 1, 64, 128, None, OK_PTR + 508, 0)]:
        refused("moe_matvec_int4", *a, OK_PTR, 1 << 30, None)
    need = moe.moe_matvec_int4_workspace_bytes(16, 128)
    assert need > 0 and moe.moe_matvec_int4_workspace_bytes(1, 128) == moe.moe_matvec_int4_workspace_bytes(17, 128) == 0
    for ws, size in ((None, 1 << 30), (OK_PTR, need - 1), (OK_PTR + 8, 1 << 30)):
        refused("moe_matvec_int4", OK_PTR, OK_PTR, 16, 64, 128, None, far, 0, ws, size, None)
    assert moe.lib().moe_matvec_int4(None, None, 0, 64, 128, None, None, 0, None, 0, None) == 0
    assert moe.lib().moe_matvec_int4(None, None, 3, 0, 128, None, None, 0, None, 0, None) == 0
    big = 1 << 40
    good = dict(x=OK_PTR, T=2, H=256, nh=4, kv=2, d=64, wq=OK_PTR, wo=OK_PTR, cache=OK_PTR, cb=big, mp=64, kl=OK_PTR,
                theta=1e4, ws=OK_PTR, wb=big)
    for b in [dict(x=None), dict(x=OK_PTR + 4), dict(T=17), dict(T=-1), dict(H=200), dict(nh=5), dict(kv=0), dict(d=80),
              dict(nh=1, kv=1), dict(wq=None), dict(wo=OK_PTR + 2), dict(cache=None), dict(cb=10), dict(mp=50),
              dict(kl=None), dict(theta=1.0), dict(theta=math.nan), dict(ws=None), dict(wb=100), dict(nh=1026, kv=2)]:
        a = {**good, **b}
        refused("moe_attention_decode_int4", a["x"], a["T"], a["H"], a["nh"], a["kv"], a["d"], a["wq"], a["wo"], a["cache"],
                a["cb"], a["mp"], a["kl"], a["theta"], a["ws"], a["wb"], None)
    assert moe.moe_attention_decode_int4_workspace_bytes(1, 256, 4, 2, 64, 64) > 0
    assert moe.moe_attention_decode_int4_workspace_bytes(17, 256, 4, 2, 64, 64) == 0
    assert moe.moe_attention_decode_int4_workspace_bytes(1, 256, 4, 2, 96, 64) == 0


def test_binding_refuses_host_tensors_and_shapes():
    cache = moe.kv4_cache(1, 2, 64, 32, device="cpu")
    k = torch.zeros((1, 2, 64))
    kl = torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        moe.moe_kv4_append(k, k, cache, kl)
    with pytest.raises(ValueError):
        moe.moe_kv4_append(k, k, cache[..., :-4], kl)
    with pytest.raises(ValueError):
        moe.moe_kv4_attention(k, cache.view(torch.int8), kl)
    with pytest.raises(ValueError):
        moe.moe_matvec_int4(torch.zeros((1, 128)), torch.zeros(64 * 64 + 128, dtype=torch.uint8), 64)


# ------------------------------------------------------------------------------------------ store (GPU) ---
def vectors(shape, gen, kind):
    x = torch.randn(shape, generator=gen)
    if kind == "wide":     # ranges of very different size, group by group
        x = x * torch.exp2(torch.randint(-60, 60, (*shape[:-1], shape[-1] // 64, 1), generator=gen).float()).expand(
            *shape[:-1], shape[-1] // 64, 64).reshape(shape)
    elif kind == "ties":   # quotients that lie on a half
        x = torch.randint(0, 31, shape, generator=gen).float() * 0.5
        x[..., 0::64], x[..., 1::64] = 0.0, 15.0
        x = x * torch.exp2(torch.randint(-3, 3, (1,), generator=gen).float())
    elif kind == "offset":  # a base far from the range
        x = x * 0.01 + 100.0
    elif kind == "equal":   # no range at all, in some groups
        x[..., :64] = x[..., :1]
    elif kind == "tiny":
        x = x * 2.0 ** -124
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,n_kv", [(64, 1), (128, 3), (192, 2), (256, 2)])
@pytest.mark.parametrize("kind", ["normal", "wide", "ties", "offset", "equal", "tiny"])
def test_append_then_read_gives_the_defined_values(dtype, d, n_kv, kind):
    gen = torch.Generator().manual_seed(d + n_kv)
    ls = [1, 31, 32, 33, 100, 0, 64]
    ks = [vectors((L, n_kv, d), gen, kind).to(dtype) for L in ls]
    vs = [vectors((L, n_kv, d), gen, kind).to(dtype) for L in ls]
    cache = fill(moe.kv4_cache(len(ls), n_kv, d, 128))
    put(ks, vs, cache, dtype)
    qs, kl, T = batch(ls, ls)
    k, v = moe.moe_kv4_read(cache, kl, T, q_start=qs, dtype=dtype)
    moe.moe_sync_check()
    assert torch.equal(k.cpu(), held(torch.cat(ks)).float().to(dtype))
    assert torch.equal(v.cpu(), held(torch.cat(vs)).float().to(dtype))


@pytest.mark.gpu
def test_append_in_pieces_equals_at_once_and_leaves_the_rest():
    """Tokens that start and end inside a block, one at a time and in chunks: the same bytes as in one call."""
    gen = torch.Generator().manual_seed(5)
    n_kv, d, L = 2, 128, 150
    k, v = (torch.randn((L, n_kv, d), generator=gen).cuda() for _ in range(2))
    whole, parts = (moe.kv4_cache(1, n_kv, d, 160) for _ in range(2))
    whole.zero_()
    parts.zero_()
    moe.moe_kv4_append(k, v, whole, torch.tensor([L], dtype=torch.int32).cuda(),
                       q_start=torch.tensor([0, L], dtype=torch.int32).cuda())
    at = 0
    for n in [1, 1, 5, 30, 1, 33, 64, 14, 1]:
        at += n
        moe.moe_kv4_append(k[at - n:at], v[at - n:at], parts, torch.tensor([at], dtype=torch.int32).cuda(),
                           q_start=torch.tensor([0, n], dtype=torch.int32).cuda())
    assert at == L and torch.equal(whole, parts)
    before = parts.clone()
    moe.moe_kv4_append(k[:1], v[:1], parts, torch.tensor([40], dtype=torch.int32).cuda())
    kl = torch.tensor([L], dtype=torch.int32).cuda()
    qs = torch.tensor([0, L], dtype=torch.int32).cuda()
    a, b = moe.moe_kv4_read(before, kl, L, q_start=qs), moe.moe_kv4_read(parts, kl, L, q_start=qs)
    for x, y, src in ((a[0], b[0], k), (a[1], b[1], v)):
        assert torch.equal(torch.cat([x[:39], x[40:]]), torch.cat([y[:39], y[40:]]))
        assert torch.equal(y[39].cpu(), held(src[:1].cpu()).float().to(BF16)[0])
    moe.moe_sync_check()


@pytest.mark.gpu
def test_store_padding_untouched_rows_strides_and_bad_lengths():
    gen = torch.Generator().manual_seed(6)
    n_kv, d = 3, 64
    ns, ls = [4, 0, 3, 2], [2, 7, 40, 2]  # the first sequence's first two tokens are padding
    qs, kl, T = batch(ns, ls, extra=3)    # three rows behind the last sequence
    wide = torch.randn((T, 5, n_kv, d), generator=gen).cuda()
    k, v = wide[:, 1], wide[:, 3]         # tokens strided, as in a fused projection
    cache = fill(moe.kv4_cache(4, n_kv, d, 64))
    moe.moe_kv4_append(k, v, cache, kl, q_start=qs)
    out = torch.full((T, 2, n_kv, d), 7.0, device="cuda")
    moe.moe_kv4_read(cache, kl, T, q_start=qs, k_out=out[:, 0], v_out=out[:, 1])
    moe.moe_sync_check()
    for x, y in ((k, out[:, 0]), (v, out[:, 1])):
        ref = held(x.cpu()).float()
        ref[:2] = 0
        ref[9:] = 7.0
        assert torch.equal(y.cpu(), ref)
    # a length past the cache stores nothing and reads as zeros; a token range that does not fit is empty
    before = cache.clone()
    bad_len = torch.tensor([2, 7, 65, -1], dtype=torch.int32).cuda()
    moe.moe_kv4_append(k[4:], v[4:], cache, bad_len, q_start=torch.tensor([0, 0, 0, 3, 5], dtype=torch.int32).cuda())
    with pytest.raises(moe.MoeError) as e:
        moe.moe_sync_check()
    assert e.value.code == -2 and torch.equal(before, cache)
    for start in ([0, 0, 0, 0, 99], [-1, 0, 0, 0, 0], [0, 4, 2, 2, 2], [0, 0, 0, 0, 5]):
        kw = dict(max_q=4) if start[-1] == 5 else {}
        got = torch.full((6, n_kv, d), 7.0, device="cuda")
        moe.moe_kv4_read(cache, kl, 6, q_start=torch.tensor(start, dtype=torch.int32).cuda(), k_out=got, **kw)
        with pytest.raises(moe.MoeError) as e:
            moe.moe_sync_check()
        assert e.value.code == -2
        bad = [i for i in range(4) if start[i] < 0 or start[i + 1] < start[i] or start[i + 1] > 6 or start[i + 1] - start[i] > kw.get("max_q", 6)]
        for i in range(4):
            if i in bad and start[i] >= 0 and start[i + 1] > start[i]:
                assert (got[start[i]:] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3.4e38])
def test_append_of_values_that_are_not_finite(value):
    gen = torch.Generator().manual_seed(7)
    k, v = torch.randn((40, 2, 128), generator=gen), torch.randn((40, 2, 128), generator=gen)
    k[3, 1, 70], v[35, 0, 1] = value, value
    if value == 3.4e38:  # finite, but the range is not
        k[3, 1, 71], v[35, 0, 2] = -value, -value
    cache = fill(moe.kv4_cache(1, 2, 128, 64))
    qs, kl, T = batch([40], [40])
    moe.moe_kv4_append(k.cuda(), v.cuda(), cache, kl, q_start=qs)
    with pytest.raises(moe.MoeError) as e:
        moe.moe_sync_check()
    assert e.value.code == -3
    a, b = moe.moe_kv4_read(cache, kl, T, q_start=qs, dtype=F32)
    assert (a[3, 1, 64:] == 0).all() and (b[35, 0, :64] == 0).all()
    assert torch.equal(a.cpu(), held(k).float()) and torch.equal(b.cpu(), held(v).float())
    moe.moe_sync_check()


# -------------------------------------------------------------------------------------- attention (GPU) ---
CASES = [  # (d, n_kv, group, tokens, lengths, max_pos, window)
    (128, 2, 8, [1, 1, 1], [1, 33, 300], 512, 0),
    (128, 1, 16, [1], [97], 128, 0),
    (64, 2, 1, [1, 1], [64, 5], 64, 0),
    (64, 3, 7, [3, 5, 0, 2], [3, 200, 9, 41], 224, 0),
    (128, 2, 3, [20, 1, 7], [20, 70, 64], 96, 0),
    (128, 1, 8, [70], [133], 160, 0),
    (128, 1, 20, [2, 9], [150, 9], 160, 0),
    (192, 1, 4, [1, 6], [40, 66], 96, 0),
    (256, 2, 2, [1, 17], [65, 40], 96, 0),
    (256, 1, 8, [5], [45], 64, 0),
    (128, 2, 4, [1, 40], [200, 100], 256, 33),
    (64, 1, 2, [4, 4], [130, 64], 160, 1),
    (64, 2, 4, [6, 5, 3, 1], [2, 0, 3, 0], 32, 0),      # padded tokens, sequences without a position
    (128, 1, 4, [40, 1], [7, 0], 64, 5),
    # hundreds of rows on many heads
    (128, 16, 4, [40, 33, 70, 5], [40, 100, 200, 3], 224, 0),
    (64, 16, 8, [16, 1, 17], [300, 1, 64], 320, 0),
    (128, 16, 8, [31, 16, 40, 2], [64, 20, 17, 1], 96, 0),
    (64, 16, 4, [33, 40, 64, 20], [130, 65, 64, 7], 160, 48),
    (128, 64, 4, [33, 32, 31, 40], [97, 32, 10, 160], 160, 0),
    (64, 64, 2, [64, 80, 70, 3], [70, 80, 200, 0], 224, 33),
    (192, 16, 4, [40, 33, 70, 5], [40, 100, 200, 3], 224, 0),
    (192, 16, 8, [33, 20, 17, 1], [130, 65, 64, 7], 160, 48),
    (256, 16, 4, [40, 33, 70, 5], [40, 100, 200, 3], 224, 0),
    (256, 32, 3, [43, 64, 1, 44], [31, 160, 0, 129], 160, 33),
    # the same over long caches, whose positions are split
    (128, 8, 4, [40, 33, 70, 5], [1500, 700, 2000, 3], 2048, 0),
    (128, 32, 2, [100, 64], [1100, 64], 2048, 600),
    (64, 16, 8, [33, 20, 17, 0], [1300, 2048, 1, 64], 2048, 0),
    (64, 2, 8, [256, 200], [1300, 600], 1312, 0),
    (192, 8, 4, [40, 33, 70, 5], [1500, 700, 2000, 3], 2048, 900),
    (256, 8, 4, [70, 33], [1057, 1056], 1088, 0),
    # more sequences than a wave has lanes, split
    (64, 1, 4, [1] * 70, [(37 * i) % 600 for i in range(70)], 608, 0),
    (64, 1, 8, [16 - i % 3 for i in range(70)], [16 + (53 * i) % 590 for i in range(70)], 608, 0),
    (128, 2, 1, [3] * 33 + [0] * 33 + [2] * 33, [(71 * i) % 700 for i in range(99)], 704, 100),
]


def attention_case(d, n_kv, G, ns, ls, max_pos, window, dtype, seed=0, scale=None, amplitude=1.0):
    gen = torch.Generator().manual_seed(seed + d)
    ks = [torch.randn((L, n_kv, d), generator=gen) * amplitude + 0.3 for L in ls]
    vs = [torch.randn((L, n_kv, d), generator=gen) for L in ls]
    cache = fill(moe.kv4_cache(len(ls), n_kv, d, max_pos))
    put(ks, vs, cache, F32)
    q = torch.randn((sum(ns), n_kv * G, d), generator=gen).to(dtype)
    ref, amount, shift = attend(q.double(), ks, vs, ns, ls, G, window, d ** -0.5 if scale is None else scale, dtype)
    return cache, q, ref, attention_tolerance(ref, amount, shift, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_matches_the_plain_form(case, dtype):
    d, n_kv, G, ns, ls, max_pos, window = CASES[case]
    cache, q, ref, tol = attention_case(*CASES[case], dtype)
    qs, kl, T = batch(ns, ls)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns), window=window)
    moe.moe_sync_check()
    assert out.dtype is dtype
    err = (out.cpu().double() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())
    t = 0
    for n, L in zip(ns, ls):  # padding gives exact zeros
        assert (out[t:t + max(0, n - L)] == 0).all()
        t += n
    if all(n == 1 for n in ns):  # the form without q_start, and a looser bound on the tokens
        assert torch.equal(moe.moe_kv4_attention(q.cuda(), cache, kl, window=window), out)
    # twice the same bits
    assert torch.equal(moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns), window=window), out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strides_rows_behind_and_loose_max_q(dtype):
    case = (128, 2, 4, [3, 1, 2], [40, 1, 90], 96, 0)
    cache, q, ref, tol = attention_case(*case, dtype)
    qs, kl, T = batch(case[3], case[4], extra=2)
    wide = torch.full((T, 24, 128), float("nan"), dtype=dtype, device="cuda")
    wide[:6, 8:16] = q.cuda()
    out = torch.full((T, 16, 128), 3.0, dtype=dtype, device="cuda")
    moe.moe_kv4_attention(wide[:, 8:16], cache, kl, q_start=qs, out=out[:, 4:12])
    moe.moe_sync_check()
    assert ((out[:6, 4:12].cpu().double() - ref).abs() <= tol).all()
    assert (out[6:] == 3).all() and (out[:, :4] == 3).all() and (out[:, 12:] == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_attention_scales(dtype, scale):
    """Scores that are all equal, turned round, and so far apart that few positions count."""
    for case in ((128, 1, 4, [2, 1], [70, 40], 96, 0), (128, 1, 16, [2, 1], [70, 40], 96, 0),
                 (64, 16, 8, [33, 20, 17, 1], [70, 40, 100, 1], 128, 0)):
        cache, q, ref, tol = attention_case(*case, dtype, scale=scale)
        qs, kl, _ = batch(case[3], case[4])
        out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(case[3]), scale=scale)
        assert ((out.cpu().double() - ref).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k_size,v_size", [(2.0 ** -30, 2.0 ** -55), (2.0 ** 30, 2.0 ** 38), (1.0, 2.0 ** -20)])
def test_attention_range(dtype, k_size, v_size):
    """Keys and values far from one, the scores kept where they are by the scale."""
    for d, n_kv, G, ns, ls in ((128, 2, 4, [1, 1], [70, 200]), (64, 2, 12, [3, 1], [70, 40]), (128, 16, 8, [20, 33, 17, 1], [70, 40, 100, 1]),
                              (192, 16, 8, [20, 33, 17, 1], [70, 40, 100, 1]), (256, 16, 8, [20, 33, 17, 1], [70, 40, 100, 1])):
        gen = torch.Generator().manual_seed(d)
        ks = [torch.randn((L, n_kv, d), generator=gen) * k_size for L in ls]
        vs = [torch.randn((L, n_kv, d), generator=gen) * v_size for L in ls]
        cache = fill(moe.kv4_cache(len(ls), n_kv, d, 224))
        put(ks, vs, cache, F32)
        q = torch.randn((sum(ns), n_kv * G, d), generator=gen).to(dtype)
        scale = d ** -0.5 / k_size
        ref, amount, shift = attend(q.double(), ks, vs, ns, ls, G, 0, scale, dtype)
        qs, kl, _ = batch(ns, ls)
        out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns), scale=scale)
        err, tol = (out.cpu().double() - ref).abs(), attention_tolerance(ref, amount, shift, dtype)
        assert (err <= tol).all(), float((err / tol).max())
    moe.moe_sync_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n_kv,G,n", [(2, 4, 1), (2, 12, 1), (2, 12, 3), (16, 8, 40)])
@pytest.mark.parametrize("order", [1, -1])
def test_attention_over_keys_and_values_of_changing_size(dtype, n_kv, G, n, order):
    """Keys and values that grow (or shrink) by 2^16 from one run of positions to the next, run by run."""
    gen = torch.Generator().manual_seed(n + G)
    d, L = 128, 450
    size = torch.exp2(torch.tensor([-8, -3, 0, 8, -8, 2, 5, 8, 1, -5][::order]).float()).repeat_interleave(45)[:, None, None]
    v = torch.randn((L, n_kv, d), generator=gen) * size
    k = torch.randn((L, n_kv, d), generator=gen) * size.rsqrt().clamp(max=4)
    ks, vs, ns, ls = [k, k[:90]], [v, v[:90]], [n, n], [L, 90]
    cache = fill(moe.kv4_cache(2, n_kv, d, 480))
    put(ks, vs, cache, F32)
    q = torch.randn((2 * n, n_kv * G, d), generator=gen).to(dtype)
    ref, amount, shift = attend(q.double(), ks, vs, ns, ls, G, 0, 0.02, dtype)
    qs, kl, _ = batch(ns, ls)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=n, scale=0.02)
    moe.moe_sync_check()
    err, tol = (out.cpu().double() - ref).abs(), attention_tolerance(ref, amount, shift, dtype)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 9])
def test_attention_long_and_split(n):
    """Enough positions that they are split over blocks, and a maximum that moves from split to split."""
    gen = torch.Generator().manual_seed(11)
    d, n_kv, G, L = 128, 1, 2, 5000
    k = torch.randn((L, n_kv, d), generator=gen) * 0.2
    k[4321] += 2.0
    v = torch.randn((L, n_kv, d), generator=gen)
    cache = fill(moe.kv4_cache(1, n_kv, d, 5024))
    put([k], [v], cache, F32)
    q = torch.randn((n, G, d), generator=gen)
    qs, kl, _ = batch([n], [L])
    assert moe.moe_kv4_attention_workspace_bytes(n, 1, G, n_kv, d, n, 5024) > 0
    for dtype in (F32, BF16):
        qd = q.to(dtype)
        ref, amount, shift = attend(qd.double(), [k], [v], [n], [L], G, 0, d ** -0.5, dtype)
        out = moe.moe_kv4_attention(qd.cuda(), cache, kl, q_start=qs, max_q=n)
        err = (out.cpu().double() - ref).abs()
        tol = attention_tolerance(ref, amount, shift, dtype)
        assert (err <= tol).all(), float((err / tol).max())
    moe.moe_sync_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_bad_batch_and_values(dtype):
    case = (64, 1, 2, [2, 1, 1], [10, 40, 3], 64, 0)
    cache, q, ref, tol = attention_case(*case, dtype)
    qs, kl, T = batch(case[3], case[4])
    bad = kl.clone()
    bad[1] = 65
    out = moe.moe_kv4_attention(q.cuda(), cache, bad, q_start=qs)
    with pytest.raises(moe.MoeError) as e:
        moe.moe_sync_check()
    assert e.value.code == -2
    assert (out[2] == 0).all()
    good = [0, 1, 3]
    assert ((out.cpu().double() - ref).abs() <= tol)[good].all()
    out = torch.full_like(out, 5.0)
    moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=torch.tensor([0, 2, 1, 9], dtype=torch.int32).cuda(), out=out)
    with pytest.raises(moe.MoeError) as e:
        moe.moe_sync_check()
    assert e.value.code == -2 and (out[2:] == 5).all()
    assert ((out.cpu().double() - ref).abs() <= tol)[:2].all()
    # a query that is not finite spoils its own head's row and no other
    for value in (math.nan, math.inf):
        qb = q.clone()
        qb[0, 1, 5] = value
        out = moe.moe_kv4_attention(qb.cuda(), cache, kl, q_start=qs).cpu().double()
        ok = torch.ones((T, 2), dtype=torch.bool)
        ok[0, 1] = False
        assert ((out - ref).abs() <= tol)[ok].all() and not torch.isfinite(out[0, 1]).any()
    # nor in a call of many rows
    case = (64, 16, 8, [33, 20, 17, 1], [70, 40, 100, 1], 128, 0)
    cache, q, ref, tol = attention_case(*case, dtype)
    qs, kl, T = batch(case[3], case[4])
    q[40, 77, 5], q[3, 0, 0] = math.nan, math.inf
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=33).cpu().double()
    ok = torch.ones((T, 128), dtype=torch.bool)
    ok[40, 77] = ok[3, 0] = False
    assert ((out - ref).abs() <= tol)[ok].all() and not torch.isfinite(out[~ok]).any()
    moe.moe_sync_check()


# ----------------------------------------------------------------------------------- int4 products (GPU) ---
def matvec_reference(x, w, add, norm):
    """Value and bound: the tokens' values within 2^-22 of the token's largest, exact products of q s x in fp32 sums:
    a group's sum of at most 12 partial results, the groups' scaled sums (K / 128 of them), the terms and the
    norm: 2^-24 of what they amount to for each of at most 32 + K / 128 roundings (2^-22 where a matrix
    product rounds towards zero)."""
    h = x.double()
    r = torch.ones((x.shape[0], 1), dtype=torch.float64)
    if norm:
        r = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
    K = x.shape[1]
    q, s = w
    y = (h * r) @ (q * s).T
    amount = (h.abs() * r) @ (q.abs() * s.abs()).T
    largest = (h.abs().amax(1, keepdim=True) * r) @ (q.abs() * s.abs()).sum(1)[None]
    tol = amount * (32 + K // 128) * 2.0 ** -22 + largest * 2.0 ** -22 + y.abs() * 2.0 ** -21
    if add is not None:
        y = y + add.double()
    return y, tol + y.abs() * 2.0 ** -24


def int4_parts(raw, N, K):
    b = raw[:N * K // 2].to(torch.int32)
    q = torch.stack([b & 15, b >> 4], -1).flatten().view(N, K)
    q = torch.where(q > 7, q - 16, q).double()
    s = raw[N * K // 2:].clone().view(BF16).double().view(N, K // 128).repeat_interleave(128, 1)
    return q, s


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 5, 6, 8, 11, 16])
@pytest.mark.parametrize("N,K", [(1, 128), (15, 256), (17, 2048), (100, 1408), (33, 4224), (16, 8192), (100, 2560)])
def test_matvec_matches_the_plain_form(T, N, K):
    gen = torch.Generator().manual_seed(T * 1000 + N)
    raw, _ = int4_matrix(N, K, gen)
    parts = int4_parts(raw, N, K)
    x = torch.randn((T, K), generator=gen) * torch.exp2(torch.randint(-20, 20, (T, 1), generator=gen).float())
    add = torch.randn((T, N), generator=gen)
    wd, xd, ad = raw.cuda(), x.cuda(), add.cuda()
    for norm in (False, True):
        for a in (None, add):
            y = moe.moe_matvec_int4(xd, wd, N, add=None if a is None else ad, rmsnorm=norm)
            ref, tol = matvec_reference(x, parts, a, norm)
            err = (y.cpu().double() - ref).abs()
            assert (err <= tol).all(), float((err / tol).max())
    y = ad.clone()  # in place on what is added
    moe.moe_matvec_int4(xd, wd, N, y=y, add=y)
    assert torch.equal(y, moe.moe_matvec_int4(xd, wd, N, add=ad))


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(40007, 512), (20001, 1408), (16400, 4352), (135000, 128), (270000, 128),
                                 (9001, 1024), (8300, 2048), (16400, 2176), (8300, 2304)])
@pytest.mark.parametrize("T", [1, 7, 8, 9, 16])
def test_matvec_many_rows(T, N, K):
    """Enough rows that waves and blocks take several items."""
    gen = torch.Generator().manual_seed(T)
    raw, _ = int4_matrix(N, K, gen)
    parts = int4_parts(raw, N, K)
    x = torch.randn((T, K), generator=gen)
    y = torch.full((T * N + 64,), 9.0, device="cuda")
    moe.moe_matvec_int4(x.cuda(), raw.cuda(), N, y=y[:T * N].view(T, N), rmsnorm=True)
    ref, tol = matvec_reference(x, parts, None, True)
    err = (y[:T * N].view(T, N).cpu().double() - ref).abs()
    assert (err <= tol).all() and (y[T * N:] == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2, 9])
@pytest.mark.parametrize("N", [40, 33000])
def test_matvec_values_that_are_not_finite_or_huge(T, N):
    gen = torch.Generator().manual_seed(3)
    K = 256
    raw, _ = int4_matrix(N, K, gen)
    q, s = int4_parts(raw, N, K)
    x = torch.randn((T, K), generator=gen)
    x[0, 5] = math.inf
    x[1] = x[1] * 1e38
    y = moe.moe_matvec_int4(x.cuda(), raw.cuda(), N).cpu().double()
    w0 = (q * s)[:, 5]
    assert torch.equal(torch.isnan(y[0]), w0 == 0)
    assert (y[0][w0 > 0] == math.inf).all() and (y[0][w0 < 0] == -math.inf).all()
    ref, tol = matvec_reference(x[1:], (q, s), None, False)
    fits = ref.abs() < 3.0e38  # (what does not fit may come out infinite)
    assert ((y[1:] - ref).abs() <= tol)[fits].all()


# ------------------------------------------------------------------------- graphs, streams, together (GPU) ---
@pytest.mark.gpu
def test_captured_decode_step_replays_with_new_lengths():
    """Projection, append and attention of a batch captured once: replays at other lengths and inputs, with eager
    work of the same kind between them, equal the eager calls."""
    gen = torch.Generator().manual_seed(21)
    B, n_kv, G, d, H, max_pos = 3, 2, 4, 64, 256, 2048
    rows = (G + 2) * n_kv * d
    raw, _ = int4_matrix(rows, H, gen, 0.1)
    raw = raw.cuda()
    cache = fill(moe.kv4_cache(B, n_kv, d, max_pos))
    lens = [5, 700, 1900]
    put([torch.randn((L, n_kv, d), generator=gen) for L in lens], [torch.randn((L, n_kv, d), generator=gen) for L in lens],
        cache, F32)
    x = torch.randn((B, H), generator=gen).cuda()
    kv_len = torch.tensor(lens, dtype=torch.int32).cuda() + 1
    ws = torch.empty(max(256, moe.moe_kv4_attention_workspace_bytes(B, B, G * n_kv, n_kv, d, 1, max_pos)),
                     dtype=torch.uint8, device="cuda")
    qkv, out = torch.empty((B, rows), device="cuda"), torch.empty((B, G * n_kv, d), device="cuda")

    def step(cache, x, kv_len, qkv, out, ws):
        moe.moe_matvec_int4(x, raw, rows, y=qkv, rmsnorm=True)
        t = qkv.view(B, -1, d)
        moe.moe_kv4_append(t[:, G * n_kv:(G + 1) * n_kv], t[:, (G + 1) * n_kv:], cache, kv_len)
        moe.moe_kv4_attention(t[:, :G * n_kv], cache, kv_len, out=out, workspace=ws)

    eager = cache.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(cache, x, kv_len, qkv, out, ws)
    ref = torch.empty_like(out)
    for i in range(4):
        x.copy_(torch.randn((B, H), generator=gen))
        if i:
            kv_len += 1
        graph.replay()
        step(eager, x, kv_len, torch.empty_like(qkv), ref, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    assert torch.equal(cache, eager)
    moe.moe_sync_check()


@pytest.mark.gpu
def test_captured_prompts_replay_with_new_lengths():
    """Prompts over a long cache, whose split goes by the lengths on the device, and a product of nine tokens, captured
    once; a query that is not finite spoils its own row in every piece and no other."""
    gen = torch.Generator().manual_seed(23)
    n_kv, G, d, max_pos, ns, ls = 8, 4, 128, 2048, [40, 33], [1400, 90]
    cache = fill(moe.kv4_cache(2, n_kv, d, max_pos))
    k = [torch.randn((2000, n_kv, d), generator=gen) for _ in ns]
    put(k, k, cache, BF16)
    qs, kl, T = batch(ns, ls)
    q = torch.randn((T, n_kv * G, d), generator=gen).bfloat16().cuda()
    raw, _ = int4_matrix(500, 2048, gen)
    raw, x = raw.cuda(), torch.randn((9, 2048), generator=gen).cuda()
    n = moe.moe_kv4_attention_workspace_bytes(T, 2, n_kv * G, n_kv, d, 40, max_pos)
    assert n > 0 and moe.moe_matvec_int4_workspace_bytes(9, 2048) > 0
    ws, ws9 = (torch.empty(b, dtype=torch.uint8, device="cuda") for b in (n, moe.moe_matvec_int4_workspace_bytes(9, 2048)))
    out, y = torch.empty_like(q), torch.empty((9, 500), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        moe.moe_kv4_attention(q, cache, kl, q_start=qs, max_q=40, out=out, workspace=ws)
        moe.moe_matvec_int4(x, raw, 500, y=y, rmsnorm=True, workspace=ws9)
    for i, lens in enumerate(([1400, 90], [40, 1990], [0, 33], [2000, 2000])):
        kl.copy_(torch.tensor(lens, dtype=torch.int32))
        x.mul_(1.5)
        graph.replay()
        ref = moe.moe_kv4_attention(q, cache, kl, q_start=qs, max_q=40)
        assert torch.equal(out, ref) and torch.equal(y, moe.moe_matvec_int4(x, raw, 500, rmsnorm=True))
    bad = q.clone()
    bad[5, 7, 3], bad[60, 0, 0] = math.nan, math.inf
    spoilt = moe.moe_kv4_attention(bad, cache, kl, q_start=qs, max_q=40)
    ok = torch.ones((T, n_kv * G), dtype=torch.bool)
    ok[5, 7] = ok[60, 0] = False
    assert torch.equal(spoilt.cpu()[ok], ref.cpu()[ok]) and not torch.isfinite(spoilt.cpu()[~ok]).any()
    moe.moe_sync_check()


@pytest.mark.gpu
def test_calls_on_another_stream():
    gen = torch.Generator().manual_seed(22)
    k = torch.randn((64, 2, 128), generator=gen).cuda()
    q = torch.randn((64, 4, 128), generator=gen).cuda()
    qs, kl, T = batch([64], [64])
    cache, other = moe.kv4_cache(1, 2, 128, 64), moe.kv4_cache(1, 2, 128, 64)
    moe.moe_kv4_append(k, k, cache, kl, q_start=qs)
    ref = moe.moe_kv4_attention(q, cache, kl, q_start=qs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    moe.moe_kv4_append(k, k, other, kl, q_start=qs, stream=side)
    out = moe.moe_kv4_attention(q, other, kl, q_start=qs, stream=side.cuda_stream)
    back = moe.moe_kv4_read(other, kl, T, q_start=qs, stream=side)
    side.synchronize()
    assert torch.equal(out, ref) and torch.equal(back[0], moe.moe_kv4_read(cache, kl, T, q_start=qs)[0])
    moe.moe_sync_check(side)


def rope(v, p, theta):
    d = v.shape[-1]
    ang = p * theta ** (-2 * torch.arange(d // 2, dtype=torch.float64) / d)
    a, b = v[..., :d // 2], v[..., d // 2:]
    return torch.cat([a * torch.cos(ang) - b * torch.sin(ang), b * torch.cos(ang) + a * torch.sin(ang)], -1)


def normed(v):
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)


@pytest.mark.gpu
@pytest.mark.parametrize("d,n_kv,G,lens", [(128, 2, 4, [1, 70, 33]), (64, 1, 2, [100]), (256, 1, 2, [5, 64]), (192, 2, 1, [40]),
                                           (128, 1, 8, [0, 12, 96, 31, 32, 1])])
def test_block_matches_its_parts(d, n_kv, G, lens):
    """The block's new keys and values lie within a step of the quantiser of the 64-bit ones, and its output is that
    of 64-bit attention over what the cache then holds."""
    gen = torch.Generator().manual_seed(d + G)
    T, H, nh, max_pos, theta = len(lens), 256, G * n_kv, 128, 1.0e4
    rows = (nh + 2 * n_kv) * d
    rq, wq = int4_matrix(rows, H, gen, 0.05)
    ro, wo = int4_matrix(H, nh * d, gen, 0.05)
    cache = fill(moe.kv4_cache(T, n_kv, d, max_pos))
    put([torch.randn((max(L - 1, 0), n_kv, d), generator=gen) for L in lens],
        [torch.randn((max(L - 1, 0), n_kv, d), generator=gen) for L in lens], cache, F32)
    x = torch.randn((T, H), generator=gen)
    xd, kl = x.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    moe.moe_attention_decode_int4(xd, rq.cuda(), ro.cuda(), cache, kl, nh, theta)
    moe.moe_sync_check()
    qs, _, n = batch(lens, lens)
    K, V = (t.cpu().double() for t in moe.moe_kv4_read(cache, kl, n, q_start=qs, dtype=F32))
    qkv = (normed(x.double()) @ wq.T).view(T, -1, d)
    y = x.double().clone()
    at = 0
    for t, L in enumerate(lens):
        if L:
            q = rope(normed(qkv[t, :nh]), L - 1, theta)
            kn, vn = rope(normed(qkv[t, nh:nh + n_kv]), L - 1, theta), qkv[t, nh + n_kv:]
            for got, want in ((K[at + L - 1], kn), (V[at + L - 1], vn)):
                w = want.view(n_kv, -1, GROUP)
                step = (w.amax(-1, keepdim=True) - w.amin(-1, keepdim=True)) / 15
                # half a step, the scale's rounding over 15 steps, the base's
                bound = step * (0.5 + 15 * 2.0 ** -8) + w.abs().amax(-1, keepdim=True) * 2.0 ** -8 + 1e-5
                assert ((got.view_as(w) - w).abs() <= bound).all()
            att = torch.empty((nh, d), dtype=torch.float64)
            for h in range(nh):
                p = torch.softmax(K[at:at + L, h // G] @ q[h] / math.sqrt(d), 0)
                att[h] = p @ V[at:at + L, h // G]
            y[t] += wo @ att.flatten()
        at += L
    # probabilities and scores within 2^-16 and the projections' sums, on outputs of sum |w| |att|
    tol = wo.abs().sum(1).max() * 4.0 * 2.0 ** -14 / math.sqrt(nh * d) + 1e-5
    assert ((xd.cpu().double() - y).abs() <= tol).all(), float((xd.cpu().double() - y).abs().max() / tol)
    for t, L in enumerate(lens):
        if L == 0:
            assert torch.equal(xd[t].cpu(), x[t])


@pytest.mark.gpu
def test_block_bad_length_changes_nothing_else():
    gen = torch.Generator().manual_seed(1)
    d, n_kv, G, H, T = 64, 2, 2, 128, 2
    rq, _ = int4_matrix((G + 2) * n_kv * d, H, gen)
    ro, _ = int4_matrix(H, G * n_kv * d, gen)
    cache = moe.kv4_cache(T, n_kv, d, 32)
    cache.zero_()
    x = torch.randn((T, H), generator=gen).cuda()
    one, good = x.clone(), cache.clone()
    moe.moe_attention_decode_int4(one, rq.cuda(), ro.cuda(), good, torch.tensor([4, 0], dtype=torch.int32).cuda(), G * n_kv)
    moe.moe_sync_check()
    for L in (33, -2):
        y, c = x.clone(), cache.clone()
        moe.moe_attention_decode_int4(y, rq.cuda(), ro.cuda(), c, torch.tensor([4, L], dtype=torch.int32).cuda(), G * n_kv)
        with pytest.raises(moe.MoeError) as e:
            moe.moe_sync_check()
        assert e.value.code == -2
        assert torch.equal(y, one) and torch.equal(c, good)


@pytest.mark.gpu
def test_stack_with_int4_attention_equals_its_blocks():
    """A decode stack with int4 attention blocks: every step is the block, then a stack of that layer alone."""
    gen = torch.Generator().manual_seed(31)
    L, H, I, E, k, d, n_kv, G, max_pos, steps = 2, 256, 128, 8, 2, 64, 2, 2, 64, 5
    nh = G * n_kv
    expert = 3 * H * I * 2
    host = moe.PinnedBuffer(L * E * expert)
    w = (torch.randn(L * E * 3 * H * I, generator=gen) * 0.02).to(BF16)
    host.array[:] = w.view(torch.uint8).numpy()
    router = [(torch.randn((E, H), generator=gen) * 0.05).to(BF16).cuda() for _ in range(L)]
    wq = [int4_matrix((nh + 2 * n_kv) * d, H, gen)[0].cuda() for _ in range(L)]
    wo = [int4_matrix(H, nh * d, gen)[0].cuda() for _ in range(L)]

    def cache_of(l0, n):
        return moe.ExpertCache(n, E, expert, n * E * expert, host.ptr + l0 * E * expert, E * expert, expert, preload=True)

    kv = [moe.kv4_cache(1, n_kv, d, max_pos) for _ in range(L)]
    for c in kv:
        c.zero_()
    ref_kv = [c.clone() for c in kv]
    att = dict(n_heads=nh, n_kv=n_kv, head_dim=d, max_pos=max_pos, theta=1.0e4, start_pos=0, w_qkv=wq, w_o=wo, cache=kv, int4=True)
    both = cache_of(0, L)
    stack = moe.MoeStack(both, H, I, E, k, moe.MOE_BF16, moe.MOE_BF16, router, attention=att)
    singles = [moe.MoeStack(cache_of(l, 1), H, I, E, k, moe.MOE_BF16, moe.MOE_BF16, router[l:l + 1]) for l in range(L)]
    for t in range(steps):
        x0 = torch.randn((1, H), generator=gen)
        x, y = x0.cuda(), x0.cuda()
        (stack.decode_graph if t == 3 else stack.decode_step)(t, x)
        kl = torch.tensor([t + 1], dtype=torch.int32).cuda()
        for l in range(L):
            moe.moe_attention_decode_int4(y, wq[l], wo[l], ref_kv[l], kl, nh, 1.0e4)
            singles[l].decode_step(t, y)
        torch.cuda.synchronize()
        assert torch.equal(x, y)
        assert all(torch.equal(a, b) for a, b in zip(kv, ref_kv))
    assert stack.kernel_time(4, 5) > 0
    moe.moe_sync_check()
    full = dict(att, start_pos=max_pos - 1)
    stack = moe.MoeStack(both, H, I, E, k, moe.MOE_BF16, moe.MOE_BF16, router, attention=full)
    stack.decode_step(0, torch.zeros((1, H), device="cuda"))
    with pytest.raises(moe.MoeError):
        stack.decode_step(1, torch.zeros((1, H), device="cuda"))
    for bad in (dict(max_pos=48), dict(head_dim=48), dict(start_pos=max_pos), dict(cache=[moe.kv4_cache(2, n_kv, d, max_pos)] * 2)):
        with pytest.raises((moe.MoeError, ValueError)):
            moe.MoeStack(both, H, I, E, k, moe.MOE_BF16, moe.MOE_BF16, router, attention=dict(att, **bad))


# ------------------------------------------------------------------- windows over what was never written (GPU) ---
def relative_rms(out, ref):
    return float((out.cpu().double() - ref).square().mean().sqrt() / ref.square().mean().sqrt())


# Largest relative rms error of an attention over values of one size and scores of a few units.
#   fp32: probabilities times scales in two fp16 terms and scores of up to 16 in log2 units, each within 2^-22 with both
#   signs; the exponential's last place; about 5e-7 together.
#   bf16: the output's rounding, 2^-8 at most and evenly spread (2^-8 / sqrt 3 = 2.26e-3), and three fp16 roundings
#   (probabilities, keys, values; 2^-11 / sqrt 3 each): 2.31e-3 together.
RMS = {F32: 1e-6, BF16: 2.5e-3}

WINDOWS = [  # (d, n_kv, group, tokens per sequence, sequences, window, first length, step of the lengths, max_pos)
    (64, 1, 4, 1, 32, 40, 81, 1, 128),        # every offset of the window's start in its block of 32
    (128, 1, 4, 1, 32, 40, 81, 1, 128),
    (64, 2, 16, 1, 32, 70, 300, 1, 512),      # (positions split)
    (128, 1, 12, 3, 32, 200, 1000, 1, 1056),
    (192, 1, 2, 2, 32, 33, 100, 1, 160),
    (256, 1, 2, 1, 32, 1, 64, 1, 128),
    (256, 2, 12, 2, 16, 64, 400, 7, 512),
    (64, 4, 8, 40, 32, 45, 90, 1, 128),       # hundreds of rows
    (64, 4, 8, 40, 8, 640, 900, 5, 1024),
    (128, 4, 8, 40, 8, 97, 900, 5, 1024),
    (128, 16, 8, 40, 5, 50, 90, 9, 128),
    (192, 4, 8, 40, 8, 97, 900, 5, 1024),
    (256, 4, 8, 40, 8, 640, 900, 5, 1024),
    (256, 16, 8, 40, 5, 50, 90, 9, 128),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(WINDOWS)))
def test_attention_window_over_positions_never_written(case, dtype):
    """Only the positions that the tokens see are in the cache; in front of them lie NaN, or large finite scales."""
    d, n_kv, G, n, B, window, L0, step, max_pos = WINDOWS[case]
    gen = torch.Generator().manual_seed(case)
    ls = [L0 + step * i for i in range(B)]
    kept = [min(L, n + window - 1) for L in ls]  # what the sequence's first token sees, and its tokens
    ks, vs = ([torch.randn((m, n_kv, d), generator=gen) for m in kept] for _ in range(2))
    q = torch.randn((n * B, n_kv * G, d), generator=gen).to(dtype)
    # (the same distances: the positions in front are left out of the reference)
    ref, amount, shift = attend(q.double(), ks, vs, [n] * B, kept, G, window, d ** -0.5, dtype)
    tol = attention_tolerance(ref, amount, shift, dtype)
    new, kl, T = batch(kept, ls)
    qs = batch([n] * B, ls)[0]
    k, v = torch.cat(ks).cuda(), torch.cat(vs).cuda()
    for byte in (0xFF, 0x7F, 0x60):  # NaN, 3e38, 6e19
        cache = fill(moe.kv4_cache(B, n_kv, d, max_pos), byte)
        moe.moe_kv4_append(k, v, cache, kl, q_start=new)
        out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=n, window=window)
        moe.moe_sync_check()
        err = (out.cpu().double() - ref).abs()
        assert (err <= tol).all(), (byte, float((err / tol).max()))
        assert relative_rms(out, ref) <= RMS[dtype], (byte, relative_rms(out, ref))


# ------------------------------------------------------------------------------------ scores of any size (GPU) ---
FAR = [  # (d, n_kv, group, tokens, lengths, max_pos)
    (64, 1, 4, [1, 1], [70, 1], 96),                  # a tile of up to 8 rows
    (128, 2, 8, [1, 1, 1], [900, 33, 500], 1024),     # (positions split)
    (128, 1, 12, [3, 1], [70, 40], 96),
    (256, 1, 3, [9, 4], [600, 4], 640),
    (64, 16, 8, [33, 20, 17, 1], [33, 40, 100, 1], 128),
    (128, 16, 4, [40, 33, 70], [40, 100, 200], 224),  # hundreds of rows
    (128, 8, 4, [40, 33], [1500, 700], 2048),
    (256, 8, 4, [70, 33], [1057, 1056], 1088),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q_exp,k_exp,scale", [
    (100, -60, 2.0 ** 32), (100, 40, 2.0 ** 32), (100, -60, 2.0 ** 18), (100, 40, -(2.0 ** -40)),
    (14, 14, 0.125), (12, 10, 0.125), (40, 20, 1.0), (-60, 40, 2.0 ** 32)])
@pytest.mark.parametrize("case", range(len(FAR)))
def test_attention_of_far_scores(case, q_exp, k_exp, scale, dtype):
    """Queries, keys and scales up to their limits: each token takes the value at its largest score."""
    d, n_kv, G, ns, ls, max_pos = FAR[case]
    gen = torch.Generator().manual_seed(case)
    ks = [torch.randn((L, n_kv, d), generator=gen) * 2.0 ** (k_exp - 2 if k_exp > 0 else k_exp) for L in ls]
    vs = [torch.randn((L, n_kv, d), generator=gen) for L in ls]
    cache = fill(moe.kv4_cache(len(ls), n_kv, d, max_pos))
    put(ks, vs, cache, F32)
    q = torch.randn((sum(ns), n_kv * G, d), generator=gen)
    q = (q / q.abs().amax(-1, keepdim=True) * 2.0 ** q_exp).to(dtype)
    scale = float(np.float32(scale))
    ref = torch.zeros((sum(ns), n_kv * G, d), dtype=torch.float64)
    most = torch.zeros_like(ref)
    clear = torch.ones((sum(ns), n_kv * G, 1), dtype=torch.bool)  # the largest score is one by more than its rounding
    t0 = 0
    for n, L, k, v in zip(ns, ls, ks, vs):
        at = torch.arange(L - n, L).view(-1, 1, 1)
        see = torch.arange(L) <= at
        for h in range(n_kv):
            cols = slice(h * G, (h + 1) * G)
            x, K = q[t0:t0 + n, cols].double(), held(k[:, h])
            z = torch.where(see, x @ K.T * scale, torch.tensor(-math.inf, dtype=torch.float64))
            top = z.topk(min(2, L), -1).values
            # what fp32 scores, from queries within 2^-22 and keys within 2^-11 in calls of many bf16 rows, can be off by
            err = (x.abs() @ K.abs().T * abs(scale)).amax(-1, keepdim=True) * (2.0 ** -17 if dtype is F32 else 2.0 ** -10)
            if L > 1:
                clear[t0:t0 + n, cols] = (top[..., :1] - top[..., 1:] > err + 40) | (top[..., 1:] == -math.inf)
            best = z.argmax(-1)
            ref[t0:t0 + n, cols], most[t0:t0 + n, cols] = held(v[:, h])[best], magnitude(v[:, h])[best]
        t0 += n
    assert clear.double().mean() > 0.5 or q_exp + k_exp < 24
    qs, kl, _ = batch(ns, ls)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns), scale=scale)
    moe.moe_sync_check()
    out = out.cpu().double()
    assert torch.isfinite(out).all()
    # (the probability is one, all others below 2^-40: one value in two fp16 terms, or three fp16 roundings)
    tol = most * (2.0 ** -20 if dtype is F32 else 3 * 2.0 ** -11) + ref.abs() * torch.finfo(dtype).eps / 2
    assert ((out - ref).abs() <= tol)[clear.expand_as(ref)].all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(FAR)))
def test_attention_far_scores_leave_other_rows_alone(case, dtype):
    """Every third head's queries are 2^40 times the others', which keep their precision; and scores that become far
    only late in the cache."""
    d, n_kv, G, ns, ls, max_pos = FAR[case]
    gen = torch.Generator().manual_seed(100 + case)
    ks = [torch.randn((L, n_kv, d), generator=gen) for L in ls]
    vs = [torch.randn((L, n_kv, d), generator=gen) for L in ls]
    cache = fill(moe.kv4_cache(len(ls), n_kv, d, max_pos))
    put(ks, vs, cache, F32)
    q = torch.randn((sum(ns), n_kv * G, d), generator=gen)
    far = torch.arange(n_kv * G) % 3 == 1
    q[:, far] *= 2.0 ** 40
    q = q.to(dtype)
    near = q.clone()
    near[:, far] = 0
    ref, amount, shift = attend(near.double(), ks, vs, ns, ls, G, 0, d ** -0.5, dtype)
    tol = attention_tolerance(ref, amount, shift, dtype)
    qs, kl, _ = batch(ns, ls)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns)).cpu().double()
    assert torch.isfinite(out).all()
    assert ((out - ref).abs() <= tol)[:, ~far].all()
    assert relative_rms(out[:, ~far], ref[:, ~far]) <= RMS[dtype]
    # the last position's key 2^26 times the others' along every query, its value the only one that counts where
    # its score is the largest
    for k in ks:
        k[-1] *= 2.0 ** 26
    put(ks, vs, cache, F32)
    q = torch.randn((sum(ns), n_kv * G, d), generator=gen).to(dtype)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns)).cpu().double()
    assert torch.isfinite(out).all()
    t0 = 0
    for n, L, k, v in zip(ns, ls, ks, vs):
        for h in range(n_kv):
            x = q[t0 + n - 1, h * G:(h + 1) * G].double()
            z = x @ held(k[-1:, h])[0] * d ** -0.5
            o, V, m = out[t0 + n - 1, h * G:(h + 1) * G], held(v[-1:, h]), magnitude(v[-1:, h])
            tol = m * (2.0 ** -20 if dtype is F32 else 3 * 2.0 ** -11) + V.abs() * torch.finfo(dtype).eps / 2
            assert ((o - V).abs() <= tol)[z > 2.0 ** 16].all()
        t0 += n
    moe.moe_sync_check()


def test_cache_whose_size_has_no_number():
    """A cache of more bytes than 64 bits count (or any device holds) is refused, not checked against what is left."""
    shape = (65535, 65535, 256, 1 << 26)  # 8.3e19 bytes
    assert moe.moe_kv4_cache_bytes(*shape) == 0
    with pytest.raises(moe.MoeError):
        moe.kv4_cache(*shape, device="cpu")
    n_seq, n_kv, d, max_pos = shape
    left = n_seq * n_kv * (max_pos // 32) * 36 * d % (1 << 64)
    refused("moe_kv4_append", OK_PTR, OK_PTR, 0, n_kv * d, n_kv * d, 1, n_seq, n_kv, d, max_pos, OK_PTR, 1, OK_PTR, OK_PTR,
            left, None)
    refused("moe_kv4_read", OK_PTR, left, 1, n_seq, n_kv, d, max_pos, OK_PTR, 1, OK_PTR, OK_PTR, OK_PTR, 0, n_kv * d,
            n_kv * d, None)
    assert moe.moe_kv4_attention_workspace_bytes(1, n_seq, n_kv, n_kv, d, 1, max_pos) == 0
    refused("moe_kv4_attention", OK_PTR, 0, n_kv * d, OK_PTR, left, 1, n_seq, n_kv, n_kv, d, max_pos, OK_PTR, 1, OK_PTR, 0,
            1.0, OK_PTR, n_kv * d, OK_PTR, left, None)
    assert moe.moe_kv4_cache_bytes(1024, 64, 256, 1 << 26) > 0


# ------------------------------------------------------------------------------- int4 products, more (GPU) ---
@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 3, 4, 16])
@pytest.mark.parametrize("N,K", [(40, 256), (33, 4224), (33000, 256)])
def test_matvec_norm_of_values_whose_squares_do_not_fit(T, N, K):
    """The norm of values up to the largest of fp32, and of values whose squares vanish."""
    gen = torch.Generator().manual_seed(T)
    raw, _ = int4_matrix(N, K, gen)
    parts = int4_parts(raw, N, K)
    x = torch.randn((T, K), generator=gen).clamp(-3, 3) / 3
    for size in (2.0 ** 64, 2.0 ** 100, 3.4e38, 2.0 ** -90):
        for token in range(T):
            y = x.clone()
            y[token] *= size
            out = moe.moe_matvec_int4(y.cuda(), raw.cuda(), N, rmsnorm=True).cpu().double()
            ref, tol = matvec_reference(y, parts, None, True)
            assert ((out - ref).abs() <= tol).all(), (size, token, float(((out - ref).abs() / tol).max()))


def test_matvec_refuses_what_is_added_half_over_the_output():
    """`add` is y itself or apart from it: one that overlaps it elsewhere would be read after it was written."""
    y = OK_PTR + (1 << 30)
    for add in (y + 4, y + 64 * 4, y + 2 * 64 * 4 - 4, y - 4, y - 64 * 4):
        refused("moe_matvec_int4", OK_PTR, OK_PTR + (1 << 20), 2, 64, 128, add, y, 0, None, 0, None)


def test_stack_attention_needs_an_entry_per_layer():
    """Lists shorter than the stack (the library would read past their arrays) are refused before anything is."""
    n_kv, d, H, max_pos = 2, 64, 256, 64
    router = [torch.zeros((8, H)) for _ in range(3)]
    whole = dict(w_qkv=[torch.zeros(1)] * 3, w_o=[torch.zeros(1)] * 3)
    caches = [moe.kv4_cache(1, n_kv, d, max_pos, device="cpu")] * 3
    shape = dict(n_heads=4, n_kv=n_kv, head_dim=d, max_pos=max_pos)
    for form in (dict(cache=caches, int4=True), dict(k_cache=caches, v_cache=caches)):
        for name in ("w_qkv", "w_o", *[nm for nm in form if nm != "int4"]):
            att = {**shape, **whole, **form}
            for entries in (att[name][:2], att[name] + att[name][:1], []):
                with pytest.raises(ValueError, match=f"{name} .* 3 layers"):
                    moe.MoeStack(None, H, 128, 8, 2, moe.MOE_BF16, moe.MOE_BF16, router, attention={**att, name: entries})


def test_stack_refuses_int4_attention_buffers_out_of_alignment():
    """As moe_attention_decode_int4 does: its kernels load 16 bytes at a time."""
    layers = 2
    pointers = lambda off: (C.c_void_p * layers)(OK_PTR, OK_PTR + off)
    cast = lambda a: C.cast(a, C.POINTER(C.c_void_p))
    router = pointers(0)
    for bad in range(3):
        for off in (8, 2):
            arrays = [pointers(off if i == bad else 0) for i in range(3)]
            att = binding.AttentionDesc(4, 2, 64, 64, 1.0e4, 0, cast(arrays[0]), cast(arrays[1]), cast(arrays[2]), None, 1)
            desc = binding.StackDesc(layers, 256, 128, 8, 2, moe.MOE_BF16, moe.MOE_BF16, cast(router), None, None, 1, 0, 0, 0, 0,
                                     C.pointer(att), 0)
            out = C.c_void_p()
            assert moe.lib().moe_stack_create(C.byref(desc), C.byref(out)) == -1 and not out.value
            assert b"aligned" in moe.lib().moe_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(8, 2432), (5, 4096), (8, 4096), (16, 2048)])
@pytest.mark.parametrize("N", [131100, 65600])
def test_matvec_many_rows_of_tokens_that_fill_the_lds(T, K, N):
    """Tokens whose terms leave a unit room for one block, which then takes several tiles of rows at a time."""
    gen = torch.Generator().manual_seed(K + T)
    on = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.randint(0, 256, (N * K // 2,), generator=on, device="cuda", dtype=torch.uint8)
    scales = (torch.rand((N * (K // 128),), generator=on, device="cuda") * 0.01 + 0.001).to(BF16)
    x, add = torch.randn((T, K), generator=gen), torch.randn((T, N), generator=gen)
    y = torch.full((T * N + 64,), 9.0, device="cuda")
    moe.moe_matvec_int4(x.cuda(), torch.cat([codes, scales.view(torch.uint8)]), N, y=y[:T * N].view(T, N), add=add.cuda(), rmsnorm=True)
    rows = torch.cat([torch.arange(0, 130), torch.randint(0, N, (300,), generator=gen), torch.arange(N - 130, N)])
    raw = torch.cat([codes.view(N, -1)[rows.cuda()].flatten(), scales.view(N, -1)[rows.cuda()].flatten().view(torch.uint8)]).cpu()
    ref, tol = matvec_reference(x, int4_parts(raw, len(rows), K), add[:, rows], True)
    out = y[:T * N].view(T, N).cpu()
    err = (out[:, rows].double() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())
    assert torch.isfinite(out).all() and (y[T * N:] == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_keeps_its_precision(case, dtype):
    """The stated roundings over all of a case's outputs together: one left out of fp32's two terms (2^-11) or twice
    bf16's would show, where a bound for the worst element leaves room."""
    _, _, _, ns, ls, _, window = CASES[case]
    cache, q, ref, _ = attention_case(*CASES[case], dtype, seed=1000 + case)
    qs, kl, _ = batch(ns, ls)
    out = moe.moe_kv4_attention(q.cuda(), cache, kl, q_start=qs, max_q=max(ns), window=window)
    moe.moe_sync_check()
    if ref.abs().amax() == 0:
        assert (out == 0).all()
    else:
        assert relative_rms(out, ref) <= RMS[dtype], relative_rms(out, ref)


def test_the_precision_bound_sees_a_dropped_term():
    """Outputs whose probabilities are rounded once to fp16 are far past fp32's bound (and within bf16's)."""
    gen = torch.Generator().manual_seed(0)
    p = torch.softmax(torch.randn((64, 300), generator=gen, dtype=torch.float64), -1)
    v = torch.randn((300, 128), generator=gen, dtype=torch.float64)
    ref = p @ v
    top = p.amax(-1, keepdim=True)
    assert relative_rms((p / top).half().double() * top @ v, ref) > 20 * RMS[F32]
    assert relative_rms((p / top).half().double() * top @ v, ref) < RMS[BF16]


def test_binding_refuses_numbers_that_do_not_fit_the_library():
    """A window or max_q past 32 bits is refused, not cut to its low bits."""
    cache = moe.kv4_cache(1, 2, 64, 32, device="cpu")
    q, kl, qs = torch.zeros((1, 2, 64)), torch.ones(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for window in ((1 << 32) + 5, 1 << 32, -(1 << 32), (1 << 30) + 1, -1):
        with pytest.raises(ValueError, match="window"):
            moe.moe_kv4_attention(q, cache, kl, window=window)
    for max_q in ((1 << 32) + 1, 1 << 31, 0, -1):
        for call in (lambda: moe.moe_kv4_attention(q, cache, kl, q_start=qs, max_q=max_q),
                     lambda: moe.moe_kv4_append(q, q, cache, kl, q_start=qs, max_q=max_q),
                     lambda: moe.moe_kv4_read(cache, kl, 1, q_start=qs, max_q=max_q)):
            with pytest.raises(ValueError, match="max_q"):
                call()
    for shape in ((1 << 32, 2, 64, 32), ((1 << 32) + 1, 2, 64, 32), (1, 2, (1 << 32) + 64, 32), (1, 2, 64, (1 << 32) + 32)):
        with pytest.raises(moe.MoeError):
            moe.kv4_cache(*shape, device="meta")


@pytest.mark.gpu
def test_binding_no_tokens_is_a_no_op():
    cache, kl = moe.kv4_cache(2, 2, 64, 32), torch.zeros(2, dtype=torch.int32, device="cuda")
    none, qs = torch.zeros((0, 2, 64), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    before = cache.clone()
    for max_q in (None, 0, 7):
        moe.moe_kv4_append(none, none, cache, kl, q_start=qs, max_q=max_q)
        assert moe.moe_kv4_attention(none, cache, kl, q_start=qs, max_q=max_q).shape == (0, 2, 64)
        assert moe.moe_kv4_read(cache, kl, 0, q_start=qs, max_q=max_q)[0].shape == (0, 2, 64)
    moe.moe_sync_check()
    assert torch.equal(cache, before)


def test_block_refuses_rows_longer_than_its_products_take():
    """The block's projections have the limits of moe_matvec_int4: at most 2^24 columns."""
    assert moe.moe_attention_decode_int4_workspace_bytes(1, 1 << 24, 4, 2, 64, 64) > 0
    assert moe.moe_attention_decode_int4_workspace_bytes(1, (1 << 24) + 128, 4, 2, 64, 64) == 0
    refused("moe_attention_decode_int4", OK_PTR, 1, 1 << 25, 4, 2, 64, OK_PTR, OK_PTR, OK_PTR, 1 << 40, 64, OK_PTR, 1.0e4,
            OK_PTR, 1 << 40, None)
