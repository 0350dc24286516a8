"""Differential attention: against its formula in 64 bits on every kernel that serves it, and what the call refuses."""
import ctypes
import math

import pytest
import torch

from paper_2605_26636_b200 import build as jv_build
from paper_2605_26636_b200 import jetvit as jv
from tests._util import guarded_empty

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def _tensors(B, H, Hkv, Nq, Nk, D=64, dtype=torch.bfloat16, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed + 7 * Nq + Nk)
    r = lambda *s: torch.randn(*s, generator=g)
    return (r(B, H, Nq, D).to(dtype).to(device), r(B, Hkv, Nk, D).to(dtype).to(device), r(B, Hkv, Nk, D).to(dtype).to(device),
            (0.1 * r(4, D)).to(device), (1 + 0.2 * r(2 * D)).to(device))


def _reference(q, k, v, lam4, init, w, eps, causal, kv_len, q_pos, scale):
    """o in 64 bits, and a bound of the error that the arithmetic may add to the rounding of o.

    A probability is off by at most E of itself (bf16 tensors: its rounding, 2^-8, and 2^-12 for exponentials, scores and
    sums in 32 bits; f32: the scores' 2 D roundings and the sums' Nk), so a map's product by E a, a = P |v|; both maps and lambda:
    dx = E (a0 + |lambda| a1).  The norm turns dx into r (dx + |x| r^2 mean(|x| dx)) to first order; dx is taken a tenth larger
    for the second."""
    B, H, Nq, D = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    f = H // Hkv
    rep = lambda t: t.reshape(B, Hkv // 2, 2, Nk, D).repeat_interleave(f, 1)
    qd, kd, vd = q.double().reshape(B, H // 2, 2, Nq, D), rep(k.double()), rep(v.double())
    len_ = torch.full((B,), Nk, device=q.device) if kv_len is None else kv_len.clamp(0, Nk)
    pos = torch.full((B,), Nk - Nq, device=q.device) if q_pos is None else q_pos
    j, i = torch.arange(Nk, device=q.device), torch.arange(Nq, device=q.device)
    seen = (j < len_[:, None])[:, None, :].expand(B, Nq, Nk)
    if causal:
        seen = seen & (j <= (i[None] + pos[:, None])[..., None])
    seen = seen[:, None, None]
    kd, vd = (torch.where((j < len_[:, None])[:, None, None, :, None], t, 0.0) for t in (kd, vd))
    vv = vd.transpose(2, 3).reshape(B, H // 2, 1, Nk, 2 * D)
    scale = scale if scale > 0 else D ** -0.5
    s = torch.where(seen, qd @ kd.transpose(3, 4) * scale, -math.inf)
    empty = ~seen.any(-1, keepdim=True)
    p = torch.where(empty, 0.0, torch.softmax(s, -1))
    l4 = lam4.double()
    lam = (l4[0] @ l4[1]).exp() - (l4[2] @ l4[3]).exp() + init
    x2, a = p @ vv, p @ vv.abs()
    x = x2[:, :, 0] - lam * x2[:, :, 1]
    big = float((qd.abs() @ kd.abs().transpose(3, 4)).max()) * scale
    E = 2.0 ** -8 + 2.0 ** -12 if q.dtype == torch.bfloat16 else (2 * D * big + 2 * Nk + 32) * U
    dx = 1.1 * E * (a[:, :, 0] + lam.abs() * a[:, :, 1])
    if w is not None:
        r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
        c = abs(1 - init) * w.double().abs()
        dx = c * r * (dx + x.abs() * r * r * (x.abs() * dx).mean(-1, keepdim=True)) + 16 * U * c * r * x.abs()
        x = (1 - init) * w.double() * x * r
    back = lambda t: t.reshape(B, H // 2, Nq, 2, D).transpose(2, 3).reshape(B, H, Nq, D)
    return back(x), back(dx)


def _check(q, k, v, lam4, w, init=0.8, eps=1e-5, causal=False, kv_len=None, q_pos=None, scale=0.0, rms=True):
    out, guard = guarded_empty(q.shape, q.dtype, q.device)
    out.fill_(math.nan)
    o = jv.diff_attn(q, k, v, lam4, init, norm_weight=w, norm_eps=eps, causal=causal, kv_len=kv_len, q_pos=q_pos, scale=scale, out=out)
    guard()
    assert jv.device_status() == jv.JV_OK
    ref, bound = _reference(q, k, v, lam4, init, w, eps, causal, kv_len, q_pos, scale)
    d = (o.double() - ref).abs()
    assert torch.isfinite(o).all()
    assert (d <= HALF[q.dtype] * (ref.abs() + bound) + bound + 1e-30).all(), float((d - HALF[q.dtype] * ref.abs() - bound).max())
    if rms and q.dtype == torch.bfloat16 and ref.numel() >= 4096:
        # independent roundings of P and of o: 2^-8 / sqrt(3) of the values each, 3.2e-3 together, a quarter more for the sample
        assert d.square().mean().sqrt() <= 4e-3 * ref.square().mean().sqrt()
    return o


# one key and one query; fewer and more keys than a tile; odd everything; single tokens and a few against long caches; many queries
SIZES = [(1, 1), (1, 5), (1, 128), (1, 129), (1, 1370), (3, 700), (16, 2049), (33, 64), (64, 1000), (100, 100), (128, 128),
         (129, 129), (257, 511), (300, 40), (640, 640)]


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(2, 2), (8, 8), (8, 4), (12, 2)])
@pytest.mark.parametrize("Nq,Nk", SIZES)
def test_sizes_and_shared_heads(Nq, Nk, heads):
    for B in (1, 3):
        q, k, v, lam, w = _tensors(B, *heads, Nq, Nk)
        _check(q, k, v, lam, w)
        _check(q, k, v, lam, None, init=0.3)
        _check(q, k, v, lam, w, causal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.float32, 20), (torch.bfloat16, 32), (torch.bfloat16, 8)])
@pytest.mark.parametrize("Nq,Nk", [(1, 1), (1, 333), (70, 70), (65, 200), (40, 17)])
def test_other_types_and_widths(Nq, Nk, dtype, D):
    q, k, v, lam, w = _tensors(2, 8, 4, Nq, Nk, D, dtype)
    lens = torch.tensor([Nk, Nk // 2], dtype=torch.int32, device="cuda")
    for causal in (False, True):
        _check(q, k, v, lam, w, causal=causal)
        _check(q, k, v, lam, None, causal=causal, kv_len=lens)


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk", [(1, 700), (7, 300), (200, 700), (384, 384)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_positions_and_garbage_behind_them(Nq, Nk, causal):
    """Ragged sequences, none at all among them; rows that see nothing are zeros; what lies behind a length may be anything."""
    q, k, v, lam, w = _tensors(7, 4, 2, Nq, Nk)
    lens = torch.tensor([Nk, Nk - 1, 1, 0, 129, -5, Nk + 9], dtype=torch.int32, device="cuda")
    pos = torch.tensor([Nk - Nq, 3, 0, 0, -Nq // 2, 5, 1 << 30], dtype=torch.int32, device="cuda")
    for t in (k, v):
        for b in range(7):
            n = min(max(int(lens[b]), 0), Nk)
            t[b, :, n:] = (math.nan, math.inf, -math.inf)[b % 3]
    o = _check(q, k, v, lam, w, causal=causal, kv_len=lens, q_pos=pos, rms=False)
    assert (o[3] == 0).all() and (o[5] == 0).all()
    if causal and Nq > 1:
        assert (o[4, :, :Nq // 2] == 0).all() and (o[4, :, (Nq + 1) // 2 + 1:] != 0).any()


@pytest.mark.gpu
@pytest.mark.parametrize("H,Nq,Nk,dtype,D", [(4, 1, 700, torch.bfloat16, 64), (4, 9, 700, torch.bfloat16, 64), (4, 200, 2000, torch.bfloat16, 64),
                                             (300, 128, 128, torch.bfloat16, 64), (4, 40, 90, torch.float32, 64), (4, 40, 90, torch.bfloat16, 32)])
def test_rows_without_keys_are_zeros_whatever_the_norm_makes_of_them(H, Nq, Nk, dtype, D):
    """A norm without eps, and with a weight of infinity: 0 times infinity in rows that see no key.  Few queries, tiles in parts and whole,
    fp32 arithmetic."""
    q, k, v, lam, w = _tensors(2, H, H, Nq, Nk, D, dtype)
    lens = torch.tensor([0, Nk], dtype=torch.int32, device="cuda")
    pos = torch.tensor([-Nq // 2, -Nq], dtype=torch.int32, device="cuda")
    some = (Nq + 1) // 2                                      # rows of the first sequence ahead of its first key
    for top in (1.0, math.inf):
        w[3] = top
        call = lambda **kw: jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w, norm_eps=0.0, **kw)
        o = call(kv_len=lens)
        assert (o[0] == 0).all() and torch.isfinite(o[1, 1::2]).all() and (o[1] != 0).any()
        o = call(causal=True, q_pos=pos)
        assert (o[1] == 0).all() and (o[0, :, :some] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk,dtype", [(1, 700, torch.bfloat16), (200, 700, torch.bfloat16), (5, 90, torch.float32)])
def test_positions_at_the_ends_of_their_type(Nq, Nk, dtype):
    q, k, v, lam, w = _tensors(5, 4, 2, Nq, Nk, dtype=dtype)
    pos = torch.tensor([-1 << 31, (1 << 31) - 1, (-1 << 31) + 70, -Nq, (1 << 31) - Nq], dtype=torch.int32, device="cuda")
    o = _check(q, k, v, lam, w, causal=True, q_pos=pos, rms=False)
    assert (o[0] == 0).all() and (o[2] == 0).all() and (o[3] == 0).all() and (o[1] != 0).any()


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk", [(1, 2000), (256, 500)])
def test_results_on_another_stream_do_not_lie_where_earlier_work_still_writes(Nq, Nk):
    q, k, v, lam, w = _tensors(2, 8, 4, Nq, Nk)
    want = jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w)
    shape = _shape(2, 8, 4, Nq, Nk)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    late = [torch.empty_like(q), torch.empty(jv.lib().jv_diff_attn_workspace_bytes(ctypes.byref(shape)), dtype=torch.uint8, device="cuda")]
    torch.cuda._sleep(1 << 26)
    for t in late:
        t.fill_(7)
    del late, t
    got = jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk", [(1, 900), (260, 260)])
def test_layouts(Nq, Nk):
    q, k, v, lam, w = _tensors(2, 4, 4, Nq, Nk)
    want = jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w)
    rows = lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)             # [B, N, H, D]
    assert torch.equal(jv.diff_attn(rows(q), rows(k), rows(v), lam, 0.8, norm_weight=w), want)
    kv = torch.stack((k, v)).permute(1, 3, 0, 2, 4).contiguous()                          # [B, N, 2, H, D]
    ks, vs = (kv[:, :, i].permute(0, 2, 1, 3) for i in (0, 1))
    assert torch.equal(jv.diff_attn(rows(q), ks, vs, lam, 0.8, norm_weight=w), want)
    cache = torch.full((2, 2, 4, Nk + 100, 64), math.nan, dtype=k.dtype, device="cuda")   # a longer cache, used up to Nk
    cache[0, :, :, :Nk], cache[1, :, :, :Nk] = k, v
    assert torch.equal(jv.diff_attn(q, cache[0, :, :, :Nk], cache[1, :, :, :Nk], lam, 0.8, norm_weight=w), want)
    lens = torch.full((2,), Nk, dtype=torch.int32, device="cuda")
    got = jv.diff_attn(q, cache[0], cache[1], lam, 0.8, norm_weight=w, kv_len=lens)
    d = (got.double() - want.double()).abs()
    assert (d <= 2 * 2.0 ** -8 * want.double().abs() + 2e-2).all()      # another cut of the keys: other roundings


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk", [(1, 1000), (20, 300), (256, 384)])
def test_scores_far_apart_and_no_numbers(Nq, Nk):
    q, k, v, lam, w = _tensors(1, 4, 4, Nq, Nk, seed=5)
    _check(16 * q, k, v, lam, w, rms=False)               # near one-hot maps
    _check(q, k, v, lam, None, scale=3.0, rms=False)
    base = jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w)
    bad = q.clone()
    bad[0, 1, 0] = math.nan                                # map 1 of pair 0, one row
    o = jv.diff_attn(bad, k, v, lam, 0.8, norm_weight=w)
    assert torch.isnan(o[0, :2, 0]).all() and torch.equal(o[0, 2:], base[0, 2:]) and torch.equal(o[0, :2, 1:], base[0, :2, 1:])
    # a key that scores -inf for every query weighs nothing wherever it lies: as if it were not there
    for at in (0, 63, Nk - 1):
        qq, kk = q.abs() + 0.1, k.clone()
        kk[0, :, at] = -math.inf
        o = jv.diff_attn(qq, kk, v, lam, 0.8, norm_weight=None)
        keep = [j for j in range(Nk) if j != at]
        ref, bound = _reference(qq, kk[:, :, keep], v[:, :, keep], lam, 0.8, None, 1e-5, False, None, None, 0.0)
        assert ((o.double() - ref).abs() <= HALF[q.dtype] * (ref.abs() + bound) + bound).all()
        kk[0, :, at] = math.inf
        assert torch.isnan(jv.diff_attn(qq, kk, v, lam, 0.8, norm_weight=None)).all()
    kk = torch.full_like(k, -math.inf)
    assert torch.isnan(jv.diff_attn(q.abs() + 0.1, kk, v, lam, 0.8)).all()
    _check(q, torch.zeros_like(k), v, lam, w, rms=False)  # all keys alike


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,Nk", [(1, 3000), (130, 1000)])
def test_streams_capture_and_repeats(Nq, Nk):
    q, k, v, lam, w = _tensors(2, 8, 4, Nq, Nk, seed=9)
    lens = torch.tensor([Nk, Nk // 3], dtype=torch.int32, device="cuda")
    call = lambda **kw: jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w, causal=Nq > 1, kv_len=lens, **kw)
    want = call()
    for _ in range(20):
        assert torch.equal(call(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [call(stream=side) for _ in range(3)] + [call()]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out)
    lens.copy_(torch.tensor([Nk // 2, Nk], dtype=torch.int32))           # lengths are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, call()) and not torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(10))
def test_equal_shares_of_unequal_sequences(seed):
    """Blocks take equal shares of all sequences' keys, cut wherever they come: many and few sequences, more of them than a block has
    threads, lengths from none to all, several pairs, prompts and single tokens."""
    g = torch.Generator().manual_seed(seed)
    pick = lambda *a: a[int(torch.randint(len(a), (1,), generator=g))]
    Nq, Hkv = pick(1, 1, 3, 150, 300), pick(2, 2, 4, 6)
    H = Hkv * pick(1, 2)
    B, Nk = ((pick(700, 900), 200) if seed < 2 else (pick(5, 11, 37), pick(130, 900, 1500)))
    Nq = 1 if seed < 2 else Nq
    q, k, v, lam, w = _tensors(B, H, Hkv, Nq, Nk, seed=seed)
    lens = (torch.rand(B, generator=g) ** 2 * (Nk + 1)).int().cuda()
    pos = (lens - torch.randint(0, Nq + 40, (B,), generator=g).cuda()).int()
    _check(q, k, v, lam, w, kv_len=lens, rms=False)
    _check(q, k, v, lam, None, causal=True, kv_len=lens, q_pos=pos, rms=False)


@pytest.mark.gpu
@pytest.mark.parametrize("H,Nq,Nk", [(64, 256, 384), (2, 140, 3000), (2, 1, 3000), (300, 128, 256)])
def test_scores_that_outgrow_the_first_keys(H, Nq, Nk):
    """Scores far above, or below, those of the first 64 keys, and values too large to be squared: rows that are done again, of items that
    one block has whole (many pairs) and of items in parts (few)."""
    q, k, v, lam, w = _tensors(1, H, H, Nq, Nk, seed=3)
    up = torch.ones(Nk)
    up[:64] = 0.02
    up[200:] = 8.0
    kk = (k.float() * up[:, None].cuda()).to(k.dtype)
    _check(8 * q, kk, v, lam, None, rms=False)                                   # maxima grow by some hundred
    _check(8 * q, kk, v, lam, w, causal=Nq > 1, rms=False)
    _check(8 * q, kk.flip(2), v, lam, w, rms=False)                              # and fall
    some = q.clone()
    some[:, :, ::3] *= 8                                                       # every third row only
    _check(some, kk, v, lam, None, rms=False)
    few = k.abs() * 2.0
    few[:, :, :64] = -few[:, :, :64]
    _check(4 * q.abs(), few, v, lam, None, rms=False)                            # first keys far below every other
    first = few.clone()
    first[:, :, :64] = -math.inf                                                # and such as weigh nothing
    out = jv.diff_attn(4 * q.abs() + 1, first, v, lam, 0.8)
    ref, bound = _reference(4 * q.abs() + 1, few[:, :, 64:], v[:, :, 64:], lam, 0.8, None, 1e-5, False, None, None, 0.0)
    assert ((out.double() - ref).abs() <= HALF[q.dtype] * (ref.abs() + bound) + bound).all()
    big = (v.float() * 1e22).to(v.dtype)                                       # (without a norm: its squares leave fp32)
    o = jv.diff_attn(q, k, big, lam, 0.8)
    ref, bound = _reference(q, k, big, lam, 0.8, None, 1e-5, False, None, None, 0.0)
    assert ((o.double() - ref).abs() <= HALF[q.dtype] * (ref.abs() + bound) + bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("size,eps", [(1e22, 1e-5), (1e25, 0.0), (1e-25, 0.0), (1e-18, 1e-38)])
@pytest.mark.parametrize("H,Nq,Nk,dtype,D", [(4, 1, 700, torch.bfloat16, 64), (2, 1, 70, torch.bfloat16, 64), (4, 200, 2000, torch.bfloat16, 64),
                                             (300, 128, 128, torch.bfloat16, 64), (4, 40, 90, torch.float32, 64), (4, 40, 90, torch.bfloat16, 32)])
def test_norms_of_rows_whose_squares_leave_fp32(H, Nq, Nk, dtype, D, size, eps):
    q, k, v, lam, w = _tensors(2, H, H, Nq, Nk, D, dtype)
    _check(q, k, (v.float() * size).to(dtype), lam, w, eps=eps, rms=False)


def _cancelling(H, Nq, Nk, which, half, device):
    """Inputs whose result hangs on the last bits of the probabilities of map ``which``: scores that are exact in 32 bits (one product of
    powers of 2 and values of 6 bits), values of neighbouring keys that cancel but for a difference of their scores of 1/32.  Keys of
    the other map weigh alike, so that its result is nothing.  half: only the first 32 of every 64 keys weigh anything."""
    g = torch.Generator().manual_seed(Nk + Nq)
    q, k = torch.zeros(1, H // 2, 2, Nq, 64), torch.zeros(1, H // 2, 2, Nk, 64)
    q[:, :, which, :, 0] = 2.0 ** -torch.randint(0, 3, (1, H // 2, Nq), generator=g).float()
    k0 = torch.randint(-32, 32, (1, H // 2, Nk // 2), generator=g) / 32
    k[:, :, which, :, 0] = torch.stack((k0, k0 + torch.randint(0, 2, k0.shape, generator=g) / 16 - 1 / 32), -1).flatten(2)
    q[..., 1] = 1.0
    if half:
        k[..., torch.arange(Nk) % 64 >= 32, 1] = -200.0           # exp(-200): nothing in 32 bits
    v0 = torch.randn(1, H, Nk // 2, 64, generator=g).to(torch.bfloat16)
    v = torch.stack((v0, -v0), 3).flatten(2, 3)
    return [t.reshape(1, H, -1, 64).to(torch.bfloat16).to(device) for t in (q, k, v)]


def _cancelling_reference(q, k, v):
    """The result for lambda = 1 (x = P0 v - P1 v) in 64 bits, and what the arithmetic may add to its rounding: a probability's two
    terms 2^-16 of it; its exponential and argument (4 at most) 2^-22 and 8 U, the sum of 256 of them 256 U, its products' 32 U and
    partial sums: below 2^-14 together."""
    o, bound = _reference(q, k, v, torch.zeros(4, 64, device=q.device), 1.0, None, 0.0, False, None, None, 1.0)
    single = 1.1 * (2.0 ** -8 + 2.0 ** -12)                          # (what _reference grants a probability, of both maps)
    return o, bound / single * 2.0 ** -14


CANCELLING = [(2, 1, 256, 0, False), (2, 1, 256, 1, False), (4, 7, 200, 0, False), (4, 16, 130, 1, False), (12, 3, 64, 1, False),     # rows
              (2, 128, 256, 0, True), (4, 200, 128, 0, True), (300, 33, 64, 0, True)]                                                # tiles


@pytest.mark.gpu
@pytest.mark.parametrize("H,Nq,Nk,which,half", CANCELLING)
def test_second_terms_of_the_probabilities(H, Nq, Nk, which, half):
    """Few queries have them for all keys of both maps, tiles of queries for the first 32 of every 64 keys of map 0."""
    q, k, v = _cancelling(H, Nq, Nk, which, half, "cuda")
    ref, bound = _cancelling_reference(q, k, v)
    o = jv.diff_attn(q, k, v, torch.zeros(4, 64, device="cuda"), 1.0, scale=1.0)
    assert ((o.double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + bound) + bound).all()


@pytest.mark.parametrize("H,Nq,Nk,which,half", [c for c in CANCELLING if c[0] < 100])
def test_second_terms_decide_that_comparison(H, Nq, Nk, which, half):
    """Probabilities in 64 bits rounded as the kernels round them: with both terms within the bound; with one, or with the second at
    another key's values, a good part of the results is not."""
    q, k, v = _cancelling(H, Nq, Nk, which, half, "cpu")
    ref, bound = _cancelling_reference(q, k, v)
    s = q.double().reshape(1, H // 2, 2, Nq, 64) @ k.double().reshape(1, H // 2, 2, Nk, 64).transpose(3, 4)
    vv = v.double().reshape(1, H // 2, 2, Nk, 64).transpose(2, 3).reshape(1, H // 2, 1, Nk, 128)
    p = (s - s.amax(-1, keepdim=True)).exp()
    hi = p.to(torch.bfloat16).double()
    lo = (p - hi).to(torch.bfloat16).double()

    def share(x):
        x = x[:, :, 0] - x[:, :, 1]
        o = x.reshape(1, H // 2, Nq, 2, 64).transpose(2, 3).reshape(1, H, Nq, 64)
        o = o.to(torch.bfloat16).double()
        return float(((o - ref).abs() > 2.0 ** -8 * (ref.abs() + bound) + bound).double().mean())

    total = p.sum(-1, keepdim=True)
    assert share((hi @ vv + lo @ vv) / total) == 0
    assert share(hi @ vv / total) > 0.2
    assert share((hi @ vv + lo @ vv.roll(8, 3)) / total) > 0.2


@pytest.mark.gpu
@pytest.mark.parametrize("Nq", [1, 130])
def test_calls_while_the_status_word_is_set(Nq):
    q, k, v, lam, w = _tensors(3, 4, 4, Nq, 1700, seed=8)
    call = lambda out: jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w, out=out)
    good = call(torch.empty_like(q))
    assert jv.device_status() == jv.JV_OK
    jv.selftest_wait_timeout(1000)
    kept = call(torch.full_like(q, 1234.5))
    torch.cuda.synchronize()
    assert (kept == 1234.5).all()
    assert jv.device_status() == jv.JV_ERR_TIMEOUT and jv.device_status() == jv.JV_OK
    assert torch.equal(call(torch.empty_like(q)), good)


@pytest.mark.gpu
@pytest.mark.parametrize("Nq,dtype", [(1, torch.bfloat16), (140, torch.bfloat16), (3, torch.float32)])
def test_a_cache_whose_offsets_pass_32_bits(Nq, dtype):
    B, H, Nk, far = 3, 4, 333, (1 << 31) // 2 + 4096          # elements between batch elements: the third begins behind 2^31
    q, k, v, lam, w = _tensors(B, H, H, Nq, Nk, dtype=dtype, seed=4)
    pool = torch.empty(2 * far + 2 * H * Nk * 64, dtype=dtype, device="cuda")
    ks = pool.as_strided((B, H, Nk, 64), (far, Nk * 64, 64, 1))
    vs = pool.as_strided((B, H, Nk, 64), (far, Nk * 64, 64, 1), H * Nk * 64)
    ks.copy_(k)
    vs.copy_(v)
    assert torch.equal(jv.diff_attn(q, ks, vs, lam, 0.8, norm_weight=w), jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w))


@pytest.mark.gpu
def test_forced_generic_kernel():
    q, k, v, lam, w = _tensors(2, 4, 2, 70, 150)
    prev = jv.set_force_generic(True)
    try:
        _check(q, k, v, lam, w, causal=True)
    finally:
        jv.set_force_generic(prev)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
def test_between_norm_and_projections(causal):
    """norm -> QKV projection -> differential attention -> output projection, as a block runs them."""
    B, H, N, C = 2, 6, 333, 384
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g)
    x = r(B, N, C).to(torch.bfloat16).cuda()
    wq, wo = (r(3 * C, C) * C ** -0.5).to(torch.bfloat16).cuda(), (r(C, C) * C ** -0.5).to(torch.bfloat16).cuda()
    lam, w = (0.1 * r(4, 64)).cuda(), torch.ones(128, device="cuda")
    xn = jv.layer_norm(x)
    q, k, v = jv.qkv_proj(xn, wq, None, H, 1, N)
    o = jv.diff_attn(q, k, v, lam, 0.8, norm_weight=w, causal=causal)
    y = jv.out_proj(o, wo, None, 1, N)
    ref, bound = _reference(q, k, v, lam, 0.8, w, 1e-5, causal, None, None, 0.0)
    assert ((o.double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + bound) + bound).all()
    xd = x.double()
    want = ((xd - xd.mean(-1, keepdim=True)) * (xd.var(-1, unbiased=False, keepdim=True) + 1e-6).rsqrt())
    assert ((xn.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
    yr = o.double().permute(0, 2, 1, 3).reshape(B, N, C) @ wo.double().T
    mag = o.double().abs().permute(0, 2, 1, 3).reshape(B, N, C) @ wo.double().abs().T
    assert ((y.double() - yr).abs() <= 2.0 ** -8 * yr.abs() + C * U * mag).all()


# ---- refusals, on the host ------------------------------------------------------------------------------------------
Q, K, V, O, LAM, W, WS, LEN = (i << 26 for i in range(1, 9))


@pytest.fixture(scope="module")
def L():
    jv_build.build()
    return jv.lib()


def _shape(B=2, H=4, Hkv=2, Nq=8, Nk=16, D=64, dtype=jv.JV_BF16, causal=0, qs=(0, 0, 0), ks=(0, 0, 0)):
    return jv.JvDiffShape(B, H, Hkv, Nq, Nk, D, dtype, causal, qs, ks)


def _call(L, shp=None, q=Q, k=K, v=V, o=O, lam=LAM, init=0.8, w=W, eps=1e-5, kv_len=None, ws=WS, n=1 << 30, diff=True):
    shp = _shape() if shp is None else shp
    d = jv.JvDiff(lam, init, w, eps, kv_len, None)
    return L.jv_diff_attn(q, k, v, o, ctypes.byref(shp), ctypes.byref(d) if diff else None, 0.0, ws, n, None)


def test_refusals(L):
    bad = jv.JV_ERR_INVALID_ARG
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(diff=False), dict(lam=None), dict(init=math.nan), dict(eps=-1.0),
               dict(q=Q + 8), dict(lam=LAM + 2), dict(w=W + 4), dict(kv_len=LEN + 1), dict(o=Q), dict(o=V - 16), dict(o=W),
               dict(shp=_shape(B=0)), dict(shp=_shape(Nk=0)), dict(shp=_shape(Nq=0)), dict(shp=_shape(H=3, Hkv=3)), dict(shp=_shape(H=4, Hkv=1)),
               dict(shp=_shape(H=6, Hkv=4)), dict(shp=_shape(dtype=5)), dict(shp=_shape(causal=2)), dict(shp=_shape(qs=(64, 0, 0))),
               dict(shp=_shape(qs=(-64, 512, 2048))), dict(shp=_shape(ks=(68, 1088, 2176)))):
        assert _call(L, **kw) == bad, kw
    for shp in (_shape(D=128), _shape(D=12), _shape(Nk=(1 << 24) + 1), _shape(B=40000)):
        assert _call(L, shp=shp) == jv.JV_ERR_UNSUPPORTED
        assert L.jv_diff_attn_workspace_bytes(ctypes.byref(shp)) == 0
    need = L.jv_diff_attn_workspace_bytes(ctypes.byref(_shape()))
    if need:
        for kw in (dict(ws=None), dict(ws=WS + 16), dict(n=need - 1)):
            assert _call(L, **kw) == jv.JV_ERR_WORKSPACE, kw
        assert _call(L, ws=O) == bad and _call(L, ws=K) == bad
    if not torch.cuda.is_available():
        assert _call(L) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)
        assert _call(L, w=None, eps=-1.0, kv_len=LEN) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)


def test_work_that_a_block_cannot_count(L):
    n = 1 << 24
    for B, H, Nq, Nk, ok in ((1, 8, n, n, True), (1, 10, n, n, False), (1000, 64, n, n, False), (1000, 64, 1, n, True), (2, 64, n // 16, n, True)):
        shp = _shape(B=B, H=H, Hkv=2, Nq=Nq, Nk=Nk)
        assert (L.jv_diff_attn_workspace_bytes(ctypes.byref(shp)) > 0) == ok, (B, H, Nq, Nk)
        if not ok:
            assert _call(L, shp) == jv.JV_ERR_UNSUPPORTED


@pytest.mark.parametrize("Nq", [8, 9, 300])
def test_workspace_refusals(L, Nq):
    """Of the few queries' plan (16 rows on a pair of keys) and of the tiles'."""
    shp = _shape(Nq=Nq, Nk=640)
    need = L.jv_diff_attn_workspace_bytes(ctypes.byref(shp))
    assert need > 0
    for kw in (dict(ws=None), dict(ws=WS + 16), dict(n=need - 1), dict(n=0)):
        assert _call(L, shp, **kw) == jv.JV_ERR_WORKSPACE, kw
    for p in (Q, K, V, O, LAM, W):
        assert _call(L, shp, ws=p) == jv.JV_ERR_INVALID_ARG
    assert _call(L, shp, kv_len=WS + 4 * (need // 8)) == jv.JV_ERR_INVALID_ARG      # an input inside it
    if not torch.cuda.is_available():
        assert _call(L, shp, n=need) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)


def test_binding_refuses():
    t = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        jv.diff_attn(t, t, t, torch.zeros(4, 64), 0.8)
    with pytest.raises(ValueError):
        jv.diff_attn(t, t[:, :, :, :32], t, torch.zeros(4, 64), 0.8)
