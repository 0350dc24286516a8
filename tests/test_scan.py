"""The state-space mixer's calls, its short causal convolution and its selective scan: against their recurrences in 64 bits."""
import ctypes
import math

import pytest
import torch

from paper_2605_26636_b200 import build as jv_build
from paper_2605_26636_b200 import jetvit as jv
from tests._util import guarded_empty

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
CANARY = 77.0


def _conv_reference(x, w, b, state, lens, silu):
    """u, its bound beside the rounding of u, the new state.  K + 1 roundings of sums, of slope 1.1 at most through the activation; the
    exponential: 2^-22 and 1.5 |s| 2^-24 of itself, three roundings more."""
    B, L, C = x.shape
    K = w.shape[1]
    past = torch.zeros(B, K - 1, C, dtype=torch.float64, device=x.device) if state is None else state.double()
    seq = torch.cat([past, x.double()], 1)
    win = seq.unfold(1, K, 1)                                  # [B, L, C, K]
    bias = 0.0 if b is None else b.double()
    s = (win * w.double()).sum(-1) + bias
    mag = (win.abs() * w.double().abs()).sum(-1) + (0.0 if b is None else b.double().abs())
    u = s * torch.sigmoid(s) if silu else s
    bound = 1.1 * (K + 1) * U * mag + u.abs() * (8 + 2 * s.abs()) * U
    new = torch.stack([seq[i, int(n):int(n) + K - 1] for i, n in enumerate(lens)])
    return u, bound, new


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", [1, 7, 64, 100, 264, 2048])
@pytest.mark.parametrize("L", [1, 2, 3, 5, 37, 400])
def test_conv(L, C, dtype):
    g = torch.Generator().manual_seed(L + C)
    r = lambda *s: torch.randn(*s, generator=g)
    for K in (2, 3, 4):
        B = 4
        wide = r(B, L, 2 * C).to(dtype).cuda()
        x = wide[..., :C]
        w, b, st = (0.5 * r(C, K)).cuda(), (0.1 * r(C)).cuda(), r(B, K - 1, C).to(dtype).cuda()
        for lens in (None, torch.tensor([L, 0, min(1, L), max(L - 1, 0)], dtype=torch.int32, device="cuda")):
            n = [L] * B if lens is None else [min(int(i), L) for i in lens]
            for state, silu, bias in ((st, True, b), (None, False, None)):
                out, guard = guarded_empty((B, L, C), dtype, "cuda")
                out.fill_(CANARY)
                new = torch.empty(B, K - 1, C, dtype=dtype, device="cuda")
                jv.causal_conv(x, w, bias, state=state, state_out=new, lens=lens, silu=silu, out=out)
                guard()
                u, bound, ns = _conv_reference(x, w, bias, state, n, silu)
                for i in range(B):
                    d = (out[i, :n[i]].double() - u[i, :n[i]]).abs()
                    assert (d <= HALF[dtype] * (u[i, :n[i]].abs() + bound[i, :n[i]]) + bound[i, :n[i]]).all()
                    assert (out[i, n[i]:] == CANARY).all()
                assert torch.equal(new.double(), ns)
        # the state in its own place, token by token: the same numbers as the whole sequence
        if L > 1:
            whole = jv.causal_conv(x, w, b, state=st)
            run = st.clone()
            parts = [jv.causal_conv(x[:, t:t + 1], w, b, state=run, state_out=run) for t in range(min(L, 6))]
            assert torch.equal(torch.cat(parts, 1), whole[:, :min(L, 6)])


def _scan_inputs(B, L, C, Ns, dtype, seed=0, extra=3):
    g = torch.Generator().manual_seed(seed + 31 * L + C + Ns)
    r = lambda *s: torch.randn(*s, generator=g)
    uz = r(B, L, 2 * C).to(dtype).cuda()
    low = r(B, L, extra + 2 * Ns).to(dtype).cuda()
    step = torch.exp(torch.rand(C, generator=g) * math.log(100.0) + math.log(1e-3))
    return dict(u=uz[..., :C], z=uz[..., C:], dt=(0.5 * r(B, L, C)).to(dtype).cuda(), Bm=low[..., extra:extra + Ns], Cm=low[..., extra + Ns:],
                A=-torch.exp(0.3 * r(C, Ns) + torch.log(torch.arange(1.0, Ns + 1))).cuda(), D=r(C).cuda(),
                dt_bias=(step + torch.log(-torch.expm1(-step))).cuda(), state=r(B, C, Ns).cuda())


def _scan_reference(i, n, softplus=True):
    """y, its bound, the state and its bound by the recurrence in 64 bits, with the error of every step carried along beside the state:
    a step's d is off by 16 roundings (its exponential and logarithm), exp(d A) by 2^-22 and what d A is, a product or sum by one.
    A sequence cut into chunks carries its state by exp(A sum d), the sum off by L roundings: at most 0.37 L U of the state."""
    u, dt, A = i["u"].double(), i["dt"].double(), i["A"].double()
    B, L, C = u.shape
    raw = dt + (i["dt_bias"].double() if i["dt_bias"] is not None else 0.0)
    d = torch.nn.functional.softplus(raw, threshold=700.0) if softplus else raw
    ed = 16 * U if softplus else 2 * U
    edd = ed * d.abs() + U * raw.abs() + 2 * U * dt.abs()
    h = torch.zeros(B, C, A.shape[1], dtype=torch.float64, device=u.device) if i["state"] is None else i["state"].double().clone()
    e = torch.zeros_like(h)
    Bm, Cm = i["Bm"].double(), i["Cm"].double()
    y, ey = torch.zeros_like(u), torch.zeros_like(u)
    cut = 0.37 * L * U if L > 4 else 0.0
    top = h.abs()
    for t in range(L):
        live = torch.tensor([t < k for k in n], device=u.device)[:, None]
        dd, ddd = d[:, t, :, None], edd[:, t, :, None]
        a = torch.exp(dd * A)
        f = dd * u[:, t, :, None] * Bm[:, t, None, :]
        rel = 2.0 ** -22 + 3 * U * (dd * A).abs() + 2 * U + (ddd * A).abs()
        ne = a * e + a * h.abs() * rel + f.abs() * 4 * U + ddd * (u[:, t, :, None] * Bm[:, t, None, :]).abs()
        nh = a * h + f
        h, e = torch.where(live[..., None], nh, h), torch.where(live[..., None], ne, e)
        top = torch.maximum(top, h.abs())
        es = e + cut * top
        y[:, t] = (h * Cm[:, t, None, :]).sum(-1)
        ey[:, t] = (es * Cm[:, t, None, :].abs()).sum(-1) + (A.shape[1] + 4) * U * (h * Cm[:, t, None, :]).abs().sum(-1)
    if i["D"] is not None:
        y, ey = y + i["D"].double() * u, ey + 2 * U * ((i["D"].double() * u).abs() + y.abs())
    if i["z"] is not None:
        z = i["z"].double()
        gate = z * torch.sigmoid(z)
        y, ey = y * gate, gate.abs() * (ey + y.abs() * (10 + 2 * z.abs()) * U)
    return y, ey, h, e + cut * top + 2 * U * h.abs()


def _scan_check(i, dtype, lens=None, softplus=True):
    B, L, C = i["u"].shape
    out, guard = guarded_empty((B, L, C), dtype, "cuda")
    out.fill_(CANARY)
    h1 = torch.full((B, C, i["A"].shape[1]), math.nan, device="cuda")
    jv.selective_scan(**i, state_out=h1, lens=lens, softplus=softplus, out=out)
    guard()
    n = [L] * B if lens is None else [min(max(int(k), 0), L) for k in lens]
    y, ey, h, eh = _scan_reference(i, n, softplus)
    assert ((h1.double() - h).abs() <= eh + 1e-30).all()
    for b in range(B):
        d = (out[b, :n[b]].double() - y[b, :n[b]]).abs()
        assert (d <= HALF[dtype] * (y[b, :n[b]].abs() + ey[b, :n[b]]) + ey[b, :n[b]] + 1e-30).all()
        assert (out[b, n[b]:] == CANARY).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("C", [1, 63, 64, 200, 520])
@pytest.mark.parametrize("L", [1, 2, 4, 5, 31, 33, 200])
def test_scan(L, C, dtype):
    for Ns in (16, 5) if L < 100 else (16,):
        i = _scan_inputs(4, L, C, Ns, dtype)
        _scan_check(i, dtype)
        lens = torch.tensor([L, 0, L // 2, L + 3], dtype=torch.int32, device="cuda")
        _scan_check(dict(i, state=None, D=None), dtype, lens)
        _scan_check(dict(i, z=None, dt_bias=None, dt=i["dt"].abs()), dtype, softplus=False)


@pytest.mark.gpu
@pytest.mark.parametrize("Ns", [1, 3, 4, 8, 17, 32, 64])
def test_state_sizes(Ns):
    for L in (1, 70):
        _scan_check(_scan_inputs(2, L, 72, Ns, torch.float32, extra=0), torch.float32)
        _scan_check(_scan_inputs(2, L, 72, Ns, torch.bfloat16), torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("B,L,C", [(1, 3000, 64), (1, 1000, 384), (2, 2048, 256), (40, 300, 256)])
def test_long_sequences(B, L, C):
    """Few channels (chunks of the sequence over the chip) and many (one pass)."""
    lens = torch.tensor([L if b % 2 == 0 else (L * b) // B + 1 for b in range(B)], dtype=torch.int32, device="cuda")
    _scan_check(_scan_inputs(B, L, C, 16, torch.float32), torch.float32, lens)


@pytest.mark.gpu
def test_prompt_then_tokens():
    """convolution -> scan over a prompt, then single tokens on the states in their own places: as the whole sequence at once."""
    B, L, C, Ns, more = 2, 90, 128, 16, 5
    i = _scan_inputs(B, L + more, C, Ns, torch.float32)
    g = torch.Generator().manual_seed(1)
    w, b = (0.5 * torch.randn(C, 4, generator=g)).cuda(), (0.1 * torch.randn(C, generator=g)).cuda()
    x = torch.randn(B, L + more, C, generator=g).cuda()

    def mixer(t0, t1, cs, hs):
        part = {k: v[:, t0:t1] for k, v in i.items() if k in ("dt", "Bm", "Cm", "z")}
        u = jv.causal_conv(x[:, t0:t1], w, b, state=cs, state_out=cs)
        return jv.selective_scan(u, A=i["A"], D=i["D"], dt_bias=i["dt_bias"], state=hs, state_out=hs, **part)

    new = lambda: (torch.zeros(B, 3, C, device="cuda"), torch.zeros(B, C, Ns, device="cuda"))
    cs, hs = new()
    whole = mixer(0, L + more, cs, hs)
    cs2, hs2 = new()
    parts = [mixer(0, L, cs2, hs2)] + [mixer(t, t + 1, cs2, hs2) for t in range(L, L + more)]
    assert torch.equal(cs, cs2)
    got = torch.cat(parts, 1)
    # two cuts of the same sum, each within some 40 roundings of values of order ten
    assert ((got - whole).abs() <= 1e-4 * (1 + whole.abs())).all() and ((hs - hs2).abs() <= 1e-4 * (1 + hs.abs())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("L", [1, 40])
def test_sequences_whose_offsets_pass_32_bits(L):
    B, C, Ns, far = 3, 72, 16, (1 << 31) // 2 + 64              # elements between batch elements: the third begins behind 2^31
    i = _scan_inputs(B, L, C, Ns, torch.bfloat16)
    pool = torch.empty(2 * far + 4096 * 8, dtype=torch.bfloat16, device="cuda")
    place = lambda t, at: pool.as_strided(t.shape, (far, t.shape[2], 1), at * 4096).copy_(t)
    moved = dict(i, **{n: place(i[n], at) for at, n in enumerate(("u", "dt", "z", "Bm", "Cm"))})
    assert torch.equal(jv.selective_scan(**moved), jv.selective_scan(**i))
    w = torch.randn(C, 4, device="cuda")
    assert torch.equal(jv.causal_conv(moved["u"], w), jv.causal_conv(i["u"], w))


@pytest.mark.gpu
@pytest.mark.parametrize("B,L,C,Ns", [(3, 500, 2100, 16), (2, 300, 1024, 40), (1, 900, 100, 33)])
def test_lanes_and_chunks(B, L, C, Ns):
    """Four lanes a channel, eight, eight with chunks; channels that end within a block."""
    for dtype in (torch.bfloat16, torch.float32):
        lens = torch.tensor([L - 7 * b for b in range(B)], dtype=torch.int32, device="cuda")
        _scan_check(_scan_inputs(B, L, C, Ns, dtype), dtype, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Ns", [5, 8, 16, 32, 40])
@pytest.mark.parametrize("B,L,off", [(2, 90, 0), (5, 300, 0), (2, 90, -3), (2, 90, -8)])
def test_eight_lanes_in_one_pass(B, L, off, Ns, dtype):
    """Channels that fill two thirds of the SMs in blocks of 32, not in blocks of 64; whole blocks and a remainder, on 16-byte boundaries and
    off them; lengths, and the state in its own place."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    C = 32 * -(-5 * sms // (6 * B)) + off                                    # a quarter more blocks of 32 than that takes
    blocks = lambda n: B * -(-C // n)
    assert 3 * blocks(64) < 2 * sms <= 3 * blocks(32)
    for softplus in (0, 1):
        shape = jv.JvScanShape(B, L, C, Ns, jv.JV_BF16 if dtype is torch.bfloat16 else jv.JV_F32, softplus)
        assert jv.lib().jv_selective_scan_workspace_bytes(ctypes.byref(shape)) == 0        # one pass
    i = _scan_inputs(B, L, C, Ns, dtype)
    _scan_check(i, dtype)
    lens = torch.tensor([L - 31 * b for b in range(B)], dtype=torch.int32, device="cuda")
    _scan_check(dict(i, D=None), dtype, lens)
    want, h, run = torch.full((B, L, C), CANARY, dtype=dtype, device="cuda"), torch.empty_like(i["state"]), i["state"].clone()
    got = want.clone()
    jv.selective_scan(**i, lens=lens, out=want, state_out=h)
    jv.selective_scan(**dict(i, state=run), lens=lens, out=got, state_out=run)
    assert torch.equal(got, want) and torch.equal(run, h)


@pytest.mark.gpu
def test_far_values_and_no_numbers():
    i = _scan_inputs(1, 40, 64, 16, torch.float32)
    big = dict(i, dt=torch.where(torch.rand_like(i["dt"]) < 0.1, 60.0, -90.0))     # steps of 60 (the state forgets all) and of nothing
    _scan_check(big, torch.float32)
    bad = dict(i, u=i["u"].clone())
    bad["u"][0, 7, 3] = math.nan
    y, y0 = jv.selective_scan(**bad), jv.selective_scan(**i)
    assert torch.isnan(y[0, 7:, 3]).all() and torch.equal(y[0, :7], y0[0, :7])
    keep = [c for c in range(64) if c != 3]
    assert torch.equal(y[0][:, keep], y0[0][:, keep])
    lens = torch.tensor([7], dtype=torch.int32, device="cuda")                       # what lies behind a sequence is not read
    out, h = torch.zeros_like(y0), torch.empty(1, 64, 16, device="cuda")
    jv.selective_scan(**bad, lens=lens, out=out, state_out=h)
    assert torch.equal(out[0, :7], y0[0, :7]) and (out[0, 7:] == 0).all() and torch.isfinite(h).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,C,Ns", [(2, 1, 100, 16), (2, 37, 5000, 16), (3, 1000, 64, 16), (2, 600, 100, 33)])
def test_states_that_are_forgotten_at_once(B, L, C, Ns, dtype):
    """A of minus infinity: what any A gives that forgets within a step; tokens and chunks past the end leave the state alone."""
    i = _scan_inputs(B, L, C, Ns, dtype)
    lens = torch.tensor([max(1, L - 401 * b) for b in range(B)], dtype=torch.int32, device="cuda")
    i["A"][:, 1::3] = -1e30
    _scan_check(i, dtype, lens)
    at_once = dict(i, A=torch.where(i["A"] == -1e30, -math.inf, i["A"]))
    h, hw = (torch.empty_like(i["state"]) for _ in range(2))
    out, want = (torch.zeros(B, L, C, dtype=dtype, device="cuda") for _ in range(2))
    jv.selective_scan(**at_once, lens=lens, out=out, state_out=h)
    jv.selective_scan(**i, lens=lens, out=want, state_out=hw)
    assert torch.equal(out, want) and torch.equal(h, hw) and torch.isfinite(h).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,C,Ns", [(2, 1, 100, 16), (2, 4, 100, 16), (2, 37, 5000, 16), (3, 1000, 64, 16), (2, 600, 100, 33)])
def test_steps_of_nothing_leave_the_state_for_any_A(B, L, C, Ns, dtype):
    """A of either infinity with steps of 0, and with sequences that end inside a tile or ahead of a chunk."""
    i = _scan_inputs(B, L, C, Ns, dtype)
    i["A"][:, 1::3], i["A"][:, 2::3] = math.inf, -math.inf
    i["dt"], i["dt_bias"] = torch.full_like(i["dt"], -200.0), None                 # softplus: exactly 0
    lens = torch.tensor([max(1, L - 401 * b) for b in range(B)], dtype=torch.int32, device="cuda")
    h, y = torch.empty_like(i["state"]), torch.zeros(B, L, C, dtype=dtype, device="cuda")
    jv.selective_scan(**i, lens=lens, out=y, state_out=h)
    assert torch.equal(h, i["state"]) and torch.isfinite(y).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Ns", [1, 3, 4, 5, 17, 33, 40])
@pytest.mark.parametrize("B,L,C", [(1, 3, 64), (2, 90, 2048), (1, 700, 64), (3, 60, 5000)])
def test_infinities_with_fewer_states_than_lanes_hold(B, L, C, Ns, dtype):
    """All of a channel's own terms plus infinity: so are its results from there on, whatever number of states lanes are left without.
    Single tokens, one pass on eight lanes and on four, chunks."""
    i = _scan_inputs(B, L, C, Ns, dtype)
    for name in ("Bm", "Cm", "z", "D", "state"):
        i[name] = i[name].abs() + 0.1
    i["A"] = torch.full_like(i["A"], -0.01)
    at = L // 2
    for name in ("u", "dt"):
        j = dict(i, **{name: i[name].abs()})
        j[name][:, at, 3] = math.inf
        if name == "dt":
            j["u"], j["A"] = i["u"].abs() + 0.1, torch.full_like(i["A"], 0.01)   # (a step of infinity: the state too grows beyond all)
        clean = jv.selective_scan(**dict(j, **{name: i[name].abs()}))
        h = torch.empty_like(i["state"])
        y = jv.selective_scan(**j, state_out=h)
        assert (y[:, at:, 3] == math.inf).all() and (h[:, 3] == math.inf).all()
        assert torch.equal(y[:, :at], clean[:, :at]) and torch.equal(y[:, :, 4:], clean[:, :, 4:]) and torch.isfinite(y[:, :, :3]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("step,start", [(-3.0, 1e-33), (-40.0, 0.0), (3.0, 1e33)])
def test_chunks_whose_steps_together_leave_fp32(step, start):
    """Steps of the first 32 tokens (a chunk's) that multiply the state by e^96 or e^-96 together: as one by one, a state that is back
    within fp32 is kept, and none stays none."""
    L, C, Ns = 1000, 64, 16
    i = _scan_inputs(1, L, C, Ns, torch.float32)
    i.update(A=torch.full((C, Ns), -1.0, device="cuda"), u=torch.zeros(1, L, C, device="cuda"), dt=torch.zeros(1, L, C, device="cuda"),
             dt_bias=None, state=torch.full((1, C, Ns), start, device="cuda"))
    i["dt"][:, :32] = step
    if start == 0.0:
        i["u"][:, 500:], i["dt"][:, 500:] = 1.0, 0.01
    assert jv.lib().jv_selective_scan_workspace_bytes(ctypes.byref(jv.JvScanShape(1, L, C, Ns, jv.JV_F32, 0))) > 0     # in chunks
    h = torch.empty_like(i["state"])
    y = jv.selective_scan(**i, softplus=False, state_out=h)
    assert torch.isfinite(y).all()
    _, _, want, bound = _scan_reference(i, [L], softplus=False)
    # beside what the recurrence carries along: the three factors, 2^-22 and the rounding of a third of 139 binary orders each, two products
    bound = bound + (3 * (2.0 ** -22 + 47 * U) + 4 * U) * want.abs()
    assert ((h.double() - want).abs() <= bound).all() and (h != 0).all()


@pytest.mark.gpu
def test_results_on_another_stream_do_not_lie_where_earlier_work_still_writes():
    i = _scan_inputs(1, 1000, 256, 16, torch.float32)
    w = torch.randn(256, 4, device="cuda")
    want, want_c = jv.selective_scan(**i), jv.causal_conv(i["u"], w)
    shape = jv.JvScanShape(1, 1000, 256, 16, jv.JV_F32, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    late = [torch.empty_like(want), torch.empty_like(want),
            torch.empty(jv.lib().jv_selective_scan_workspace_bytes(ctypes.byref(shape)), dtype=torch.uint8, device="cuda")]
    torch.cuda._sleep(1 << 26)
    for t in late:
        t.fill_(7)
    del late, t
    got, got_c = jv.selective_scan(**i, stream=side), jv.causal_conv(i["u"], w, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_c, want_c)


@pytest.mark.gpu
@pytest.mark.parametrize("B,L,C", [(2, 1, 300), (1, 700, 192)])
def test_streams_and_capture(B, L, C):
    i = _scan_inputs(B, L, C, 16, torch.bfloat16)
    st = i.pop("state")
    h = torch.empty_like(st)
    want, hw = jv.selective_scan(**i, state=st, state_out=h), None
    hw = h.clone()
    for _ in range(5):
        assert torch.equal(jv.selective_scan(**i, state=st, state_out=h), want) and torch.equal(h, hw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [jv.selective_scan(**i, state=st, stream=side) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)
    out, run = torch.empty_like(want), st.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jv.selective_scan(**i, state=run, state_out=run, out=out)
    run.copy_(st)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(run, hw)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, jv.selective_scan(**i, state=hw))


# ---- refusals, on the host ------------------------------------------------------------------------------------------
P = [i << 26 for i in range(1, 16)]


@pytest.fixture(scope="module")
def L():
    jv_build.build()
    return jv.lib()


def test_conv_refusals(L):
    S = jv.JvConvShape
    ok = S(2, 8, 64, 4, jv.JV_F32, 1)
    call = lambda shp=ok, x=P[0], w=P[1], b=P[2], si=P[3], u=P[4], so=P[3], lens=P[5]: L.jv_causal_conv(
        x, w, b, si, u, so, lens, ctypes.byref(shp) if shp else None, None)
    for kw in (dict(shp=None), dict(x=None), dict(w=None), dict(u=None), dict(x=P[0] + 2), dict(w=P[1] + 1), dict(lens=P[5] + 2), dict(u=P[0]), dict(u=P[3]),
               dict(so=P[0]), dict(so=P[3] + 16), dict(so=P[1]), dict(shp=S(0, 8, 64, 4, 0, 1)), dict(shp=S(2, 0, 64, 4, 0, 1)),
               dict(shp=S(2, 8, 64, 4, 3, 1)), dict(shp=S(2, 8, 64, 4, 0, 2)), dict(shp=S(2, 8, 64, 4, 0, 1, (63, 0))),
               dict(shp=S(2, 8, 64, 4, 0, 1, (64, -512)))):
        assert call(**kw) == jv.JV_ERR_INVALID_ARG, kw
    for shp in (S(2, 8, 64, 1, 0, 1), S(2, 8, 64, 5, 0, 1), S(70000, 8, 64, 4, 0, 1)):
        assert call(shp=shp) == jv.JV_ERR_UNSUPPORTED
    far = S(65535, 8, 64, 4, 0, 1, (64, 1 << 55))                      # extents that 64 bits of bytes do not hold
    assert call(shp=far) == jv.JV_ERR_UNSUPPORTED
    if not torch.cuda.is_available():
        assert call() in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)
    t = torch.zeros(1, 4, 8)
    with pytest.raises(ValueError):
        jv.causal_conv(t, torch.zeros(8, 4))


def test_scan_refusals(L):
    S = jv.JvScanShape
    ok = S(2, 800, 64, 16, jv.JV_F32, 1)
    need = L.jv_selective_scan_workspace_bytes(ctypes.byref(ok))
    assert need > 0

    def call(shp=ok, ws=P[12], n=need, **kw):
        p = dict(u=P[0], dt=P[1], A=P[2], Bm=P[3], Cm=P[4], D=P[5], z=P[6], bias=P[7], si=P[8], y=P[9], so=P[8], lens=P[10])
        p.update(kw)
        return L.jv_selective_scan(*p.values(), ctypes.byref(shp) if shp else None, ws, n, None)

    bad = [dict([(k, None)]) for k in ("u", "dt", "A", "Bm", "Cm", "y", "shp")] + [dict([(k, P[11] + 2)]) for k in ("u", "D", "si", "so", "lens")]
    bad += [dict(y=P[0]), dict(y=P[8]), dict(so=P[8] + 64), dict(so=P[2]), dict(ws=P[9]), dict(ws=P[8])]
    bad += [dict(shp=s) for s in (S(0, 8, 64, 16, 0, 1), S(2, 8, 64, 0, 0, 1), S(2, 8, 64, 16, 9, 1), S(2, 8, 64, 16, 0, 2),
                                  S(2, 8, 64, 16, 0, 1, (32, 0)), S(2, 8, 64, 16, 0, 1, (0, 0), (0, 0), (15, 0)))]
    for kw in bad:
        assert call(**kw) == jv.JV_ERR_INVALID_ARG, kw
    assert call(shp=S(2, 8, 64, 65, 0, 1)) == jv.JV_ERR_UNSUPPORTED
    assert call(shp=S(65535, 8, 64, 16, 0, 1, (64, 1 << 55))) == jv.JV_ERR_UNSUPPORTED
    for kw in (dict(ws=None), dict(ws=P[12] + 8), dict(n=need - 1)):
        assert call(**kw) == jv.JV_ERR_WORKSPACE, kw
    one = S(2, 1, 64, 16, jv.JV_F32, 1)
    assert L.jv_selective_scan_workspace_bytes(ctypes.byref(one)) == 0
    if not torch.cuda.is_available():
        assert call() in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED) and call(shp=one, ws=None, n=0) in (jv.JV_ERR_CUDA, jv.JV_ERR_UNSUPPORTED)
