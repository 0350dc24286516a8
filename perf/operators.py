"""The operators around the mixers, by the calls a user makes of them and in plain form.

``kind`` names the operator of a case:

* ``norm``, ``norm_grad``: layer norm of token rows, in front of a block's projections, and its gradient;
* ``diff``: differential attention on heads in pairs, for prompts and for single tokens against a cache;
* ``scan``: the two calls of a state-space mixer, its short causal convolution and its selective scan, for prompts and for
  single tokens.  The projection that lies between them in a model is not part of a pass: the scan's inputs, like the
  convolution's, are there already.

Sizes are those of this repository's configurations, tests and benchmark (16 x 16 up to 128 x 128 tokens, heads of 64
channels, widths of 384 to 1024, twice that inside the state-space mixer) and the ranges between them.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
NORM_EPS = 1e-5
LAMBDA_INIT = 0.8


def _norm(kind, rows, C, dtype):
    return {"kind": kind, "rows": rows, "C": C, "dtype": dtype}


def _diff(B, H, Hkv, Nq, Nk, causal, ragged, layout="bhnd"):
    # ragged: every sequence has its own number of keys; the last query of a causal one sits on its last key
    return {"kind": "diff", "B": B, "H": H, "Hkv": Hkv, "Nq": Nq, "Nk": Nk, "causal": causal, "ragged": ragged, "layout": layout}


def _scan(B, L, C, Ns, K, dtype, ragged, start):
    # start: a state of earlier tokens goes in
    return {"kind": "scan", "B": B, "L": L, "C": C, "Ns": Ns, "K": K, "dtype": dtype, "ragged": ragged, "start": start}


def listed():
    named = {
        # One 518 x 518 image of a small model at patch 14, class token included: the smallest norm, all latency.
        "norm_image": _norm("norm", 1370, 384, "bf16"),
        # Eight 1024 x 1024 images of a large model.
        "norm_batch": _norm("norm", 32768, 1024, "bf16"),
        # The same in a fine-tuning step.
        "norm_grad_batch": _norm("norm_grad", 32768, 1024, "bf16"),
        # A step in fp32 on four 1022 x 1022 images at patch 14 of a base-size model: a row count that nothing divides.
        "norm_grad_f32": _norm("norm_grad", 21316, 768, "f32"),
        # Causal prompts of 4096 tokens, 16 heads.
        "diff_prompt": _diff(2, 16, 16, 4096, 4096, True, False),
        # 73 x 73 tokens of four images, every token sees every other, inputs left in the projection's token-major layout: the largest.
        "diff_grid": _diff(4, 16, 16, 5329, 5329, False, False, "bnhd"),
        # 256 further tokens of one long sequence against its cache, heads sharing keys two by two: few rows, many keys.
        "diff_chunk": _diff(1, 16, 8, 256, 16384, True, True),
        # One token for each of 32 sequences of all lengths up to 16384, four query heads to a key head.
        "diff_token": _diff(32, 16, 4, 1, 16384, False, True),
        # One token of one short sequence: latency.
        "diff_token_one": _diff(1, 12, 12, 1, 1370, False, False),
        # Two prompts of 4096 tokens through a mixer twice as wide as the model.
        "scan_prompt": _scan(2, 4096, 2048, 16, 4, "bf16", False, False),
        # fp32, five sequences of different lengths that continue earlier ones.
        "scan_ragged": _scan(5, 1369, 768, 16, 4, "f32", True, True),
        # One token for each of 64 sequences.
        "scan_token": _scan(64, 1, 2048, 16, 4, "bf16", False, True),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    what = rng.choice(["norm", "norm", "diff", "diff", "diff", "scan", "scan"])
    if what == "norm":
        C = rng.choice([64 * rng.randint(1, 32), 8 * rng.randint(8, 256), rng.randint(33, 2048)])
        rows = _log(rng, 1, 40000 * 1024 // max(C, 1024))
        return _norm(rng.choice(["norm", "norm_grad"]), rows, C, rng.choice(["bf16", "bf16", "f32"]))
    if what == "diff":
        Hkv = 2 * rng.randint(1, 8)
        H = Hkv * rng.choice([1, 1, 2, 4])
        form = rng.choice(["prompt", "chunk", "token"])
        if form == "prompt":
            N = _log(rng, 1, 5329)
            B = max(1, min(rng.randint(1, 8), int(64 * 5329 ** 2 / (H * N * N))))
            while H * N * N * B > 64 * 5329 ** 2 and H > 2:
                Hkv, H = 2, max(2, H // 2 // 2 * 2)
            return _diff(B, H, Hkv, N, N, rng.random() < 0.5, rng.random() < 0.5, rng.choice(["bhnd", "bnhd"]))
        Nk = _log(rng, 1, 16384)
        if form == "chunk":
            return _diff(rng.randint(1, 2), H, Hkv, _log(rng, 2, 512), Nk, rng.random() < 0.7, rng.random() < 0.5, rng.choice(["bhnd", "bnhd"]))
        return _diff(_log(rng, 1, 32), H, Hkv, 1, Nk, False, rng.random() < 0.7, rng.choice(["bhnd", "bnhd"]))
    C = rng.choice([64 * rng.randint(1, 32), rng.randint(1, 2048)])
    Ns, K = rng.choice([4, 8, 16, 16, 16, 32]), rng.randint(2, 4)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if rng.random() < 0.4:
        return _scan(_log(rng, 1, 128), 1, C, Ns, K, dtype, False, rng.random() < 0.7)
    return _scan(rng.randint(1, 6), _log(rng, 2, 2048), C, Ns, K, dtype, rng.random() < 0.5, rng.random() < 0.5)


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _heads(t, layout):
    """[B, H, N, 64] values in the case's layout: contiguous, or token-major rows seen as [B, H, N, 64]."""
    if layout == "bhnd":
        return t
    return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    if case["kind"] in ("norm", "norm_grad"):
        rows, C, dt = case["rows"], case["C"], DTYPES[case["dtype"]]
        # residual streams: a few channels much larger than the others, and off zero
        gain = torch.exp(0.5 * _rand(gen, C)) * torch.where(_rand(gen, C) > 2.3, 10.0, 1.0)
        x = (_rand(gen, rows, C) * gain + 0.3 * _rand(gen, C)).to(dt)
        s = {"case": case, "x": x, "w": 1 + 0.1 * _rand(gen, C), "b": 0.1 * _rand(gen, C)}
        if case["kind"] == "norm_grad":
            s["dy"] = _rand(gen, rows, C).to(dt)
            x64 = x.double()
            mean = x64.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = ((x64 - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
        return s
    if case["kind"] == "diff":
        B, H, Hkv, Nq, Nk, lay = (case[k] for k in ("B", "H", "Hkv", "Nq", "Nk", "layout"))
        s = {"case": case, "kv_len": None, "q_pos": None,
             "q": _heads(_rand(gen, B, H, Nq, 64).to(torch.bfloat16), lay),
             "k": _heads(_rand(gen, B, Hkv, Nk, 64).to(torch.bfloat16), lay),
             "v": _heads(_rand(gen, B, Hkv, Nk, 64).to(torch.bfloat16), lay),
             "lam": 0.1 * _rand(gen, 4, 64), "w": 1 + 0.1 * _rand(gen, 128)}
        if case["ragged"]:
            lens = rng.integers(max(1, Nk // 4), Nk + 1, B)
            lens[rng.integers(0, B)] = Nk
            s["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
            if case["causal"]:
                s["q_pos"] = (s["kv_len"] - Nq).to(torch.int32)
        return s
    B, L, C, Ns, K, dt = (case[k] for k in ("B", "L", "C", "Ns", "K", "dtype"))
    dt = DTYPES[dt]
    xz = _rand(gen, B, L, 2 * C).to(dt)          # what an input projection leaves: the mixer's input beside its gate
    r = max(1, C // 32)
    low = _rand(gen, B, L, r + 2 * Ns).to(dt)    # what the inner projection leaves: the step's low rank, B, C
    step = torch.exp(_rand(gen, C).sigmoid() * math.log(100.0) + math.log(1e-3))     # steps of 0.001 to 0.1
    s = {"case": case, "x": xz[..., :C], "z": xz[..., C:], "Bm": low[..., r:r + Ns], "Cm": low[..., r + Ns:],
         "dt": (0.5 * _rand(gen, B, L, C)).to(dt), "dt_bias": step + torch.log(-torch.expm1(-step)),
         "A": -torch.exp(torch.log(torch.arange(1.0, Ns + 1, device="cuda")) + 0.2 * _rand(gen, C, Ns)),
         "D": 1 + 0.1 * _rand(gen, C), "cw": 0.5 * _rand(gen, C, K), "cb": 0.1 * _rand(gen, C), "lens": None, "h0": None, "s0": None}
    if case["ragged"]:
        lens = rng.integers(0, L + 1, B)
        lens[rng.integers(0, B)] = L
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["start"]:
        s["h0"] = 0.1 * _rand(gen, B, C, Ns)
        s["s0"] = _rand(gen, B, K - 1, C).to(dt)
    s["us"] = torch.nn.functional.silu(_rand(gen, B, L, C)).to(dt)        # the scan's own input
    # buffers that a serving loop keeps: padding rows of u and y stay as they are
    s["u"] = torch.zeros(B, L, C, dtype=dt, device="cuda")
    s["y"] = torch.zeros(B, L, C, dtype=dt, device="cuda")
    s["h1"] = torch.empty(B, C, Ns, device="cuda")
    s["s1"] = torch.empty(B, K - 1, C, dtype=dt, device="cuda")
    return s


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _own(s):
    from paper_2605_26636_b200 import jetvit as jv
    kind = s["case"]["kind"]
    if kind == "norm":
        return jv.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
    if kind == "norm_grad":
        return jv.layer_norm_grad(s["dy"], s["x"], s["w"], s["mean"], s["rstd"])
    if kind == "diff":
        return jv.diff_attn(s["q"], s["k"], s["v"], s["lam"], LAMBDA_INIT, norm_weight=s["w"], norm_eps=NORM_EPS,
                            causal=s["case"]["causal"], kv_len=s["kv_len"], q_pos=s["q_pos"])
    u = jv.causal_conv(s["x"], s["cw"], s["cb"], state=s["s0"], state_out=s["s1"], lens=s["lens"], out=s["u"])
    y = jv.selective_scan(s["us"], s["dt"], s["A"], s["Bm"], s["Cm"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], state=s["h0"],
                          state_out=s["h1"], lens=s["lens"], out=s["y"])
    return {"u": u, "y": y, "conv_state": s["s1"], "state": s["h1"]}


# ---- plain forms --------------------------------------------------------------------------------------------------

def _plain_norm(s):
    x = s["x"].float()
    xc = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    return (xc * r * s["w"] + s["b"]).to(s["x"].dtype)


def _plain_norm_grad(s):
    x, dy = s["x"].float(), s["dy"].float()
    r = s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * r
    g = dy * s["w"]
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    # sums over all rows in 64 bits: tens of thousands of terms that nearly cancel
    return dx.to(s["x"].dtype), (dy * xh).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()


def _plain_diff(s):
    c = s["case"]
    B, H, Hkv, Nq, Nk = (c[k] for k in ("B", "H", "Hkv", "Nq", "Nk"))
    lam = torch.exp((s["lam"][0] * s["lam"][1]).sum()) - torch.exp((s["lam"][2] * s["lam"][3]).sum()) + LAMBDA_INIT
    pairs, share = H // 2, H // Hkv
    kv = torch.arange(pairs, device="cuda") // share             # the key pair of each query pair
    j = torch.arange(Nk, device="cuda")
    out = torch.empty(B, H, Nq, 64, dtype=s["q"].dtype, device="cuda")
    for b in range(B):
        q = s["q"][b].float().reshape(pairs, 2, Nq, 64)
        k = s["k"][b].float().reshape(Hkv // 2, 2, Nk, 64)[kv]
        v = s["v"][b].float().reshape(Hkv // 2, 2, Nk, 64)[kv].transpose(1, 2).reshape(pairs, Nk, 128)
        seen = torch.ones(Nq, Nk, dtype=torch.bool, device="cuda")
        if s["kv_len"] is not None:
            seen = seen & (j < s["kv_len"][b])
        if c["causal"]:
            first = Nk - Nq if s["q_pos"] is None else s["q_pos"][b]
            seen = seen & (j[None, :] <= torch.arange(Nq, device="cuda")[:, None] + first)
        some = seen.any(1)[:, None]
        p = (q @ k.transpose(2, 3)) * 0.125
        p = torch.where(seen, p, -math.inf)
        p = torch.exp(p - torch.where(some, p.amax(3, keepdim=True), 0.0))
        p = p / torch.where(some, p.sum(3, keepdim=True), 1.0)
        x = (p[:, 0] - lam * p[:, 1]) @ v
        x = (1 - LAMBDA_INIT) * s["w"] * x * torch.rsqrt((x * x).mean(2, keepdim=True) + NORM_EPS)
        out[b] = x.reshape(pairs, Nq, 2, 64).transpose(1, 2).reshape(H, Nq, 64).to(out.dtype)
    return out


def _plain_scan(s):
    c = s["case"]
    B, L, C, Ns, K = (c[k] for k in ("B", "L", "C", "Ns", "K"))
    dt = s["x"].dtype
    before = torch.zeros(B, K - 1, C, dtype=dt, device="cuda") if s["s0"] is None else s["s0"]
    lens = torch.full((B,), L, device="cuda") if s["lens"] is None else s["lens"].long()
    xx = torch.cat([before, s["x"]], 1)
    u = s["cb"] + sum(xx[:, i:i + L].float() * s["cw"][:, i] for i in range(K))
    live = (torch.arange(L, device="cuda") < lens[:, None])[..., None]
    u = torch.where(live, u / (1 + torch.exp(-u)), 0.0).to(dt)
    s1 = torch.gather(xx, 1, (lens[:, None] + torch.arange(K - 1, device="cuda"))[..., None].expand(B, K - 1, C))
    uf = s["us"].float()
    raw = s["dt"].float() + s["dt_bias"]
    step = torch.where(raw > 20, raw, torch.log1p(torch.exp(torch.clamp(raw, max=20))))
    step = torch.where(live, step, 0.0)                       # padding leaves the state alone
    su = step * uf
    bm, cm = s["Bm"].float(), s["Cm"].float()
    h = torch.zeros(B, C, Ns, device="cuda") if s["h0"] is None else s["h0"].clone()
    y = torch.empty(B, L, C, device="cuda")
    for t in range(L):
        h = torch.exp(step[:, t, :, None] * s["A"]) * h + su[:, t, :, None] * bm[:, t, None, :]
        y[:, t] = (h * cm[:, t, None, :]).sum(2)
    z = s["z"].float()
    y = (y + s["D"] * uf) * z / (1 + torch.exp(-z))
    return {"u": u, "y": torch.where(live, y, 0.0).to(dt), "conv_state": s1, "state": h}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "diff": _plain_diff, "scan": _plain_scan}[state["case"]["kind"]](state)


def work(case):
    e = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if case["kind"] == "norm":
        n = case["rows"] * case["C"]
        return {"bytes": 2 * n * e + 8 * case["C"], "flops": 8 * n}
    if case["kind"] == "norm_grad":
        n = case["rows"] * case["C"]
        return {"bytes": 3 * n * e + 8 * case["rows"] + 12 * case["C"], "flops": 14 * n}
    if case["kind"] == "diff":
        B, H, Hkv, Nq, Nk = (case[k] for k in ("B", "H", "Hkv", "Nq", "Nk"))
        keys = Nk * (0.625 if case["ragged"] and B > 1 else 1.0)          # lengths between a quarter of the cache and all of it
        seen = keys - (min(Nq, Nk) - 1) / 2 if case["causal"] else keys   # keys of a row
        # scores of two maps, one product of their difference with the values
        return {"bytes": int(2 * 64 * B * (2 * H * Nq + 2 * Hkv * keys)), "flops": int(B * H // 2 * Nq * max(seen, 1.0) * 512)}
    B, L, C, Ns, K = (case[k] for k in ("B", "L", "C", "Ns", "K"))
    n = B * L * C * (0.6 if case["ragged"] else 1.0)
    states = (2 if case["start"] else 1) * B * C * (4 * Ns + e * (K - 1))
    # x, the scan's u, dt and z read, u and y written; B and C; the states
    return {"bytes": int(6 * n * e + 2 * B * L * Ns * e + states + 4 * C * (Ns + K + 3)), "flops": int(n * (2 * K + 7 * Ns + 12))}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_diff(s):
    c = s["case"]
    B, H, Hkv, Nq, Nk = (c[k] for k in ("B", "H", "Hkv", "Nq", "Nk"))
    l64 = s["lam"].double()
    lam = float(torch.exp(l64[0] @ l64[1]) - torch.exp(l64[2] @ l64[3])) + LAMBDA_INIT
    lens = [Nk] * B if s["kv_len"] is None else s["kv_len"].tolist()
    first = [Nk - Nq] * B if s["q_pos"] is None else s["q_pos"].tolist()
    out = torch.zeros(B, H, Nq, 64, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = lens[b]
        for p in range(H // 2):
            g = 2 * (p // (H // Hkv))
            v = torch.cat([s["v"][b, g, :n], s["v"][b, g + 1, :n]], 1).double()
            for r0 in range(0, Nq, 2048):
                rows = torch.arange(r0, min(Nq, r0 + 2048), device="cuda")
                diff = 0.0
                for m, sign in ((0, 1.0), (1, -lam)):
                    a = s["q"][b, 2 * p + m, rows].double() @ s["k"][b, g + m, :n].double().T / 8.0
                    if c["causal"]:
                        a.masked_fill_(torch.arange(n, device="cuda")[None] > rows[:, None] + first[b], -math.inf)
                    diff = diff + sign * torch.nan_to_num(torch.softmax(a, 1), nan=0.0)      # a row without keys
                x = diff @ v
                x = x / torch.sqrt(x.pow(2).mean(1, keepdim=True) + NORM_EPS) * s["w"].double() * (1 - LAMBDA_INIT)
                out[b, 2 * p, rows], out[b, 2 * p + 1, rows] = x[:, :64], x[:, 64:]
    return out


def _exact_scan(s):
    c = s["case"]
    B, L, C, Ns, K = (c[k] for k in ("B", "L", "C", "Ns", "K"))
    lens = [L] * B if s["lens"] is None else s["lens"].tolist()
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")
    u, y, s1, h1 = new(B, L, C), new(B, L, C), new(B, K - 1, C), new(B, C, Ns)
    for b in range(B):
        n = lens[b]
        past = new(K - 1, C) if s["s0"] is None else s["s0"][b].double()
        seq = torch.cat([past, s["x"][b, :n].double()])
        s1[b] = seq[n:]
        h0 = new(C, Ns) if s["h0"] is None else s["h0"][b].double()
        if n == 0:
            h1[b] = h0
            continue
        pre = (seq.unfold(0, K, 1) * s["cw"].double()).sum(2) + s["cb"].double()
        u[b, :n] = pre * torch.sigmoid(pre)
        for c0 in range(0, C, 256):                             # (slices of channels: the states of all tokens at once)
            ch = slice(c0, min(C, c0 + 256))
            uu = s["us"][b, :n, ch].double()
            d = torch.nn.functional.softplus(s["dt"][b, :n, ch].double() + s["dt_bias"][ch].double(), threshold=700.0)
            a = torch.exp(d[:, :, None] * s["A"][ch].double())
            f = (d * uu)[:, :, None] * s["Bm"][b, :n].double()[:, None, :]
            f[0] += a[0] * h0[ch]
            w = 1
            while w < n:                                        # prefix composition of the maps h -> a h + f by doubling
                f = torch.cat([f[:w], f[w:] + a[w:] * f[:-w]])
                a = torch.cat([a[:w], a[w:] * a[:-w]])
                w *= 2
            h1[b, ch] = f[-1]
            zz = s["z"][b, :n, ch].double()
            y[b, :n, ch] = (torch.einsum("tcs,ts->tc", f, s["Cm"][b, :n].double()) + s["D"][ch].double() * uu) * zz * torch.sigmoid(zz)
    return {"u": u, "y": y, "conv_state": s1, "state": h1}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "diff":
        return _exact_diff(s)
    if case["kind"] == "scan":
        return _exact_scan(s)
    x, w = s["x"].double(), s["w"].double()
    if case["kind"] == "norm":
        mean = x.mean(1, keepdim=True)
        return (x - mean) / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS) * w + s["b"].double()
    C = case["C"]
    xh, r = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None], s["rstd"].double()[:, None]
    dy = s["dy"].double()
    dxh = dy * w
    dx = r / C * (C * dxh - dxh.sum(1, keepdim=True) - xh * (dxh * xh).sum(1, keepdim=True))
    return dx, torch.einsum("rc,rc->c", dy, xh), dy.sum(0)
