"""The sequence operators of the library as cases to be timed and compared: spike trains counted into the steps of a
sequence, the short causal convolution, the selective state-space scan, their 8-bit activation checkpoints, and the
class that a readout answers with.

A case names its operator in ``op``; what else it holds are sizes.  With ``own`` false ``run`` computes the operator from
elementary torch operations in 32 bits (64 where a border decides), with ``own`` true through
``paper_2501_07331_amd.SequenceLayer`` and ``paper_2501_07331_amd.Sampler``.

The formulas, per sample, with t counting its steps:

  bin      dst[t, c]  = number of spikes of neuron c in steps [t f, (t + 1) f)
  conv     pre[t, c]  = bias[c] + sum_k w[c, k] x[t - (K - 1) + k, c],  y = pre sigmoid(pre)
  scan     delta'     = log(1 + exp(delta + bias)),  a = exp(delta' A),  h[t] = a h[t - 1] + delta' u B[t],
           y[t, c]    = (sum_n C[t, n] h[t, c, n] + D[c] u[t, c]) z sigmoid(z)
  pack     x[t, c]    = scale[t, c / 128] q[t, c], q in e4m3, the scale the smallest power of two that keeps q in range
  sample   the first index (in index order) whose running sum of the kept exp((z - max z) / temperature) passes u times
           their sum; kept: the top_k largest (ties: lowest index first), those before which less than top_p of the mass
           lies in that order, and those of at least min_p times the largest
"""
import math

import torch

own = False

BLOCK = 128          # channels that share a scale in the 8-bit form
F32, BF16, F16 = "float32", "bfloat16", "float16"


def _case(name, op, **kw):
    c = dict(kw, op=op)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the audio benchmark's input, 700 channels and 1000 steps of 1 ms at its full batch, in bins of 4 ms
        _case("bin audio input", "bin", B=256, T=1000, C=700, factor=4, rate=0.0115, dtype=BF16, records=False),
        # the hidden spikes of the small tactile network as its forward pass records them, an odd batch, every step kept
        _case("bin tactile records", "bin", B=37, T=300, C=128, factor=1, rate=0.045, dtype=F32, records=True),
        # training: the convolution and its gradients at the wide network's 1024 channels on a rank's batch
        _case("conv train", "conv", B=32, T=1000, C=1024, K=4, dtype=BF16, ragged=False),
        # serving: one step of the convolution for a full batch of streams
        _case("conv one step", "conv_step", B=256, C=1024, K=4, dtype=BF16),
        # a single long recording: one row of work, only the time axis is long
        _case("scan long recording", "scan", B=1, T=16384, C=1024, N=16, G=1, dtype=BF16, gate=True, ragged=False,
              train=False),
        # training: the scan and every gradient, same sizes as the convolution's
        _case("scan train", "scan", B=32, T=1000, C=1024, N=16, G=1, dtype=BF16, gate=True, ragged=False, train=True),
        # sizes that fill no tile, in 32 bits, with trials of different lengths and three groups of channels
        _case("scan train odd", "scan", B=5, T=333, C=150, N=12, G=3, dtype=F32, gate=False, ragged=True, train=True),
        # serving: one step of the scan for a full batch of streams
        _case("scan one step", "scan_step", B=256, C=1024, N=16, G=1, dtype=BF16, gate=True),
        # training with what the backward pass reads kept in 8 bits: the scan over a fine grid's longer trials
        _case("scan train packed", "scan_packed", B=16, T=4000, C=256, N=16, G=1, dtype=BF16),
        # an activation kept in 8 bits and read back
        _case("pack and unpack", "pack", B=64, T=1000, C=512, dtype=BF16),
        # the answer of the audio network's readout: a class for each of its trials
        _case("sample readout", "sample", rows=256, V=20, dtype=F32),
        # a wide head: a long row needs the filters' selection, few rows leave most of the chip to each
        _case("sample wide head", "sample", rows=32, V=65536, dtype=BF16),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["bin", "conv", "conv_packed", "conv_step", "scan", "scan", "scan", "scan_packed", "scan_step", "pack",
                     "sample", "sample"])
    dt = rng.choice([BF16, BF16, F16, F32])
    if op == "bin":
        return _case(None, op, B=log(1, 256), T=log(100, 1000), C=log(10, 1024), factor=rng.randint(1, 10),
                     rate=rng.uniform(0.005, 0.05), dtype=dt, records=rng.choice([False, True]))
    if op in ("conv", "conv_packed"):
        return _case(None, op, B=log(1, 32), T=log(100, 1000), C=log(64, 1024), K=rng.randint(2, 6), dtype=dt,
                     ragged=rng.choice([False, True]))
    if op == "conv_step":
        return _case(None, op, B=log(1, 512), C=log(64, 2048), K=rng.randint(2, 6), dtype=dt)
    if op in ("scan", "scan_packed"):
        G = rng.choice([1, 1, 1, 2, 4])
        sizes = dict(B=log(1, 32), T=log(16, 1000), C=G * log(64 // G, 1024 // G), N=rng.choice([4, 8, 16, 16, 16, 24, 32]), G=G,
                     dtype=dt)
        if sizes["N"] > 16:
            sizes["T"] = min(sizes["T"], 500)
        if op == "scan_packed":
            return _case(None, op, **sizes)
        sizes.update(gate=rng.choice([True, True, False]), ragged=rng.choice([False, False, True]),
                     train=rng.choice([True, True, False]))
        if rng.random() < 0.25:
            sizes.update(B=rng.randint(1, 2), T=log(1000, 16384), train=False)
            sizes["N"] = min(sizes["N"], 16)
        return _case(None, op, **sizes)
    if op == "scan_step":
        G = rng.choice([1, 1, 2])
        return _case(None, op, B=log(1, 512), C=G * log(64, 1024 // G), N=rng.choice([8, 16, 16, 32]), G=G, dtype=dt,
                     gate=rng.choice([True, False]))
    if op == "pack":
        return _case(None, op, B=log(1, 64), T=log(16, 1000), C=log(64, 512), dtype=dt)
    return _case(None, op, rows=log(1, 256), V=log(2, 8000), dtype=dt) if rng.random() < 0.5 else \
        _case(None, op, rows=log(1, 32), V=log(8000, 65536), dtype=dt)


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = getattr(torch, c["dtype"])

    def randn(*n, dtype=dt, std=1.0):
        return (torch.randn(*n, device="cuda", generator=g) * std).to(dtype)

    def rand(*n):
        return torch.rand(*n, device="cuda", generator=g)

    s = {"case": c}
    if c["op"] == "bin":
        B, T, C = c["B"], c["T"], c["C"]
        hit = rand(B, T, C) < c["rate"]
        b, t, n = torch.nonzero(hit, as_tuple=True)
        count = hit.sum((1, 2)).to(torch.int32)
        off = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        off[1:] = torch.cumsum(count, 0)
        if c["records"]:
            cap = 64 * C
            s["step"] = torch.full((B, cap), -1, dtype=torch.int32, device="cuda")
            s["neuron"] = torch.full((B, cap), -1, dtype=torch.int32, device="cuda")
            k = torch.arange(b.numel(), device="cuda") - off[:-1].long()[b]
            keep = k < cap
            s["step"][b[keep], k[keep]] = t[keep].to(torch.int32)
            s["neuron"][b[keep], k[keep]] = n[keep].to(torch.int32)
            s["count"] = count
        else:
            s["offsets"], s["step"], s["neuron"] = off, t.to(torch.int32), n.to(torch.int32)
        s["y"] = torch.empty(B, -(-T // c["factor"]), C, dtype=dt, device="cuda")
    elif c["op"] in ("conv", "conv_packed"):
        B, T, C, K = c["B"], c["T"], c["C"], c["K"]
        s["x"] = randn(B, T, 2 * C)[:, :, :C]      # one half of a projection's output
        s["w"] = randn(C, K, dtype=torch.float32, std=K ** -0.5)
        s["bias"] = randn(C, dtype=torch.float32, std=0.1)
        s["dy"] = randn(B, T, C)
        s["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=g, dtype=torch.int32) if c["ragged"] else None
    elif c["op"] == "conv_step":
        B, C, K = c["B"], c["C"], c["K"]
        s["x"] = randn(B, 2 * C)[:, :C]
        s["w"] = randn(C, K, dtype=torch.float32, std=K ** -0.5)
        s["bias"] = randn(C, dtype=torch.float32, std=0.1)
        s["state"] = randn(B, K - 1, C)
    elif c["op"] in ("scan", "scan_packed", "scan_step"):
        B, T, C, N, G = c["B"], c.get("T", 1), c["C"], c["N"], c["G"]
        s["u"] = randn(B, T, C)
        s["delta"] = randn(B, T, C, std=0.5)
        bc = randn(B, T, 16 + 2 * G * N)             # B and C are parts of one projection's output
        s["Bm"] = bc[:, :, 16:16 + G * N]
        s["Cm"] = bc[:, :, 16 + G * N:]
        s["z"] = randn(B, T, 2 * C)[:, :, C:] if c.get("gate", True) else None
        s["A"] = -(torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * (0.5 + rand(C, 1)))
        s["D"] = 0.5 + rand(C)
        lo = torch.exp(rand(C) * (math.log(0.1) - math.log(1e-3)) + math.log(1e-3))     # steps of 0.001 to 0.1
        s["delta_bias"] = torch.log(torch.expm1(lo))
        s["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=g, dtype=torch.int32) if c.get("ragged") else None
        if c["op"] == "scan_step":
            s["h"] = randn(B, C, N, dtype=torch.float32)
            for k in ("u", "delta", "Bm", "Cm", "z"):
                s[k] = None if s[k] is None else s[k][:, 0]
        else:
            s["h0"] = randn(B, C, N, dtype=torch.float32, std=0.1)
            if c.get("train", True):
                s["dy"] = randn(B, T, C)
    elif c["op"] == "pack":
        # channels of different sizes, as activations have them
        s["x"] = (randn(c["B"], c["T"], c["C"], dtype=torch.float32) * torch.exp(2.0 * randn(c["C"], dtype=torch.float32))).to(dt)
    else:
        R, V = c["rows"], c["V"]
        s["logits"] = randn(R, V, std=2.0)
        s["logits"][rand(R, V) < 0.05] = float("-inf")
        s["temperature"] = 0.5 + rand(R)
        s["top_k"] = torch.randint(0, max(2, min(V, 64)), (R,), device="cuda", generator=g, dtype=torch.int32)
        s["top_k"][rand(R) < 0.5] = 0                # half of the rows keep any number
        s["top_p"] = 1.0 - 0.5 * rand(R)
        s["top_p"][rand(R) < 0.25] = 1.0
        s["min_p"] = 0.1 * rand(R)
        s["min_p"][rand(R) < 0.5] = 0.0
        s["u"] = rand(R)
    if own:
        import paper_2501_07331_amd as snn
        if c["op"] == "sample":
            s["sampler"] = snn.Sampler(c["rows"], c["V"])
            s["token"] = torch.empty(c["rows"], dtype=torch.int32, device="cuda")
            s["logprob"] = torch.empty(c["rows"], device="cuda")
        else:
            s["layer"] = snn.SequenceLayer(c["B"], c.get("T", 1), c["C"], state=c.get("N", 1), groups=c.get("G", 1),
                                           taps=c.get("K", 1), train="dy" in s, recompute=c["op"] == "scan_packed")
    return s


# ------------------------------------------------------------------ plain forms


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _dsilu(x):
    p = 1.0 / (1.0 + torch.exp(-x))
    return p * (1.0 + x * (1.0 - p))


def _valid(T, lengths, like):
    """[B, T, 1] truth of the steps inside each sample."""
    B = like.shape[0]
    if lengths is None:
        return torch.ones(B, T, 1, dtype=torch.bool, device=like.device)
    return (torch.arange(T, device=like.device)[None, :] < lengths[:, None])[:, :, None]


def _recur(a, x):
    """h[t] = a[t] h[t - 1] + x[t] along axis 1, by doubling."""
    d = 1
    while d < x.shape[1]:
        x = torch.cat([x[:, :d], x[:, d:] + a[:, d:] * x[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return x


def _plain_bin(s):
    c = s["case"]
    B, C, f = c["B"], c["C"], c["factor"]
    S = -(-c["T"] // f)
    if c["records"]:
        keep = torch.arange(s["step"].shape[1], device="cuda")[None, :] < s["count"][:, None]
        b = torch.nonzero(keep, as_tuple=True)[0]
        step, neuron = s["step"][keep], s["neuron"][keep]
    else:
        b = torch.repeat_interleave(torch.arange(B, device="cuda"), (s["offsets"][1:] - s["offsets"][:-1]).long())
        step, neuron = s["step"], s["neuron"]
    at = (b * S + step.long() // f) * C + neuron.long()
    y = torch.zeros(B * S * C, device="cuda")
    y.index_add_(0, at, torch.ones(at.numel(), device="cuda"))
    return y.view(B, S, C).to(getattr(torch, c["dtype"]))


def _windows(x, K):
    return torch.nn.functional.pad(x, (0, 0, K - 1, 0)).unfold(1, K, 1)      # [B, T, C, K]


def _plain_conv(s, x, dt):
    c = s["case"]
    T, K = c["T"], c["K"]
    ok = _valid(T, s["lengths"], x)
    x = torch.where(ok, x.float(), 0.0)
    win = _windows(x, K)
    pre = (win * s["w"]).sum(-1) + s["bias"]
    y = torch.where(ok, _silu(pre), 0.0).to(dt)
    dpre = torch.where(ok, s["dy"].float() * _dsilu(pre), 0.0)
    dx = (torch.nn.functional.pad(dpre, (0, 0, 0, K - 1)).unfold(1, K, 1) * s["w"].flip(1)).sum(-1)
    dx = torch.where(ok, dx, 0.0).to(dt)
    return {"y": y, "dx": dx, "dw": (dpre[..., None] * win).sum((0, 1)), "dbias": dpre.sum((0, 1))}


def _plain_conv_step(s):
    win = torch.cat([s["state"], s["x"][:, None]], 1)
    pre = (win.float() * s["w"].t()).sum(1) + s["bias"]
    return {"y": _silu(pre).to(s["x"].dtype), "state": win[:, 1:].contiguous()}


def _per_channel(m, c):
    """[B, T, G N] of the groups as [B, T, C, N] in 32 bits."""
    B, T = m.shape[:2]
    return m.float().view(B, T, c["G"], c["N"]).repeat_interleave(c["C"] // c["G"], 2)


def _plain_scan(s, u, delta, z, out):
    """The scan from inputs in 32 bits; gradients where the state has dy."""
    c = s["case"]
    B, T, C, G, N = c["B"], c["T"], c["C"], c["G"], c["N"]
    dt = s["u"].dtype
    ok = _valid(T, s["lengths"], u)
    u, raw = torch.where(ok, u, 0.0), torch.where(ok, delta, 0.0) + s["delta_bias"]
    d = torch.where(raw > 20.0, raw, torch.log1p(torch.exp(torch.clamp(raw, max=20.0))))
    gate = _silu(torch.where(ok, z, 0.0)) if z is not None else 1.0
    Bc = torch.where(ok[..., None], _per_channel(s["Bm"], c), 0.0)
    Cc = torch.where(ok[..., None], _per_channel(s["Cm"], c), 0.0)
    a = torch.where(ok[..., None], torch.exp(d[..., None] * s["A"]), 1.0)
    x = (d * u)[..., None] * Bc
    x[:, 0] += a[:, 0] * s["h0"]
    h = _recur(a, x)
    del x
    y0 = (h * Cc).sum(-1) + s["D"] * u
    if "y" in out:
        out["y"] = torch.where(ok, y0 * gate, 0.0).to(dt)
        out["h"] = h[:, -1].contiguous()
    if "du" not in out:
        return out
    dy = torch.where(ok, s["dy"].float(), 0.0)
    if z is not None:
        out["dz"] = (dy * y0 * _dsilu(torch.where(ok, z, 0.0))).to(dt)
    dy = dy * gate
    out["dD"] = (dy * u).sum((0, 1))
    out["dC"] = (dy[..., None] * h).view(B, T, G, C // G, N).sum(3).view(B, T, G * N).to(dt)
    back = torch.cat([a[:, 1:], a[:, :1]], 1).flip(1)
    g = _recur(back, (dy[..., None] * Cc).flip(1)).flip(1)
    del back, Cc
    hp = a * torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    out["dh0"] = a[:, 0] * g[:, 0]
    del a, h
    out["dB"] = (g * (d * u)[..., None]).view(B, T, G, C // G, N).sum(3).view(B, T, G * N)
    out["dB"] = torch.where(ok, out["dB"], 0.0).to(dt)
    gB = (g * Bc).sum(-1)
    del Bc
    g = g * hp
    del hp
    g = torch.where(ok[..., None], g, 0.0)
    out["dA"] = (g * d[..., None]).sum((0, 1))
    dd = ((g * s["A"]).sum(-1) + gB * u) / (1.0 + torch.exp(-raw))
    dd = torch.where(ok, dd, 0.0)
    out["ddelta"] = dd.to(dt)
    out["ddelta_bias"] = dd.sum((0, 1))
    out["du"] = torch.where(ok, s["D"] * dy + d * gB, 0.0).to(dt)
    return out


def _scan_outputs(c, forward=True, backward=True):
    names = ["y", "h"] if forward else []
    if backward:
        names += ["du", "ddelta", "dB", "dC", "dA", "dD", "ddelta_bias", "dh0"] + (["dz"] if c.get("gate", True) else [])
    return dict.fromkeys(names)


def _plain_scan_step(s):
    c = s["case"]
    N, per = c["N"], c["C"] // c["G"]
    u, raw = s["u"].float(), s["delta"].float() + s["delta_bias"]
    d = torch.where(raw > 20.0, raw, torch.log1p(torch.exp(torch.clamp(raw, max=20.0))))
    Bc = s["Bm"].float().view(-1, c["G"], N).repeat_interleave(per, 1)
    Cc = s["Cm"].float().view(-1, c["G"], N).repeat_interleave(per, 1)
    h = torch.exp(d[..., None] * s["A"]) * s["h"] + (d * u)[..., None] * Bc
    y = (h * Cc).sum(-1) + s["D"] * u
    return {"y": (y * _silu(s["z"].float()) if s["z"] is not None else y).to(s["u"].dtype), "h": h}


def _plain_pack(x):
    """(e4m3 values, scales): the scale 2^k, k the least with max |x| <= 448 2^k over a block's finite values."""
    B, T, C = x.shape
    nb = -(-C // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - C)).view(B, T, nb, BLOCK)
    m, e = torch.frexp(torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1))
    k = torch.where(m == 0.0, 0, torch.where(m > 0.875, e - 8, e - 9)).clamp(min=-126)
    scale = torch.ldexp(torch.ones_like(m), k)
    q = torch.where(torch.isfinite(x), x / scale[..., None], float("nan")).to(torch.float8_e4m3fn)
    return q, scale


def _plain_unpack(q, scale, C):
    v = q.float() * scale[..., None]
    return v.view(v.shape[0], v.shape[1], -1)[:, :, :C]


def _packed(x):
    return _plain_unpack(*_plain_pack(x), x.shape[2])


def _plain_sample(s):
    z = s["logits"].double()
    V = z.shape[1]
    top = z.amax(1, keepdim=True)
    w = torch.exp((z - top) / s["temperature"].double()[:, None])
    order = torch.sort(z, dim=1, descending=True, stable=True)[1]
    ws = torch.gather(w, 1, order)
    before = torch.cumsum(ws, 1) - ws
    total = ws.sum(1, keepdim=True)
    k = torch.where(s["top_k"] > 0, s["top_k"], V)
    keep = torch.arange(V, device=z.device)[None, :] < k[:, None]
    keep &= (before < s["top_p"].double()[:, None] * total) | (s["top_p"] >= 1.0)[:, None]
    keep &= ws >= s["min_p"].double()[:, None]
    keep &= ws > 0.0
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0.0))
    run_ = torch.cumsum(kept, 1)
    past = (run_ > s["u"].double()[:, None] * run_[:, -1:]) & (kept > 0.0)
    first = torch.argmax(past.to(torch.int32), 1)
    last = V - 1 - torch.argmax((kept > 0.0).to(torch.int32).flip(1), 1)
    token = torch.where(past.any(1), first, last)
    some = (kept > 0.0).any(1)                     # a row of nothing but -inf has no answer
    logprob = torch.log(torch.gather(kept, 1, token[:, None])[:, 0] / run_[:, -1])
    return {"token": torch.where(some, token, -1).to(torch.int32),
            "logprob": torch.where(some, logprob, -math.inf).float()}


def _plain(s):
    op = s["case"]["op"]
    if op == "bin":
        return _plain_bin(s)
    if op == "conv":
        return _plain_conv(s, s["x"], s["x"].dtype)
    if op == "conv_packed":
        out = _plain_conv(s, _packed(s["x"]), s["x"].dtype)
        out["y"] = _plain_conv(s, s["x"], s["x"].dtype)["y"]
        return out
    if op == "conv_step":
        return _plain_conv_step(s)
    if op == "scan":
        return _plain_scan(s, s["u"].float(), s["delta"].float(), s["z"].float() if s["z"] is not None else None,
                           _scan_outputs(s["case"], True, s["case"]["train"]))
    if op == "scan_packed":
        # the forward pass reads the activations; the backward pass takes u, delta and z, and the states that they give, from 8 bits
        out = _plain_scan(s, s["u"].float(), s["delta"].float(), s["z"].float(), _scan_outputs(s["case"], True, False))
        return dict(out, **_plain_scan(s, _packed(s["u"]), _packed(s["delta"]), _packed(s["z"]),
                                       _scan_outputs(s["case"], False, True)))
    if op == "scan_step":
        return _plain_scan_step(s)
    if op == "pack":
        q, scale = _plain_pack(s["x"])
        return {"scale": scale, "x": _plain_unpack(q, scale, s["case"]["C"]).to(s["x"].dtype)}
    return _plain_sample(s)


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    import paper_2501_07331_amd as snn
    c, op = s["case"], s["case"]["op"]
    if op == "sample":
        s["sampler"].sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"],
                            top_p=s["top_p"], min_p=s["min_p"], logprob=s["logprob"])
        return {"token": s["token"], "logprob": s["logprob"]}
    L = s["layer"]
    if op == "bin":
        if c["records"]:
            L.bin_records(s["count"], s["step"], s["neuron"], s["y"], factor=c["factor"])
        else:
            L.bin_spikes(s["offsets"], s["step"], s["neuron"], s["y"], factor=c["factor"])
        return s["y"]
    if op == "pack":
        q, y = snn.Packed.like(s["x"]), torch.empty_like(s["x"])
        L.pack(s["x"], q)
        L.unpack(q, y)
        return {"scale": q.scale, "x": y}
    if op == "conv_step":
        y, state = torch.empty(c["B"], c["C"], dtype=s["x"].dtype, device="cuda"), torch.empty_like(s["state"])
        L.conv_step(s["x"], s["w"], s["bias"], s["state"], state, y)
        return {"y": y, "state": state}
    if op in ("conv", "conv_packed"):
        y, dx = torch.empty_like(s["dy"]), torch.empty_like(s["dy"])
        dw, dbias = torch.empty_like(s["w"]), torch.empty_like(s["bias"])
        x = s["x"]
        L.conv_forward(x, s["w"], s["bias"], y, lengths=s["lengths"])
        if op == "conv_packed":
            x = snn.Packed.like(x)
            L.pack(s["x"], x)
        L.conv_backward(x, s["w"], s["bias"], s["dy"], dx, dw, dbias, lengths=s["lengths"])
        return {"y": y, "dx": dx, "dw": dw, "dbias": dbias}
    if op == "scan_step":
        y, h = torch.empty_like(s["u"]), torch.empty_like(s["h"])
        L.scan_step(s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["h"], h, y, D=s["D"], z=s["z"], delta_bias=s["delta_bias"])
        return {"y": y, "h": h}
    u, delta, z = s["u"], s["delta"], s["z"]
    # the states of packed activations are computed again with them
    saved = torch.empty(L.saved_shape, device="cuda") if "dy" in s and op != "scan_packed" else None
    out = {"y": torch.empty_like(u), "h": torch.empty_like(s["h0"])}
    L.scan_forward(u, delta, s["A"], s["Bm"], s["Cm"], out["y"], D=s["D"], z=z, delta_bias=s["delta_bias"], h0=s["h0"],
                   hT=out["h"], saved=saved, lengths=s["lengths"])
    if "dy" not in s:
        return out
    if op == "scan_packed":
        u, delta, z = (snn.Packed.like(x) for x in (u, delta, z))
        for x, q in ((s["u"], u), (s["delta"], delta), (s["z"], z)):
            L.pack(x, q)
    act = s["dy"].dtype
    dB = torch.empty(c["B"], c["T"], c["G"] * c["N"], dtype=act, device="cuda")
    out.update(du=torch.empty_like(s["dy"]), ddelta=torch.empty_like(s["dy"]), dB=dB, dC=torch.empty_like(dB),
               dA=torch.empty_like(s["A"]), dD=torch.empty_like(s["D"]), ddelta_bias=torch.empty_like(s["D"]),
               dh0=torch.empty_like(s["h0"]))
    if z is not None:
        out["dz"] = torch.empty_like(s["dy"])
    L.scan_backward(u, delta, s["A"], s["Bm"], s["Cm"], s["dy"], saved, out["du"], out["ddelta"], out["dA"], out["dB"],
                    out["dC"], D=s["D"], z=z, delta_bias=s["delta_bias"], dD=out["dD"], dz=out.get("dz"),
                    ddelta_bias=out["ddelta_bias"], h0=s["h0"], dh0=out["dh0"], lengths=s["lengths"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c, op = case, case["op"]
    e = 4 if c["dtype"] == F32 else 2
    if op == "sample":
        n = c["rows"] * c["V"]
        return {"bytes": n * e + 28 * c["rows"], "flops": 4 * n}
    if op == "bin":
        spikes = int(c["B"] * c["T"] * c["C"] * c["rate"])
        return {"bytes": 8 * spikes + e * c["B"] * -(-c["T"] // c["factor"]) * c["C"], "flops": spikes}
    rows = c["B"] * c.get("T", 1)
    n = rows * c["C"]
    if op == "pack":
        return {"bytes": n * (2 * e + 2) + 8 * rows * -(-c["C"] // BLOCK), "flops": 4 * n}
    if op == "conv_step":
        return {"bytes": n * e * 2 * c["K"] + c["C"] * 4 * (c["K"] + 1), "flops": n * (2 * c["K"] + 6)}
    if op in ("conv", "conv_packed"):
        # x and dy in, y and dx out; the packed form is written and read
        return {"bytes": n * (4 * e + (2 if op == "conv_packed" else 0)) + 8 * c["C"] * (c["K"] + 1),
                "flops": n * (8 * c["K"] + 24)}
    N, gate = c["N"], bool(c.get("gate", True))
    state = c["B"] * c["C"] * N * 4
    small = c["C"] * (N + 2) * 4
    if op == "scan_step":
        return {"bytes": n * e * (3 + gate) + 2 * rows * c["G"] * N * e + 2 * state + small, "flops": n * (7 * N + 20)}
    groups = 2 * rows * c["G"] * N * e
    forward = {"bytes": n * e * (3 + gate) + groups + 2 * state + small, "flops": n * (7 * N + 20)}
    if op == "scan" and not c["train"]:
        return forward
    # dy in, du, ddelta and dz out, the gradients of B, C, the first state and the parameters
    back = {"bytes": n * e * (3 + gate) + groups + state + small, "flops": n * (20 * N + 40)}
    return {"bytes": forward["bytes"] + back["bytes"] + (6 * n if op == "scan_packed" else 0),
            "flops": forward["flops"] + back["flops"]}


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_scan(s, u, delta, z, forward, backward):
    """Step by step along the time axis, one state at a time."""
    c = s["case"]
    B, T, C, G, N = c["B"], c["T"], c["C"], c["G"], c["N"]
    f64 = dict(dtype=torch.float64, device="cuda")
    A, D, bias = s["A"].double(), s["D"].double(), s["delta_bias"].double()
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    h = s["h0"].double()
    y0 = torch.zeros(B, T, C, **f64)
    kept = torch.zeros(T, B, C, N, **f64) if backward else None
    out = {}

    def at(t):
        live = (t < length)[:, None]
        ut, dt_ = u[:, t].double(), torch.logaddexp(torch.zeros((), **f64), delta[:, t].double() + bias)
        bt = s["Bm"][:, t].double().reshape(B, G, 1, N).expand(B, G, C // G, N).reshape(B, C, N)
        ct = s["Cm"][:, t].double().reshape(B, G, 1, N).expand(B, G, C // G, N).reshape(B, C, N)
        return live, ut, dt_, bt, ct

    for t in range(T):
        live, ut, dt_, bt, ct = at(t)
        if backward:
            kept[t] = h
        nxt = torch.exp(dt_[..., None] * A) * h + (dt_ * ut)[..., None] * bt
        h = torch.where(live[..., None], nxt, h)
        y0[:, t] = torch.where(live, (ct * h).sum(-1) + D * ut, 0.0)
    mask = (torch.arange(T, device="cuda")[None, :] < length[:, None])[..., None]
    zz = torch.where(mask, z.double(), 0.0) if z is not None else None
    if forward:
        out["y"] = y0 * (zz * torch.sigmoid(zz)) if z is not None else y0
        out["h"] = h
    if not backward:
        return out
    dy = torch.where(mask, s["dy"].double(), 0.0)
    if z is not None:
        p = torch.sigmoid(zz)
        out["dz"] = dy * y0 * (p + zz * p * (1.0 - p))
        dy = dy * zz * p
    for k in ("du", "ddelta"):
        out[k] = torch.zeros(B, T, C, **f64)
    for k in ("dB", "dC"):
        out[k] = torch.zeros(B, T, G * N, **f64)
    dA, dD = torch.zeros(C, N, **f64), torch.zeros(C, **f64)
    g = torch.zeros(B, C, N, **f64)
    for t in reversed(range(T)):
        live, ut, dt_, bt, ct = at(t)
        a = torch.exp(dt_[..., None] * A)
        ht = a * kept[t] + (dt_ * ut)[..., None] * bt
        gt = torch.where(live[..., None], g + dy[:, t, :, None] * ct, 0.0)
        out["dC"][:, t] = torch.where(live[..., None], dy[:, t, :, None] * ht, 0.0).view(B, G, C // G, N).sum(2).view(B, G * N)
        out["dB"][:, t] = (gt * (dt_ * ut)[..., None]).view(B, G, C // G, N).sum(2).view(B, G * N)
        ga = gt * a * kept[t]
        dA += (ga * dt_[..., None]).sum(0)
        dD += torch.where(live, dy[:, t] * ut, 0.0).sum(0)
        gb = (gt * bt).sum(-1)
        out["du"][:, t] = torch.where(live, D * dy[:, t] + dt_ * gb, 0.0)
        out["ddelta"][:, t] = ((ga * A).sum(-1) + ut * gb) * torch.sigmoid(delta[:, t].double() + bias)
        g = torch.where(live[..., None], a * gt, g)
    out.update(dA=dA, dD=dD, ddelta_bias=out["ddelta"].sum((0, 1)), dh0=g)
    return out


def _exact_conv(s, x):
    c = s["case"]
    B, T, C, K = c["B"], c["T"], c["C"], c["K"]
    w = s["w"].double()
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    ok = (torch.arange(T, device="cuda")[None, :] < length[:, None])[..., None]
    x = torch.where(ok, x.double(), 0.0)
    pre = s["bias"].double().expand(B, T, C).clone()
    for k in range(min(K, T)):                     # the tap that looks k steps back
        pre[:, k:] += w[:, K - 1 - k] * x[:, :T - k]
    p = torch.sigmoid(pre)
    dpre = torch.where(ok, s["dy"].double() * (p + pre * p * (1.0 - p)), 0.0)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for k in range(min(K, T)):
        dx[:, :T - k] += w[:, K - 1 - k] * dpre[:, k:]
        dw[:, K - 1 - k] = (dpre[:, k:] * x[:, :T - k]).sum((0, 1))
    return {"y": torch.where(ok, pre * p, 0.0), "dx": torch.where(ok, dx, 0.0), "dw": dw, "dbias": dpre.sum((0, 1))}


def _exact_pack(x):
    """The nearest e4m3 value (ties to the even one) of each x over its block's scale, by searching the sorted values."""
    B, T, C = x.shape
    code = torch.arange(127, device="cuda")
    mant, exp = (code % 8).double(), (code // 8).double()
    grid = torch.where(exp == 0, mant * 2.0 ** -9, (1.0 + mant / 8.0) * torch.exp2(exp - 7.0))
    x = x.double()
    pad = torch.cat([x, torch.zeros(B, T, -C % BLOCK, dtype=torch.float64, device="cuda")], 2).view(B, T, -1, BLOCK)
    top = pad.abs().amax(-1)
    k = torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0))
    k = torch.where(torch.exp2(k) * 448.0 < top, k + 1, k)
    k = torch.where((torch.exp2(k - 1) * 448.0 >= top) & (top > 0), k - 1, k)
    scale = torch.exp2(k)
    v = pad.abs() / scale[..., None]
    hi = torch.searchsorted(grid, v.contiguous()).clamp(1, 126)
    low, high = grid[hi - 1], grid[hi]
    up = (v - low > high - v) | ((v - low == high - v) & (hi % 2 == 0))
    v = torch.where(up, high, low) * torch.sign(pad) * scale[..., None]
    return v.view(B, T, -1)[:, :, :C], scale


def _exact_sample(s):
    """The answers' log-probabilities, from the row's values in falling order."""
    z = s["logits"].double()
    R, V = z.shape
    val, idx = torch.sort(z, dim=1, descending=True, stable=True)
    p = torch.softmax(val / s["temperature"].double()[:, None], 1)
    rank = torch.arange(V, device=z.device).expand(R, V)
    inside = torch.cat([torch.zeros(R, 1, dtype=torch.float64, device=z.device), torch.cumsum(p, 1)[:, :-1]], 1)
    out = (rank >= s["top_k"][:, None]) & (s["top_k"] > 0)[:, None]
    out |= (inside >= s["top_p"].double()[:, None]) & (s["top_p"] < 1.0)[:, None]
    out |= (p < s["min_p"].double()[:, None] * p[:, :1]) | torch.isinf(val)
    p = torch.where(out, 0.0, p)
    by_index = torch.zeros_like(p).scatter_(1, idx, p)
    share = by_index / by_index.sum(1, keepdim=True)
    token = (torch.cumsum(share, 1) <= s["u"].double()[:, None]).sum(1).clamp(max=V - 1)
    none = torch.isinf(val[:, 0])
    return {"token": None, "logprob": torch.where(none, -math.inf, torch.log(torch.gather(share, 1, token[:, None])[:, 0]))}


def _exact_bin(s):
    c = s["case"]
    B, S, C = c["B"], -(-c["T"] // c["factor"]), c["C"]
    n = s["count"].tolist() if c["records"] else (s["offsets"][1:] - s["offsets"][:-1]).tolist()
    rows = []
    for b in range(B):
        at = slice(0, n[b]) if c["records"] else slice(sum(n[:b]), sum(n[:b + 1]))
        step, neuron = (s[k][b] if c["records"] else s[k] for k in ("step", "neuron"))
        bins = torch.div(step[at].long(), c["factor"], rounding_mode="floor") * C + neuron[at].long()
        rows.append(torch.bincount(bins, minlength=S * C).view(S, C))
    return torch.stack(rows).double()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "bin":
        return _exact_bin(s)
    if op == "sample":
        return _exact_sample(s)
    if op == "pack":
        v, scale = _exact_pack(s["x"])
        return {"scale": scale, "x": v}
    if op == "conv":
        return _exact_conv(s, s["x"])
    if op == "conv_packed":
        return dict(_exact_conv(s, _exact_pack(s["x"])[0]), y=_exact_conv(s, s["x"])["y"])
    if op == "conv_step":
        x, K = s["x"].double(), case["K"]
        pre = s["bias"].double() + s["w"][:, K - 1].double() * x
        for k in range(K - 1):
            pre = pre + s["w"][:, k].double() * s["state"][:, k].double()
        return {"y": pre * torch.sigmoid(pre), "state": torch.cat([s["state"], s["x"][:, None]], 1)[:, 1:].double()}
    if op == "scan":
        return _exact_scan(s, s["u"], s["delta"], s["z"], True, case["train"])
    if op == "scan_packed":
        f = _exact_scan(s, s["u"], s["delta"], s["z"], True, False)
        return dict(f, **_exact_scan(s, *(_exact_pack(s[k])[0] for k in ("u", "delta", "z")), False, True))
    G, per = case["G"], case["C"] // case["G"]
    u, d = s["u"].double(), torch.logaddexp(torch.zeros((), dtype=torch.float64, device="cuda"),
                                            s["delta"].double() + s["delta_bias"].double())
    Bc, Cc = (s[k].double().reshape(-1, G, 1, case["N"]).expand(-1, G, per, case["N"]).reshape(-1, G * per, case["N"])
              for k in ("Bm", "Cm"))
    h = torch.exp(d[..., None] * s["A"].double()) * s["h"].double() + (d * u)[..., None] * Bc
    y = (h * Cc).sum(-1) + s["D"].double() * u
    z = s["z"].double() if s["z"] is not None else None
    return {"y": y * z * torch.sigmoid(z) if z is not None else y, "h": h}
