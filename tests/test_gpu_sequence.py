"""The sequence operators (include/snn_seq.h, paper_2501_07331_amd.SequenceLayer)
against their fp64 oracle.

Tolerances.  An output of type t is rounded once: eps_t / 2 of its value.
Before that it is an fp32 sum of products along a chain of at most n roundings,
each at most 2^-24 of a partial result, which the sum of the terms' absolute
values (the oracle's ``absolute`` run) bounds: n 2^-24 of that.  A decay
exp(x) counts |x| / ln 2 roundings more, from its argument; |x| stays below 16
here.  Values below the smallest normal fp16 are rounded to 2^-25.
"""
import numpy as np
import pytest

from oracle import sequence as seq

pytestmark = pytest.mark.gpu

TYPES = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def _torch():
    import torch
    return torch


def _dev(x, dtype="float32", strided=False, behind=None):
    """x on the GPU; strided: the middle of a wider tensor; behind: lengths past which NaN stands."""
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype))
    if behind is not None:
        for b, n in enumerate(behind):
            t[b, max(0, n):] = float("nan")
    t = t.cuda()
    if strided:
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 5), float("nan"), dtype=t.dtype, device="cuda")
        wide[..., 3:3 + t.shape[-1]] = t
        t = wide[..., 3:3 + t.shape[-1]]
    return t


def _cast(x, dtype):
    """x rounded to a type, in fp64."""
    torch = _torch()
    return torch.from_numpy(np.ascontiguousarray(x)).to(getattr(torch, dtype)).double().numpy()


class Out:
    """An output inside a wider buffer whose other values must stay (768: a value of every type)."""

    def __init__(self, shape, dtype="float32", strided=False):
        torch = _torch()
        pad = 7 if strided else 0
        self.wide = torch.full((*shape[:-1], shape[-1] + pad), 768.0, dtype=getattr(torch, dtype), device="cuda")
        self.t = self.wide[..., 2:2 + shape[-1]] if strided else self.wide
        if pad:
            self.t.fill_(float("nan"))

    def get(self):
        w = self.wide.double().cpu().numpy()
        if self.wide.shape != self.t.shape:
            n = self.t.shape[-1]
            assert (w[..., :2] == 768.0).all() and (w[..., 2 + n:] == 768.0).all()
            return w[..., 2:2 + n]
        return w


def _close(name, got, ref, size, dtype, n):
    assert got.shape == ref.shape, name
    tol = TYPES[dtype] * np.abs(ref) + n * 2.0 ** -24 * size + (2.0 ** -25 if dtype == "float16" else 2.0 ** -126)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.abs(got - ref)[bad][:4], tol[bad][:4], ref[bad][:4])


def _layer(B, T, C, **kw):
    import paper_2501_07331_amd as snn
    print(f"[seq] B={B} T={T} C={C} {kw}", flush=True)
    return snn.SequenceLayer(B, T, C, **kw)


def _len(lengths, T):
    return None if lengths is None else _torch().tensor(lengths, dtype=_torch().int32, device="cuda")


# ------------------------------------------------------------------ convolution

CONV = [
    # B, T, C, K, dtype, lengths, state, silu, strided
    (1, 1, 1, 1, "float32", None, False, True, False),
    (2, 5, 3, 4, "float32", None, True, True, True),
    (3, 40, 130, 4, "bfloat16", [40, 0, 2], True, True, True),
    (2, 300, 65, 3, "float16", [299, 17], False, True, False),
    (2, 17, 256, 8, "float32", [3, 99], True, False, True),
    (3, 33, 24, 2, "bfloat16", [1, -4, 33], True, False, False),
    (1, 520, 16, 5, "float32", None, False, True, False),
    (2, 19, 9, 6, "float16", None, True, True, True),
    (2, 16, 8, 7, "bfloat16", [16, 5], True, True, False),
]


@pytest.mark.parametrize("B,T,C,K,dtype,lengths,state,silu,strided", CONV)
@pytest.mark.parametrize("packed", [False, True])
def test_conv(B, T, C, K, dtype, lengths, state, silu, strided, packed):
    import paper_2501_07331_amd as snn
    r = np.random.default_rng(B * 1000 + T + K)
    x, dy = _cast(r.normal(size=(B, T, C)), dtype), _cast(r.normal(size=(B, T, C)), dtype)
    w, bias = _cast(r.normal(size=(C, K)) * K ** -0.5, "float32"), _cast(r.normal(size=C), "float32")
    st = _cast(r.normal(size=(B, K - 1, C)), dtype) if state else None
    ds = _cast(r.normal(size=(B, K - 1, C)), dtype) if state else None
    L = _layer(B, T, C, taps=K, train=True)
    behind = None if lengths is None else [min(max(n, 0), T) for n in lengths]
    gx, gdy = _dev(x, dtype, strided, behind), _dev(dy, dtype, strided, behind)
    gw, gb, gst = _dev(w), _dev(bias), None if st is None else _dev(st, dtype)
    y, so = Out((B, T, C), dtype, strided), Out((B, K - 1, C), dtype) if K > 1 else None
    L.conv_forward(gx, gw, gb, y.t, lengths=_len(lengths, T), state=gst, state_out=so.t if so else None, silu=silu)
    ref = seq.conv(x, w, bias, lengths, st, silu)
    size = seq.conv(x, w, bias, lengths, st, silu, absolute=True)
    _close("y", y.get(), ref["y"], 1.1 * size["y"], dtype, K + 16)
    if so:
        assert np.array_equal(so.get(), ref["state_out"])
    if packed:
        q = snn.Packed.like(gx)
        L.pack(gx, q)
        gx = q
        code, scale = seq.pack(np.where(np.isfinite(x), x, 0))
        x = seq.unpack(code, scale)
        if behind is not None:       # the blocks behind a sample's end hold NaN
            for b, n in enumerate(behind):
                x[b, n:] = 0
    dx, dw, db, dst = Out((B, T, C), dtype, strided), Out((C, K)), Out((C,)), Out((B, K - 1, C), dtype) if K > 1 else None
    L.conv_backward(gx, gw, gb, gdy, dx.t, dw.t, db.t, lengths=_len(lengths, T), state=gst,
                    dstate_out=None if ds is None or K == 1 else _dev(ds, dtype), dstate=dst.t if dst else None, silu=silu)
    ref = seq.conv(x, w, bias, lengths, st, silu, dy, ds)
    size = seq.conv(x, w, bias, lengths, st, silu, dy, ds, absolute=True)
    _close("dx", dx.get(), ref["dx"], size["dx"], dtype, 2 * K + 32)
    _close("dw", dw.get(), ref["dw"], size["dw"], "float32", K + 32 + B * T)
    _close("dbias", db.get(), ref["dbias"], size["dbias"], "float32", K + 32 + B * T)
    if dst:
        _close("dstate", dst.get(), ref["dstate"], size["dstate"], dtype, 2 * K + 32)


@pytest.mark.parametrize("dtype,K", [("float32", 4), ("bfloat16", 2), ("float16", 8), ("float32", 1)])
def test_conv_steps_are_the_convolution(dtype, K):
    torch = _torch()
    r = np.random.default_rng(K)
    B, T, C = 3, 11, 37
    x, st = _cast(r.normal(size=(B, T, C)), dtype), _cast(r.normal(size=(B, K - 1, C)), dtype)
    w, bias = _cast(r.normal(size=(C, K)), "float32"), _cast(r.normal(size=C), "float32")
    L = _layer(B, T, C, taps=K)
    gx, gw, gb, state = _dev(x, dtype, True), _dev(w), _dev(bias), _dev(st, dtype)
    y, so = torch.empty(B, T, C, dtype=gx.dtype, device="cuda"), torch.empty_like(state)
    L.conv_forward(gx, gw, gb, y, state=state, state_out=so if K > 1 else None)
    for t in range(T):
        o = torch.empty(B, C, dtype=gx.dtype, device="cuda")
        L.conv_step(gx[:, t], gw, gb, state if K > 1 else None, state if K > 1 else None, o)
        assert torch.equal(o, y[:, t])
    assert torch.equal(state, so)


# ------------------------------------------------------------------ scan

SCAN = [
    # B, T, C, N, G, dtype, lengths, gate, plus, strided
    (1, 1, 1, 1, 1, "float32", None, True, True, False),
    (2, 17, 5, 3, 1, "float32", None, True, True, True),
    (3, 40, 6, 5, 3, "bfloat16", [40, 0, 16], True, True, True),
    (2, 33, 130, 16, 2, "float16", [31, 33], False, True, False),
    (2, 64, 70, 16, 1, "bfloat16", None, True, True, True),
    (1, 50, 20, 20, 1, "float32", [37], True, False, False),
    (2, 48, 33, 64, 1, "float32", [48, 1], False, True, True),
    (1, 300, 8, 8, 2, "float32", None, True, True, False),          # parts of the time axis
    (2, 200, 24, 12, 1, "bfloat16", [70, 200], True, True, True),   # a part behind a sample's end
    (1, 130, 3, 33, 1, "float16", None, True, True, True),
    (2, 96, 4, 4, 4, "float32", [64, -1], False, False, False),
    (1, 2300, 3, 4, 1, "float32", None, True, True, False),         # more parts than their workgroups join themselves
    (2, 2200, 2, 9, 1, "bfloat16", [2200, 1234], False, True, False),
]


def _scan_inputs(B, T, C, N, G, dtype, gate, plus, seed):
    r = np.random.default_rng(seed)
    v = dict(u=_cast(r.normal(size=(B, T, C)), dtype),
             delta=_cast(r.normal(size=(B, T, C)) if plus else r.uniform(0.01, 1.0, size=(B, T, C)), dtype),
             A=_cast(-r.uniform(0.02, 2.0, size=(C, N)), "float32"),
             Bm=_cast(r.normal(size=(B, T, G, N)), dtype), Cm=_cast(r.normal(size=(B, T, G, N)), dtype),
             D=_cast(r.normal(size=C), "float32"), z=_cast(r.normal(size=(B, T, C)), dtype) if gate else None,
             delta_bias=_cast(r.uniform(-3, 1, size=C) if plus else r.uniform(0, 0.2, size=C), "float32"),
             h0=_cast(r.normal(size=(B, C, N)), "float32"))
    return v, _cast(r.normal(size=(B, T, C)), dtype), _cast(r.normal(size=(B, C, N)), "float32")


def _run_scan(L, v, dy, dhT, dtype, lengths, plus, strided, recompute=False, packed=(), forward=True):
    """(forward outputs, gradients) of the library."""
    import paper_2501_07331_amd as snn
    torch = _torch()
    B, T, C = v["u"].shape
    G, N = v["Bm"].shape[2:]
    behind = None if lengths is None else [min(max(n, 0), T) for n in lengths]
    g = {k: _dev(v[k], dtype, strided, behind) if v[k] is not None else None for k in ("u", "delta", "z")}
    for k in ("Bm", "Cm"):
        g[k] = _dev(v[k].reshape(B, T, G * N), dtype, strided, behind)
    g.update({k: _dev(v[k]) for k in ("A", "D", "delta_bias", "h0")})
    gdy = _dev(dy, dtype, strided, behind)
    gl = _len(lengths, T)
    y, hT = Out((B, T, C), dtype, strided), Out((B, C, N))
    saved = None if recompute else torch.full(L.saved_shape, float("nan"), device="cuda")
    opt = dict(D=g["D"], z=g["z"], delta_bias=g["delta_bias"], lengths=gl, softplus=plus)
    L.scan_forward(g["u"], g["delta"], g["A"], g["Bm"], g["Cm"], y.t, h0=g["h0"], hT=hT.t, saved=saved, **opt)
    for k in packed:
        q = snn.Packed.like(g[k])
        L.pack(g[k], q)
        g[k] = q
    opt["z"] = g["z"]
    o = {k: Out((B, T, C), dtype, strided) for k in ("du", "ddelta")}
    o.update({k: Out((B, T, G * N), dtype, strided) for k in ("dB", "dC")})
    o.update(dA=Out((C, N)), dD=Out((C,)), ddelta_bias=Out((C,)), dh0=Out((B, C, N)))
    if v["z"] is not None:
        o["dz"] = Out((B, T, C), dtype, strided)
    L.scan_backward(g["u"], g["delta"], g["A"], g["Bm"], g["Cm"], gdy, saved, o["du"].t, o["ddelta"].t, o["dA"].t,
                    o["dB"].t, o["dC"].t, dD=o["dD"].t, dz=o["dz"].t if "dz" in o else None,
                    ddelta_bias=o["ddelta_bias"].t, h0=g["h0"] if recompute else None, dhT=_dev(dhT), dh0=o["dh0"].t, **opt)
    return {"y": y.get(), "hT": hT.get()}, {k: x.get() for k, x in o.items()}


def _check_scan(got, ref, size, B, T, C, G, N, dtype):
    n = 32 * T + 64
    for k, x in got.items():
        whole = k in ("hT", "dA", "dD", "ddelta_bias", "dh0")
        r, s = (ref[k], size[k]) if x.ndim == ref[k].ndim else (ref[k].reshape(x.shape), size[k].reshape(x.shape))
        _close(k, x, r, s, "float32" if whole else dtype, 2 * n + C + B * T)


@pytest.mark.parametrize("B,T,C,N,G,dtype,lengths,gate,plus,strided", SCAN)
@pytest.mark.parametrize("recompute", [False, True])
def test_scan(B, T, C, N, G, dtype, lengths, gate, plus, strided, recompute):
    v, dy, dhT = _scan_inputs(B, T, C, N, G, dtype, gate, plus, B * 1000 + T + N)
    L = _layer(B, T, C, state=N, groups=G, train=True, recompute=recompute)
    fwd, grad = _run_scan(L, v, dy, dhT, dtype, lengths, plus, strided, recompute)
    ref = seq.scan(**v, lengths=lengths, plus=plus, dy=dy, dhT=dhT)
    size = seq.scan(**v, lengths=lengths, plus=plus, dy=dy, dhT=dhT, absolute=True)
    _check_scan(dict(fwd, **grad), ref, size, B, T, C, G, N, dtype)


@pytest.mark.parametrize("packed", [("u", "delta", "z"), ("delta",), ("z",)])
@pytest.mark.parametrize("dtype,lengths", [("float16", None), ("bfloat16", [70, 35]), ("float32", [20, 70])])
@pytest.mark.parametrize("C,N,G", [(150, 16, 1), (402, 24, 3), (273, 3, 1), (258, 7, 2), (129, 40, 1)])
def test_scan_from_packed_activations(packed, dtype, lengths, C, N, G):
    """Among them groups that start inside a block of 128, so that a vector of channels has two scales."""
    B, T = 2, 70
    v, dy, dhT = _scan_inputs(B, T, C, N, G, dtype, True, True, 9)
    L = _layer(B, T, C, state=N, groups=G, train=True, recompute=True)
    _, grad = _run_scan(L, v, dy, dhT, dtype, lengths, True, True, True, packed)
    for k in packed:
        v[k] = seq.unpack(*seq.pack(v[k]))
    ref = seq.scan(**v, lengths=lengths, dy=dy, dhT=dhT)
    size = seq.scan(**v, lengths=lengths, dy=dy, dhT=dhT, absolute=True)
    _check_scan(grad, ref, size, B, T, C, G, N, dtype)


@pytest.mark.parametrize("N,dtype,recompute", [(16, "bfloat16", False), (16, "float32", True), (8, "float16", True),
                                               (3, "float32", False), (30, "bfloat16", True)])
def test_scan_of_a_batch_that_fills_the_chip(N, dtype, recompute):
    """Enough rows for an undivided time axis, of many tiles: a thousand copies of two samples, whose outputs are
    theirs and whose parameter gradients are five hundred times their sums."""
    torch = _torch()
    B, T, C, copies = 2, 90, 70, 512
    v, dy, dhT = _scan_inputs(B, T, C, N, 1, dtype, True, True, N)
    rep = lambda x: np.tile(x, (copies,) + (1,) * (x.ndim - 1))     # noqa: E731
    many = {k: rep(x) if k in ("u", "delta", "Bm", "Cm", "z", "h0") else x for k, x in v.items()}
    L = _layer(B * copies, T, C, state=N, train=True, recompute=recompute)
    lengths = [T, 77]
    fwd, grad = _run_scan(L, many, rep(dy), rep(dhT), dtype, lengths * copies, True, False, recompute)
    ref = seq.scan(**v, lengths=lengths, dy=dy, dhT=dhT)
    size = seq.scan(**v, lengths=lengths, dy=dy, dhT=dhT, absolute=True)
    got = dict(fwd, **grad)
    for k in got:
        if k in ("dA", "dD", "ddelta_bias"):
            got[k] = got[k] / copies
        else:
            assert np.array_equal(got[k][:B], got[k][-B:]), k
            got[k] = got[k][B:2 * B]
    _check_scan(got, ref, size, B * copies, T, C, 1, N, dtype)


def test_offsets_past_32_bits():
    """Samples 2^30 elements apart: the third one's offsets pass 2^31 elements."""
    torch = _torch()
    B, T, C, N, far = 3, 40, 16, 4, 2 ** 30 + 8
    v, dy, dhT = _scan_inputs(B, T, C, N, 1, "bfloat16", True, True, 21)
    wide = torch.empty(2 * far + 8 * T * C, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(wide)
    place = iter(range(8))

    def at(x, buf=wide):
        n = x.shape[-1]
        t = buf[next(place) * T * C:].as_strided((B, T, n), (far, n, 1))
        t.copy_(torch.from_numpy(np.ascontiguousarray(x.reshape(B, T, n))).bfloat16())
        return t

    u, delta, z, gdy, Bm, Cm = (at(x) for x in (v["u"], v["delta"], v["z"], dy, v["Bm"], v["Cm"]))
    A, D, bias, h0 = (_dev(v[k]) for k in ("A", "D", "delta_bias", "h0"))
    place = iter(range(8))
    nan = np.full((B, T, C), np.nan)
    y, du, dd, dz, cy, cdx = (at(nan, out) for _ in range(6))
    dB, dC = at(nan[:, :, :N], out), at(nan[:, :, :N], out)
    L = _layer(B, T, C, state=N, taps=4, train=True)
    saved, hT = torch.empty(L.saved_shape, device="cuda"), torch.empty(B, C, N, device="cuda")
    dA, dD, db, dh0 = (torch.empty_like(x) for x in (A, D, bias, h0))
    opt = dict(D=D, z=z, delta_bias=bias)
    L.scan_forward(u, delta, A, Bm, Cm, y, h0=h0, hT=hT, saved=saved, **opt)
    L.scan_backward(u, delta, A, Bm, Cm, gdy, saved, du, dd, dA, dB, dC, dD=dD, dz=dz, ddelta_bias=db, dhT=_dev(dhT),
                    dh0=dh0, **opt)
    got = {k: x.double().cpu().numpy() for k, x in dict(y=y, hT=hT, du=du, ddelta=dd, dz=dz, dB=dB, dC=dC, dA=dA, dD=dD,
                                                        ddelta_bias=db, dh0=dh0).items()}
    ref, size = seq.scan(**v, dy=dy, dhT=dhT), seq.scan(**v, dy=dy, dhT=dhT, absolute=True)
    _check_scan(got, ref, size, B, T, C, 1, N, "bfloat16")
    w, dw = _dev(np.random.default_rng(1).normal(size=(C, 4))), torch.empty(C, 4, device="cuda")
    L.conv_forward(u, w, None, cy)
    L.conv_backward(u, w, None, gdy, cdx, dw)
    hw = w.double().cpu().numpy()
    ref, size = seq.conv(v["u"], hw, dy=dy), seq.conv(v["u"], hw, dy=dy, absolute=True)
    _close("y", cy.double().cpu().numpy(), ref["y"], 1.1 * size["y"], "bfloat16", 20)
    _close("dx", cdx.double().cpu().numpy(), ref["dx"], size["dx"], "bfloat16", 40)


def test_scan_without_what_may_be_left_out():
    torch = _torch()
    B, T, C, N = 2, 20, 9, 4
    v, dy, _ = _scan_inputs(B, T, C, N, 1, "float32", False, True, 2)
    v.update(D=None, delta_bias=None, h0=None)
    L = _layer(B, T, C, state=N, train=True)
    u, delta, A, Bm, Cm, gdy = (_dev(x) for x in (v["u"], v["delta"], v["A"], v["Bm"].reshape(B, T, N),
                                                  v["Cm"].reshape(B, T, N), dy))
    y, saved = torch.empty_like(u), torch.empty(L.saved_shape, device="cuda")
    L.scan_forward(u, delta, A, Bm, Cm, y, saved=saved)
    o = {k: torch.empty_like(t) for k, t in dict(du=u, ddelta=u, dA=A, dB=Bm, dC=Cm).items()}
    L.scan_backward(u, delta, A, Bm, Cm, gdy, saved, **o)
    ref, size = seq.scan(**v, dy=dy), seq.scan(**v, dy=dy, absolute=True)
    got = {k: x.double().cpu().numpy() for k, x in dict(o, y=y).items()}
    _check_scan(got, ref, size, B, T, C, 1, N, "float32")


@pytest.mark.parametrize("dtype,N,G", [("float32", 16, 1), ("bfloat16", 5, 3), ("float16", 64, 1), ("float32", 4, 2)])
def test_scan_steps_and_parts_are_the_scan(dtype, N, G):
    """One step at a time, and a sequence in two calls, from the state of the one before."""
    torch = _torch()
    B, T, C = 2, 21, 12
    v, _, _ = _scan_inputs(B, T, C, N, G, dtype, True, True, N)
    ref, size = seq.scan(**v), seq.scan(**v, absolute=True)
    L, first, rest = _layer(B, T, C, state=N, groups=G), _layer(B, 8, C, state=N, groups=G), _layer(B, T - 8, C, state=N, groups=G)
    u, delta, z = (_dev(v[k], dtype, True) for k in ("u", "delta", "z"))
    Bm, Cm = (_dev(v[k].reshape(B, T, G * N), dtype, True) for k in ("Bm", "Cm"))
    A, D, bias, h = (_dev(v[k]) for k in ("A", "D", "delta_bias", "h0"))
    h2, y = h.clone(), torch.empty(B, T, C, dtype=u.dtype, device="cuda")
    for t in range(T):
        o = torch.empty(B, C, dtype=u.dtype, device="cuda")
        L.scan_step(u[:, t], delta[:, t], A, Bm[:, t], Cm[:, t], h, h, o, D=D, z=z[:, t], delta_bias=bias)
        y[:, t] = o
    _close("y", y.double().cpu().numpy(), ref["y"], size["y"], dtype, 32 * T + 64)
    _close("h", h.double().cpu().numpy(), ref["hT"], size["hT"], "float32", 32 * T + 64)
    mid, end = torch.empty_like(h2), torch.empty_like(h2)
    first.scan_forward(u[:, :8], delta[:, :8], A, Bm[:, :8], Cm[:, :8], y[:, :8], D=D, z=z[:, :8], delta_bias=bias, h0=h2, hT=mid)
    rest.scan_forward(u[:, 8:], delta[:, 8:], A, Bm[:, 8:], Cm[:, 8:], y[:, 8:], D=D, z=z[:, 8:], delta_bias=bias, h0=mid, hT=end)
    _close("y", y.double().cpu().numpy(), ref["y"], size["y"], dtype, 32 * T + 64)
    _close("h", end.double().cpu().numpy(), ref["hT"], size["hT"], "float32", 32 * T + 64)


@pytest.mark.parametrize("T", [700, 4000])
def test_states_that_grow_from_zero(T):
    """exp(A sum delta') over a part of the time axis overflows, and what it multiplies is zero: the states before the
    inputs begin, the adjoints behind the last gradient.  Four steps of decays with 4.7 roundings of their argument and
    four more each, sums over 5 states and 40 channels: 128 roundings hold them."""
    torch = _torch()
    B, C, N = 1, 40, 5
    r = np.random.default_rng(T)
    f = lambda *s: torch.from_numpy(r.normal(size=s)).float()           # noqa: E731
    L = _layer(B, T, C, state=N, train=True)
    A = torch.from_numpy(r.uniform(2.8, 3.2, size=(C, N))).float()
    A[::2] *= -1
    u, dy, zero = torch.zeros(B, T, C), torch.zeros(B, T, C), torch.zeros(B, T, C)
    u[:, -4:], dy[:, :3], delta = f(B, 4, C), f(B, 3, C), torch.ones(B, T, C)
    Bm, Cm = f(B, T, N), f(B, T, N)
    g = {k: x.cuda() for k, x in dict(u=u, dy=dy, zero=zero, delta=delta, A=A, B=Bm, C=Cm).items()}
    y, hT, saved = torch.empty(B, T, C, device="cuda"), torch.empty(B, C, N, device="cuda"), torch.empty(L.saved_shape, device="cuda")
    o = dict(du=torch.empty_like(y), ddelta=torch.empty_like(y), dA=torch.empty(C, N, device="cuda"),
             dB=torch.empty(B, T, N, device="cuda"), dC=torch.empty(B, T, N, device="cuda"))

    def oracle(u, dy=None):
        v = [x.double().numpy() for x in (u, delta, A, Bm.view(B, T, 1, N), Cm.view(B, T, 1, N))]
        return [seq.scan(*v, plus=False, dy=None if dy is None else dy.double().numpy(), absolute=x) for x in (False, True)]

    L.scan_forward(g["u"], g["delta"], g["A"], g["B"], g["C"], y, hT=hT, softplus=False)
    ref, size = oracle(u)
    for k, x in dict(y=y, hT=hT).items():
        _close(k, x.double().cpu().numpy(), ref[k], size[k], "float32", 128)
    L.scan_forward(g["zero"], g["delta"], g["A"], g["B"], g["C"], y, saved=saved, softplus=False)
    L.scan_backward(g["zero"], g["delta"], g["A"], g["B"], g["C"], g["dy"], saved, softplus=False, **o)
    ref, size = oracle(zero, dy)
    for k, x in o.items():
        _close(k, x.double().cpu().numpy(), ref[k].reshape(x.shape), size[k].reshape(x.shape), "float32", 128)


@pytest.mark.parametrize("order", ["time first", "broadcast"])
def test_strides_of_other_orders(order):
    """[T][B][n] memory, and inputs that all samples share: the same results as from [B][T][n], bit for bit."""
    torch = _torch()
    B, T, C, N = 3, 45, 24, 8
    t, outs = _train_tensors(B, T, C, N, 31)
    if order == "broadcast":
        for k in ("delta", "B", "C", "dy", "x"):
            t[k] = t[k][:1].expand(B, -1, -1).contiguous()
    L = _layer(B, T, C, state=N, train=True)
    t["saved"] = torch.empty(L.saved_shape, device="cuda")
    _train_step(L, t)
    other = dict(t)
    for k, v in t.items():
        if k == "saved" or v.dim() != 3 or v.shape[:2] != (B, T):
            other[k] = v if k not in outs else torch.empty_like(v)
        elif order == "time first":
            m = torch.empty(T, B, v.shape[2], dtype=v.dtype, device="cuda").transpose(0, 1)
            other[k] = m.copy_(v) if k not in outs else m
        else:
            other[k] = v[:1].expand(B, -1, -1) if k in ("delta", "B", "C", "dy", "x") else v if k not in outs else torch.empty_like(v)
    _train_step(L, other)
    for k in outs:
        assert torch.equal(t[k], other[k]), k


def test_scan_gradients_are_the_same_from_call_to_call():
    torch = _torch()
    B, T, C, N = 3, 90, 100, 16
    v, dy, dhT = _scan_inputs(B, T, C, N, 1, "bfloat16", True, True, 11)
    L = _layer(B, T, C, state=N, train=True)
    a = _run_scan(L, v, dy, dhT, "bfloat16", [90, 3, 55], True, False)
    torch.cuda.synchronize()
    b = _run_scan(L, v, dy, dhT, "bfloat16", [90, 3, 55], True, False)
    for x, y in zip(a, b):
        for k in x:
            assert np.array_equal(x[k], y[k]), k


# ------------------------------------------------------------------ packed form, counts


@pytest.mark.parametrize("dtype,n", [("float32", 1), ("float32", 300), ("bfloat16", 128), ("float16", 135), ("bfloat16", 1000)])
def test_pack_and_unpack(dtype, n):
    import paper_2501_07331_amd as snn
    torch = _torch()
    r = np.random.default_rng(n)
    x = r.normal(size=(2, 5, n)) * np.exp(r.normal(size=n) * (1 if dtype == "float16" else 6))
    x[0, 0] = 0.0
    x[0, 1, n // 2], x[1, 1, 0], x[1, 3, n - 1] = np.inf, np.nan, -np.inf
    x[1, 0] = np.where(r.random(n) < 0.5, 448.0, -17.0)
    x[1, 2] = 1e-41
    x = _cast(x, dtype)
    L = _layer(2, 5, 1)
    gx = _dev(x, dtype, True)
    q = snn.Packed.like(gx)
    L.pack(gx, q)
    code, scale = seq.pack(x)
    assert np.array_equal(q.scale.double().cpu().numpy(), scale)
    got = q.data.cpu().numpy()
    nan = code & 0x7F == 0x7F
    assert np.array_equal(got[~nan], code[~nan]) and (got[nan] & 0x7F == 0x7F).all()
    back = Out((2, 5, n), dtype, True)
    L.unpack(q, back.t)
    want = seq.unpack(code, scale)
    fine = ~nan
    v = back.get()
    assert np.isnan(v[nan]).all()
    assert (np.abs(v - want)[fine] <= np.abs(want)[fine] * TYPES[dtype] + (2.0 ** -25 if dtype == "float16" else 0)).all()


@pytest.mark.parametrize("B,T,n,factor,dtype", [(1, 1, 1, 1, "float32"), (3, 50, 700, 4, "bfloat16"), (2, 100, 9000, 7, "float16"),
                                                (4, 33, 130, 33, "float32"), (2, 1000, 20, 3, "bfloat16")])
def test_bin(B, T, n, factor, dtype):
    torch = _torch()
    r = np.random.default_rng(n)
    lists = []
    for b in range(B):
        hit = r.random((T, n)) < (0.0 if b == 1 else 0.1)
        s, c = np.nonzero(hit)
        lists.append((s, c))
    want = seq.bin_spikes(lists, T, n, factor)
    L = _layer(B, T, 1)
    i32 = lambda v: torch.from_numpy(np.asarray(v, np.int32)).cuda()   # noqa: E731
    off = np.concatenate([[0], np.cumsum([len(s) for s, _ in lists])])
    out = Out(want.shape, dtype, True)
    L.bin_spikes(i32(off), i32(np.concatenate([s for s, _ in lists])), i32(np.concatenate([c for _, c in lists])), out.t, factor)
    assert np.array_equal(out.get(), want)
    # records: a capacity that the last sample exceeds, stale entries behind each count
    cap = max(1, len(lists[-1][0]) - 2)
    step, neuron = np.zeros((B, cap), np.int32), np.zeros((B, cap), np.int32)
    for b, (s, c) in enumerate(lists):
        k = min(cap, len(s))
        step[b, :k], neuron[b, :k] = s[:k], c[:k]
    want = seq.bin_spikes([(s[:cap], c[:cap]) for s, c in lists], T, n, factor)
    out = Out(want.shape, dtype, True)
    L.bin_records(i32([len(s) for s, _ in lists]), i32(step), i32(neuron), out.t, factor)
    assert np.array_equal(out.get(), want)


def test_bin_leaves_out_events_outside():
    torch = _torch()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    L = _layer(1, 6, 1)
    out = torch.full((1, 3, 4), -1.0, device="cuda")
    L.bin_spikes(i32([0, 99]), i32([-3, 0, 1, 1, 5, 6, 70]), i32([0, 4, -1, 2, 3, 0, 1]), out, 2)
    want = torch.zeros(1, 3, 4, device="cuda")
    want[0, 0, 2] = want[0, 2, 3] = 1
    assert torch.equal(out, want)


# ------------------------------------------------------------------ streams, graphs, refusals


def _train_step(L, t):
    L.conv_forward(t["x"], t["w"], t["b"], t["u"], lengths=t["len"])
    L.scan_forward(t["u"], t["delta"], t["A"], t["B"], t["C"], t["y"], z=t["z"], saved=t["saved"], lengths=t["len"])
    L.scan_backward(t["u"], t["delta"], t["A"], t["B"], t["C"], t["dy"], t["saved"], t["du"], t["dd"], t["dA"], t["dB"],
                    t["dC"], z=t["z"], dz=t["dz"], lengths=t["len"])
    L.conv_backward(t["x"], t["w"], t["b"], t["du"], t["dx"], t["dw"], t["db"], lengths=t["len"])


def _train_tensors(B, T, C, N, seed):
    torch = _torch()
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    t = {k: f(B, T, C).bfloat16() for k in ("x", "delta", "z", "dy")}
    t.update(B=f(B, T, N).bfloat16(), C=f(B, T, N).bfloat16(), A=-torch.exp(f(C, N)), w=f(C, 4), b=f(C),
             len=torch.tensor([T] + [T // 2] * (B - 1), dtype=torch.int32, device="cuda"))
    outs = dict(u=t["x"], y=t["x"], du=t["x"], dd=t["x"], dz=t["x"], dx=t["x"], dA=t["A"], dB=t["B"], dC=t["C"], dw=t["w"], db=t["b"])
    t.update({k: torch.empty_like(v) for k, v in outs.items()})
    return t, list(outs)


def test_training_step_in_a_graph():
    """Captured once, replayed on new inputs with eager calls in between: every replay equals the eager result."""
    torch = _torch()
    B, T, C, N = 2, 150, 70, 16
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        L, E = _layer(B, T, C, state=N, train=True), _layer(B, T, C, state=N, train=True)
        t, outs = _train_tensors(B, T, C, N, 1)
        t["saved"] = torch.empty(L.saved_shape, device="cuda")
        _train_step(L, t)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            _train_step(L, t)
        for seed in (2, 3, 4):
            n, _ = _train_tensors(B, T, C, N, seed)
            n["saved"] = torch.empty(L.saved_shape, device="cuda")
            for k in n:
                if k not in outs and k != "saved":
                    t[k].copy_(n[k])
            for k in outs:
                t[k].fill_(float("nan"))
            graph.replay()
            _train_step(E, n)
            s.synchronize()
            for k in outs:
                assert torch.equal(t[k], n[k]), (seed, k)


def test_a_capture_on_another_stream_takes_the_handle_s_in():
    torch = _torch()
    B, T, C, N = 2, 64, 40, 16
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()
    L, E = _layer(B, T, C, state=N, train=True, stream=mine), _layer(B, T, C, state=N, train=True)
    t, outs = _train_tensors(B, T, C, N, 6)
    t["saved"] = torch.empty(L.saved_shape, device="cuda")
    _train_step(E, t)
    want = {k: t[k].clone() for k in outs}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        _train_step(L, t)
    for _ in range(3):
        for k in outs:
            t[k].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for k in outs:
            assert torch.equal(t[k], want[k]), k


def test_calls_under_another_stream_are_ordered():
    torch = _torch()
    B, T, C, N = 2, 64, 128, 16
    L = _layer(B, T, C, state=N, train=True)
    t, outs = _train_tensors(B, T, C, N, 5)
    t["saved"] = torch.empty(L.saved_shape, device="cuda")
    _train_step(L, t)
    want = {k: t[k].clone() for k in outs}
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        late = {k: torch.zeros_like(v) for k, v in t.items()}
        for k, v in t.items():          # the inputs are written on this stream, just before
            late[k].copy_(v)
        late["len"] = t["len"]
        _train_step(L, late)
        got = {k: late[k].clone() for k in outs}
    other.synchronize()
    for k in outs:
        assert torch.equal(got[k], want[k]), k


def test_default_stream_handles_refuse_a_capture():
    torch = _torch()
    L = _layer(1, 4, 8)
    if L.stream.cuda_stream != 0:
        pytest.skip("the current stream is not the default stream")
    s = torch.cuda.Stream()
    x, w = torch.zeros(1, 4, 8, device="cuda"), torch.zeros(8, 4, device="cuda")
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="default stream"):
        with torch.cuda.graph(graph, stream=s):
            L.conv_forward(x, w, None, y)
    torch.cuda.synchronize()


def test_refusals():
    import paper_2501_07331_amd as snn
    torch = _torch()
    B, T, C, N = 2, 10, 6, 4
    L = _layer(B, T, C, state=N, groups=2)
    f = lambda *s, **k: torch.zeros(*s, device="cuda", **k)   # noqa: E731
    x, w, y = f(B, T, C), f(C, 4), f(B, T, C)
    bc, A, st = f(B, T, 2 * N), f(C, N), f(B, C, N)
    saved = f(*L.saved_shape)
    grads = dict(du=f(B, T, C), ddelta=f(B, T, C), dA=f(C, N), dB=f(B, T, 2 * N), dC=f(B, T, 2 * N))
    q = snn.Packed.like(x)
    bad = [
        lambda: L.conv_forward(x[:, :5], w, None, y),                       # wrong number of steps
        lambda: L.conv_forward(x.double(), w, None, y),                     # a type that is not taken
        lambda: L.conv_forward(x.cpu(), w, None, y),                        # host memory
        lambda: L.conv_forward(x, w[:, :3], None, y),                       # not contiguous, wrong size
        lambda: L.conv_forward(x, w.double(), None, y),
        lambda: L.conv_forward(q, w, None, y),                              # packed where it is not taken
        lambda: L.conv_forward(x, w, None, y.bfloat16()),                   # two types in a call
        lambda: L.conv_forward(x, w, None, y, lengths=torch.zeros(B, dtype=torch.int64, device="cuda")),
        lambda: L.conv_forward(x, w, None, y[:1].expand(B, T, C)),          # an output's samples on one another
        lambda: L.conv_forward(x[:, :1].expand(B, T, C), w, None, y),       # steps on one another
        lambda: L.conv_forward(x.transpose(1, 2).contiguous().transpose(1, 2), w, None, y),
        lambda: L.conv_backward(x, w, None, x, y, f(C, 4)),                 # made without train
        lambda: L.scan_forward(x, x, A, bc[:, :, :N].contiguous(), bc, y),  # one group's B for two groups
        lambda: L.scan_forward(x, x, A, bc, bc, y, h0=st, hT=st),
        lambda: L.scan_forward(x, x, A, bc, bc, y, saved=saved.view(-1)[1:]),
        lambda: L.scan_forward(x, x, f(C, N + 1), bc, bc, y),
        lambda: L.scan_backward(x, x, A, bc, bc, x, saved, **grads),
        lambda: L.scan_step(x[:, 0], x[:, 0], A, bc[:, 0], bc[:, 0], None, None, y[:, 0]),
        lambda: L.bin_spikes(f(B, dtype=torch.int32), f(1, dtype=torch.int32), f(1, dtype=torch.int32), y),
        lambda: L.bin_spikes(f(B + 1, dtype=torch.int32), f(1, dtype=torch.int32), f(1, dtype=torch.int32), y, factor=0),
        lambda: L.bin_spikes(f(B + 1, dtype=torch.int32), f(1, dtype=torch.int32), f(1, dtype=torch.int32), y, factor=11),
        lambda: L.conv_forward(x, w, None, x),                              # in place
        lambda: L.scan_forward(x, x, A, bc, bc, x),
        lambda: L.scan_step(x[:, 0], x[:, 0], A, bc[:, 0], bc[:, 0], st, st, x[:, 0]),
        lambda: L.pack(x, x),
        lambda: L.pack(x, snn.Packed.like(f(B, T, C + 1))),
        lambda: snn.Packed(f(B, T, C, dtype=torch.uint8), f(B, T, 2)),
    ]
    R = _layer(B, T, C, state=N, groups=2, train=True)
    bad += [
        lambda: R.scan_backward(x, x, A, bc, bc, x, None, **grads),         # no states, and no memory for them
        lambda: R.scan_backward(x, x, A, bc, bc, x, saved, z=x, **grads),   # a gate without its gradient
        lambda: R.scan_backward(x, x, A, bc, bc, x, saved, dz=y, **grads),
        lambda: R.scan_backward(x, x, A, bc, bc, q, saved, **grads),
        lambda: R.scan_backward(x, x, A, bc, bc, x, saved, **dict(grads, ddelta=grads["du"])),      # two outputs in one
        lambda: R.scan_backward(x, x, A, bc, bc, x, saved, **dict(grads, dB=f(B, T, 2 * N).half())),
    ]
    for i, call in enumerate(bad):
        print(f"[seq] refusal {i}", flush=True)
        with pytest.raises((ValueError, snn.SNNError)):
            call()
    L.conv_forward(x, w, None, y)          # and the handle is fine
    torch.cuda.synchronize()
    for kw in (dict(state=65), dict(groups=4), dict(taps=9), dict(T=0), dict(batch=0), dict(channels=0), dict(state=0),
               dict(recompute=True)):
        with pytest.raises(snn.SNNError):
            snn.SequenceLayer(**dict(dict(batch=B, T=T, channels=C), **kw))


def test_outputs_that_are_inputs_and_sizes_past_a_launch_are_refused():
    import paper_2501_07331_amd as snn
    torch = _torch()
    B, T, C = 2, 10, 6
    L = _layer(B, T, C)
    x = torch.zeros(B, T, C, device="cuda")
    scale = torch.zeros(B, T, 1, device="cuda")
    same = snn.Packed(x.view(-1).view(torch.uint8)[:B * T * C].view(B, T, C), scale)
    onto = snn.Packed(torch.zeros(B, T, C, dtype=torch.uint8, device="cuda"), x.view(-1)[:B * T].view(B, T, 1))
    i32 = x.view(-1).view(torch.int32)
    ids = torch.zeros(60, dtype=torch.int32, device="cuda")
    R = snn.Sampler(4, 5)
    z, t = x.view(-1)[20:40].view(4, 5), torch.zeros(4, dtype=torch.int32, device="cuda")
    u = x.view(-1)[:4]
    bad = [lambda: L.pack(x, same), lambda: L.pack(x, onto), lambda: L.unpack(same, x), lambda: L.unpack(onto, x),
           lambda: L.bin_spikes(i32[:B + 1], ids, ids, x), lambda: L.bin_records(ids[:B], i32[:B].view(B, 1), ids[:B].view(B, 1), x),
           lambda: L.conv_forward(torch.ones_like(x), torch.zeros(C, 4, device="cuda"), None, x, lengths=i32[:B]),
           lambda: R.sample(z, u, i32[:4]), lambda: R.sample(z, u, i32[20:24]), lambda: R.sample(z, u, t, logprob=u),
           lambda: R.sample(z, u, t, top_k=t), lambda: R.sample(z, u, t, logprob=t.view(torch.float32)),
           # batch x channels, batch x taps x channels, the sums of a training pass, rows
           lambda: snn.SequenceLayer(65535, 1, 65536, state=8, taps=1), lambda: snn.SequenceLayer(65535, 1, 65536, state=4, taps=3),
           lambda: snn.SequenceLayer(64, 65536, 64, state=64, groups=16, train=True), lambda: snn.Sampler(1 << 22, 4)]
    for i, call in enumerate(bad):
        print(f"[seq] refusal {i}", flush=True)
        with pytest.raises(snn.SNNError) as e:
            call()
        assert "EINVAL" in str(e.value), (i, e.value)
    R.sample(z, u, t)
    torch.cuda.synchronize()


@pytest.mark.parametrize("N", [4, 16])
def test_a_step_with_states_at_odd_addresses(N):
    torch = _torch()
    B, C = 3, 10
    L = _layer(B, 1, C, state=N)
    f = lambda *s: torch.randn(*s, device="cuda")   # noqa: E731
    torch.manual_seed(N)
    x, d, bc, A, h = f(B, C), f(B, C), f(B, N), -f(C, N).abs(), f(B, C, N)
    y, hT, y1 = f(B, C), f(B, C, N), f(B, C)
    L.scan_step(x, d, A, bc, bc, h, hT, y)
    off = [f(v.numel() + 1)[1:].view(v.shape) for v in (A, h, hT)]
    off[0].copy_(A), off[1].copy_(h)
    L.scan_step(x, d, off[0], bc, bc, off[1], off[2], y1)
    assert torch.equal(y, y1) and torch.equal(hT, off[2])
