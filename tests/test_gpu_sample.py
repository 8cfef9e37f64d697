"""Sampling (include/snn_seq.h, paper_2501_07331_amd.Sampler) against its oracle:
the same class in every row, its log-probability to fp32's rounding."""
import numpy as np
import pytest

from oracle import sequence as seq

pytestmark = pytest.mark.gpu


def _run(z, u, dtype, strided=False, **kw):
    import torch
    import paper_2501_07331_amd as snn
    print(f"[sample] {z.shape} {dtype} {sorted(kw)}", flush=True)
    t = torch.from_numpy(z).to(getattr(torch, dtype)).cuda()
    R, V = t.shape
    if strided:
        wide = torch.full((R, V + 3), float("inf"), dtype=t.dtype, device="cuda")
        wide[:, 1:1 + V] = t
        t = wide[:, 1:1 + V]
    s = snn.Sampler(R, V)
    f = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in kw.items()}
    token = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    logprob = torch.full((R,), float("nan"), device="cuda")
    s.sample(t, torch.tensor(u, dtype=torch.float32, device="cuda"), token, logprob=logprob, **f)
    zz = t.double().cpu().numpy()
    got, lp = token.cpu().numpy(), logprob.double().cpu().numpy()
    for r in range(R):
        row = {k: float(f[k][r]) if k != "top_k" else int(f[k][r]) for k in f}
        want, wlp, _ = seq.sample(zz[r], float(np.float32(u[r])), **row)
        assert got[r] == want, (r, row, u[r], got[r], want)
        # each of V weights is rounded to a multiple of 2^-s, V <= 2^(62 - s), their sum is at least 1; then fp32
        half = V * 2.0 ** -(63 - np.ceil(np.log2(V)))
        assert (lp[r] == wlp) or abs(lp[r] - wlp) <= 2.0 ** -24 * abs(wlp) + half + 1e-12, (r, lp[r], wlp)


@pytest.mark.parametrize("V", [1, 2, 20, 63, 64, 65, 128, 200, 256, 257, 1000, 4097, 9001, 16384, 20011])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_every_filter(V, dtype):
    r = np.random.default_rng(V)
    R = 24
    z = (r.normal(size=(R, V)) * r.choice([0.1, 2.0, 8.0], size=(R, 1))).astype(np.float32)
    z[r.random((R, V)) < 0.1] = -np.inf
    _run(z, r.random(R), dtype, True, temperature=r.uniform(0.3, 2, R),
         top_k=np.where(r.random(R) < 0.5, r.integers(1, max(2, min(V, 50)), R), 0),
         top_p=np.where(r.random(R) < 0.5, r.uniform(0.3, 1, R), 1.0), min_p=np.where(r.random(R) < 0.5, r.uniform(0, 0.2, R), 0.0))


@pytest.mark.parametrize("V", [5, 300, 5000])
def test_one_filter_at_a_time(V):
    r = np.random.default_rng(V + 1)
    R = 9
    z, u = r.normal(size=(R, V)).astype(np.float32) * 3, r.random(R)
    _run(z, u, "float32")
    _run(z, u, "float32", top_k=np.arange(1, R + 1))
    _run(z, u, "float32", top_k=[V, V + 1, V - 1, -1, 0, 1, 2, 3, 2 ** 31 - 1])
    _run(z, u, "bfloat16", top_p=np.linspace(0, 1, R))
    _run(z, u, "float16", min_p=np.linspace(0, 1, R))
    _run(z, u, "float32", temperature=[0.0, -1.0, 1e-30, 1e-3, 1e30, np.inf, 1.0, 0.5, 2.0])


@pytest.mark.parametrize("V", [7, 100, 256, 300, 4500, 17001])
def test_ties_are_cut_by_index(V):
    """Rows of one value, and of three: the limits fall inside values that many classes share.  Weights of 1 have exact
    sums, so a border that top-p meets is met exactly."""
    r = np.random.default_rng(V)
    R = 12
    z = np.zeros((R, V), np.float32)
    z[6:] = r.choice([0.0, 1.0, -2.0], size=(6, V))
    z[0, ::2] = -0.0                      # equal to 0
    u = r.random(R)
    _run(z, u, "float32", top_k=r.integers(1, V, R))
    _run(z[:6], u[:6], "bfloat16", top_p=np.full(6, 0.5))
    _run(z, u, "bfloat16", top_k=np.full(R, max(1, V // 2)), top_p=r.uniform(0.2, 0.9, R))


@pytest.mark.parametrize("V", [40, 150, 600, 5000, 16400])
def test_values_that_are_no_scores(V):
    r = np.random.default_rng(3)
    z = r.normal(size=(9, V)).astype(np.float32)
    z[0] = -np.inf
    z[1] = np.nan
    z[2, ::3] = np.nan
    z[3, 5] = z[3, 9] = np.inf
    z[4, :V - 1] = -np.inf
    z[5] = np.finfo(np.float32).min
    z[6, 0], z[6, 1] = np.finfo(np.float32).max, np.finfo(np.float32).min
    z[7] = np.float32(1e-45) * np.arange(V)
    z[8, 3] = np.inf
    z[8, 4:] = np.nan
    u = r.random(9)
    _run(z, u, "float32")
    _run(z, u, "float32", top_k=np.full(9, 2), top_p=np.full(9, 0.9), min_p=np.full(9, 0.05))
    _run(z, u, "float32", temperature=np.zeros(9))
    nan = np.full(9, np.nan)
    import torch
    import paper_2501_07331_amd as snn
    s = snn.Sampler(9, V)
    f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")   # noqa: E731
    a, b = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    s.sample(f(z), f(np.zeros(9)), a)
    s.sample(f(z), f(nan), b, temperature=f(nan), top_p=f(nan), min_p=f(nan))       # NaN: the defaults
    assert torch.equal(a, b)
    s.sample(f(z), f(np.full(9, 5.0)), a)                                          # u outside [0, 1)
    s.sample(f(z), f(np.full(9, 1.0 - 2.0 ** -24)), b)
    assert torch.equal(a, b)


def test_a_long_row_and_the_ends_of_u():
    r = np.random.default_rng(8)
    z = r.normal(size=(6, 70001)).astype(np.float32)
    z[4] = 1.5
    z[5] = np.linspace(-1e-3, 1e-3, 70001)
    u = [0.0, 1 - 2.0 ** -24, 0.5, 2.0 ** -30, 0.999, 0.25]
    _run(z, u, "float32")
    _run(z, u, "bfloat16", top_p=np.full(6, 0.95), top_k=[0, 0, 1000, 60000, 12345, 0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_few_equal_scores_far_apart(dtype):
    """The limits fall among a few elements that three close values share, all over a long row: each place of the border,
    and draws from the first element to the last one kept."""
    r = np.random.default_rng(21)
    R, V, few = 48, 33001, 40
    z = (r.normal(size=(R, V)) * 0.5 - 12).astype(np.float32)
    for k in range(R):
        z[k, r.choice(V, few, replace=False)] = r.choice([2.0, 2.015625, 2.03125], few)
    u = np.where(np.arange(R) % 3 == 0, 1 - 2.0 ** -24, np.where(np.arange(R) % 3 == 1, 0.0, r.random(R)))
    _run(z, u, dtype, True, top_k=np.arange(1, R + 1))
    _run(z, u, dtype, top_p=np.linspace(0.0, 1.0, R))
    _run(z, u, dtype, top_k=np.full(R, few + 5), top_p=r.uniform(0.3, 1, R), min_p=np.where(np.arange(R) % 2, 0.98, 0.0))


def test_many_scores_near_the_border():
    """Thousands of scores within a hundredth of the one that the kept ones end at, all different or of a few values."""
    r = np.random.default_rng(31)
    R, V = 14, 130001
    u = np.where(np.arange(R) % 3 == 0, 1 - 2.0 ** -24, r.random(R))
    flat = (r.normal(size=(R, V)) * 0.3).astype(np.float32)
    few = (r.integers(0, 200, size=(R, V)) * 0.003).astype(np.float32)
    for z in (flat, few):
        _run(z, u, "float32", top_p=np.linspace(0.01, 0.99, R))
        _run(z, u, "float32", top_k=np.linspace(2, V - 1, R).astype(np.int64))
        _run(z, u, "bfloat16", top_p=np.linspace(0.05, 0.95, R), top_k=np.full(R, V // 2), min_p=np.full(R, 0.3))


def test_a_handle_serves_smaller_calls():
    """Rows and scores below the handle's: a row is divided otherwise for each call."""
    import torch
    import paper_2501_07331_amd as snn
    r = np.random.default_rng(12)
    s = snn.Sampler(200, 40000)
    for R, V in ((200, 40000), (128, 16384), (7, 40000), (1, 33333), (3, 70), (90, 16383)):
        z, u = r.normal(size=(R, V)).astype(np.float32) * 2, r.random(R).astype(np.float32)
        p = r.uniform(0.5, 1, R).astype(np.float32)
        t, token = torch.from_numpy(z).cuda(), torch.empty(R, dtype=torch.int32, device="cuda")
        s.sample(t, torch.from_numpy(u).cuda(), token, top_p=torch.from_numpy(p).cuda())
        got = token.cpu().numpy()
        for i in range(0, R, max(1, R // 10)):
            assert got[i] == seq.sample(z[i], float(u[i]), top_p=float(p[i]))[0], (R, V, i)


def test_draws_in_a_graph():
    """Replayed on new scores and numbers: every replay equals the eager call (the divided row's histograms are cleared by each)."""
    import torch
    import paper_2501_07331_amd as snn
    r = np.random.default_rng(13)
    R, V = 4, 20000
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        s, eager = snn.Sampler(R, V), snn.Sampler(R, V)
        z, u = torch.zeros(R, V, device="cuda"), torch.zeros(R, device="cuda")
        p = torch.full((R,), 0.9, device="cuda")
        token = torch.empty(R, dtype=torch.int32, device="cuda")
        want = torch.empty_like(token)
        s.sample(z, u, token, top_p=p)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.sample(z, u, token, top_p=p)
        for _ in range(4):
            z.copy_(torch.from_numpy(r.normal(size=(R, V)).astype(np.float32) * 3))
            u.copy_(torch.from_numpy(r.random(R).astype(np.float32)))
            g.replay()
            eager.sample(z, u, want, top_p=p)
            st.synchronize()
            assert torch.equal(token, want)


def test_the_network_answers():
    """Network.sample draws from the z of the network's own forward pass; a spiking output layer has no scores."""
    import torch
    import paper_2501_07331_amd as snn
    from workloads import make_workload
    from .gpu_util import make_gpu_net, to_device
    wl = make_workload(1, weight_scale=6.0)
    net, d = make_gpu_net(wl), to_device(wl)
    dev, B, C, cap = torch.device("cuda"), wl.B, wl.cfg.n_classes, net.record_capacity
    recs = [(torch.zeros(B, dtype=torch.int32, device=dev), torch.zeros(B, cap, dtype=torch.int32, device=dev),
             torch.zeros(B, cap, dtype=torch.int32, device=dev)) for _ in net.lif_layers]
    loss, z = torch.zeros(B + 1, device=dev), torch.zeros(B, C, device=dev)
    net.forward(d["off"], d["step"], d["neuron"], d["W"], d["D"], d["labels"], recs, loss, z)
    u, token, lp = torch.rand(B, device=dev), torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, device=dev)
    net.sample(z, u, token, logprob=lp)
    p = torch.softmax(z.double(), 1)
    for b in range(B):
        assert int(token[b]) == seq.sample(z[b].double().cpu().numpy(), float(u[b]))[0]
        assert abs(float(lp[b]) - float(torch.log(p[b, token[b].long()]))) < 1e-6
    # the drawn classes' log-probabilities under labels = token are the loss of the same forward pass
    net.forward(d["off"], d["step"], d["neuron"], d["W"], d["D"], token, recs, loss, z)
    torch.testing.assert_close(loss[:B], -lp, rtol=1e-5, atol=1e-6)
    spiking = snn.Network([(3, 0, 0), (4, 1, 0), (2, 1, 0)], 20.0, 5.0, 1.0, 1.0, 2, 2, 10, snn.SNN_LOSS_DMSE, 0.1, 8)
    with pytest.raises(ValueError):
        spiking.sample(torch.zeros(2, 2, device=dev), u[:2], token[:2])


def test_refusals():
    import torch
    import paper_2501_07331_amd as snn
    s = snn.Sampler(4, 10)
    z, u, t = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: s.sample(torch.zeros(5, 10, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")),
                 lambda: s.sample(torch.zeros(4, 11, device="cuda"), u, t),
                 lambda: s.sample(z.double(), u, t), lambda: s.sample(z.cpu(), u, t), lambda: s.sample(z, None, t),
                 lambda: s.sample(z, u.double(), t), lambda: s.sample(z, u, t.long()), lambda: s.sample(z, u, t[:3]),
                 lambda: s.sample(z[0], u, t), lambda: s.sample(torch.zeros(10, 4, device="cuda").t(), u, t),
                 lambda: s.sample(z[:1].expand(4, 10), u, t), lambda: s.sample(z, u, t, top_k=u),
                 lambda: snn.Sampler(0, 5), lambda: snn.Sampler(3, 0), lambda: snn.Sampler(3, snn.SNN_SAMPLE_MAX_N + 1)):
        with pytest.raises((ValueError, snn.SNNError)):
            call()
    s.sample(z, u, t)
    torch.cuda.synchronize()
