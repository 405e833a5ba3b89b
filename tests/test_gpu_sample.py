"""mirror_sample against the oracle: tokens and counts exactly, the distribution to fp32."""
import numpy as np
import pytest
import torch

from oracle import rows as O
from paper_2510_13161_b200 import binding
from tests.rows_helpers import make

pytestmark = pytest.mark.gpu


def logits_of(M, V, seed, std=2.5, leaders=12):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((M, V)).astype(np.float32) * np.float32(std)
    for r in range(M):
        x[r, rng.choice(V, min(leaders, V), replace=False)] += np.float32(rng.uniform(3, 12))
    return x


def check(x, T=None, k=None, p=None, mp=None, seed=0, ctx_T=1.0, strided=False, u=None):
    M, V = x.shape
    m = make(2, 2, 64, vocab=V, temperature=ctx_T)
    ctx_T = float(np.float32(ctx_T))                               # (the context holds it in 32 bits)
    rng = np.random.default_rng(seed + 99)
    u = rng.random(M).astype(np.float32) if u is None else np.asarray(u, np.float32)
    dev = lambda a, t: None if a is None else torch.tensor(np.broadcast_to(np.asarray(a), (M,)).astype(t)).cuda()  # noqa: E731
    xd = torch.from_numpy(x).cuda()
    if strided:
        wide = torch.full((M, V + 5), 1e9, device="cuda")
        wide[:, :V] = xd
        xd = wide[:, :V]
    got = m.mirror_sample(xd, torch.from_numpy(u).cuda(), dev(T, np.float32), dev(k, np.int32), dev(p, np.float32), dev(mp, np.float32),
                          want_probs=True, want_logits=True)
    bare = m.mirror_sample(xd, torch.from_numpy(u).cuda(), dev(T, np.float32), dev(k, np.int32), dev(p, np.float32), dev(mp, np.float32))
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    got = {n: t.cpu().numpy() for n, t in got.items()}
    for n in ("token", "n_kept", "logprob"):
        np.testing.assert_array_equal(got[n], bare[n].cpu().numpy())
    at = lambda a, r, default, t=np.float32: default if a is None else float(np.broadcast_to(np.asarray(a, t), (M,))[r])  # noqa: E731
    for r in range(M):
        tok, n, ids, pr = O.sample_row(x[r], at(T, r, ctx_T), int(at(k, r, 0, np.int32)), at(p, r, 1.0), at(mp, r, 0.0), float(u[r]))
        assert got["n_kept"][r] == n, (r, got["n_kept"][r], n)
        assert got["token"][r] == tok, (r, got["token"][r], tok)
        want = np.zeros(V)
        want[ids] = pr
        # exponential and sum are good to 1e-10, one rounding to fp32 (subnormal ones to half of theirs)
        np.testing.assert_allclose(got["probs"][r], want, rtol=2.0 ** -24 + 1e-9, atol=1e-45)
        kept = np.zeros(V, bool)
        kept[ids] = True
        assert np.isneginf(got["logits"][r][~kept]).all()
        if n:
            z = x[r][ids].astype(np.float64) - x[r][ids[0]] if np.isfinite(x[r][ids[0]]) else np.zeros(n)
            t = at(T, r, ctx_T)
            z = z / t if t > 0 else z
            ln = z - np.log(np.exp(z).sum())
            want = ln * ctx_T
            want[want < -float(np.finfo(np.float32).max)] = -np.inf       # (what fp32 does not hold)
            np.testing.assert_allclose(got["logits"][r][ids], want, rtol=2.0 ** -24 + 1e-9, atol=1e-9)
            lp = float(ln[list(ids).index(tok)])
            assert abs(got["logprob"][r] - lp) <= 2.0 ** -23 * abs(lp) + 1e-7
        else:
            assert np.isneginf(got["logprob"][r])


@pytest.mark.parametrize("V", [1, 2, 31, 1000, 4097, 32000, 128256])
def test_no_filter(V):
    check(logits_of(5, V, V), T=[0.3, 0.7, 1.0, 1.6, 5.0], seed=V)


@pytest.mark.parametrize("V", [3, 1000, 50257, 151936])
@pytest.mark.parametrize("k,p,mp", [(1, None, None), (50, None, None), (40, 0.9, None), (None, 0.5, None), (None, 0.95, None), (None, None, 0.05),
                                    (200, 0.8, 0.01), (None, 0.9, 0.002), (3000, 0.97, None)])
def test_filters(V, k, p, mp):
    check(logits_of(4, V, V + 7), T=[0.6, 0.9, 1.0, 1.4], k=k, p=p, mp=mp, seed=V)


def test_open_rows_keep_more_than_fits_the_list():
    """Flat rows: fronts of thousands of ids, by rank, by share and by both."""
    x = logits_of(6, 30000, 5, std=0.7, leaders=0)
    check(x, k=[0, 5000, 20000, 3000, 29999, 2500], p=[0.6, 0.9, 1.0, 0.4, 0.999, 1.0], mp=[0.0, 0.0, 0.0, 0.001, 0.05, 0.12])


@pytest.mark.parametrize("V", [300001, 655360])
def test_the_largest_vocabularies(V):
    check(logits_of(2, V, V), T=[0.7, 1.3], k=[60, 0], p=[0.9, 0.95], seed=1)
    check(logits_of(2, V, V + 1), T=[0.9, 1.1], seed=2)


def test_many_rows_that_are_open_tied_or_masked():
    """More rows than are kept in shared memory: every way through the kernel that the small batches take, too."""
    M = 60
    x = logits_of(M, 9004, 21, std=0.8, leaders=3)
    x[1] = 0.0
    x[2] = np.round(x[2] * 2) / 2
    x[3, 100:] = -np.inf
    x[4] = -np.inf
    x[5] = np.nan
    x[6, ::3] = np.nan
    x[7, [5, 77]] = np.inf
    rng = np.random.default_rng(3)
    k = rng.choice([0, 1, 700, 1500, 4000, 9003], M)
    p = rng.choice([0.3, 0.9, 0.999, 1.0], M)
    mp = rng.choice([0.0, 0.0, 0.02, 0.4], M)
    check(x, T=rng.uniform(0.3, 1.5, M), k=k, p=p, mp=mp, seed=4)
    check(x, T=rng.uniform(0.3, 1.5, M), p=0.95, seed=5)
    check(x[:, :9001].copy(), T=rng.uniform(0.3, 1.5, M), k=2500, p=0.9, seed=6)


@pytest.mark.parametrize("T", [1e-44, 1e-38, 3e38, np.inf])
def test_temperatures_at_the_ends_of_fp32(T):
    x = logits_of(3, 5000, 30)
    x[1] = 3.0
    x[2, :2500] = 2.0
    for k, p, mp in ((None, None, None), (1, None, None), (3000, None, None), (None, 0.7, None), (None, None, 0.5)):
        check(x, T=T, k=k, p=p, mp=mp, seed=6)


def test_settings_differ_by_row():
    M = 40
    rng = np.random.default_rng(1)
    check(logits_of(M, 9001, 2), T=rng.uniform(0.2, 2.0, M), k=rng.integers(-3, 300, M), p=rng.uniform(-0.1, 1.2, M), mp=rng.uniform(-0.05, 0.3, M))


def test_ties():
    """Equal logits: the lower ids stay."""
    x = np.round(logits_of(4, 5000, 3) * 2) / 2
    check(x.astype(np.float32), k=[7, 100, 3000, 0], p=[1.0, 0.7, 0.8, 0.9])
    check(np.zeros((4, 20000), np.float32), k=[0, 11, 6000, 0], p=[0.5, 1.0, 0.25, 1.0], u=[0.0, 0.5, 0.999, 0.37])
    check(np.array([[0.0, -0.0, 0.0, -1.0]], np.float32), k=2)


def test_masked_infinite_and_missing_logits():
    x = logits_of(8, 3000, 4)
    x[0, 5:] = -np.inf
    x[1] = -np.inf
    x[2, ::2] = np.nan
    x[3] = np.nan
    x[4, [17, 900, 2999]] = np.inf
    x[5, :2990] = np.finfo(np.float32).min
    x[6] = -np.inf
    x[6, 2999] = -3e38
    x[7, 11] = 3e38
    for k, p, mp in ((None, None, None), (4, None, None), (None, 0.9, None), (None, None, 0.1), (9, 0.7, 0.01)):
        check(x, T=0.8, k=k, p=p, mp=mp, seed=11)


@pytest.mark.parametrize("M", [3, 40])
@pytest.mark.parametrize("k", [1, 2, 255, 256, 257, 800, 1023, 1024, 1025, 1399, 1400, 1401, 1600, 2047, 2048, 2049])
def test_fronts_of_every_length_of_list(M, k):
    """Few candidates are compared each with each, more are sorted, and fronts that are longer than the list are found by their end."""
    x = logits_of(M, 40961, k, std=1.5, leaders=0)
    check(x, k=k, seed=k)
    check(x[:3], T=1.2, k=k, p=[0.9, 0.3, 1.0], mp=[0.0, 0.0, 0.04], seed=k + 1)


@pytest.mark.parametrize("V", [257, 2048, 2049])
def test_rows_as_long_as_the_list(V):
    check(logits_of(4, V, V, std=0.5, leaders=0), k=[0, 300, 0, 256], p=[0.9, 1.0, 0.99, 0.8], mp=[0.0, 0.0, 0.3, 0.05], seed=V)


@pytest.mark.parametrize("M", [2, 40])
def test_leaders_that_lie_together(M):
    """The largest logits side by side, in order, or in one thread's reach: the candidates of few groups are many."""
    x = logits_of(M, 60000, 77, leaders=0)
    x[0, 1000:6000] += 30
    x[1] = np.sort(x[1])
    if M > 2:
        x[2] = np.sort(x[2])[::-1]
        x[3, 128 * np.arange(16)] += 30
        x[4, 59990:] += 30
        x[5, :3000] = 9.0
    for k, p, mp in ((50, None, None), (1000, 0.9, None), (None, None, 0.2), (None, 0.6, 0.3), (1, None, None)):
        check(x[:6], T=0.9, k=k, p=p, mp=mp, seed=M)
    check(x, k=200, seed=M + 1)


def test_uniforms_at_their_ends_and_greedy_rows():
    x = logits_of(6, 2000, 6)
    check(x, u=[0.0, np.nextafter(np.float32(1), np.float32(0)), 0.5, 1e-30, 0.25, 0.75], p=0.9)
    check(x, T=[0.0, -1.0, 1e-30, 1e30, 0.5, 0.01], u=[0.9] * 6)
    check(x, T=[0.0, -1.0, 1e-30, 1e30, 0.5, 0.01], p=0.6, k=20, u=[0.9] * 6)


@pytest.mark.parametrize("M", [1, 3, 20, 150, 700])
def test_row_counts(M):
    check(logits_of(M, 5003, M), p=0.85, seed=M)


def test_strided_rows_and_the_contexts_temperature():
    check(logits_of(5, 4003, 8), k=30, strided=True, ctx_T=0.6)
    check(logits_of(5, 4000, 8), p=0.8, ctx_T=1.7)


def test_out_of_place_equals_in_place():
    m = make(2, 2, 64, vocab=1000)
    x = torch.from_numpy(logits_of(3, 1000, 9)).cuda()
    u, p = torch.rand(3, device="cuda"), torch.full((3,), 0.8, device="cuda")
    want = m.mirror_sample(x, u, top_p=p, want_probs=True)
    tok = torch.empty(3, dtype=torch.int32, device="cuda")
    assert m.lib.mirror_sample(m._ctx, x.data_ptr(), 1000, 3, None, None, p.data_ptr(), None, u.data_ptr(), tok.data_ptr(), None, None, x.data_ptr(),
                               None, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(x, want["probs"]) and torch.equal(tok, want["token"])


@pytest.mark.parametrize("M,V", [(2, 30004), (60, 30004), (60, 30001), (300, 700)])
@pytest.mark.parametrize("k,p", [(50, 1.0), (0, 0.9), (3000, 0.7), (0, 1.0)])
@pytest.mark.parametrize("what", ["probs", "logits"])
def test_every_way_in_place(M, V, k, p, what):
    m = make(2, 2, 64, vocab=V)
    x = torch.from_numpy(logits_of(M, V, V + k, std=1.0)).cuda()
    u, pd, kd = torch.rand(M, device="cuda"), torch.full((M,), p, device="cuda"), torch.full((M,), k, dtype=torch.int32, device="cuda")
    want = m.mirror_sample(x, u, top_k=kd, top_p=pd, want_probs=what == "probs", want_logits=what == "logits")
    tok = torch.empty(M, dtype=torch.int32, device="cuda")
    out = (x.data_ptr(), None) if what == "probs" else (None, x.data_ptr())
    assert m.lib.mirror_sample(m._ctx, x.data_ptr(), V, M, None, kd.data_ptr(), pd.data_ptr(), None, u.data_ptr(), tok.data_ptr(), None, None, *out,
                               torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(x, want[what]) and torch.equal(tok, want["token"])


def test_captured_and_replayed():
    m = make(2, 2, 64, vocab=3001)
    x = torch.from_numpy(logits_of(4, 3001, 10)).cuda()
    u, p = torch.rand(4, device="cuda"), torch.full((4,), 0.8, device="cuda")
    want = m.mirror_sample(x, u, top_p=p)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = m.mirror_sample(x, u, top_p=p)
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got["token"], want["token"]) and torch.equal(got["logprob"], want["logprob"])


def test_draws_follow_the_distribution():
    """20,000 draws from one row: each id's share within five standard deviations of its probability."""
    V, M = 64, 20000
    x = np.repeat(logits_of(1, V, 12, std=1.0, leaders=3), M, 0)
    m = make(2, 2, 64, vocab=V)
    got = m.mirror_sample(torch.from_numpy(x).cuda(), (torch.arange(M, device="cuda") + 0.5) / M)["token"].cpu().numpy()
    pr = np.exp(x[0].astype(np.float64) - x[0].max())
    pr /= pr.sum()
    share = np.bincount(got, minlength=V) / M
    assert (np.abs(share - pr) <= 5 * np.sqrt(pr / M) + 1.0 / M).all()


def test_refusals():
    m = make(2, 2, 64, vocab=100)
    x, u = torch.zeros((4, 100), device="cuda"), torch.zeros(4, device="cuda")
    for bad in (x[:, :99], x.double(), x.t(), x.cpu()):
        with pytest.raises((ValueError, IndexError)):
            m.mirror_sample(bad, u)
    for name in ("temperature", "top_k", "top_p", "min_p"):
        with pytest.raises(ValueError):
            m.mirror_sample(x, u, **{name: torch.zeros(3, dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda")})
        with pytest.raises(ValueError):
            m.mirror_sample(x, u, **{name: torch.zeros(4, dtype=torch.int64, device="cuda")})
    call = lambda logits=x.data_ptr(), ld=100, M=4, u=u.data_ptr(), token=u.data_ptr(), probs=None, lg=None: m.lib.mirror_sample(  # noqa: E731
        m._ctx, logits, ld, M, None, None, None, None, u, token, None, None, probs, lg, None)
    assert call(logits=None) == 1 and call(u=None) == 1 and call(token=None) == 1 and call(M=-1) == 1
    assert call(ld=99) == 2 and call(probs=x.data_ptr(), lg=x.data_ptr()) == 1 and call(probs=x.data_ptr(), ld=104) == 1
    assert call(logits=x.data_ptr() + 2) == 1
    assert call(M=0) == 0
    big = make(2, 2, 64, vocab=16 * 40960 + 1)
    assert big.lib.mirror_sample(big._ctx, x.data_ptr(), 16 * 40960 + 1, 1, None, None, None, None, u.data_ptr(), u.data_ptr(), None, None, None, None, None) == 2
    assert binding.MirrorError


@pytest.mark.parametrize("V", [2049, 4097, 8193, 8200])
@pytest.mark.parametrize("M", [1, 9, 30])
def test_clusters_whose_last_ctas_have_few_ids_or_none(V, M):
    """Rows so short that the last CTAs of a cluster have nothing to load and are through with it long before the others have begun: call
    after call, the same tokens."""
    x = logits_of(M, V, V + M)
    check(x, k=20, seed=V)
    m = make(2, 2, 64, vocab=V)
    xd, u = torch.from_numpy(x).cuda(), torch.rand(M, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))
    want = [int(O.sample_row(x[r], u=float(u[r]))[0]) for r in range(M)]
    got = [m.mirror_sample(xd, u)["token"] for _ in range(200)]
    assert (torch.stack(got).cpu() == torch.tensor(want, dtype=torch.int32)).all()


@pytest.mark.parametrize("V,crowd", [(300, 300), (32000, 500), (32000, 32000), (128256, 1000), (655360, 800), (655360, 655360)])
@pytest.mark.parametrize("M", [2, 60])
def test_min_p_below_a_step_of_the_sums(V, crowd, M):
    """Thresholds of 10^-12 to 10^-30, where a weight is less than one of the steps that sums are counted in, or a few of them: what stays goes
    by the weight itself.  `crowd` ids lie up to 80 nats below the largest, the others further down."""
    if M * V > 1 << 24:
        M = 25                                                   # (more rows than two large CTAs an SM hold, at this size)
    mp = np.resize(np.float32([1e-12, 1e-15, 3e-13, 1e-30, 1e-18]), M)
    x = logits_of(M, V, V + crowd, std=1.0, leaders=0) - np.float32(200.0)
    rng = np.random.default_rng(crowd)
    for r in range(M):
        x[r, rng.choice(V, crowd, replace=False)] = -rng.uniform(0.0, 80.0, crowd).astype(np.float32)
        z = x[r].astype(np.float64) - x[r].max()
        assert np.abs(z - np.log(float(mp[r]))).min() > 1e-9     # (no id so close to the threshold that the last bits of exp decide)
    check(x, mp=mp, seed=V)
    check(x[:2], p=[0.999, 1.0], mp=mp[:2], seed=V + 1)
    check(x[:2], k=[40, 1000], mp=mp[:2], seed=V + 2)


@pytest.mark.parametrize("M,V", [(3, 9), (3, 40000), (60, 40000)])
def test_min_p_of_one_and_more(M, V):
    """Of ids with the largest logit all have one times the largest probability, none has more: the first alone stays then."""
    x = logits_of(M, V, V, std=0.5, leaders=0)
    x[0, V // 3:] = 7.0
    x[1, [2, V - 1]] = 9.0
    for p in (None, 0.7):
        check(x, p=p, mp=np.resize(np.float32([1.0, 1.0, 1.0, 1.0, 1.0001, np.inf, 3.0]), M), seed=V)
        check(x, p=p, k=30000, mp=np.resize(np.float32([1.5, np.inf, 1.0001, 0.5]), M), seed=V + 1)
        check(x, p=p, T=0.0, mp=1.5, seed=V + 2)
