"""mirror_attn_causal against the oracle in 64 bits; everything that no row sees is NaN in the cache."""
import numpy as np
import pytest
import torch

from paper_2510_13161_b200 import binding
from tests.rows_helpers import PAGE, Case, check_attention, make

pytestmark = pytest.mark.gpu

LENS = [0, 1, 15, 16, 17, 31, 130, 500, 0, 999]


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (5, 1), (14, 2), (16, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens(hq, hkv, d):
    check_attention(make(hq, hkv, d), Case(hq, hkv, d, LENS, [1] * 10, layers=2, pad=2, seed=hq), False)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 16), (40, 3), (100, 33), (100, 200), (5000, 4)])
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_under_a_window(window, sinks, d):
    check_attention(make(8, 2, d), Case(8, 2, d, LENS, [1] * 10, window=window, sinks=sinks, seed=window), False)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 2), (9, 5), (64, 17)])
def test_a_few_rows(window, sinks):
    counts = [2, 4, 0, 1, 3, 4, 4, 2, 0, 4]
    check_attention(make(8, 2, 128), Case(8, 2, 128, LENS, counts, layers=2, pad=5, window=window, sinks=sinks, seed=4), False)
    check_attention(make(2, 2, 64), Case(2, 2, 64, LENS, [c * 4 for c in counts], window=window, sinks=sinks, seed=5), False)


def test_a_long_context_cut_over_all_ctas():
    check_attention(make(8, 1, 128), Case(8, 1, 128, [20000], [1], seed=1), False)
    check_attention(make(8, 2, 64), Case(8, 2, 64, [12345, 3, 0, 7000], [2, 1, 0, 2], seed=2, window=6000, sinks=40), False)


def test_many_requests():
    check_attention(make(2, 1, 64), Case(2, 1, 64, [(b * 13) % 90 for b in range(1024)], [b % 3 for b in range(1024)], seed=3), False)


@pytest.mark.parametrize("spread", [8.0, 0.0])
def test_scores_far_apart_and_all_alike(spread):
    """Scores of +-100 and more: weights underflow, and the running maximum moves again and again."""
    check_attention(make(8, 2, 128), Case(8, 2, 128, [700, 40], [1, 2], seed=6, spread=spread), False)


def test_a_scale_of_its_own_and_uniform_rows():
    check_attention(make(4, 2, 64, scale=0.3), Case(4, 2, 64, [33, 70, 5], [2, 2, 2], seed=7, uniform=True), False, scale=0.3)


COUNTS = [1, 100, 16, 0, 300, 33, 128, 15, 257, 64]


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (5, 1), (14, 2), (32, 1), (144, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_prompts(hq, hkv, d):
    check_attention(make(hq, hkv, d), Case(hq, hkv, d, LENS, COUNTS, pad=2, seed=hq), True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 16), (40, 3), (100, 33), (100, 200), (300, 0), (5000, 4)])
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_under_a_window(window, sinks, d):
    check_attention(make(8, 2, d), Case(8, 2, d, LENS, COUNTS, window=window, sinks=sinks, seed=window), True)
    check_attention(make(2, 2, d), Case(2, 2, d, [0, 700, 33], [400, 129, 256], window=window, sinks=sinks, seed=window + 1), True)


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (7, 2 ** 31 - 1), (2 ** 30 + 5, 3)])
def test_the_widest_windows_and_sinks(window, sinks):
    check_attention(make(8, 2, 64), Case(8, 2, 64, LENS, [1] * 10, window=window, sinks=sinks, seed=3), False)
    check_attention(make(8, 2, 64), Case(8, 2, 64, LENS, COUNTS, window=window, sinks=sinks, seed=4), True)


def test_prompts_of_every_length_around_a_tile():
    for n in (17, 31, 32, 33, 63, 64, 65, 127, 128, 129):
        check_attention(make(4, 1, 64), Case(4, 1, 64, [n, 0, 128 - n % 128], [n, n + 1, 1], seed=n), True)


def test_a_prompt_cut_over_all_ctas_and_several_layers():
    check_attention(make(8, 1, 128), Case(8, 1, 128, [9000], [40], seed=1), True)
    check_attention(make(8, 2, 64), Case(8, 2, 64, [5000, 3, 0], [50, 600, 1], layers=3, seed=2), True)
    check_attention(make(4, 4, 128), Case(4, 4, 128, [0], [1500], seed=3), True)


def test_many_requests_with_prompts():
    check_attention(make(4, 1, 64), Case(4, 1, 64, [(b * 13) % 90 for b in range(1024)], [(b * 5) % 11 for b in range(1024)], seed=3), True)


@pytest.mark.parametrize("spread", [8.0, 0.0])
def test_prompts_with_scores_far_apart_and_all_alike(spread):
    check_attention(make(8, 2, 128), Case(8, 2, 128, [700, 40], [70, 200], seed=6, spread=spread), True)


def test_twice_and_on_another_stream_the_same():
    m = make(8, 2, 128)
    for counts in ([1, 1], [40, 300]):
        again(m, Case(8, 2, 128, [3000, 77], counts, seed=8), counts[0] > 1)


def again(m, c, p_rounded):
    a, la = check_attention(m, c, p_rounded)
    s = torch.cuda.Stream()
    out, lse = torch.empty_like(a), torch.empty_like(la)
    q = c.q.cuda()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.mirror_attn_causal(c.kv, c.rows, q, out=out, lse_out=lse)
    s.synchronize()
    assert torch.equal(a, out) and torch.equal(la, lse)


@pytest.mark.parametrize("n", [1, 30])
def test_captured_and_replayed_with_other_lengths(n):
    """The partition is made on the device: a captured call follows the lengths that it finds."""
    m = make(8, 2, 128)
    c = Case(8, 2, 128, [1500, 900], [n, n], seed=9)
    kv, rows = c.device(m)
    q, out = c.q.cuda(), torch.empty((1, 2 * n, 8, 128), dtype=torch.bfloat16, device="cuda")
    m.mirror_attn_causal(kv, rows, q, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.mirror_attn_causal(kv, rows, q, out=out)
    lens = kv._refs[3]
    for a, b in ((1500, 900), (3, 870), (0, 17)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        g.replay()
        got = out.clone()
        m.mirror_attn_causal(kv, rows, q, out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and not out.isnan().any()
    assert m.device_status() == (0, 0)


@pytest.mark.parametrize("n", [1, 20])
def test_a_cache_beyond_four_gigabytes(n):
    """Pages at the far end of a pool whose elements do not count in 32 bits: the same rows as in a small pool."""
    hq, hkv, d, pages = 16, 8, 128, 150_000
    m = make(hq, hkv, d)
    c = Case(hq, hkv, d, [37, 100], [n, n], seed=11)
    want, _ = check_attention(m, c, n * 2 > 16)
    big = [torch.zeros((1, pages, hkv, PAGE, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.from_numpy(c.table).cuda()
    moved = torch.where(table < 1000, pages - 1 - table, table)
    used = c.k.shape[1]
    for far, near in zip(big, (c.kd, c.vd)):
        far[:, pages - used:] = near.flip(1)
    kv = m.kv(*big, moved, torch.tensor(c.lens, dtype=torch.int32).cuda())
    assert torch.equal(m.mirror_attn_causal(kv, c.rows, c.q.cuda())[:, :2 * n], want[:, :2 * n])
    # the rows' own keys and values once more, appended there
    k = torch.randn((1, 2 * n, hkv, d), device="cuda").to(torch.bfloat16)
    m.mirror_kv_append(kv, c.rows, k, k)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    for b, t in enumerate(c.lens):
        for i in range(n):
            page = int(moved[b, (t + i) // PAGE])
            assert torch.equal(big[1][0, page, :, (t + i) % PAGE], k[0, b * n + i])


@pytest.mark.parametrize("n", [1, 20])
def test_in_place(n):
    """The output may take the queries' place."""
    m = make(8, 2, 64)
    c = Case(8, 2, 64, [3000, 77, 5], [n, n, n], seed=12)
    want, _ = check_attention(m, c, n > 4)
    q = c.q.cuda()
    got = m.mirror_attn_causal(c.kv, c.rows, q, out=q)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("n", [1, 20])
def test_two_contexts_at_once(n):
    """Calls of two contexts on two streams, side by side."""
    ms = [make(8, 2, 128), make(8, 2, 128)]
    cs = [Case(8, 2, 128, [900, 40, 2000], [n, n, n], seed=13 + i) for i in range(2)]
    want = [check_attention(m, c, n > 4)[0] for m, c in zip(ms, cs)]
    qs, streams = [c.q.cuda() for c in cs], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for m, c, q, s in zip(ms, cs, qs, streams):
            with torch.cuda.stream(s):
                got.append(m.mirror_attn_causal(c.kv, c.rows, q))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n", [1, 20])
def test_reports(n):
    m = make(4, 2, 64)
    c = Case(4, 2, 64, [20, 5], [n, n], seed=1)
    kv, rows = c.device(m)
    q = c.q.cuda()
    lens, table = kv._refs[3], kv._refs[2]
    for name, change, code in (("length", lambda: lens.fill_(1000), 831), ("negative", lambda: lens.fill_(-1), 831), ("page", lambda: table.fill_(99), 832),
                               ("page", lambda: table.fill_(-1), 832)):
        kept = lens.clone(), table.clone()
        table[table > 90] = 0
        change()
        m.mirror_attn_causal(kv, rows, q)
        torch.cuda.synchronize()
        assert m.device_status() == (6, code), name
        lens.copy_(kept[0]), table.copy_(kept[1])
    rows._refs[0].copy_(torch.tensor([0, n + 1, n], dtype=torch.int32))          # a request with more rows than max_rows
    table[table > 90] = 0
    m.mirror_attn_causal(kv, rows, q)
    torch.cuda.synchronize()
    assert m.device_status() == (6, 830)


def test_refusals():
    m = make(4, 2, 64)
    c = Case(4, 2, 64, [20, 5], [1, 1])
    kv, rows = c.device(m)
    q = c.q.cuda()
    with pytest.raises(binding.MirrorError) as e:
        m.mirror_attn_causal(kv, rows, q, window=-1)
    assert e.value.code == 1
    with pytest.raises(binding.MirrorError) as e:
        m.mirror_attn_causal(kv, rows, q, sinks=-1)
    assert e.value.code == 1
    for bad in (q[:, :1], q.float(), q.transpose(1, 2)):
        with pytest.raises(ValueError):
            m.mirror_attn_causal(kv, rows, bad)
    with pytest.raises(ValueError):
        m.mirror_attn_causal(kv, rows, q, lse_out=torch.empty((1, 4, 2), device="cuda"))
    m2 = make(4, 2, 64)
    import ctypes as C
    assert m2.lib.mirror_attn_causal(m2._ctx, C.byref(kv), C.byref(rows), 0, 0, q.data_ptr(), q.data_ptr(), None, None) == 4        # no workspace


SPOILED = [(8, 2, LENS, [1] * 10, 0, 0, False), (8, 2, LENS, [1, 2, 3, 4, 4, 2, 4, 4, 0, 3], 0, 0, False), (8, 1, [20000], [2], 0, 0, False), (8, 2, LENS, [2] * 10, 40, 3, False),
           (8, 2, LENS, [1, 100, 16, 0, 300, 33, 128, 15, 257, 64], 0, 0, True), (8, 2, LENS, [1, 100, 16, 0, 300, 33, 128, 15, 257, 64], 40, 3, True),
           (8, 1, [9000], [40], 0, 0, True), (4, 4, [0, 3000], [1500, 20], 0, 0, True)]


@pytest.mark.parametrize("hq,hkv,lens,counts,window,sinks,p_rounded", SPOILED)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["query nan", "query inf", "key nan", "key inf", "key -inf", "all -inf"])
def test_scores_that_are_no_numbers(hq, hkv, lens, counts, window, sinks, p_rounded, d, what):
    """NaN or an infinity in a query, or in a key that some rows see: the rows whose softmax has no value are NaN, as in 64 bits, whether
    their unit was cut or not, and all others are as they would be."""
    m = make(hq, hkv, d)
    c = Case(hq, hkv, d, lens, counts, window=window, sinks=sinks, seed=31)
    s = 1 / np.sqrt(d)
    b = int(np.argmax(np.asarray(lens) + 1000 * np.asarray(counts)))
    row, pos = int(c.start[b]) + counts[b] // 2, lens[b] + counts[b] // 2                       # a row in the middle, and its own key
    if what.startswith("query"):
        c.q[0, row, 1, 5] = float(what.split()[1])
    elif what.startswith("key"):
        c.k[0, c.table[b, pos // PAGE], 0, pos % PAGE, 5] = float(what.split()[1])
    else:                                                        # one row's query meets only keys of the other sign
        c.q[0, row, 1] = 0.0
        c.q[0, row, 1, 5] = float("-inf")
        for j in range(lens[b] + counts[b]):
            page = c.table[b, j // PAGE]
            if page < c.k.shape[1]:
                c.k[0, page, 0, j % PAGE, 5] = c.k[0, page, 0, j % PAGE, 5].abs() + 0.125
    largest = lambda t: float(t.float().nan_to_num(0.0, 0.0, 0.0).norm(dim=-1).max())  # noqa: E731
    moved = d * 2.0 ** -24 * s * largest(c.q) * largest(c.k)
    kv, rows = c.device(m)
    lse = torch.full((1, c.R, hq), 7.0, device="cuda")
    out = m.mirror_attn_causal(kv, rows, c.q.cuda(), window=window, sinks=sinks, lse_out=lse)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    with np.errstate(invalid="ignore"):
        want, want_lse, spread = c.expect(0, s)
    got, gl, none = out[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), np.isnan(want)
    assert not none.all() and np.array_equal(none.any(-1), none.all(-1))
    assert np.array_equal(np.isnan(got), none)
    assert not np.isfinite(gl[none.all(-1)]).any()
    # (tolerances of check_attention)
    ok = ~none
    tol = 2.0 ** -8 * np.abs(want) + ((2.0 ** -8 if p_rounded else 2.0 ** -15) + 2 * moved + 1e-6) * spread + 1e-30
    assert (np.abs(got - want)[ok] <= tol[ok]).all()
    ok = ~none.all(-1)
    assert (np.abs(gl - want_lse)[ok] <= moved + 2e-6 * (1 + np.abs(want_lse[ok]))).all()


@pytest.mark.parametrize("hkv,n", [(1, 6000), (1, 8300), (2, 6000)])
def test_more_tiles_than_can_be_counted(hkv, n):
    """A page table of 2^27 tokens and thousands of rows behind them: 1048511 tiles for each pair of row tiles (two rows of 128 heads, or four of
    64 a KV head), which over the pairs and heads is past 2^31, or past 2^32.  Such a call is reported, and its rows are left as they are."""
    m = make(128, hkv, 64)
    pools = [torch.zeros((1, 4, hkv, PAGE, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pages = 1 << 23
    prefix = pages * PAGE - n
    tiles = n // (2 * hkv) * (prefix // 128) * hkv               # at least
    assert tiles > 1 << (32 if n == 8300 else 31)
    kv = m.kv(*pools, torch.zeros((1, pages), dtype=torch.int32, device="cuda"), torch.tensor([prefix], dtype=torch.int32, device="cuda"))
    q = torch.zeros((1, n, 128, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((1, n, 128), 7.0, device="cuda")
    m.mirror_attn_causal(kv, m.rows(None, n, n, 1), q, out=out, lse_out=lse)
    torch.cuda.synchronize()
    assert m.device_status() == (6, 833)
    assert (out == 7.0).all() and (lse == 7.0).all()


def test_rows_that_are_not_in_order():
    """Every other request claims all rows: reported, and no plan of 32 times the work is made."""
    m = make(4, 1, 64)
    B, R = 64, 4096
    pools = [torch.zeros((1, 4, 1, PAGE, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kv = m.kv(*pools, torch.zeros((B, 300), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"))
    start = torch.tensor([0, R] * (B // 2) + [0], dtype=torch.int32, device="cuda")
    q = torch.zeros((1, R, 4, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    m.mirror_attn_causal(kv, m.rows(start, R, R), q, out=out)
    torch.cuda.synchronize()
    assert m.device_status() == (6, 830)
    assert (out == 7.0).all()
    start.copy_(torch.arange(B + 1, dtype=torch.int32) * (R // B))
    m.mirror_attn_causal(kv, m.rows(start, R, R), q, out=out)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0) and (out == 0.0).all()
