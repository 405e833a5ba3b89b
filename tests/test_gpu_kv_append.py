"""mirror_kv_append against the oracle: every layout of the rotation, ragged rows, strided inputs, what is refused and reported."""
import numpy as np
import pytest
import torch

from oracle import rows as O
from paper_2510_13161_b200 import binding
from tests.rows_helpers import PAGE, make

pytestmark = pytest.mark.gpu


def run(m, lens, counts, layers=1, pad=0, rope=None, with_q=True, fused=False, in_place=False, seed=0, far=0):
    """-> (inputs, pools before, pools after, q_out) as float64 numpy, table, start."""
    hq, hkv, d = m.desc.n_q_heads, m.desc.n_kv_heads, m.desc.head_dim
    g = torch.Generator(device="cuda").manual_seed(seed)
    bf = lambda *s: torch.randn(s, dtype=torch.bfloat16, device="cuda", generator=g)  # noqa: E731
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    R = int(start[-1]) + pad
    if fused:
        qkv = bf(layers, R, hq + 2 * hkv, d)
        q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    else:
        q, k, v = bf(layers, R, hq, d), bf(layers, R, hkv, d), bf(layers, R, hkv, d)
    lens = [t + far for t in lens]
    most = max(-(-(t + n) // PAGE) for t, n in zip(lens, counts))
    rng = np.random.default_rng(seed)
    mine = [range(t // PAGE, -(-(t + n) // PAGE)) for t, n in zip(lens, counts)]
    order = rng.permutation(sum(len(r) for r in mine) + 2)
    table, at = np.full((len(lens), most), -7, np.int32), 0
    for b, r in enumerate(mine):
        table[b, list(r)] = order[at:at + len(r)]
        at += len(r)
    kp, vp = bf(layers, len(order), hkv, PAGE, d), bf(layers, len(order), hkv, PAGE, d)
    k0, v0 = kp.clone(), vp.clone()
    kv = m.kv(kp, vp, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    rows = m.rows(torch.from_numpy(start).cuda(), R, max(max(counts), 1))
    q_before = q.double().cpu().numpy()
    q_out = q if in_place else torch.full((layers, R, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    m.mirror_kv_append(kv, rows, k, v, q=q if with_q else None, rope=rope, q_out=q_out if with_q else None)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    return dict(q=q_before, k=n(k), v=n(v), k0=n(k0), v0=n(v0), k1=n(kp), v1=n(vp), q_out=n(q_out), table=table, start=start, lens=lens, R=R)


def check(m, r, freq, interleaved, amplitude, with_q=True, in_place=False):
    """A turned element: half a bf16 step of its size, and fp32 products of a sine and cosine good to a few 2^-24 of the pair."""
    places = O.row_places(r["start"], r["lens"])
    k1, v1 = r["k0"].copy(), r["v0"].copy()
    n = len(places)
    rows, pos = [p[0] for p in places], [p[2] for p in places]
    for layer in range(r["k"].shape[0]):
        def held(got, x):
            want = O.turn(x, pos, freq, interleaved, amplitude) if n else x
            pair = 4 * 2.0 ** -23 * amplitude * np.abs(x).max(-1, keepdims=True)
            assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + pair).all()
            np.testing.assert_array_equal(got[..., 2 * len(freq):], x[..., 2 * len(freq):])
        got_k = np.stack([r["k1"][layer, r["table"][b, p // PAGE], :, p % PAGE] for _, b, p in places])
        held(got_k, r["k"][layer, rows])
        for row, b, p in places:
            page = r["table"][b, p // PAGE]
            k1[layer, page, :, p % PAGE] = r["k1"][layer, page, :, p % PAGE]
            v1[layer, page, :, p % PAGE] = r["v"][layer, row]
        if with_q:
            held(r["q_out"][layer, rows], r["q"][layer, rows])
            rest = r["q_out"][layer, n:]
            np.testing.assert_array_equal(rest, r["q"][layer, n:] if in_place else np.full_like(rest, 7.0))
    np.testing.assert_array_equal(r["k1"], k1)                     # nothing else of the pools was touched
    np.testing.assert_array_equal(r["v1"], v1)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 32), (128, 112)])
def test_layouts_and_parts_of_the_head(d, rotary, interleaved):
    m = make(6, 2, d)
    rope = m.rope(rotary_dim=rotary, interleaved=interleaved, theta=1e4)
    r = run(m, [0, 15, 100, 7], [1, 40, 17, 0], layers=2, pad=3, rope=rope, seed=rotary)
    check(m, r, O.rope_frequencies(rotary, 1e4), interleaved, 1.0)


@pytest.mark.parametrize("scaling,high", [("linear", 32.0), ("turns", 4.0), ("pairs", 32.0)])
def test_scalings_at_far_positions(scaling, high):
    m = make(4, 4, 128)
    a = dict(theta=1e6, scaling=scaling, factor=16.0, original_len=8192, low=1.0, high=high, amplitude=1.2)
    r = run(m, [0, 3, 900], [5, 1, 9], rope=m.rope(**a), seed=3, far=1_000_000)
    check(m, r, O.rope_frequencies(128, 1e6, scaling, 16.0, 8192, 1.0, high), False, 1.2)


@pytest.mark.parametrize("counts", [[1], [1] * 33, [3, 0, 0, 2, 1], [0, 0, 4], [700, 1, 301]])
@pytest.mark.parametrize("fused", [False, True])
def test_ragged_rows_and_columns_of_one_projection(counts, fused):
    m = make(8, 8, 64)
    lens = [(37 * b) % 101 for b in range(len(counts))]
    r = run(m, lens, counts, layers=3, pad=len(counts) % 2, rope=m.rope(theta=5e5), fused=fused, seed=len(counts))
    check(m, r, O.rope_frequencies(64, 5e5), False, 1.0)


def test_many_requests():
    m = make(2, 1, 64)
    counts = [(b * 7) % 3 for b in range(1024)]
    r = run(m, [b % 50 for b in range(1024)], counts, rope=m.rope())
    check(m, r, O.rope_frequencies(64, 1e6), False, 1.0)


def test_without_rotation_without_queries_and_in_place():
    m = make(10, 2, 128)
    r = run(m, [5, 60], [20, 3], rope=None)
    check(m, r, np.zeros(0), False, 1.0)
    np.testing.assert_array_equal(r["q_out"][:, :23], r["q"][:, :23])
    r = run(m, [5, 60], [20, 3], rope=m.rope(), with_q=False)
    check(m, r, O.rope_frequencies(128, 1e6), False, 1.0, with_q=False)
    r = run(m, [5, 60], [20, 3], rope=m.rope(), in_place=True, pad=2)
    check(m, r, O.rope_frequencies(128, 1e6), False, 1.0, in_place=True)


def test_uniform_rows_and_an_empty_call():
    m = make(2, 2, 64)
    k = torch.randn((1, 9, 2, 64), device="cuda").to(torch.bfloat16)
    pools = [torch.zeros((1, 4, 2, PAGE, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    kv = m.kv(*pools, table, torch.tensor([14, 3], dtype=torch.int32, device="cuda"))
    m.mirror_kv_append(kv, m.rows(None, 9, 4, 2), k, k)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    v = pools[1][0]
    assert torch.equal(v[0, :, 14:16].transpose(0, 1), k[0, :2]) and torch.equal(v[1, :, :2].transpose(0, 1), k[0, 2:4])
    assert torch.equal(v[2, :, 3:7].transpose(0, 1), k[0, 4:8]) and v[3].abs().sum() == 0
    before = m.launch_count()
    m.mirror_kv_append(kv, m.rows(torch.zeros(3, dtype=torch.int32, device="cuda"), 0, 1), k[:, :0], k[:, :0])
    assert m.launch_count() == before


def test_positions_and_pages_outside_are_reported_and_skipped():
    m = make(2, 2, 64)
    for lens, table in (([31, 0], [[0, 1], [2, 3]]), ([-3, 0], [[0, 1], [2, 3]]), ([0, 0], [[4, 1], [2, 3]]), ([0, 0], [[-1, 1], [2, 3]])):
        k = torch.randn((1, 8, 2, 64), device="cuda").to(torch.bfloat16)
        pools = [torch.zeros((1, 4, 2, PAGE, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        kv = m.kv(*pools, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        m.mirror_kv_append(kv, m.rows(None, 8, 4, 2), k, k, rope=m.rope())
        torch.cuda.synchronize()
        assert m.device_status() == (6, 820)
        assert torch.equal(pools[1][0, 2, :, :4].transpose(0, 1), k[0, 4:8])             # the other request's rows are there
        good = [i for i in range(4) if 0 <= lens[0] + i < 32 and 0 <= table[0][(lens[0] + i) // 16] < 4]
        assert int((pools[1] != 0).any(-1).any(2).sum()) == 4 + len(good)


def test_refusals():
    m = make(4, 2, 64)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    pools = [torch.zeros((2, 4, 2, PAGE, 64), **bf) for _ in range(2)]
    kv = m.kv(*pools, torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"))
    k, q = torch.zeros((2, 8, 2, 64), **bf), torch.zeros((2, 8, 4, 64), **bf)
    rows = m.rows(None, 8, 4, 2)
    for bad in (k[:1], k[:, :7], q, k.float(), k.transpose(1, 2), torch.zeros((2, 8, 2, 128), **bf)[..., ::2]):
        with pytest.raises(ValueError):
            m.mirror_kv_append(kv, rows, bad, k)
    with pytest.raises(ValueError):
        m.mirror_kv_append(kv, rows, k, torch.zeros((2, 8, 4, 64), **bf)[:, :, :2])      # other strides than k's
    with pytest.raises(ValueError):
        m.mirror_kv_append(kv, rows, k, k, q=q, q_out=q[:, :, :2])
    with pytest.raises(ValueError):
        m.rope(scaling="other")
    with pytest.raises(ValueError):
        m.rows(None, 8, 4)

    def code(rows, k=k, kv_row=128, kv_layer=1024, q=None, q_out=None, q_row=256, rope=None):
        with pytest.raises(binding.MirrorError) as e:
            binding._check(m.lib.mirror_kv_append(m._ctx, kv_ref, rows_ref(rows), rope, q, q_row, 2048, q_out, k.data_ptr() if hasattr(k, "data_ptr") else k, pools[0].data_ptr(),
                                                  kv_row, kv_layer, None), "mirror_kv_append")
        return e.value.code
    import ctypes as C
    kv_ref, rows_ref = C.byref(kv), C.byref
    assert code(m.rows(None, 7, 4, 2)) == 2                              # rows that do not fit
    assert code(m.rows(None, 8, 0, 2)) == 1 and code(m.rows(None, -1, 4, 2)) == 1 and code(m.rows(None, 8, 4, 0)) == 1
    assert code(m.rows(None, 8192, 4, 1025)) == 2
    assert code(rows, kv_row=132) == 2 and code(rows, kv_row=64) == 2 and code(rows, kv_layer=1028) == 2 and code(rows, kv_layer=-8) == 2
    assert code(rows, k=k.data_ptr() + 2) == 1
    assert code(rows, q=q.data_ptr()) == 1 and code(rows, q=q.data_ptr(), q_out=q.data_ptr(), q_row=128) == 2
    bad = m.rope()
    for value in (0, 24, 80):
        bad.rotary_dim = value
        assert code(rows, rope=C.byref(bad)) == 2


def test_in_place_only_where_the_queries_are_contiguous():
    m = make(4, 2, 64)
    import ctypes as C
    bf = dict(dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k, q = torch.zeros((2, 8, 2, 64), **bf), torch.zeros((2, 16, 4, 64), **bf)

    def code(L, R, q_row, q_layer, q_out=None):
        pools = [torch.zeros((L, 4, 2, PAGE, 64), **bf) for _ in range(2)]
        kv, rows = m.kv(*pools, table, lens), m.rows(None, R, R, 1)
        got = m.lib.mirror_kv_append(m._ctx, C.byref(kv), C.byref(rows), None, q.data_ptr(), q_row, q_layer, q.data_ptr() if q_out is None else q_out,
                                     k.data_ptr(), k.data_ptr(), 128, 1024, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return got
    assert code(2, 8, 256, 2048) == 0 and code(1, 8, 256, 0) == 0 and code(2, 1, 512, 256) == 0
    other = torch.empty((2, 8, 4, 64), **bf).data_ptr()
    for L, R, q_row, q_layer in ((1, 8, 512, 0), (2, 8, 256, 4096), (2, 8, 256, 0), (2, 8, 512, 4096), (2, 1, 256, 512)):
        assert code(L, R, q_row, q_layer) == 1
        assert code(L, R, q_row, q_layer, other) == 0              # (the same queries, out of place)


def test_rows_beyond_max_rows_are_reported_and_skipped():
    """As mirror_attn_causal does: what it would not see is not appended."""
    m = make(2, 2, 64)
    k, q = (torch.randn((1, 9, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    pools = [torch.zeros((1, 4, 2, PAGE, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kv = m.kv(*pools, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([14, 0], dtype=torch.int32, device="cuda"))
    start = torch.tensor([0, 5, 8], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    m.mirror_kv_append(kv, m.rows(start, 9, 3), k, k, q=q, q_out=out)
    torch.cuda.synchronize()
    assert m.device_status() == (6, 830)
    v = pools[1][0]
    assert torch.equal(v[0, :, 14:].transpose(0, 1), k[0, :2]) and torch.equal(v[1, :, :1].transpose(0, 1), k[0, 2:3])
    assert torch.equal(v[2, :, :3].transpose(0, 1), k[0, 5:8]) and int((pools[1] != 0).any(-1).any(2).sum()) == 6
    assert torch.equal(out[0, [0, 1, 2, 5, 6, 7]], q[0, [0, 1, 2, 5, 6, 7]]) and (out[0, [3, 4, 8]] == 7.0).all()
    m.mirror_kv_append(kv, m.rows(start, 9, 5), k, k, q=q, q_out=out)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0) and torch.equal(out[0, :8], q[0, :8])
