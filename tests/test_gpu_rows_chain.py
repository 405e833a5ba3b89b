"""Appending, attention without a tree and sampling together, as a server uses them, and beside the calls that were there."""
import math

import numpy as np
import pytest
import torch

from oracle import rows as O
from paper_2510_13161_b200 import binding, inputs as I
from tests.rows_helpers import PAGE, make

pytestmark = pytest.mark.gpu


def cache(L, B, pages, hkv, d, dev="cuda"):
    """Zeroed pools, and a table with pages of its own for each request, in no order."""
    order = torch.randperm(B * pages, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    z = lambda: torch.zeros((L, B * pages, hkv, PAGE, d), dtype=torch.bfloat16, device=dev)  # noqa: E731
    return z(), z(), order.view(B, pages).to(dev)


def test_prompt_chunks_and_tokens_give_what_one_prompt_gives():
    """A prompt at once, the same in three chunks, and the same token by token: one cache, one attention, to the rounding of P and
    of the output (each half a bf16 step: of the value, or of the weights' sum of |v|)."""
    L, B, hq, hkv, d, n = 2, 3, 10, 2, 128, 150
    m = make(hq, hkv, d)
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = torch.randn((L, B, n, hq + 2 * hkv, d), device="cuda", generator=g).to(torch.bfloat16)
    rope = m.rope(theta=1e5, interleaved=True, rotary_dim=64)
    results = []
    for cuts in ([0, n], [0, 1, 65, n], list(range(0, n + 1))):
        k_pool, v_pool, table = cache(L, B, 10, hkv, d)
        out = torch.empty((L, B, n, hq, d), dtype=torch.bfloat16, device="cuda")
        for a, b in zip(cuts, cuts[1:]):
            kv = m.kv(k_pool, v_pool, table, torch.full((B,), a, dtype=torch.int32, device="cuda"))
            rows = m.rows(None, B * (b - a), b - a, B)
            x = qkv[:, :, a:b].reshape(L, B * (b - a), hq + 2 * hkv, d)
            q = m.mirror_kv_append(kv, rows, x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], q=x[:, :, :hq], rope=rope)
            out[:, :, a:b] = m.mirror_attn_causal(kv, rows, q, window=100, sinks=3).view(L, B, b - a, hq, d)
        torch.cuda.synchronize()
        assert m.device_status() == (0, 0)
        results.append((k_pool, v_pool, out))
    v_most = float(qkv[..., hq + hkv:, :].abs().max())
    for k_pool, v_pool, out in results[1:]:
        assert torch.equal(k_pool, results[0][0]) and torch.equal(v_pool, results[0][1])
        a, b = out.double(), results[0][2].double()
        assert ((a - b).abs() <= 2 * 2.0 ** -8 * b.abs() + (2.0 ** -8 + 1e-5) * v_most).all()


@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 64, 5), (10, 2, 128, 17), (16, 2, 128, 2)])
def test_verify_attention_of_a_chain_is_the_attention_of_its_appended_rows(hq, hkv, d, n):
    """mirror_attn_verify of a chain of n nodes over a prompt's cache, and mirror_attn_causal of the same rows appended to it."""
    L, B, lens = 2, 2, [70, 33]
    m = make(hq, hkv, d)
    g = torch.Generator(device="cuda").manual_seed(n)
    bf = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    k_pool, v_pool, table = cache(L, B, 8, hkv, d)
    k_pool.copy_(bf(*k_pool.shape)), v_pool.copy_(bf(*v_pool.shape))
    kv = m.kv(k_pool, v_pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q, k, v = bf(L, B, n, hq, d), bf(L, B, n, hkv, d), bf(L, B, n, hkv, d)
    tree = m.tree(torch.zeros((B, n), dtype=torch.int32, device="cuda"), 1, n - 1)
    want = m.mirror_attn_verify(kv, tree, q, k, v)
    rows = m.rows(None, B * n, n, B)
    flat = lambda t: t.view(L, B * n, t.shape[3], d)  # noqa: E731
    m.mirror_kv_append(kv, rows, flat(k), flat(v))
    got = m.mirror_attn_causal(kv, rows, flat(q)).view(L, B, n, hq, d)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    # both round P (2^-8 of the weights' sum of |v| each) and the output
    assert ((got.double() - want.double()).abs() <= 2 * 2.0 ** -8 * want.double().abs() + (2 * 2.0 ** -8 + 1e-5) * float(v.abs().max().clamp(min=v_pool.abs().max()))).all()


def test_a_prompt_then_a_verify_step_with_a_sampled_draft():
    """Fill the cache with a prompt, sample a draft chain from filtered distributions, verify it with the target's logits filtered alike:
    the draft's distribution is the target's, so everything is accepted, and the extra token comes from the kept ids."""
    V, gamma, B = 3000, 4, 2
    m = make(4, 2, 64, vocab=V)
    g = torch.Generator(device="cuda").manual_seed(5)
    logits = torch.randn((B, gamma + 1, V), device="cuda", generator=g) * 3
    u = torch.rand((B, gamma + 1), device="cuda", generator=g)
    T, k, p = (torch.full((B * (gamma + 1),), x, device="cuda", dtype=t) for x, t in ((0.8, torch.float32), (40, torch.int32), (0.9, torch.float32)))
    s = m.mirror_sample(logits.view(-1, V), u.view(-1), temperature=T, top_k=k, top_p=p, want_probs=True, want_logits=True)
    token, probs = s["token"].view(B, gamma + 1), s["probs"].view(B, gamma + 1, V)
    tokens = torch.cat((torch.zeros((B, 1), dtype=torch.int32, device="cuda"), token[:, :gamma]), 1).contiguous()
    tree = m.tree(tokens, 1, gamma)
    n = gamma + 1
    acc = m.accept_in(binding.ACCEPT_SPEC_SAMPLING, True, logits=s["logits"], lse=torch.zeros(B * n, device="cuda"), q_probs=probs[:, :gamma].contiguous(),
                      u_accept=torch.rand((B, n), device="cuda", generator=g) * 0.999, u_resample=torch.rand((B, n), device="cuda", generator=g))
    res = m.mirror_accept_select(tree, acc)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    got = res.cpu()
    assert got["n_accepted"].tolist() == [gamma] * B and got["n_emitted"].tolist() == [gamma + 1] * B
    for b in range(B):
        assert got["emitted"][b, :gamma].tolist() == token[b, :gamma].tolist()
        assert probs[b, gamma, got["emitted"][b, gamma]] > 0
    # the distribution is the oracle's, and a kept row sums to one
    want = O.sample_row(logits[0, 0].cpu().numpy(), float(np.float32(0.8)), 40, float(np.float32(0.9)), 0.0, float(u[0, 0]))
    assert want[0] == int(token[0, 0]) and want[1] == int(s["n_kept"][0])
    assert torch.allclose(probs.sum(-1), torch.ones((B, n), device="cuda"), atol=1e-5)


def test_a_layer_of_a_prompt_through_the_framework():
    """RMSNorm, projection, append, attention, output projection with residual: one layer of a prompt and then of a single token, against
    64 bits.  Every stored tensor is rounded to bf16 once: the oracle takes the stored ones, so each step is held on its own."""
    H, hq, hkv, d, B, lens = 256, 4, 2, 64, 2, [40, 9]
    m = make(hq, hkv, d)
    g = torch.Generator(device="cuda").manual_seed(3)
    bf = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).to(torch.bfloat16)  # noqa: E731
    w_qkv, w_o, gamma_w = bf((hq + 2 * hkv) * d, H, std=H ** -0.5), bf(H, hq * d, std=(hq * d) ** -0.5), bf(H)
    k_pool, v_pool, table = cache(1, B, 5, hkv, d)
    rope = m.rope(theta=1e4)
    freq = O.rope_frequencies(d, 1e4)
    done = [0, 0]
    for counts in (lens, [1, 1]):
        start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        R = int(start[-1])
        x = bf(R, H)
        h = m.mirror_rmsnorm(x, gamma_w)
        qkv = m.mirror_linear(h, w_qkv).view(1, R, hq + 2 * hkv, d)
        kv = m.kv(k_pool, v_pool, table, torch.tensor(done, dtype=torch.int32, device="cuda"))
        rows = m.rows(torch.from_numpy(start).cuda(), R, max(counts))
        q = m.mirror_kv_append(kv, rows, qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], q=qkv[:, :, :hq], rope=rope)
        a = m.mirror_attn_causal(kv, rows, q)
        y = m.mirror_linear(a.view(R, hq * d), w_o, residual=x)
        torch.cuda.synchronize()
        assert m.device_status() == (0, 0)
        n = lambda t: t.double().cpu().numpy()  # noqa: E731
        places = O.row_places(start, done)
        pos = [p for _, _, p in places]
        want_q = O.turn(n(qkv[0, :, :hq]), pos, freq, False)
        assert (np.abs(n(q[0]) - want_q) <= 2.0 ** -8 * np.abs(want_q) + 1e-5).all()
        want_k = O.turn(n(qkv[0, :, hq:hq + hkv]), pos, freq, False)
        tb = table.cpu().numpy()
        got_k = np.stack([n(k_pool[0, tb[b, p // PAGE], :, p % PAGE]) for _, b, p in places])
        assert (np.abs(got_k - want_k) <= 2.0 ** -8 * np.abs(want_k) + 1e-5).all()
        want_a, _ = O.causal_attention(n(q[0]), n(k_pool[0]), n(v_pool[0]), tb, done, start, 0, 0, d ** -0.5)
        v_most = float(v_pool.abs().max())
        assert (np.abs(n(a[0]) - want_a) <= 2.0 ** -8 * np.abs(want_a) + (2.0 ** -8 + 1e-5) * v_most).all()
        want_y = n(a.view(R, hq * d)) @ n(w_o).T + n(x)
        assert (np.abs(n(y) - want_y) <= 2.0 ** -8 * np.abs(want_y) + 1e-3).all()
        done = [t + c for t, c in zip(done, counts)]
    assert math.isfinite(float(y.float().sum())) and I.PAGE_SIZE == PAGE


def test_the_whole_chain_captured_and_replayed():
    """Append, attention and sampling of a single token in one graph: replayed, it repeats what it gave."""
    V, hq, hkv, d, B = 1000, 8, 2, 64, 3
    m = make(hq, hkv, d, vocab=V)
    g = torch.Generator(device="cuda").manual_seed(9)
    bf = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    k_pool, v_pool, table = cache(1, B, 6, hkv, d)
    k_pool.copy_(bf(*k_pool.shape)), v_pool.copy_(bf(*v_pool.shape))
    lens = torch.tensor([80, 0, 17], dtype=torch.int32, device="cuda")
    kv, rows, rope = m.kv(k_pool, v_pool, table, lens), m.rows(None, B, 1, B), m.rope()
    q, k, v, W = bf(1, B, hq, d), bf(1, B, hkv, d), bf(1, B, hkv, d), torch.randn((hq * d, V), device="cuda", generator=g) * 0.2
    u, p = torch.rand(B, device="cuda", generator=g), torch.full((B,), 0.9, device="cuda")

    def step():
        a = m.mirror_attn_causal(kv, rows, m.mirror_kv_append(kv, rows, k, v, q=q, rope=rope), window=50, sinks=2)
        return a, m.mirror_sample(a.view(B, hq * d).float() @ W, u, top_p=p)
    want_a, want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, got = step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, want_a) and torch.equal(got["token"], want["token"]) and m.device_status() == (0, 0)


def test_a_captured_call_after_the_workspace_has_grown():
    """A graph's attention keeps the workspace that it was captured with when a later call needs a larger one: its replay is right, and
    writes into nothing that was allocated since."""
    hq, hkv, d, n = 8, 2, 128, 30
    m = make(hq, hkv, d, vocab=30000)
    g = torch.Generator(device="cuda").manual_seed(2)
    bf = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    k_pool, v_pool, table = cache(1, 1, 200, hkv, d)
    k_pool.copy_(bf(*k_pool.shape)), v_pool.copy_(bf(*v_pool.shape))
    kv, rows, q = m.kv(k_pool, v_pool, table, torch.tensor([3000], dtype=torch.int32, device="cuda")), m.rows(None, n, n, 1), bf(1, n, hq, d)
    want = m.mirror_attn_causal(kv, rows, q)                     # (one request over 3030 tokens: its unit is cut, records are written)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = m.mirror_attn_causal(kv, rows, q)
    before = m._ws.data_ptr(), m._ws.numel()
    m.mirror_lmhead_reduce(bf(300, 256), bf(30000, 256))
    assert m._ws.numel() > before[1]
    torch.cuda.synchronize()
    others = [torch.full((before[1],), 7, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert all(t.data_ptr() != before[0] for t in others)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all((t == 7).all() for t in others) and m.device_status() == (0, 0)


def test_one_cache_from_the_prompt_through_a_verify_step_and_on():
    """A model of one layer (Q, K, V and logits by way of its tokens' rows of a table) over one cache: two prompts, single tokens without
    a draft, a drafted chain with its distributions, mirror_verify_step of that chain, mirror_kv_commit, and a token more.  The draft is the
    target, so all of it is accepted (u <= 0.8, and p and q differ by the roundings of P alone); what the cache then holds is what
    one prompt of the whole sequence leaves, bit for bit, and the last row's attention is that prompt's to the roundings of P and the output."""
    hq, hkv, d, V, B, gamma = 4, 2, 64, 3000, 2, 4
    H = hq * d
    m = make(hq, hkv, d, vocab=V)
    g = torch.Generator(device="cuda").manual_seed(17)
    bf = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).to(torch.bfloat16)  # noqa: E731
    qkv_of = m.mirror_linear(bf(V, H), bf((hq + 2 * hkv) * d, H, std=H ** -0.5)).view(V, hq + 2 * hkv, d)
    W, rope = bf(V, H, std=0.1), m.rope(theta=1e4)
    k_pool, v_pool, table = cache(1, B, 6, hkv, d)
    lens = [37, 9]
    i32 = dict(dtype=torch.int32, device="cuda")
    done = torch.zeros(B, **i32)
    seq = [torch.randint(0, V, (n,), device="cuda", generator=g).tolist() for n in lens]

    def forward(tokens, pools=None, at=None):
        """Appends ragged tokens, attends; -> (turned queries, attention) [1, R, hq, d]."""
        start = np.concatenate([[0], np.cumsum([len(t) for t in tokens])]).astype(np.int32)
        x = qkv_of[torch.tensor(sum(tokens, []), device="cuda")].unsqueeze(0)
        kv = m.kv(*(pools or (k_pool, v_pool)), table, done if at is None else at)
        rows = m.rows(torch.from_numpy(start).cuda(), int(start[-1]), max(len(t) for t in tokens))
        q = m.mirror_kv_append(kv, rows, x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], q=x[:, :, :hq], rope=rope)
        return q, m.mirror_attn_causal(kv, rows, q)

    def draw(a, temperature, p=1.0):
        logits = m.mirror_lmhead_reduce(a.reshape(B, H).contiguous(), W, want_logits=True)["logits"]
        f = lambda x: torch.full((B,), x, device="cuda")  # noqa: E731
        return m.mirror_sample(logits, torch.rand(B, device="cuda", generator=g), temperature=f(temperature), top_p=f(p), want_probs=True)

    # the prompts, and three tokens without a draft (the last of them stays out of the cache: the tree's root)
    _, a = forward(seq)
    a = a[0, torch.tensor(np.cumsum(lens) - 1, device="cuda")]
    done += torch.tensor(lens, **i32)
    for step in range(3):
        new = draw(a, 0.8, 0.9)["token"].tolist()
        for b in range(B):
            seq[b].append(new[b])
        if step < 2:
            _, a = forward([[t] for t in new])
            done += 1
    # the draft: it continues in the pages behind the cache's tokens, which are not counted
    root, chain, probs, qs, at = new, [], [], [], done.clone()
    for i in range(gamma + 1):
        q, a = forward([[t] for t in (root if i == 0 else chain[-1])], at=at)
        qs.append(q.view(1, B, 1, hq, d))
        at += 1
        if i < gamma:
            s = draw(a, 1.0)
            chain.append(s["token"].tolist())
            probs.append(s["probs"])
    where = (done[:, None] + torch.arange(gamma + 1, device="cuda")).long()                    # the nodes' positions
    pages, slots = table.long().gather(1, where // PAGE), where % PAGE
    k_new, v_new = (pool[:, pages, :, slots].permute(2, 0, 1, 3, 4).contiguous() for pool in (k_pool, v_pool))
    assert k_new.shape == (1, B, gamma + 1, hkv, d)
    for pool in (k_pool, v_pool):
        pool[:, pages, :, slots] = 100.0                         # (a verify step that read the draft's rows would be far off)
    tokens = torch.tensor([root] + chain, **i32).t().contiguous()
    tree, kv = m.tree(tokens, 1, gamma), m.kv(k_pool, v_pool, table, done)
    acc = m.accept_in(binding.ACCEPT_SPEC_SAMPLING, True, q_probs=torch.stack(probs, 1).contiguous(),
                      u_accept=torch.rand((B, gamma + 1), device="cuda", generator=g) * 0.8, u_resample=torch.rand((B, gamma + 1), device="cuda", generator=g))
    attn = torch.empty((1, B, gamma + 1, hq, d), dtype=torch.bfloat16, device="cuda")
    res = m.mirror_verify_step(kv, tree, torch.cat(qs, 2).contiguous(), k_new, v_new, None, W, acc, attn)
    m.mirror_kv_commit(kv, tree, k_new, v_new, res, done)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    got = res.cpu()
    assert got["n_accepted"].tolist() == [gamma] * B and got["n_emitted"].tolist() == [gamma + 1] * B
    assert got["emitted"][:, :gamma].tolist() == [[chain[i][b] for i in range(gamma)] for b in range(B)]
    assert done.tolist() == [n + 3 + gamma for n in lens]
    for b in range(B):
        seq[b] += got["emitted"][b].tolist()
    # a token more, and the whole sequence as one prompt
    _, a = forward([[s[-1]] for s in seq])
    pools, zero = tuple(torch.zeros_like(p) for p in (k_pool, v_pool)), torch.zeros(B, **i32)
    _, want = forward(seq, pools, zero)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    ends = np.cumsum([len(s) for s in seq])
    for b, s in enumerate(seq):
        assert len(s) == lens[b] + 4 + gamma and int(done[b]) == len(s) - 1
        for i in range(len(s)):
            for pool, whole in zip((k_pool, v_pool), pools):
                assert torch.equal(pool[:, table[b, i // PAGE], :, i % PAGE], whole[:, table[b, i // PAGE], :, i % PAGE]), (b, i)
    v_most = float(pools[1].abs().max())
    near = lambda x, y: ((x.double() - y.double()).abs() <= 2 * 2.0 ** -8 * y.double().abs() + (2 * 2.0 ** -8 + 1e-5) * v_most).all()  # noqa: E731
    assert near(a[0], want[0, torch.tensor(ends - 1, device="cuda")])
    for b in range(B):                                           # (the verify step's rows are that prompt's, too)
        assert near(attn[0, b], want[0, ends[b] - 2 - gamma:ends[b] - 1])
