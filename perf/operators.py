"""Operators around the verify step, as timed cases: filling the paged cache, attention without a draft tree, sampling.

The verify step takes a cache that somebody has filled, and a draft's distributions that somebody has drawn from.  These are
the calls of a serving program that does both:

  append   keys and values of new tokens (a prompt's chunk, or one token of each request) turned to their positions and put
           into the paged cache, the queries turned on the way
  attn     causal attention of those tokens over the paged cache, with or without a window and first tokens that stay visible
  sample   one token of each row of logits under a temperature, Top-k, Top-p and Min-p, from given uniforms; the filtered
           distribution as the draft's probabilities, or as the target's logits of a verification under the same filter

Values: queries, keys and values are N(0, 1).  Logits are N(0, 2.5) with a few dozen leaders per row, some rows nearly
decided and some open, as a language model's are.
"""
import math
import random

import torch

own = False

_14B = dict(hq=40, hkv=8, d=128)
_32B = dict(hq=64, hkv=8, d=128)
_SMALL = dict(hq=32, hkv=8, d=64)
_PAGE = 16


def listed():
    return [
        # One request decodes its next token: what is left is the launch.
        dict(name="append_token", kind="append", **_14B, layers=1, batch=1, rows_lo=1, rows_hi=1, lo=2048, hi=2048, pad=0,
             rotary=128, interleaved=False, scaling="none", factor=1.0),
        # A full batch of single tokens at far positions: neighbouring pairs, half of a small head, stretched by wavelength.
        dict(name="append_batch", kind="append", **_SMALL, layers=2, batch=256, rows_lo=1, rows_hi=1, lo=1000, hi=120001, pad=0,
             rotary=32, interleaved=True, scaling="turns", factor=8.0),
        # The chunks of a few prompts, one of them started before, with rows behind the last one.
        dict(name="append_prompts", kind="append", **_32B, layers=1, batch=5, rows_lo=257, rows_hi=4090, lo=0, hi=9001, pad=13,
             rotary=128, interleaved=False, scaling="pairs", factor=4.0),
        # One request with a long document behind it takes its next token.
        dict(name="attn_token_long", kind="attn", **_32B, layers=1, batch=1, rows_lo=1, rows_hi=1, lo=32768, hi=32768, pad=0, window=0, sinks=0),
        # A server's batch of single tokens, ragged contexts.
        dict(name="attn_token_batch", kind="attn", **_14B, layers=1, batch=64, rows_lo=1, rows_hi=1, lo=130, hi=8191, pad=0, window=0, sinks=0),
        # The same where a window keeps the long contexts cheap.
        dict(name="attn_token_window", kind="attn", **_SMALL, layers=2, batch=48, rows_lo=1, rows_hi=1, lo=1, hi=30011, pad=0, window=4096, sinks=4),
        # A chat prompt from its first token.
        dict(name="attn_prompt", kind="attn", **_14B, layers=1, batch=1, rows_lo=2048, rows_hi=2048, lo=0, hi=0, pad=0, window=0, sinks=0),
        # The last chunk of a long document.
        dict(name="attn_prompt_chunk", kind="attn", **_32B, layers=1, batch=1, rows_lo=2048, rows_hi=2048, lo=30720, hi=30720, pad=0, window=0, sinks=0),
        # Ragged chunks of several requests under a window.
        dict(name="attn_prompt_window", kind="attn", **_SMALL, layers=1, batch=7, rows_lo=5, rows_hi=2777, lo=0, hi=4001, pad=9, window=1000, sinks=20),
        # One request's next token under the usual three filters.
        dict(name="sample_token", kind="sample", vocab=152064, rows=1, top_k=50, top_p=0.95, min_p=0.02, out="none"),
        # A draft's batch: its tokens, and its distributions for the acceptance.
        dict(name="sample_draft", kind="sample", vocab=128256, rows=64, top_k=0, top_p=0.9, min_p=0.0, out="probs"),
        # Every node of 8 requests' trees, filtered as the target's logits.
        dict(name="sample_tree", kind="sample", vocab=128256, rows=520, top_k=1000, top_p=0.98, min_p=0.0, out="logits"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("append", "attn", "sample")}
    while True:
        kind = rng.choice(["append", "attn", "attn", "sample"])
        if kind == "sample":
            c = dict(kind=kind, vocab=_log_int(rng, 300, 256000), rows=_log_int(rng, 1, 600), top_k=rng.choice([0, 1, _log_int(rng, 2, 5000)]),
                     top_p=rng.choice([1.0, round(rng.uniform(0.05, 0.999), 3)]), min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.3), 4)]),
                     out=rng.choice(["none", "probs", "logits"]))
        else:
            c = dict(kind=kind, hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]), layers=_log_int(rng, 1, 4), batch=_log_int(rng, 1, 128))
            c["hq"] = c["hkv"] * rng.choice([1, 2, 4, 5, 7, 8, 16])
            single = rng.random() < 0.5
            c["rows_lo"] = 1 if single else _log_int(rng, 1, 2000)
            c["rows_hi"] = 1 if single else min(4000, int(c["rows_lo"] * rng.uniform(1.0, 6.0)))
            c["lo"] = rng.choice([0, _log_int(rng, 1, 20000)])
            c["hi"] = c["lo"] + _log_int(rng, 1, 12000) if c["batch"] > 1 else c["lo"]
            c["pad"] = rng.choice([0, 0, rng.randint(1, 40)])
            if kind == "append":
                c["rotary"] = rng.choice([c["d"], c["d"] // 2, 16 * rng.randint(1, c["d"] // 16)])
                c["interleaved"] = rng.random() < 0.5
                c["scaling"] = rng.choice(["none", "linear", "turns", "pairs"])
                c["factor"] = 1.0 if c["scaling"] == "none" else round(rng.uniform(1.5, 32.0), 2)
            else:
                c["window"] = rng.choice([0, _log_int(rng, 1, 8000)])
                c["sinks"] = rng.choice([0, rng.randint(1, 140)]) if c["window"] else 0
            if c["hq"] * c["d"] > 8192:
                continue
        if _cost(c) <= largest[kind] and _gigabytes(c) <= 6.0:
            return c


# ---- sizes ---------------------------------------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly apart: which request has which depends on the seed, their sum does not."""
    return [lo + (hi - lo) * i // max(n - 1, 1) for i in range(n)] if n > 1 else [hi]


def _counts(c):
    return _spread(c["rows_lo"], c["rows_hi"], c["batch"])


def _lens(c):
    return _spread(c["lo"], c["hi"], c["batch"])


def _pairing(c):
    """(rows, tokens before them) of the requests as work() counts them."""
    return list(zip(_counts(c), _lens(c)))


def _visible(n, before, window, sinks):
    """(query, key) pairs that n rows behind `before` tokens see, and distinct keys."""
    if not window:
        return n * before + n * (n + 1) // 2, before + n
    pairs = sum(min(window, p + 1) + min(sinks, max(0, p + 1 - window)) for p in range(before, before + n))
    first = max(0, before - window + 1)
    return pairs, before + n - first + min(sinks, first)


def work(case):
    c = case
    if c["kind"] == "sample":
        e = c["rows"] * c["vocab"]
        return {"bytes": 4 * e * (2 if c["out"] != "none" else 1) + 16 * c["rows"], "flops": 4 * e}
    per_row = c["d"] * 2 * c["layers"]
    if c["kind"] == "append":
        r = sum(_counts(c))
        return {"bytes": 2 * r * per_row * (c["hq"] + 2 * c["hkv"]), "flops": 3 * c["rotary"] * r * c["layers"] * (c["hq"] + c["hkv"])}
    seen = [_visible(n, t, c["window"], c["sinks"]) for n, t in _pairing(c)]
    return {"bytes": per_row * (2 * c["hkv"] * sum(k for _, k in seen) + 2 * c["hq"] * sum(_counts(c))),
            "flops": 4 * c["d"] * c["hq"] * c["layers"] * sum(p for p, _ in seen)}


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def _gigabytes(c):
    """What one pass of the plain form holds at a time, roughly."""
    if c["kind"] == "sample":
        return c["rows"] * c["vocab"] * 60 / 1e9
    b, n, t = c["batch"], c["rows_hi"], c["hi"] + c["rows_hi"]
    if c["kind"] == "append":
        return b * n * (c["hq"] + c["hkv"]) * c["d"] * 16 * c["layers"] / 1e9
    pool = b * t * c["hkv"] * c["d"] * 4 * c["layers"]
    return (pool + b * t * c["d"] * 8 + 10 * b * n * t * (c["hq"] // c["hkv"])) / 1e9


# ---- inputs --------------------------------------------------------------------------------------------------------
def _rope_args(c):
    """How a stretched rotation is set up: lengths up to 8192 seen in training, 1 to 32 turns over them blended."""
    low, high = (1.0, 4.0) if c["scaling"] == "turns" else (1.0, 32.0)
    amplitude = 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "pairs" else 1.0
    return dict(rotary_dim=c["rotary"], interleaved=c["interleaved"], theta=1e6, scaling=c["scaling"], factor=c["factor"],
                original_len=8192, low=low, high=high, amplitude=amplitude)


def _frequencies(a):
    """Radians per position of each pair, from the formulas that mirror.h gives for mirror_rope_init."""
    i = torch.arange(a["rotary_dim"] // 2, dtype=torch.float64)
    f = a["theta"] ** (-2.0 * i / a["rotary_dim"])
    if a["scaling"] == "linear":
        keep = torch.zeros_like(f)
    elif a["scaling"] == "turns":
        keep = ((f * a["original_len"] / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
    elif a["scaling"] == "pairs":
        at = lambda turns: a["rotary_dim"] * math.log(a["original_len"] / (2 * math.pi * turns)) / (2 * math.log(a["theta"]))  # noqa: E731
        first, last = max(math.floor(at(a["high"])), 0), min(math.ceil(at(a["low"])), a["rotary_dim"] - 1)
        keep = 1 - ((i - first) / max(last - first, 1e-3)).clamp(0, 1)
    else:
        keep = torch.ones_like(f)
    return f * (keep + (1 - keep) / a["factor"])


_handles = {}


def _handle(binding, c):
    """The library context that a program has for its model."""
    key = (c.get("hq", 8), c.get("hkv", 8), c.get("d", 128), c.get("vocab", 1024))
    if key not in _handles:
        _handles[key] = binding.Mirror(1024, *key)
    return _handles[key]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = random.Random(seed)
    f32 = dict(device="cuda", dtype=torch.float32, generator=g)
    s = dict(case=c)
    if c["kind"] == "sample":
        m, v = c["rows"], c["vocab"]
        z = torch.randn((m, v), **f32).mul_(2.5)
        # leaders: a few dozen ids well above the rest, by more in the rows that are nearly decided
        n = min(40, v)
        at = torch.arange(n, device="cuda") * (v // n) + torch.randint(0, v // n, (m, n), device="cuda", generator=g)
        z.scatter_(1, at, torch.rand((m, 1), **f32) * 8 + 5 + 2 * torch.randn((m, n), **f32))
        s["logits"] = z
        s["u"] = torch.rand(m, **f32)
        # each request has settings of its own around the case's
        s["temperature"] = torch.rand(m, **f32) * 0.8 + 0.5
        s["top_k"] = torch.full((m,), c["top_k"], dtype=torch.int32, device="cuda")
        s["top_p"] = torch.rand(m, **f32) * (1 - c["top_p"]) + c["top_p"]
        s["min_p"] = torch.rand(m, **f32) * c["min_p"]
        if own:
            from paper_2510_13161_b200 import binding
            s["m"] = _handle(binding, c)
        return s
    counts, lens = _counts(c), _lens(c)
    host.shuffle(counts)
    host.shuffle(lens)
    b, L, hq, hkv, d = c["batch"], c["layers"], c["hq"], c["hkv"], c["d"]
    r = sum(counts) + c["pad"]
    pages = [(t + n + _PAGE - 1) // _PAGE for t, n in zip(lens, counts)]
    most = max(pages)
    # Physical pages in no order, a few unused.  (Appending touches a request's last pages alone: the ones before share page 0.)
    skip = [t // _PAGE if c["kind"] == "append" else 0 for t in lens]
    order = list(range(1, sum(pages) - sum(skip) + 4))
    host.shuffle(order)
    table, at = torch.zeros((b, most), dtype=torch.int32), 0
    for i, k in enumerate(pages):
        table[i, skip[i]:k] = torch.tensor(order[at:at + k - skip[i]], dtype=torch.int32)
        at += k - skip[i]
    start = [0]
    for n in counts:
        start.append(start[-1] + n)
    bf = lambda *shape: torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=g)  # noqa: E731
    pool = (L, len(order) + 1, hkv, _PAGE, d)
    s.update(k_pool=bf(*pool), v_pool=bf(*pool), table=table.cuda(),
             prefix=torch.tensor(lens, dtype=torch.int32, device="cuda"), start=torch.tensor(start, dtype=torch.int32, device="cuda"),
             most_rows=max(counts), longest=max(t + n for t, n in zip(lens, counts)))
    if c["kind"] == "append":
        # the three are columns of one projection's output
        qkv = bf(L, r, hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        s["q_out"] = torch.zeros((L, r, hq, d), device="cuda", dtype=torch.bfloat16)
        s["freq"] = _frequencies(_rope_args(c)).cuda()
        s["amplitude"] = _rope_args(c)["amplitude"]
    else:
        s["q"] = bf(L, r, hq, d)
        s["out"] = torch.zeros((L, r, hq, d), device="cuda", dtype=torch.bfloat16)
        s["lse"] = torch.zeros((L, r, hq), device="cuda", dtype=torch.float32)
    if own:
        from paper_2510_13161_b200 import binding
        m = s["m"] = _handle(binding, c)
        s["kv"] = m.kv(s["k_pool"], s["v_pool"], s["table"], s["prefix"])
        s["rows"] = m.rows(s["start"], r, s["most_rows"])
        if c["kind"] == "append":
            s["rope"] = m.rope(**_rope_args(c))
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _places(s):
    """Of every row that belongs to a request: its request, and its position."""
    counts = (s["start"][1:] - s["start"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts)
    i = torch.arange(len(b), device="cuda") - s["start"].long()[b]
    return b, s["prefix"].long()[b] + i, i


def _turn(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    x = x.float()
    cos, sin = cos[None, :, None], sin[None, :, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., r:]), -1).to(torch.bfloat16)


def _append(s):
    c = s["case"]
    b, pos, _ = _places(s)
    n = len(b)
    angle = pos[:, None].double() * s["freq"]
    cos, sin = (angle.cos() * s["amplitude"]).float(), (angle.sin() * s["amplitude"]).float()
    s["q_out"][:, :n] = _turn(s["q"][:, :n], cos, sin, c["interleaved"])
    page, slot = s["table"][b, pos // _PAGE].long(), pos % _PAGE
    s["k_pool"][:, page, :, slot] = _turn(s["k"][:, :n], cos, sin, c["interleaved"]).transpose(0, 1)
    s["v_pool"][:, page, :, slot] = s["v"][:, :n].transpose(0, 1)
    return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _attn(s):
    """All requests side by side, padded to the longest; a KV head at a time, since the scores of all do not fit the card."""
    c = s["case"]
    L, hkv, d, w = c["layers"], c["hkv"], c["d"], c["window"]
    G, n, T = c["hq"] // hkv, s["most_rows"], s["longest"]
    b, _, i = _places(s)
    B, rows = len(s["prefix"]), len(b)
    pos = s["prefix"].long()[:, None] + torch.arange(n, device="cuda")                        # [B, n]
    key = torch.arange(T, device="cuda")
    sees = key <= pos[..., None]
    if w:
        sees &= (key > pos[..., None] - w) | (key < c["sinks"])
    sees = sees[:, :, None]
    q = torch.zeros((B, n, hkv, G, d), device="cuda")
    for l in range(L):
        q[b, i] = s["q"][l, :rows].float().view(rows, hkv, G, d)
        for h in range(hkv):
            k = s["k_pool"][l, :, h][s["table"].long()].flatten(1, 2)[:, :T].float()          # [B, T, d]
            v = s["v_pool"][l, :, h][s["table"].long()].flatten(1, 2)[:, :T].float()
            a = (q[:, :, h].flatten(1, 2) @ k.transpose(1, 2)).view(B, n, G, T).mul_(d ** -0.5)
            a.masked_fill_(~sees, -math.inf)
            top = a.amax(-1, keepdim=True)
            a.sub_(top).exp_()
            sums = a.sum(-1, keepdim=True)
            o = (a.flatten(1, 2) @ v).view(B, n, G, d) / sums
            s["out"][l, :rows, h * G:(h + 1) * G] = o[b, i].to(torch.bfloat16)
            s["lse"][l, :rows, h * G:(h + 1) * G] = (top + sums.log())[b, i, :, 0]
    return {"out": s["out"], "lse": s["lse"]}


def _sample(s):
    c = s["case"]
    z = s["logits"].double() / s["temperature"].double()[:, None]
    M, V = z.shape
    order = s["logits"].sort(dim=1, descending=True, stable=True).indices
    w = (z - z.amax(1, keepdim=True)).exp()
    ranked = w.gather(1, order)
    rank = torch.arange(V, device="cuda")
    if c["top_k"]:
        ranked = ranked * (rank < s["top_k"].long()[:, None])
    # the shortest front of the ranks with that share: an id stays if what comes before it is less
    before = ranked.cumsum(1) - ranked
    p = s["top_p"].double()[:, None]
    stays = (ranked > 0) & ((p >= 1) | (before < p * ranked.sum(1, keepdim=True))) & (ranked >= s["min_p"].double()[:, None])
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(stays, ranked, 0.0))
    total = kept.sum(1, keepdim=True)
    cdf = kept.cumsum(1)
    token = (cdf <= s["u"].double()[:, None] * total).sum(1)
    prob = kept / total
    got = {"token": token.int(), "n_kept": stays.sum(1).int(), "logprob": prob.gather(1, token[:, None])[:, 0].log().float()}
    if c["out"] == "probs":
        got["probs"] = prob.float()
    elif c["out"] == "logits":
        got["logits"] = prob.log().float()
    return got


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _append, "attn": _attn, "sample": _sample}[c["kind"]](s)
    m = s["m"]
    if c["kind"] == "append":
        m.mirror_kv_append(s["kv"], s["rows"], s["k"], s["v"], q=s["q"], rope=s["rope"], q_out=s["q_out"])
        return {"q": s["q_out"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    if c["kind"] == "attn":
        m.mirror_attn_causal(s["kv"], s["rows"], s["q"], window=c["window"], sinks=c["sinks"], out=s["out"], lse_out=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    got = m.mirror_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"] if c["top_k"] else None, top_p=s["top_p"],
                          min_p=s["min_p"], want_probs=c["out"] == "probs", want_logits=c["out"] == "logits")
    return {k: v for k, v in got.items() if v is not None}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "sample":
        return _exact_sample(s)
    start, lens = s["start"].tolist(), s["prefix"].tolist()
    if c["kind"] == "append":
        return _exact_append(s, start, lens)
    if work(c)["flops"] > 3e13:
        return None
    L, hkv, d = c["layers"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    out, lse = s["out"].double(), s["lse"].double()
    for r, before in enumerate(lens):
        r0, r1 = start[r], start[r + 1]
        T = before + r1 - r0
        pages = s["table"][r, :(T + _PAGE - 1) // _PAGE].long()
        j = torch.arange(T, device="cuda")
        for l in range(L):
            for h in range(hkv):
                k = s["k_pool"][l, pages, h].reshape(-1, d)[:T].double()
                v = s["v_pool"][l, pages, h].reshape(-1, d)[:T].double()
                for q0 in range(r0, r1, 512):
                    q1 = min(q0 + 512, r1)
                    p = torch.arange(before + q0 - r0, before + q1 - r0, device="cuda")[:, None]
                    hidden = j > p
                    if c["window"]:
                        hidden |= (j <= p - c["window"]) & (j >= c["sinks"])
                    x = torch.einsum("rgd,td->rgt", s["q"][l, q0:q1, h * G:(h + 1) * G].double(), k) / math.sqrt(d)
                    x.masked_fill_(hidden[:, None], -math.inf)
                    z = torch.logsumexp(x, -1)
                    out[l, q0:q1, h * G:(h + 1) * G] = torch.einsum("rgt,td->rgd", torch.exp(x - z[..., None]), v)
                    lse[l, q0:q1, h * G:(h + 1) * G] = z
    return {"out": out, "lse": lse}


def _exact_append(s, start, lens):
    c, a = s["case"], _rope_args(s["case"])
    r = c["rotary"]
    q, k_pool, v_pool = s["q_out"].double(), s["k_pool"].double(), s["v_pool"].double()
    freq = []
    for i in range(r // 2):
        f = math.exp(-2.0 * i / r * math.log(a["theta"]))
        if a["scaling"] == "linear":
            f /= a["factor"]
        elif a["scaling"] == "turns":
            t = a["original_len"] * f / (2 * math.pi)
            share = min(1.0, max(0.0, (t - a["low"]) / (a["high"] - a["low"])))
            f = share * f + (1 - share) * f / a["factor"]
        elif a["scaling"] == "pairs":
            ends = [r / 2 * math.log(a["original_len"] / (2 * math.pi * t)) / math.log(a["theta"]) for t in (a["high"], a["low"])]
            lo, hi = max(0, math.floor(ends[0])), min(r - 1, math.ceil(ends[1]))
            slow = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
            f = slow * f / a["factor"] + (1 - slow) * f
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    first = torch.arange(r // 2, device="cuda") * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else r // 2)

    def turned(x, pos):
        # a rotation as a product of complex numbers
        w = torch.polar(torch.full((len(pos), r // 2), a["amplitude"], dtype=torch.float64, device="cuda"), pos[:, None] * freq)
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * w[:, None]
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    for b, before in enumerate(lens):
        n = start[b + 1] - start[b]
        pos = torch.arange(before, before + n, device="cuda")
        page, slot = s["table"][b].long()[pos // _PAGE], pos % _PAGE
        for l in range(c["layers"]):
            rows = slice(start[b], start[b + 1])
            q[l, rows] = turned(s["q"][l, rows], pos.double())
            k_pool[l, page, :, slot] = turned(s["k"][l, rows], pos.double())
            v_pool[l, page, :, slot] = s["v"][l, rows].double()
    return {"q": q, "k_pool": k_pool, "v_pool": v_pool}


def _exact_sample(s):
    """Row by row: the kept ids as a list, in the order of their ranks."""
    c = s["case"]
    got = {"token": [], "n_kept": [], "logprob": []}
    whole = []
    for r in range(c["rows"]):
        x = s["logits"][r].double()
        ids = torch.argsort(x, descending=True, stable=True)
        if c["top_k"]:
            ids = ids[:int(s["top_k"][r])]
        p = torch.softmax(x[ids] / s["temperature"][r].double(), 0)
        n = len(ids)
        if float(s["top_p"][r]) < 1:
            n = min(n, 1 + int((p.cumsum(0) < s["top_p"][r].double()).sum()))
        n = max(1, min(n, int((p >= s["min_p"][r].double() * p[0]).sum())))
        ids, at = ids[:n].sort()
        p = p[:n][at] / p[:n].sum()
        cdf = p.cumsum(0)
        k = min(int((cdf <= s["u"][r].double() * cdf[-1]).sum()), n - 1)
        got["token"].append(int(ids[k]))
        got["n_kept"].append(n)
        got["logprob"].append(p[k].log())
        if c["out"] != "none":
            row = torch.zeros(c["vocab"], dtype=torch.float64, device="cuda")
            row[ids] = p
            whole.append(row if c["out"] == "probs" else row.log())
    res = {"token": torch.tensor(got["token"], dtype=torch.int32), "n_kept": torch.tensor(got["n_kept"], dtype=torch.int32), "logprob": torch.stack(got["logprob"])}
    if whole:
        res[c["out"]] = torch.stack(whole)
    return res
