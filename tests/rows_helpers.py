"""Inputs and checks shared by the GPU tests of rows without a tree."""
import numpy as np
import torch

from oracle import rows as O
from paper_2510_13161_b200 import binding, inputs as I

PAGE = 16


def make(hq, hkv, d, vocab=512, temperature=1.0, scale=0.0):
    return binding.Mirror(256, hq, hkv, d, vocab, softmax_scale=scale, temperature=temperature)


class Case:
    """A paged cache with ragged rows: prefixes lens[b], counts[b] new rows, `pad` rows behind the last request.  Every element that no
    row sees is NaN (K and V alike): what is masked must not leak."""

    def __init__(self, hq, hkv, d, lens, counts, layers=1, pad=0, window=0, sinks=0, seed=0, spread=1.0, uniform=False):
        g = torch.Generator().manual_seed(seed)
        self.hq, self.hkv, self.d, self.window, self.sinks = hq, hkv, d, window, sinks
        self.lens, self.counts, self.layers = list(lens), list(counts), layers
        self.start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.R = int(self.start[-1]) + pad
        need = [-(-(t + n) // PAGE) for t, n in zip(lens, counts)]
        most = max(need + [1]) + 1
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=g).numpy()
        self.table = np.full((len(lens), most), 1 << 20, np.int32)             # (entries that are not needed are not looked at)
        self.k = torch.full((layers, pages, hkv, PAGE, d), float("nan"), dtype=torch.bfloat16)
        self.v = self.k.clone()
        at = 0
        for b, (t, n) in enumerate(zip(lens, counts)):
            lo = max(0, t - window + 1) if window else 0
            for j in range(need[b]):
                keys = [key for key in range(j * PAGE, min((j + 1) * PAGE, t + n)) if key >= lo or key < sinks]
                if not keys or n == 0:
                    continue
                self.table[b, j] = order[at]
                s = [key - j * PAGE for key in keys]
                for pool in (self.k, self.v):
                    pool[:, int(order[at]), :, s] = (torch.randn((layers, hkv, len(s), d), generator=g) * (spread if pool is self.k else 1.0)).to(torch.bfloat16)
                at += 1
        self.q = torch.randn((layers, self.R, hq, d), generator=g).to(torch.bfloat16)
        self.uniform = uniform

    def device(self, m):
        self.kd, self.vd = self.k.cuda(), self.v.cuda()
        self.kv = m.kv(self.kd, self.vd, torch.from_numpy(self.table).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda())
        if self.uniform:
            self.rows = m.rows(None, self.R, max(self.counts), len(self.lens))
        else:
            self.rows = m.rows(torch.from_numpy(self.start).cuda(), self.R, max(max(self.counts), 1))
        return self.kv, self.rows

    def expect(self, layer, scale=None):
        """(out, lse, sum of p |v|) of one layer in 64 bits."""
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        f = lambda t: t[layer].double().numpy()  # noqa: E731
        args = (f(self.q), f(self.k))
        rest = (self.table, self.lens, self.start, self.window, self.sinks, scale)
        out, lse = O.causal_attention(*args, f(self.v), *rest)
        return out, lse, O.causal_attention(*args, np.abs(f(self.v)), *rest)[0]


def check_attention(m, c, p_rounded, scale=None):
    """Runs the call and holds it to the oracle.  What may differ: the output's rounding, half a bf16 step of its size; where P is one
    bf16 (p_rounded), half a step of each weight, 2^-8 sum p |v|; and fp32: a score of d products is off by at most d 2^-24 sum |q k|,
    which moves weights, and with them the output, by twice that share."""
    kv, rows = c.device(m)
    out = torch.full((c.layers, c.R, c.hq, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.layers, c.R, c.hq), 7.0, dtype=torch.float32, device="cuda")
    m.mirror_attn_causal(kv, rows, c.q.cuda(), window=c.window, sinks=c.sinks, out=out, lse_out=lse)
    torch.cuda.synchronize()
    assert m.device_status() == (0, 0)
    used = int(c.start[-1])
    assert (out[:, used:] == 7.0).all() and (lse[:, used:] == 7.0).all()       # rows behind the last request
    s = 1 / np.sqrt(c.d) if scale is None else scale
    k = c.k.float().abs().nan_to_num(0.0)
    # sum |q k| <= |q| |k| (Cauchy)
    moved = c.d * 2.0 ** -24 * s * float(c.q.float().norm(dim=-1).max()) * float(k.norm(dim=-1).max())
    for layer in range(c.layers):
        want, want_lse, spread = c.expect(layer, s)
        got = out[layer, :used].double().cpu().numpy()
        tol = 2.0 ** -8 * np.abs(want[:used]) + ((2.0 ** -8 if p_rounded else 2.0 ** -15) + 2 * moved + 1e-6) * spread[:used] + 1e-30
        bad = ~(np.abs(got - want[:used]) <= tol)
        assert not bad.any(), (layer, np.argwhere(bad)[:5], np.abs(got - want[:used])[bad][:5], tol[bad][:5])
        gl = lse[layer, :used].double().cpu().numpy()
        assert (np.abs(gl - want_lse[:used]) <= moved + 2e-6 * (1 + np.abs(want_lse[:used]))).all()
    return out, lse
