"""Plain implementations of the serving operators for the tests: fp32 with one rounding an operation where codes are pinned
(torch on the CPU, one elementary operation at a time), fp64 elsewhere.  Nothing here knows how the cache lays out its bytes."""
import math

import numpy as np
import torch

import paper_2503_01483_amd as kt

TINY = float(np.finfo(np.float32).tiny)
LEVELS = {kt.KT_Q_INT4: 7.0, kt.KT_Q_INT8: 127.0, kt.KT_Q_E4M3: 448.0}
TOP = {kt.KT_KV_U4: 15.0, kt.KT_KV_U8: 255.0}
F32 = lambda v: torch.tensor(v, dtype=torch.float32)  # noqa: E731


def norm(x, res, gain, eps, clip, fmt):
    """(h, codes as fp32 values, t, scale in fp64) of rows on the CPU."""
    h = x.float() if res is None else x.float() + res.float()
    u = h if gain is None else h * gain.float()
    rstd = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)
    if fmt == kt.KT_Q_NONE:
        return h, None, None, rstd * u.double()
    top = F32(LEVELS[fmt])
    t = (u.abs().amax(1, keepdim=True) * F32(clip)) / top
    some = t >= TINY
    z = torch.minimum(torch.maximum(u * (F32(1.0) / torch.where(some, t, torch.ones_like(t))), -top), top)
    z = torch.where(some, z, torch.zeros_like(z))
    code = z.to(torch.float8_e4m3fn).float() if fmt == kt.KT_Q_E4M3 else torch.round(z)
    return h, code, t, torch.where(some, t.double() * rstd, torch.zeros_like(rstd))


def rotate(x, pos, rope, interleaved, hadamard):
    """Position and Hadamard rotation of x [n, heads, hd] fp32, in the pinned order."""
    y = x.clone()
    hd = x.shape[-1]
    if rope is not None:
        half = rope.shape[1] // 2
        row = rope[pos.long()][:, None]
        c, s = row[..., :half], row[..., half:]
        first = torch.arange(half) * 2 if interleaved else torch.arange(half)
        second = first + 1 if interleaved else first + half
        a, b = x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    if hadamard:
        step = 1
        while step < hd:
            z = y.reshape(-1, hd // (2 * step), 2, step)
            y = torch.stack([z[:, :, 0] + z[:, :, 1], z[:, :, 0] - z[:, :, 1]], 2).reshape(x.shape)
            step *= 2
        y = y * F32(1 / math.sqrt(hd))
    return y


def held(y, fmt):
    """What the cache holds of rows y [..., hd] fp32: (values fp32, largest magnitude of a centred code times its step)."""
    if fmt == kt.KT_KV_BF16:
        return y.to(torch.bfloat16).float()
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    width = hi - lo
    s = width / F32(TOP[fmt])
    s = torch.where(s < TINY, torch.zeros_like(s), s)
    c = torch.round(((y - lo) * F32(TOP[fmt])) / torch.where(s > 0, width, torch.ones_like(s)))
    c = torch.where(s > 0, c, torch.zeros_like(c))
    bad = ~torch.isfinite(y).all(-1, keepdim=True) | ~(width * F32(TOP[fmt]) <= np.finfo(np.float32).max)
    return torch.where(bad, torch.full_like(c, math.nan), c * s + lo)


def rope_table(n_pos, rot, base=10000.0):
    angle = np.arange(n_pos)[:, None] * (base ** (-np.arange(0, rot, 2) / rot))[None]
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32))


class Batch:
    """Sequences in a cache whose pages lie anywhere, and their queries: inputs on the GPU, what is held of them in fp64."""

    def __init__(self, fmt, hd, hkv, group, lens, counts=None, prefix=0, page=64, seed=0, spread=1.0, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.hd, self.hkv, self.hq, self.page = fmt, hd, hkv, hkv * group, page
        self.lens, self.counts, self.prefix = list(lens), list(counts or [1] * len(lens)), prefix
        per = max(1, max(-(-t // page) for t in lens))
        pre = -(-prefix // page)
        n_pages = len(lens) * per + pre + 1
        order = torch.randperm(n_pages, generator=g)
        self.pages = order[:len(lens) * per].reshape(len(lens), per).to(torch.int32).cuda()
        self.prefix_pages = order[len(lens) * per:len(lens) * per + pre].to(torch.int32).cuda()
        self.cache = kt.KVCache(n_pages, page, hkv, hd, fmt)
        self.cache.data.fill_(255)        # NaN as bf16 and fp32 alike: what is not written must not matter
        self.k, self.v = [], []
        for i, t in enumerate(self.lens + [prefix]):
            table = (self.pages[i] if i < len(lens) else self.prefix_pages).cpu().long()
            k, v = (torch.randn(t, hkv, hd, generator=g) * spread for _ in range(2))
            if t:
                slots = table[torch.arange(t) // page] * page + torch.arange(t) % page
                kt.kt_kv_append(self.cache, k.cuda(), v.cuda(), slots.cuda())
            self.k.append(held(k, fmt).double())
            self.v.append(held(v, fmt).double())
        self.pk, self.pv = self.k.pop(), self.v.pop()
        self.starts = [0]
        for c in self.counts:
            self.starts.append(self.starts[-1] + c)
        self.n = self.starts[-1] + pad
        self.q = (torch.randn(self.n, self.hq, hd, generator=g) * 2).to(torch.bfloat16)
        self.single = counts is None

    def call(self, **kw):
        more = {}
        if not self.single:
            more = dict(q_starts=torch.tensor(self.starts, dtype=torch.int32, device="cuda"), max_q=max(1, max(self.counts)))
        if self.prefix:
            more.update(prefix_pages=self.prefix_pages, prefix_len=self.prefix)
        more.update(kw)
        return kt.kt_paged_attention(self.q.cuda() if "Q" not in kw else more.pop("Q"), self.cache, self.pages,
                                     torch.tensor(self.lens, dtype=torch.int32, device="cuda"), **more)

    def expected(self, scale=None):
        """out, lse in fp64, and how far a result may be off: arrays [n, hq, hd] and [n, hq].

        out: its rounding to bf16, 2^-8 of it; that of p (bf16) or p times the step (u8, u4), 2^-8 of each term, the terms being
        p times |v|, or the centred code's part of v; and what an error e of the scores does, 2 e sum p |v|.
        e: 16 roundings in fp32 of sums as large as sum |q| (|k| + 144 steps) (codes enter as 128 + c), and as many of exp and log.
        """
        scale = self.hd ** -0.5 if scale is None else scale
        G = self.hq // self.hkv
        out = torch.zeros(self.n, self.hq, self.hd, dtype=torch.float64)
        lse = torch.full((self.n, self.hq), -math.inf, dtype=torch.float64)
        tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
        for s, t in enumerate(self.lens):
            k, v = torch.cat([self.pk, self.k[s]]), torch.cat([self.pv, self.v[s]])
            for h in range(self.hq):
                kh, vh = k[:, h // G], v[:, h // G]
                step = 0.0 if self.fmt == kt.KT_KV_BF16 else (kh.amax(1) - kh.amin(1)) / TOP[self.fmt]
                for i in range(self.counts[s]):
                    row, sees = self.starts[s] + i, self.prefix + max(0, t - self.counts[s] + i + 1)
                    if sees == 0:
                        continue
                    q = self.q[row, h].double()
                    x = (kh[:sees] @ q) * scale
                    z = torch.logsumexp(x, 0)
                    p = torch.exp(x - z)
                    o = p @ vh[:sees]
                    e = 2.0 ** -20 * scale * float((q.abs().sum() * (kh[:sees].abs().amax(1) + 144 * (step if isinstance(step, float) else step[:sees]))).max()) + 2.0 ** -20
                    if self.fmt == kt.KT_KV_BF16:
                        part = p @ vh[:sees].abs()
                    else:
                        lo, hi = vh[:sees].amin(1), vh[:sees].amax(1)
                        part = (p * (hi - lo) / TOP[self.fmt] * (8 if self.fmt == kt.KT_KV_U4 else 128)).sum()
                    out[row, h], lse[row, h] = o, z
                    tol[row, h] = 2.0 ** -8 * (o.abs() + part) + 2 * e * (p @ vh[:sees].abs())
                    ltol[row, h] = e + 2.0 ** -22 * abs(z)
        return out, lse, tol, ltol

    def check(self, out, lse, scale=None):
        o, z, tol, ltol = self.expected(scale)
        n = self.starts[-1]
        d = (out.cpu().double() - o).abs()[:n]
        assert bool((d <= tol[:n]).all()), f"out off by {float((d / tol[:n].clamp_min(1e-30)).max()):.2f} of what it may"
        if lse is not None:
            l = lse.cpu().double()[:n]
            assert torch.equal(torch.isinf(l), torch.isinf(z[:n]))
            fin = torch.isfinite(z[:n])
            d = (l - z[:n]).abs()[fin]
            assert bool((d <= ltol[:n][fin]).all()), f"lse off by {float((d / ltol[:n][fin].clamp_min(1e-30)).max()):.2f} of what it may"
