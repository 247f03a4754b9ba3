"""Plain implementations of the operators for drafted tokens and budgets of cached ones, in fp64 on the CPU, and how far results may be off."""
import math

import numpy as np
import torch

import paper_2503_01483_amd as kt
from serving_util import TOP

FORMATS = [kt.KT_KV_BF16, kt.KT_KV_U8, kt.KT_KV_U4]
NAMES = {kt.KT_KV_BF16: "bf16", kt.KT_KV_U8: "u8", kt.KT_KV_U4: "u4"}


def ints(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).cuda()


def few(b, max_q):
    """Whether trees of up to max_q queries are computed by waves (p times the step to 16 bits) or as many rows are."""
    return max_q * (b.hq // b.hkv) <= {kt.KT_KV_BF16: 0, kt.KT_KV_U8: 32, kt.KT_KV_U4: 64}[b.fmt]


def random_tree(count, rng, wide=7):
    """[count][count] bool: a draft's ancestors and itself; parents are among the few in front, or none."""
    seen = np.zeros((count, count), dtype=bool)
    for i in range(count):
        p = int(rng.integers(max(-1, i - wide), i)) if i else -1
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def words_of(masks, n, words):
    """Masks [count][count] of each sequence as rows of words [n][words] int64 (rows behind the last: all bits set)."""
    out = np.full((n, words), -1, dtype=np.int64)
    at = 0
    for m in masks:
        for row in m:
            v = sum(1 << int(d) for d in np.nonzero(row)[0])
            out[at] = np.array([v >> 64 * w & (1 << 64) - 1 for w in range(words)], dtype=np.uint64).view(np.int64)
            at += 1
    return torch.from_numpy(out).cuda()


def seen_by(b, s, mask):
    """[count][len]: which of sequence s' tokens each of its queries sees under a mask of its queries."""
    t, c = b.lens[s], b.counts[s]
    j = torch.arange(t) - (t - c)
    m = torch.as_tensor(mask, dtype=torch.bool).reshape(c, c)
    return (j < 0)[None] | ((j >= 0)[None] & m[:, j.clamp(0, max(c - 1, 0))]) if c else torch.zeros(0, t, dtype=torch.bool)


def score_error(b, q, k, ks, scale):
    """Of q . k scale in fp32, and of its exponential (relative to 1): 16 roundings of sums as large as sum |q| (|k| + 144 steps), as many of exp and log."""
    return 2.0 ** -20 * (scale * q.abs().sum(-1)[..., None] * (k.abs().amax(1) + 144 * ks) + 1)


def tree_expected(b, masks, max_q=None):
    """out, lse of a serving_util.Batch whose queries see each other by `masks`, and what they may be off by; the roundings are those that
    attention_bounds.expected counts, over the tokens that a row sees."""
    scale, G, quant, pre = b.hd ** -0.5, b.hq // b.hkv, b.fmt != kt.KT_KV_BF16, b.pk.shape[0]
    out, lse = torch.zeros(b.n, b.hq, b.hd, dtype=torch.float64), torch.full((b.n, b.hq), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    waves = few(b, max(b.counts) if max_q is None else max_q)
    for s, t in enumerate(b.lens):
        rows = torch.arange(b.starts[s], b.starts[s + 1])
        if not len(rows) or t + pre == 0:
            continue
        seen = torch.cat([torch.ones(len(rows), pre, dtype=torch.bool), seen_by(b, s, masks[s])], 1)      # [rows, tokens]
        for h in range(b.hkv):
            k, v = torch.cat([b.pk[:, h], b.k[s][:, h]]), torch.cat([b.pv[:, h], b.v[s][:, h]])
            k, v = torch.where(seen.any(0)[:, None], k, 0.0), torch.where(seen.any(0)[:, None], v, 0.0)
            q = b.q[rows][:, h * G:(h + 1) * G].double()
            ks, vs = ((y.amax(1) - y.amin(1)) / TOP[b.fmt] if quant else torch.zeros(len(y), dtype=torch.float64) for y in (k, v))
            x = torch.where(seen[:, None], torch.einsum("rgd,td->rgt", q, k) * scale, -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None])
            e = score_error(b, q, k, ks, scale)
            o, size = p @ v, p @ v.abs()
            off = 2.0 ** -8 * o.abs() + (p * e) @ v.abs() + (p * e).sum(-1)[..., None] * o.abs()
            if not quant:
                off += (2.0 ** -8 + 2.0 ** -20) * size
            else:
                as_many = torch.arange(len(k)) < pre if waves else torch.ones(len(k), dtype=torch.bool)
                c, u = (8, 151) if b.fmt == kt.KT_KV_U4 else (128, 256)
                off += 2.0 ** -20 * size + (p * vs * ~as_many).sum(-1)[..., None] * (2.0 ** -16 * c + 2.0 ** -20 * u)
                own = v.abs().amax(1) * as_many
                places = torch.cat([torch.arange(pre) // 64, -(-pre // 64) + torch.arange(t) // 64])
                each = torch.where(seen, own, torch.zeros(()))
                tiles = torch.zeros(len(rows), int(places.max()) + 1, dtype=torch.float64).scatter_reduce(1, places.expand(len(rows), -1), each, "amax")
                most = torch.minimum(tiles[:, places], 128 * own)
                off += (2.0 ** -11 + 2.0 ** -15) * (p * as_many) @ v.abs() + 1.5 * 2.0 ** -11 * (p * most[:, None]).sum(-1)[..., None]
                off += 2.0 ** -31 * ((p * own).amax(-1) * seen.sum(1)[:, None])[..., None]
            out[rows, h * G:(h + 1) * G], lse[rows, h * G:(h + 1) * G] = o, z
            tol[rows, h * G:(h + 1) * G] = off
            ltol[rows, h * G:(h + 1) * G] = torch.where(torch.isinf(z), 0.0, (p * e).sum(-1) + 2.0 ** -20 + 2.0 ** -22 * z.abs())
    return out, lse, tol, ltol


def tree_check(b, out, lse, masks, max_q=None):
    o, z, tol, ltol = tree_expected(b, masks, max_q)
    n = b.starts[-1]
    d = (out.cpu().double() - o).abs()[:n]
    print(f"off by {float((d / tol[:n].clamp_min(1e-300)).max()):.3f} of what it may", flush=True)
    assert bool((d <= tol[:n]).all())
    if lse is not None:
        l = lse.cpu().double()[:n]
        assert torch.equal(torch.isinf(l), torch.isinf(z[:n]))
        fin = torch.isfinite(z[:n])
        assert bool(((l - z[:n]).abs()[fin] <= ltol[:n][fin]).all())


def mass_expected(b, lse, mass, decay):
    """mass [pages][heads][page] in fp64 after a call, and what it may be off by.

    A term is off, relatively, by the error of its score (as in attention), of scale log2(e) and of lse log2(e) (two roundings each of numbers as
    large as the score and lse, with the rounding of their difference 2^-22 of |lse| and of |score|), and of the exponential (2^-22).  The sum: a lane adds a
    sixteenth of the rows one by one, then 4 + 4 additions and the old mass' product: (rows / 16 + 12) 2^-24 of it."""
    scale, G = b.hd ** -0.5, b.hq // b.hkv
    quant = b.fmt != kt.KT_KV_BF16
    want, tol = mass.double().clone(), torch.zeros(mass.shape, dtype=torch.float64)
    pages = b.pages.cpu().long()
    for s, t in enumerate(b.lens):
        rows, ahead, tok = torch.arange(b.starts[s], b.starts[s + 1]), t - b.counts[s], torch.arange(t)
        seen = tok[None] <= ahead + torch.arange(len(rows))[:, None]
        at = pages[s][tok // b.page]
        for h in range(b.hkv):
            k, q = b.k[s][:, h], b.q[rows][:, h * G:(h + 1) * G].double()
            ks = (k.amax(1) - k.amin(1)) / TOP[b.fmt] if quant else torch.zeros(t, dtype=torch.float64)
            z = lse[rows][:, h * G:(h + 1) * G].double()
            x = torch.einsum("rgd,td->rgt", q, k) * scale
            use = seen[:, None] & torch.isfinite(z)[..., None]
            p = torch.where(use, torch.exp(x - z.nan_to_num(0.0, 0.0, 0.0)[..., None]), 0.0)
            rel = score_error(b, q, k, ks, scale) + 2.0 ** -22 * (x.abs() + z.nan_to_num(0.0, 0.0, 0.0).abs()[..., None] + 1)
            old = torch.where(tok < ahead, want[at, h, tok % b.page], 0.0) * decay if decay else torch.zeros(t, dtype=torch.float64)
            new = old + p.sum((0, 1))
            want[at, h, tok % b.page] = new
            tol[at, h, tok % b.page] = torch.where(use, p * rel, 0.0).sum((0, 1)) + (len(rows) * G / 16 + 12) * 2.0 ** -24 * (p.sum((0, 1)) + old.abs())
    return want, tol


def mass_check(b, got, lse, before, decay):
    want, tol = mass_expected(b, lse, before, decay)
    d = (got.cpu().double() - want).abs()
    d = torch.where(torch.isnan(want) & torch.isnan(got.cpu()), 0.0, d)        # (places that nothing was written to)
    print(f"off by {float((d / tol.clamp_min(1e-300)).max()):.3f} of what it may", flush=True)
    assert bool((d <= tol).all())


def select_expected(mass, lens, keep, sink, recent, most):
    """Lists [sequence][head] of the tokens that stay; mass: [sequence][head] arrays of the tokens' masses."""
    out = []
    for per_head, t, k in zip(mass, lens, keep):
        n = max(0, min(t, k, most))
        r = min(recent, n)
        f = min(sink, n - r)
        mine = []
        for x in per_head:
            x = np.asarray(x, dtype=np.float64)
            middle = np.arange(f, t - r)
            y = x[middle]
            best = middle[np.lexsort((middle, -np.nan_to_num(y, nan=0.0, posinf=np.inf, neginf=-np.inf), np.isnan(y)))[:n - r - f]]
            mine.append(np.concatenate([np.arange(f), np.sort(best), np.arange(t - r, t)]).astype(np.int32))
        out.append(mine)
    return out


class Held:
    """A cache of random tokens in every slot, and what every slot holds, as the bits of fp32 values [slots][heads][head_dim]."""

    def __init__(self, fmt, hd, heads, n_pages, page, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.cache = kt.KVCache(n_pages, page, heads, hd, fmt)
        self.cache.data.zero_()
        n = n_pages * page
        k, v = (torch.randn(n, heads, hd, generator=g) for _ in range(2))
        self.slots = torch.arange(n).cuda()
        kt.kt_kv_append(self.cache, k.cuda(), v.cuda(), self.slots)
        self.mass = torch.rand(n_pages, heads, page, generator=g).cuda()
        self.page, self.heads = page, heads

    def now(self):
        k, v = kt.kt_kv_gather(self.cache, self.slots, dtype=torch.float32)
        m = self.mass.transpose(1, 2).reshape(-1, self.heads, 1)
        return torch.cat([k, v, m], 2).cpu().view(torch.int32)

    def slot(self, table, t):
        return int(table[t // self.page]) * self.page + t % self.page
