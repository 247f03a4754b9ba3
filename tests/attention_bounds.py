"""What the documentation of kt_paged_attention allows a result to be off, rounding by rounding (fp64, on the CPU), for a serving_util.Batch."""
import math

import torch

import paper_2503_01483_amd as kt
from serving_util import TOP, held

FEW = {(kt.KT_KV_BF16, 64): 32, (kt.KT_KV_BF16, 128): 16, (kt.KT_KV_BF16, 256): 16, (kt.KT_KV_U8, 256): 32}   # else 64 rows a sequence and head


def few(b, max_q):
    return max_q * (b.hq // b.hkv) <= FEW.get((b.fmt, b.hd), 64)


def replace(b, seq, tokens, k=None, v=None):
    """Other keys / values [len(tokens), heads, hd] fp32 for tokens of a sequence, or of the prefix (seq None)."""
    at = torch.as_tensor(tokens)
    table = (b.prefix_pages if seq is None else b.pages[seq]).cpu().long()
    slots = table[at // b.page] * b.page + at % b.page
    keys, values = (b.pk, b.pv) if seq is None else (b.k[seq], b.v[seq])
    have = kt.kt_kv_gather(b.cache, slots.cuda(), dtype=torch.float32)
    new = [h.cpu() if x is None else x for x, h in zip((k, v), have)]
    kt.kt_kv_append(b.cache, new[0].cuda(), new[1].cuda(), slots.cuda())
    now = kt.kt_kv_gather(b.cache, slots.cuda(), dtype=torch.float32)
    for x, held_now, mine in zip((k, v), now, (keys, values)):
        if x is not None:
            assert torch.equal(held_now.cpu().nan_to_num(7.0), held(x, b.fmt).nan_to_num(7.0))
        mine[at] = held_now.cpu().double()       # (a row that is appended again as it was read may be held one rounding off)


def expected(b, scale=None, max_q=None):
    """out, lse in fp64 and what they may be off by.

    A score: 16 roundings in fp32 of sums as large as sum |q| (|k| + 144 steps), as many of exp and log (relative to 1); through the softmax an error e_j of
    score j moves the output by p_j e_j (|v_j| + |out|).  Output: rounded to bf16, 2^-8 of it.  Sums in fp32: 2^-20 of their terms' magnitudes.
    Products with the values:
      bf16        p to bf16: 2^-8 of p |v|
      few rows    (their own tokens) p step to 16 bits: 2^-16 of p step (a centred code: up to 8 or 128); codes enter uncentred: fp32 sums of p step (136 + 15) or p step 256
      many rows, and the tokens of a prefix in either
                  p to fp16: 2^-11 of p |v|, its exponent, score plus size, up to 512 in fp32: 2^-15; nothing below 2^-31 of the largest p |v|;  v to 1.5 x 2^-11 of the largest value that the row sees of its 64 tokens,
                  or of 2^7 times its token's own largest, whichever is less
    """
    scale = b.hd ** -0.5 if scale is None else scale
    G = b.hq // b.hkv
    out, lse = torch.zeros(b.n, b.hq, b.hd, dtype=torch.float64), torch.full((b.n, b.hq), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    quant = b.fmt != kt.KT_KV_BF16
    waves = few(b, max(b.counts) if max_q is None else max_q)
    pre = b.pk.shape[0]
    for s, t in enumerate(b.lens):
        for h in range(b.hkv):
            k, v = torch.cat([b.pk[:, h], b.k[s][:, h]]), torch.cat([b.pv[:, h], b.v[s][:, h]])
            rows = torch.arange(b.starts[s], b.starts[s + 1])
            if not len(rows) or not len(k):
                continue
            q = b.q[rows][:, h * G:(h + 1) * G].double()                            # [rows, G, hd]
            sees = pre + (t - b.counts[s] + torch.arange(len(rows)) + 1).clamp(0, t)
            seen = torch.arange(len(k))[None, :] < sees[:, None]                    # [rows, tokens]
            k, v = torch.where(seen.any(0)[:, None], k, 0.0), torch.where(seen.any(0)[:, None], v, 0.0)
            ks, vs = ((y.amax(1) - y.amin(1)) / TOP[b.fmt] if quant else torch.zeros(len(y), dtype=torch.float64) for y in (k, v))
            x = torch.einsum("rgd,td->rgt", q, k) * scale
            x = torch.where(seen[:, None], x, -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[..., None])
            e = 2.0 ** -20 * (scale * q.abs().sum(-1)[..., None] * (k.abs().amax(1) + 144 * ks) + 1)
            o, mass = p @ v, p @ v.abs()
            off = 2.0 ** -8 * o.abs() + (p * e) @ v.abs() + (p * e).sum(-1)[..., None] * o.abs()
            if not quant:
                off += (2.0 ** -8 + 2.0 ** -20) * mass
            else:
                as_many = torch.arange(len(k)) < pre if waves else torch.ones(len(k), dtype=torch.bool)
                c, u = (8, 151) if b.fmt == kt.KT_KV_U4 else (128, 256)
                off += 2.0 ** -20 * mass + (p * vs * ~as_many).sum(-1)[..., None] * (2.0 ** -16 * c + 2.0 ** -20 * u)
                own = v.abs().amax(1) * as_many                                     # [tokens]
                places = torch.cat([torch.arange(pre) // 64, -(-pre // 64) + torch.arange(t) // 64])
                each = torch.where(seen, own, torch.zeros(()))                      # [rows, tokens]
                tiles = torch.zeros(len(rows), int(places.max()) + 1, dtype=torch.float64).scatter_reduce(1, places.expand(len(rows), -1), each, "amax")
                most = torch.minimum(tiles[:, places], 128 * own)                   # [rows, tokens]
                off += (2.0 ** -11 + 2.0 ** -15) * (p * as_many) @ v.abs() + 1.5 * 2.0 ** -11 * (p * most[:, None]).sum(-1)[..., None]
                off += 2.0 ** -31 * ((p * own).amax(-1) * sees[:, None])[..., None]
            out[rows, h * G:(h + 1) * G], lse[rows, h * G:(h + 1) * G] = o, z
            tol[rows, h * G:(h + 1) * G] = off
            ltol[rows, h * G:(h + 1) * G] = torch.where(torch.isinf(z), 0.0, (p * e).sum(-1) + 2.0 ** -20 + 2.0 ** -22 * z.abs())
    return out, lse, tol, ltol


def check(b, out, lse, scale=None, max_q=None):
    o, z, tol, ltol = expected(b, scale, max_q)
    n = b.starts[-1]
    d = (out.cpu().double() - o).abs()[:n]
    print(f"off by {float((d / tol[:n].clamp_min(1e-300)).max()):.3f} of what it may", flush=True)
    assert bool((d <= tol[:n]).all())
    l = lse.cpu().double()[:n]
    assert torch.equal(torch.isinf(l), torch.isinf(z[:n]))
    fin = torch.isfinite(z[:n])
    assert bool(((l - z[:n]).abs()[fin] <= ltol[:n][fin]).all())
