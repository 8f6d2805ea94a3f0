"""New tokens over pages, behind a shared prefix, in 64 bits from the definition (CPU tensors)."""
import math

import torch

from llm_ref import assert_within, f64, half_step, scale_of

HALF = half_step(torch.bfloat16)


def flat_keys(cache, pages, n):
    """Keys 0..n-1 of a list of pages of a cache [num_pages, H_kv, page, D]: [H_kv, n, D], and which of them are there."""
    num, Hkv, page, D = cache.shape
    pages = pages.long().cpu()
    there = (pages >= 0) & (pages < num)
    x = cache.cpu()[pages.clamp(0, num - 1)].transpose(0, 1).reshape(Hkv, -1, D)[:, :n]
    return x, there.repeat_interleave(page)[:n]


def attend(q, k, v, seen, scale=None):
    """q [n, H, D]; k, v [H_kv, m, D]; seen [n, m]: O [n, H, D], LSE [n, H], sum p |v|, and scale sum |q k| at its largest."""
    n, H, D = q.shape
    G = H // k.shape[0]
    o, pv = torch.zeros(n, H, D, dtype=torch.float64), torch.zeros(n, H, D, dtype=torch.float64)
    lse, mag = torch.full((n, H), -math.inf, dtype=torch.float64), torch.zeros(n, H, dtype=torch.float64)
    if k.shape[1] == 0:
        return o, lse, pv, mag
    some = seen.any(1)
    for h in range(H):
        kk, vv = f64(k[h // G]), f64(v[h // G])
        kk, vv = torch.where(seen.any(0)[:, None], kk, 0.0), torch.where(seen.any(0)[:, None], vv, 0.0)
        x = f64(q[:, h])
        s = (scale_of(D, scale) * x @ kk.T).masked_fill(~seen, -math.inf)
        lse[:, h] = torch.logsumexp(s, 1)
        p = torch.where(some[:, None], torch.softmax(s, 1), 0.0)
        o[:, h], pv[:, h] = p @ vv, p @ vv.abs()
        mag[:, h] = torch.where(seen, scale_of(D, scale) * x.abs() @ kk.abs().T, 0.0).amax(1)
    return o, lse, pv, mag


def batch(q, kc, vc, table, starts, lens, prefix=None, plen=0, scale=None):
    """The sequences' results, each with its tokens' indices; a prefix of plen keys in the pages `prefix`."""
    page, out = kc.shape[2], []
    for b in range(table.shape[0]):
        first, n = starts[b], starts[b + 1] - starts[b]
        L = max(0, min(lens[b], table.shape[1] * page))
        k, there = flat_keys(kc, table[b], L)
        v, _ = flat_keys(vc, table[b], L)
        seen = there[None] & (torch.arange(L)[None] <= (L - n + torch.arange(n))[:, None])
        if prefix is not None:
            P = max(0, min(plen, prefix.shape[0] * page))
            pk, pt = flat_keys(kc, prefix, P)
            k, v = torch.cat((pk, k), 1), torch.cat((flat_keys(vc, prefix, P)[0], v), 1)
            seen = torch.cat((pt[None].expand(n, P), seen), 1)
        out.append((slice(first, first + n), *attend(q.cpu()[first:first + n], k, v, seen, scale)))
    return out


def check(o, lse, refs, what):
    """P is rounded to bf16 before it meets V, and O on its way out: half a step (2^-8) of p |v| summed, and of O.  q and k
    are exact, D products of them are summed in fp32 (2 D 2^-24 <= 2^-16 of their magnitudes): a score moves by at most 2^-16
    of A = scale sum |q k|, an LSE by as much, a weight by twice that of itself; exp2, log2, and fp32 sums of weights and of
    partials, add 2^-16 of p and 2^-18 (1 + |LSE|)."""
    for b, (at, O, L, pv, mag) in enumerate(refs):
        tol = 2.0 ** -16 * mag
        assert_within(o[at], O, HALF * O.abs() + (HALF + 2 * tol[..., None] + 2.0 ** -16) * pv, f"{what} O[{b}]")
        fin = torch.isfinite(L)
        got = f64(lse[at])
        assert torch.equal(torch.isneginf(got), ~fin), f"{what} LSE[{b}]"
        assert_within(got[fin], L[fin], (tol + 2.0 ** -18 * (1 + L.abs()))[fin], f"{what} LSE[{b}]")
