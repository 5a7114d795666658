"""The decode step in plain 64-bit arithmetic, request by request, from the
definitions in include/driftsched_serve.h. Tensors on the CPU in, numpy out;
shares nothing with the library."""
import math

import numpy as np
import torch


def values(x):
    """A tensor's values as float64."""
    return x.float().numpy().astype(np.float64) if x.dtype != torch.float64 else x.numpy()


def tokens_of(pool, table, n, page_size, n_pages):
    """(n, n_kv, dim) values of a request's tokens and which of them exist."""
    j = np.arange(n)
    pages = table[j // page_size].astype(np.int64)
    there = (pages >= 0) & (pages < n_pages)
    x = pool[np.where(there, pages, 0), j % page_size]
    return x, there


def attention(q, k, v, table, lens, rows=None, scale=None, window=0, sinks=0, mass=None, k_scale=None, v_scale=None):
    """Returns out, the bound on |out - exact| before out's own rounding (see
    `bound` below), and the new mass with its bound."""
    f16 = q.dtype == torch.float16
    q, k, v = values(q), values(k), values(v)
    if k_scale is not None:
        k = k * values(k_scale)[None, None, :, None]
    if v_scale is not None:
        v = v * values(v_scale)[None, None, :, None]
    table, lens = table.numpy(), lens.numpy()
    n_rows, t, n_q, dim = q.shape
    n_pages, page_size, n_kv, _ = k.shape
    group = n_q // n_kv
    scale = dim ** -0.5 if scale is None else scale
    rows = np.arange(n_rows) if rows is None else rows.numpy()
    out, off = np.zeros(q.shape), np.zeros(q.shape)
    mass = None if mass is None else values(mass).copy()
    mass_off = None if mass is None else np.zeros(mass.shape)
    eps = 2.0 ** -24
    with np.errstate(all="ignore"):
        for i, r in enumerate(rows):
            n = int(lens[r]) if 0 <= r < len(lens) else 0
            if n == 0:
                continue
            kk, there = tokens_of(k, table[r], n, page_size, n_pages)
            vv, _ = tokens_of(v, table[r], n, page_size, n_pages)
            j = np.arange(n)
            got, got_off = np.zeros((n_kv, n)), np.zeros((n_kv, n))
            for b in range(t):
                p = n - t + b
                if p < 0:
                    continue
                see = there & (j <= p)
                if window:
                    see &= (j > p - window) | (j < sinks)
                see = np.nonzero(see)[0]
                if len(see) == 0:
                    continue
                for h in range(n_q):
                    g = h // group
                    s = kk[see, g] @ q[i, b, h] * scale
                    top = s.max()
                    if top == -math.inf:
                        continue
                    w = np.exp(s - top)
                    w = w / w.sum()
                    out[i, b, h] = np.where(w > 0, w, 0 if not np.isnan(w).any() else np.nan) @ np.where(w[:, None] > 0, vv[see, g], 0.0) \
                        if not np.isnan(w).any() else np.nan
                    got[g, see] += w
                    # |score error|: dim products summed in 32 bits, the scale and the exponential's
                    # own rounding (argument and value); a weight's relative error is twice that
                    # (its own score's and the normalizer's), plus the sums over n tokens, plus what
                    # two 16-bit parts leave: 2^-17 of a bf16 pair, 2^-22 (or 2^-25 absolute) of an f16 pair
                    size = (np.abs(kk[see, g]) @ np.abs(q[i, b, h])).max() * abs(scale)
                    rel = 2 * (dim + 8) * eps * max(1.0, size) + (n + 64) * eps
                    got_off[g, see] += w * rel
                    pair = 2.0 ** -17
                    off[i, b, h] = (rel + pair) * (w @ np.abs(vv[see, g]))
                    if f16:              # (a product with 0 would be NaN where a value is infinite)
                        off[i, b, h] += n * 2.0 ** -25 * np.abs(vv[see, g]).max()
            if mass is not None:
                for g in range(n_kv):
                    new = j >= n - t
                    old = np.where(new, 0.0, mass[r, g, :n])
                    mass[r, g, :n] = old + got[g]
                    mass_off[r, g, :n] = got_off[g] + (group * t + 2) * eps * np.abs(mass[r, g, :n])
    return out, off, mass, mass_off


HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}    # half a subnormal step


def check_out(got, want, off, dtype):
    got = values(got)
    same = np.isnan(want) & np.isnan(got) | (got == want)
    with np.errstate(all="ignore"):
        near = np.abs(got - want) <= off + HALF_STEP[dtype] * (np.abs(want) + off) + SMALLEST[dtype]
    bad = ~(same | near)
    assert not bad.any(), "%d of %d off, first at %s: %r, not %r" % (
        bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0])


def check_mass(got, want, off):
    got = values(got)
    bad = ~((np.abs(got - want) <= off) | (got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), "%d of %d masses off, first at %s: %r, not %r" % (
        bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0])


def evict(lens, budget, mass, rows, sinks, recent, slack, kept_len, dst_tokens):
    """Per row: None (not cut) or an array (n_kv, keep) of kept indices."""
    res = []
    mass = values(mass)
    for r in rows:
        n, b = int(lens[r]), float(budget[r])
        if not b < n:
            res.append(None)
            continue
        keep = max(int(math.floor(b)) if b > 0 else 0, sinks + recent)
        if n <= keep + slack or keep > kept_len or keep > dst_tokens:
            res.append(None)
            continue
        got = np.zeros((mass.shape[1], keep), np.int64)
        for h in range(mass.shape[1]):
            m = np.where(np.isnan(mass[r, h, :n]), -np.inf, mass[r, h, :n])
            # NaN below every number, -inf among them
            worse = np.isnan(mass[r, h, :n])
            mid = np.arange(sinks, n - recent)
            by = mid[np.lexsort((mid, -m[mid], worse[mid]))][:keep - sinks - recent]
            got[h] = np.concatenate([np.arange(sinks), np.sort(by), np.arange(n - recent, n)])
        res.append(got)
    return res


def verify(target, draft, tokens, u, u_sample, n_draft):
    """Per row the list of emitted tokens and the accepted count."""
    p_all = values(target)
    q_all = None if draft is None else values(draft)
    tokens, u, u_sample = tokens.numpy(), u.numpy().astype(np.float64), u_sample.numpy().astype(np.float64)
    n_rows, k = tokens.shape
    vocab = p_all.shape[2]
    res = []
    with np.errstate(all="ignore"):
        for i in range(n_rows):
            m = k if n_draft is None else min(int(n_draft[i]), k)
            a = 0
            while a < m:
                x = int(tokens[i, a])
                if not 0 <= x < vocab:
                    break
                q = 1.0 if q_all is None else q_all[i, a, x]
                if not u[i, a] * q < p_all[i, a, x]:
                    break
                a += 1
            p = p_all[i, a]
            w = p.copy()
            if a < m:
                if q_all is None:
                    if 0 <= tokens[i, a] < vocab:
                        w[tokens[i, a]] = 0
                else:
                    w = p - q_all[i, a]
            w = np.where(w > 0, w, 0.0)
            if not w.sum() > 0:
                w = np.where(p > 0, p, 0.0)
            seq = [int(x) for x in tokens[i, :a]]
            if w.sum() > 0:
                sums = np.cumsum(w)
                over = np.nonzero(sums > u_sample[i] * sums[-1])[0]
                seq.append(int(over[0]) if len(over) else int(np.nonzero(w)[0][-1]))
            res.append((seq, a))
    return res
