"""Plain implementations, in 64 bits and on the host, of the operators around the base model's forward pass over a tree of drafted
tokens, and the inputs that their tests share."""
import math
from collections import Counter

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step of the last place, relative


def random_candidates(rng, B, K, n, vocab, shared=0.6, short=0.0):
    """Candidates that share prefixes: each one follows an earlier one for some tokens."""
    cand = rng.integers(0, vocab, (B, K, n))
    for b in range(B):
        for k in range(1, K):
            if rng.random() < shared:
                keep = rng.integers(0, n + 1)
                cand[b, k, :keep] = cand[b, rng.integers(0, k), :keep]
            if rng.random() < short:
                cand[b, k, rng.integers(0, n):] = -1
    return cand.astype(np.int32)


def plan(cand, last, lens, T):
    B, K, n = cand.shape
    W = (T + 31) // 32
    tok, parent = np.zeros((B, T), np.int32), np.full((B, T), -1, np.int32)
    pos, mask = np.repeat(np.asarray(lens, np.int32)[:, None], T, 1), np.zeros((B, T, W), np.uint32)
    node_of, count = np.full((B, K, n + 1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        number = {(): 0}
        tok[b, 0] = last[b]
        for k in range(K):
            node_of[b, k, 0] = 0
            for j in range(n):
                if cand[b, k, j] < 0:
                    break
                prefix = tuple(cand[b, k, :j + 1].tolist())
                if prefix not in number:
                    i = number[prefix] = len(number)
                    if i < T:
                        tok[b, i], parent[b, i], pos[b, i] = prefix[-1], number[prefix[:-1]], lens[b] + j + 1
                node_of[b, k, j + 1] = number[prefix] if number[prefix] < T else -1
        count[b] = min(len(number), T)
        for i in range(count[b]):
            at = i
            while at >= 0:
                mask[b, i, at // 32] |= np.uint32(1 << (at % 32))
                at = parent[b, at]
    return tok, pos, parent, mask.view(np.int32), node_of, count


def page_tables(lens, new, table, held, free, count, page, max_new):
    """Returns slots, table, held, count and whether pages or a row's entries ran out."""
    table, held, count = table.copy(), held.copy(), int(count)
    B, width = table.shape
    slots, short, start, stopped = np.full((B, max_new), -1, np.int64), False, count, False
    for b in range(B):
        fresh = max_new if new is None else int(new[b])
        want = -(-(int(lens[b]) + fresh) // page)
        need = max(want - int(held[b]), 0)
        if want > width:
            short, need = True, 0
        if need and (stopped or need > count):
            short = stopped = True
            need = 0
        for _ in range(need):
            count -= 1
            table[b, held[b]] = free[count]
            held[b] += 1
        for j in range(fresh):
            at = int(lens[b]) + j
            if at // page < held[b]:
                slots[b, j] = int(table[b, at // page]) * page + at % page
    return slots, table, held, count, short


def random_tree(rng, B, T, levels, empty_rows=0.0):
    """Ancestor masks [B, T, ceil(T / 32)] of random trees (levels 1: every node hangs on the root); rows without a bit."""
    seen = np.zeros((B, T, T), bool)
    for b in range(B):
        level = np.zeros(T, int)
        for i in range(T):
            if i:
                level[i] = rng.integers(1, levels + 1)
                above = np.flatnonzero(level[:i] < level[i])
                seen[b, i] = seen[b, rng.choice(above)]
            seen[b, i, i] = True
        seen[b, rng.random(T) < empty_rows] = False
    return seen


def pack_mask(seen):
    B, T, _ = seen.shape
    W = (T + 31) // 32
    bits = np.zeros((B, T, W * 32), np.uint64)
    bits[:, :, :T] = seen
    words = (bits.reshape(B, T, W, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return words.astype(np.uint32).view(np.int32)


def attention(q, k, v, k_cache, v_cache, table, lens, nodes, seen, scale):
    """Returns out, lse and the tolerance of out: rounding the probabilities and the result to the inputs' type, scores and
    exponents in fp32 (all tensors on one device, any shapes of the call; the cache as [pages, page, Hkv, D])."""
    B, T, Hq, D = q.shape
    Hkv, page, half = k.shape[2], k_cache.shape[1], HALF[q.dtype]
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=q.device)
    lse, tol = torch.zeros((B, T, Hq), dtype=torch.float64, device=q.device), torch.zeros_like(out)
    lse_tol = torch.zeros_like(lse)
    for b in range(B):
        L, N = int(lens[b]), int(nodes[b])
        at = torch.arange(L, device=q.device)
        ids = table[b].long()[at // page]
        for h in range(Hq):
            g = h // (Hq // Hkv)
            keys = torch.cat([k_cache[ids, at % page, g], k[b, :N, g]]).double()
            vals = torch.cat([v_cache[ids, at % page, g], v[b, :N, g]]).double()
            visible = torch.ones((N, L + N), dtype=torch.bool, device=q.device)
            visible[:, L:] = torch.as_tensor(seen[b, :N, :N], device=q.device)
            for i in range(N):
                kk, vv = keys[visible[i]], vals[visible[i]]
                if not len(kk):
                    lse[b, i, h] = -math.inf
                    continue
                s = scale * (kk @ q[b, i, h].double())
                size = abs(scale) * (kk.abs() @ q[b, i, h].double().abs())
                norm = torch.logsumexp(s, 0)
                p = torch.exp(s - norm)
                o = p @ vv
                out[b, i, h], lse[b, i, h] = o, norm
                # a score: D + 2 roundings of partial sums of at most `size`, three more of the exponent's argument
                err = (D + 6) * 2.0 ** -24 * size.max() + 4 * 2.0 ** -24 * (s.abs().max() + norm.abs())
                small = 2.0 ** -25 * vv.abs().sum(0) if q.dtype == torch.float16 else 0.0    # subnormal probabilities
                spread = p @ vv.abs()
                many = (len(kk) + 256) * 2.0 ** -24                                          # sums in fp32
                tol[b, i, h] = spread * (half + torch.expm1(2 * err) + many + 2.0 ** -20) * 1.01 + half * o.abs() + small + 1e-30
                if q.dtype == torch.float16:
                    tol[b, i, h] += 2.0 ** -25                                               # a subnormal result
                lse_tol[b, i, h] = 2 * err + many + 2.0 ** -20 + 2.0 ** -22 * norm.abs()
    return out, lse, tol, lse_tol


def walk(tok, parent, nodes, logits, n, hist=None, prompt=None, rep=None, freq=None, pres=None, bias=None, allow=None):
    """hist: a list of tokens per sequence; bias: a list of (token, value) per sequence; allow: bool [B, T, V]; logits float64."""
    B, T, V = logits.shape
    accept, last, nxt = np.zeros(B, np.int32), np.full(B, -1, np.int32), np.full(B, -1, np.int32)
    path = np.full((B, n + 1), -1, np.int32)
    for b in range(B):
        if nodes[b] <= 0:
            continue
        at, went = 0, []
        for step in range(n + 1):
            path[b, step] = last[b] = at
            x = np.where(np.isnan(logits[b, at]), -np.inf, logits[b, at])
            if hist is not None:
                text = [t for t in hist[b] if 0 <= t < V]
                written = [t for t in hist[b][0 if prompt is None else prompt[b]:] if 0 <= t < V] + went
                for t in set(text + went):
                    r = 1.0 if rep is None else float(rep[b])
                    x[t] = x[t] / r if x[t] > 0 else x[t] * r
                for t, times in Counter(written).items():
                    x[t] -= (0.0 if freq is None else float(freq[b])) * times
                    x[t] -= 0.0 if pres is None else float(pres[b])
            if bias is not None:
                for t, value in {t: value for t, value in bias[b] if 0 <= t < V}.items():
                    x[t] += value
            ids = np.arange(V) if allow is None else np.flatnonzero(allow[b, at])
            nxt[b] = ids[np.argmax(x[ids])] if len(ids) else -1
            down = [i for i in range(1, nodes[b]) if parent[b, i] == at and tok[b, i] == nxt[b]]
            if step == n or not down or nxt[b] < 0:
                break
            at, accept[b] = down[0], accept[b] + 1
            went.append(int(nxt[b]))
    return accept, last, nxt, path
