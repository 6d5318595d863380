"""What the operators around the base model's forward pass are measured on.

One verification step of a serving program: the drafted candidates become a tree (`plan`), the block tables grow for the
tokens that may be accepted (`tables`), every layer attends from the tree's nodes to the paged cache and the tree itself
(`attention`), the accepted path is walked in the tree's logits (`verify`), and its keys and values go to the cache
(`commit`).  A case's `op` names one of these.  `own` chooses between the library's calls and the plain form of the same
operator in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False


# ---- cases --------------------------------------------------------------------------------------------------------
def _plan(B, topk, K, T, V, name=None):
    return _named(name, {"op": "plan", "B": B, "topk": topk, "K": K, "T": T, "V": V})


def _tables(B, page, max_new, new, max_len, name=None):
    """new: "all" every sequence appends max_new tokens, "ragged" any number up to that."""
    return _named(name, {"op": "tables", "B": B, "page": page, "max_new": max_new, "new": new, "max_len": max_len})


def _attention(B, T, Hq, Hkv, D, min_len, max_len, page, dtype, layout, tree, ragged, name=None):
    """layout: "nhd" cache [pages, page, heads, D], "hnd" cache [pages, heads, page, D]; tree: levels of the tree, 0 a chain;
    ragged: trees of fewer than T nodes among them."""
    return _named(name, {"op": "attention", "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "min_len": min_len,
                         "max_len": max_len, "page": page, "dtype": dtype, "layout": layout, "tree": tree,
                         "ragged": ragged})


def _verify(B, topk, K, T, V, dtype, history, biases, grammar, name=None):
    """history: longest history that penalties look at, 0 no penalties; biases: entries per sequence."""
    return _named(name, {"op": "verify", "B": B, "topk": topk, "K": K, "T": T, "V": V, "dtype": dtype,
                         "history": history, "biases": biases, "grammar": grammar})


def _commit(L, B, T, n, H, D, page, dtype, layout, name=None):
    return _named(name, {"op": "commit", "L": L, "B": B, "T": T, "n": n, "H": H, "D": D, "page": page, "dtype": dtype,
                         "layout": layout})


def _named(name, case):
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # The trees of a 16-sequence batch at the 13B preset's branching, and of 64 sequences with four heads.
        _plan(16, "6,4,3", 32, 97, 32000, name="plan_13b"),
        _plan(64, "8,4,3,2", 64, 257, 128256, name="plan_8b"),
        # Before every decoding step: room for the n + 1 tokens that may be accepted.
        _tables(64, 16, 5, "all", 8192, name="tables_decode"),
        # A batch of prompts enters the cache: a slot for every token, ragged lengths.
        _tables(64, 64, 4096, "ragged", 1, name="tables_prompt"),
        # One token per sequence, the case that latency decides: a step without speculation.
        _attention(4, 1, 32, 8, 128, 512, 1024, 16, "bf16", "nhd", 0, False, name="attention_token"),
        # The trees of the 13B preset: as many heads of keys as of queries, ragged lengths and trees.
        _attention(16, 61, 40, 40, 128, 300, 2048, 16, "bf16", "nhd", 3, True, name="attention_tree_mha"),
        # Large trees with four query heads per key head: bound by the matrix products.
        _attention(64, 129, 32, 8, 128, 500, 4000, 64, "bf16", "hnd", 4, True, name="attention_tree_gqa"),
        # One sequence with a long context and a short chain.
        _attention(1, 5, 64, 8, 128, 131000, 131072, 16, "f16", "nhd", 0, False, name="attention_long"),
        # Plain greedy acceptance, and a large vocabulary with penalties, biases and a grammar.
        _verify(16, "6,4,3", 32, 97, 32000, "bf16", 0, 0, False, name="verify_13b"),
        _verify(64, "8,4,3,2", 32, 129, 128256, "bf16", 2048, 64, True, name="verify_constrained"),
        # The accepted tokens' keys and values of all layers: few sequences with a head per group, many with grouped heads.
        _commit(40, 4, 61, 3, 40, 128, 16, "bf16", "nhd", name="commit_13b"),
        _commit(32, 64, 33, 4, 8, 128, 16, "bf16", "hnd", name="commit_8b"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _draw_tree(rng):
    while True:
        topk = [rng.randint(1, 8) for _ in range(rng.randint(1, 5))]
        leaves = math.prod(topk)
        if leaves <= 512:
            return ",".join(map(str, topk)), _log_int(rng, 1, min(leaves, 64)), len(topk)


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["op"]] = {k: max(w[k], top.get(c["op"], w)[k]) for k in w}
    while True:
        op = rng.choice(["plan", "tables", "attention", "attention", "attention", "verify", "commit"])
        B = _log_int(rng, 1, 64)
        dtype = rng.choice(["bf16", "bf16", "f16"])
        layout = rng.choice(["nhd", "hnd"])
        page = rng.choice([1, 8, 16, 16, 24, 32, 64, 128])
        topk, K, n = _draw_tree(rng)
        nodes = 1 + K * n
        if op == "plan":
            c = _plan(B, topk, K, min(nodes, _log_int(rng, 2, 320)), _log_int(rng, 1000, 128256))
        elif op == "tables":
            c = _tables(B, page, _log_int(rng, 1, 4096), rng.choice(["all", "ragged"]), _log_int(rng, 1, 16384))
        elif op == "attention":
            Hkv = rng.choice([1, 2, 4, 5, 8, 16, 40])
            tree = rng.choice([0, 0, 2, 3, 4])
            long = _log_int(rng, 1, 131072)
            c = _attention(B, 1 if rng.random() < 0.15 else _log_int(rng, 2, 160), Hkv * rng.choice([1, 1, 3, 4, 8]), Hkv,
                           rng.choice([64, 64, 80, 96, 128, 128, 128]), rng.randint(0, long), long, page, dtype, layout, tree,
                           rng.random() < 0.5)
        elif op == "verify":
            c = _verify(B, topk, K, min(nodes, _log_int(rng, 2, 160)), _log_int(rng, 1000, 128256),
                        rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, _log_int(rng, 1, 4096)]),
                        rng.choice([0, _log_int(rng, 1, 256)]), rng.random() < 0.4)
            if 4.0 * c["B"] * c["T"] * c["V"] > 4.3e9:
                continue
        else:
            c = _commit(_log_int(rng, 1, 48), B, _log_int(rng, 1, 96), n, rng.choice([1, 2, 4, 8, 40]),
                        rng.choice([64, 80, 96, 128]), page, dtype, layout)
        w = work(c)
        if all(w[k] <= top[op][k] for k in w) and _resident(c) <= 6e9:
            return c


def _resident(c):
    if c["op"] == "attention":
        return 4.0 * c["Hkv"] * c["D"] * c["B"] * (c["max_len"] + 2.0 * c["T"] + 2 * c["page"])
    if c["op"] == "commit":
        return 4.0 * c["L"] * c["H"] * c["D"] * c["B"] * (c["T"] + 3.0 * max(c["page"], 32))
    return 0.0


# ---- inputs -------------------------------------------------------------------------------------------------------
_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def _candidates(rng, B, topk, K, V):
    """K of the leaves of a product tree per sequence, best first: siblings are distinct tokens, leaves share prefixes."""
    n = len(topk)
    leaves = math.prod(topk)
    gain = [rng.exponential(1.0, (B, math.prod(topk[:l + 1]))) for l in range(n)]
    toks = []
    for l in range(n):
        first = rng.integers(0, V, (B, math.prod(topk[:l]), 1))
        step = rng.integers(1, max(2, V // topk[l]), first.shape)
        toks.append(((first + step * np.arange(topk[l])) % V).reshape(B, -1))
    score = sum(np.repeat(gain[l], leaves // gain[l].shape[1], axis=1) for l in range(n))
    leaf = np.argsort(score, axis=1)[:, :K]
    cand = np.stack([np.take_along_axis(toks[l], leaf // (leaves // toks[l].shape[1]), axis=1) for l in range(n)], axis=2)
    return cand.astype(np.int32)


def _trie(cand, last, T):
    """Tokens and parents [B, T] of the candidates' tree on the host, at most T nodes, and their numbers [B]."""
    B, K, n = cand.shape
    tok, parent, count = np.zeros((B, T), np.int32), np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        seen, tok[b, 0], nodes = {}, last[b], 1
        for k in range(K):
            at = 0
            for t in cand[b, k]:
                key = (at, int(t))
                if key not in seen:
                    seen[key] = nodes
                    if nodes < T:
                        tok[b, nodes], parent[b, nodes] = t, at
                    nodes += 1
                at = seen[key]
        count[b] = min(nodes, T)
    return tok, parent, count


def _topk(case):
    return [int(t) for t in case["topk"].split(",")]


def _pages(rng, lengths, page, longest):
    """A pool's pages dealt to the sequences in no order: block table [B, width], pages held, free pages, pages in the pool,
    which has room for B sequences of `longest` tokens."""
    held = (np.asarray(lengths) + page - 1) // page
    width = max(1, -(-longest // page))
    total = len(held) * width + 7
    order = rng.permutation(total)
    table, at = np.full((len(held), width), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    return table, held.astype(np.int32), order[at:].astype(np.int32), total


def _cache(shape, layout, dtype, gen):
    """[..., pages, page, H, D] seen through the layout's own order in memory."""
    *lead, pages, page, H, D = shape
    if layout == "hnd":
        return _normal((*lead, pages, H, page, D), dtype, gen).transpose(-3, -2)
    return _normal(shape, dtype, gen)


def _normal(shape, dtype, gen):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for s in range(0, flat.numel(), 1 << 28):
        part = flat[s:s + (1 << 28)]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda", dtype=torch.float32 if dtype == torch.float32
                               else torch.float16))
    return out


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, rng, gen)
    s["op"] = case["op"]
    return s


def _words(*shape, dtype=torch.int32, value=0):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def _prepare_plan(c, rng, gen):
    B, topk, K, T = c["B"], _topk(c), c["K"], c["T"]
    n = len(topk)
    return {"cand": _gpu(_candidates(rng, B, topk, K, c["V"])), "T": T,
            "last": _gpu(rng.integers(0, c["V"], B), torch.int32), "len": _gpu(rng.integers(0, 8192, B), torch.int32),
            "out": (_words(B, T), _words(B, T), _words(B, T), _words(B, T, (T + 31) // 32), _words(B, K, n + 1), _words(B))}


def _prepare_tables(c, rng, gen):
    B, page, most = c["B"], c["page"], c["max_new"]
    lens = np.exp(rng.uniform(0.0, math.log(c["max_len"] + 1.0), B)).astype(np.int64) - 1
    new = np.full(B, most) if c["new"] == "all" else rng.integers(0, most + 1, B)
    table, held, free, _ = _pages(rng, lens, page, c["max_len"] + most)
    return {"len": _gpu(lens, torch.int32), "new": _gpu(new, torch.int32), "table": _gpu(table),
            "held": _gpu(held), "free": _gpu(free), "count": _gpu(np.array([len(free)], np.int32)),
            "page": page, "out": (_words(B, most, dtype=torch.int64), _words(B), _words(1))}


def _prepare_attention(c, rng, gen):
    B, T, Hq, Hkv, D, page = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], c["page"]
    dt = _TORCH[c["dtype"]]
    lens = rng.integers(c["min_len"], c["max_len"] + 1, B)
    nodes = rng.integers((T + 1) // 2, T + 1, B) if c["ragged"] else np.full(B, T)
    table, _, _, pool = _pages(rng, lens, page, c["max_len"])
    s = {"len": _gpu(lens, torch.int32), "nodes": _gpu(nodes, torch.int32), "table": _gpu(table), "mask": None,
         "q": _normal((B, T, Hq, D), dt, gen), "k": _normal((B, T, Hkv, D), dt, gen), "v": _normal((B, T, Hkv, D), dt, gen),
         "k_cache": _cache((pool, page, Hkv, D), c["layout"], dt, gen),
         "v_cache": _cache((pool, page, Hkv, D), c["layout"], dt, gen), "scale": D ** -0.5,
         "out": torch.zeros((B, T, Hq, D), dtype=dt, device="cuda"),
         "lse": torch.zeros((B, T, Hq), dtype=torch.float32, device="cuda")}
    if c["tree"]:
        level = np.zeros(T, np.int64)       # nodes of a level hang on nodes of the level before
        level[1:] = np.sort(rng.integers(1, c["tree"] + 1, T - 1))
        bits = np.zeros((B, T, (T + 31) // 32), np.uint32)
        for i in range(T):
            if i:
                above = np.flatnonzero(level[:i] < level[i])
                above = above[level[above] == level[above].max()]
                bits[:, i] = bits[np.arange(B), rng.choice(above, B)]
            bits[:, i, i // 32] |= np.uint32(1 << (i % 32))
        s["mask"] = _gpu(bits.view(np.int32))
    if own:
        from paper_2404_19124_b200 import binding
        s["ws"] = torch.empty(binding.spec_tree_attention_workspace_bytes(B, T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    return s


def _prepare_verify(c, rng, gen):
    B, topk, K, T, V = c["B"], _topk(c), c["K"], c["T"], c["V"]
    n = len(topk)
    last = rng.integers(0, V, B)
    tok, parent, count = _trie(_candidates(rng, B, topk, K, V), last, T)
    logits = _normal((B, T, V), _TORCH[c["dtype"]], gen).mul_(2.0)
    # the base model agrees with one path of the tree down to a depth of its own per sequence
    on_path = []
    for b in range(B):
        at = int(rng.integers(0, count[b]))
        while parent[b, at] >= 0:
            on_path.append((b, parent[b, at], tok[b, at]))
            at = parent[b, at]
    if on_path:
        i = _gpu(np.array(on_path), torch.int64)
        logits[i[:, 0], i[:, 1], i[:, 2]] = 40.0
    s = {"tok": _gpu(tok), "parent": _gpu(parent), "nodes": _gpu(count), "logits": logits, "n": n, "hist": None,
         "bias": None, "allow": None, "out": (_words(B), _words(B), _words(B), _words(B, n + 1))}
    if c["history"]:
        H = c["history"]
        size = rng.integers(1, H + 1, B)
        # words repeat as in text: a few tokens make up most of it
        hist = (V * rng.random((B, H)) ** 6.0).astype(np.int32)
        hist[np.arange(B), size - 1] = last
        s["hist"] = (_gpu(hist), _gpu(size, torch.int32), _gpu(rng.integers(0, size + 1), torch.int32),
                     _gpu(rng.uniform(1.0, 1.5, B), torch.float32), _gpu(rng.uniform(-0.5, 1.0, B), torch.float32),
                     _gpu(rng.uniform(-0.5, 1.0, B), torch.float32))
    if c["biases"]:
        N = c["biases"]
        s["bias"] = (_gpu(rng.integers(0, V, (B, N)), torch.int32), _gpu(rng.normal(0, 5, (B, N)), torch.float32),
                     _gpu(rng.integers(0, N + 1, B), torch.int32))
    if c["grammar"]:
        # most words of 32 tokens are open or shut as a whole, the path's tokens are allowed
        shape = (B, T, (V + 31) // 32)
        words = torch.randint(-2 ** 31, 2 ** 31, shape, generator=gen, device="cuda", dtype=torch.int64)
        kind = torch.rand(shape, generator=gen, device="cuda")
        words = torch.where(kind < 0.5, torch.zeros_like(words), torch.where(kind < 0.8, torch.full_like(words, -1), words))
        for b, r, t in on_path:
            words[int(b), int(r), int(t) // 32] = -1
        s["allow"] = words.to(torch.int32)
    return s


def _prepare_commit(c, rng, gen):
    L, B, T, n, H, D, page = (c[k] for k in ("L", "B", "T", "n", "H", "D", "page"))
    dt = _TORCH[c["dtype"]]
    lens = rng.integers(0, 33, B)
    table, _, _, pool = _pages(rng, lens + n + 1, page, 32 + n + 1)
    at = lens[:, None] + np.arange(n + 1)
    slots = np.take_along_axis(table, at // page, axis=1).astype(np.int64) * page + at % page
    accept = rng.integers(0, min(n, T - 1) + 1, B)
    path = np.full((B, n + 1), -1, np.int32)
    for b in range(B):
        path[b, 0] = 0
        path[b, 1:accept[b] + 1] = 1 + np.sort(rng.permutation(T - 1)[:accept[b]])
    return {"k": _normal((L, B, T, H, D), dt, gen), "v": _normal((L, B, T, H, D), dt, gen),
            "k_cache": _cache((L, pool, page, H, D), c["layout"], dt, gen),
            "v_cache": _cache((L, pool, page, H, D), c["layout"], dt, gen), "path": _gpu(path),
            "accept": _gpu(accept, torch.int32), "slots": _gpu(slots), "len": _gpu(lens, torch.int32), "out": _words(B)}


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(s):
    return globals()[("_own_" if own else "_plain_") + s["op"]](s)


def _own_plan(s):
    from paper_2404_19124_b200 import binding as spec
    tree = spec.spec_tree_plan(s["cand"], s["last"], s["len"], s["T"], tree=spec.SpecTree(*s["out"]))
    return tuple(tree)


def _own_tables(s):
    from paper_2404_19124_b200 import binding as spec
    slots, held, count = s["out"]
    spec.spec_page_tables(s["len"], s["new"], s["table"], s["held"], s["free"], s["count"], s["page"], slots=slots,
                          n_pages_out=held, free_count_out=count)
    return slots, s["table"], held, count


def _own_attention(s):
    from paper_2404_19124_b200 import binding as spec
    spec.spec_tree_attention(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["len"], mask=s["mask"],
                             n_nodes=s["nodes"], scale=s["scale"], out=s["out"], lse=s["lse"], workspace=s["ws"])
    return s["out"], s["lse"]


def _own_verify(s):
    from paper_2404_19124_b200 import binding as spec
    given = {}
    if s["hist"] is not None:
        given.update(zip(("hist_tok", "hist_len", "prompt_len", "repetition", "frequency", "presence"), s["hist"]))
    if s["bias"] is not None:
        given.update(zip(("bias_tok", "bias_val", "bias_len"), s["bias"]))
    accept, last, nxt, path = s["out"]
    spec.spec_verify_tree(s["tok"], s["parent"], s["nodes"], s["logits"], allow=s["allow"], accept_len=accept, last_node=last,
                          next_tok=nxt, path=path, **given)
    return s["out"]


def _own_commit(s):
    from paper_2404_19124_b200 import binding as spec
    spec.spec_kv_commit(s["k"], s["v"], s["k_cache"], s["v_cache"], s["path"], s["accept"], s["slots"], s["len"],
                        new_len=s["out"])
    return s["k_cache"], s["v_cache"], s["out"]


def _plain_plan(s):
    cand, T = s["cand"], s["T"]
    B, K, n = cand.shape
    dev = cand.device
    same = (cand[:, :, None] == cand[:, None]).to(torch.int32).cumprod(-1) > 0          # [B, K, K', n] equal prefixes
    first = same.to(torch.int32).argmax(2)                                               # lowest K' with the same prefix
    new = first == torch.arange(K, device=dev)[:, None]
    number = new.reshape(B, -1).to(torch.int64).cumsum(1).reshape(B, K, n)
    node = number.gather(1, first)
    keep = node < T
    node_of = torch.cat([torch.zeros((B, K, 1), dtype=torch.int64, device=dev), torch.where(keep, node, -1)], 2)
    above = torch.cat([torch.zeros((B, K, 1), dtype=torch.int64, device=dev), node[:, :, :-1]], 2)
    at = torch.where(keep, node, T).reshape(B, -1)                                       # what does not fit goes to column T
    put = lambda start, value: torch.full((B, T + 1), start, dtype=torch.int64, device=dev).scatter_(1, at, value.reshape(B, -1))
    tok, parent = put(0, cand.long())[:, :T], put(-1, above)[:, :T]
    depth = put(0, torch.arange(1, n + 1, device=dev).expand(B, K, n))[:, :T]
    tok[:, 0] = s["last"]
    count = 1 + new.reshape(B, -1).sum(1)
    count = count.clamp(max=T)
    sees = torch.zeros((B, T, T + 1), dtype=torch.bool, device=dev)
    up = torch.arange(T, device=dev).expand(B, T)
    for _ in range(n + 1):
        sees.scatter_(2, torch.where(up >= 0, up, T).unsqueeze(2), True)
        up = torch.where(up > 0, parent.gather(1, up.clamp(min=0)), -1)
    sees = sees[:, :, :T] & (torch.arange(T, device=dev) < count[:, None])[:, :, None]
    W = (T + 31) // 32
    bits = torch.zeros((B, T, W * 32), dtype=torch.int64, device=dev)
    bits[:, :, :T] = sees
    mask = (bits.reshape(B, T, W, 32) << torch.arange(32, device=dev)).sum(-1)
    mask = torch.where(mask >= 2 ** 31, mask - 2 ** 32, mask)
    pos = s["len"].long()[:, None] + depth
    return tuple(t.to(torch.int32) for t in (tok, pos, parent, mask, node_of, count))


def _plain_tables(s):
    slots, table, page = s["out"][0], s["table"], s["page"]
    dev = table.device
    lens, new, held = s["len"].long(), s["new"].long(), s["held"].long()
    want = (lens + new + page - 1) // page
    need = (want - held).clamp(min=0)
    before = need.cumsum(0) - need
    col = torch.arange(table.shape[1], device=dev)
    fresh = (col >= held[:, None]) & (col < want[:, None])
    from_top = s["count"].long() - 1 - (before[:, None] + col - held[:, None])
    out = torch.where(fresh, s["free"][from_top.clamp(0, s["free"].numel() - 1)], table)
    at = lens[:, None] + torch.arange(slots.shape[1], device=dev)
    slot = out.long().gather(1, (at // page).clamp(max=table.shape[1] - 1)) * page + at % page
    slot = torch.where(torch.arange(slots.shape[1], device=dev) < new[:, None], slot, -1)
    return slot, out, (held + need).to(torch.int32), (s["count"] - need.sum()).to(torch.int32)


def _plain_attention(s):
    q, T = s["q"], s["q"].shape[1]
    B, _, Hq, D = q.shape
    Hkv = s["k"].shape[2]
    G, dev = Hq // Hkv, q.device
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    page = s["k_cache"].shape[1]
    lens, nodes = s["len"].tolist(), s["nodes"].tolist()
    node = torch.arange(T, device=dev)
    for b in range(B):
        L, N = lens[b], nodes[b]
        ids = s["table"][b, :(L + page - 1) // page].long()
        gather = lambda cache, tree: torch.cat([cache[ids].reshape(-1, Hkv, D)[:L], tree[b, :N]]).float().transpose(0, 1)
        if s["mask"] is None:
            sees = node[None, :N] <= node[:N, None]
        else:
            sees = ((s["mask"][b, :N, :, None] >> torch.arange(32, device=dev)) & 1).reshape(N, -1)[:, :N] != 0
        sees = torch.cat([torch.ones((N, L), dtype=torch.bool, device=dev), sees], 1).repeat_interleave(G, 0)
        rows = q[b, :N].float().reshape(N, Hkv, G, D).transpose(0, 1).reshape(Hkv, N * G, D)
        score = torch.matmul(rows, gather(s["k_cache"], s["k"]).transpose(1, 2)) * s["scale"]
        score = torch.where(sees, score, float("-inf"))
        top = score.max(-1, keepdim=True).values
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, gather(s["v_cache"], s["v"])) / total
        out[b, :N] = o.reshape(Hkv, N, G, D).transpose(0, 1).reshape(N, Hq, D).to(out.dtype)
        lse[b, :N] = (top + torch.log(total)).reshape(Hkv, N, G).transpose(0, 1).reshape(N, Hq)
    return out, lse


def _plain_verify(s):
    tok, parent, logits, n = s["tok"].long(), s["parent"], s["logits"], s["n"]
    B, T, V = logits.shape
    dev = logits.device
    live = torch.arange(T, device=dev) < s["nodes"][:, None]
    each = torch.arange(B, device=dev)
    cur = torch.zeros(B, dtype=torch.int64, device=dev)
    accept, nxt = torch.zeros_like(cur), torch.full_like(cur, -1)
    path = torch.full((B, n + 1), -1, dtype=torch.int64, device=dev)
    walking = torch.ones(B, dtype=torch.bool, device=dev)
    if s["hist"] is not None:
        hist, size, prompt, rep, freq, pres = s["hist"]
        col = torch.arange(hist.shape[1], device=dev)
        seen = torch.zeros((B, V), dtype=torch.float32, device=dev).scatter_add_(
            1, hist.long(), (col < size[:, None]).float())
        count = torch.zeros((B, V), dtype=torch.float32, device=dev).scatter_add_(
            1, hist.long(), ((col < size[:, None]) & (col >= prompt[:, None])).float())
    if s["bias"] is not None:
        where, value, size = s["bias"]
        N = where.shape[1]
        order = torch.where(torch.arange(N, device=dev) < size[:, None], torch.arange(1, N + 1, device=dev), 0)
        entry = torch.zeros((B, V), dtype=torch.int64, device=dev).scatter_reduce_(1, where.long(), order, "amax")
        bias = torch.where(entry > 0, value.gather(1, (entry - 1).clamp(min=0)), 0.0)
    for step in range(n + 1):
        x = logits[each, cur].float()
        if s["hist"] is not None:
            x = torch.where(seen > 0, torch.where(x > 0, x / rep[:, None], x * rep[:, None]), x)
            x = x - freq[:, None] * count - pres[:, None] * (count > 0).float()
        if s["bias"] is not None:
            x = torch.where(entry > 0, x + bias, x)
        x = torch.where(x != x, float("-inf"), x)
        best = x.argmax(1)
        if s["allow"] is not None:
            ok = ((s["allow"][each, cur][:, :, None] >> torch.arange(32, device=dev)) & 1).reshape(B, -1)[:, :V] != 0
            top = torch.where(ok, x, float("-inf")).max(1, keepdim=True).values
            good = ok & (x == top)
            best = torch.where(good.any(1), good.to(torch.int32).argmax(1), -1)
        path[:, step] = torch.where(walking, cur, path[:, step])
        nxt = torch.where(walking, best, nxt)
        child = live & (parent == cur[:, None]) & (tok == best[:, None])
        walking = walking & child.any(1) & (step < n)
        cur = torch.where(walking, child.to(torch.int32).argmax(1), cur)
        accept += walking
        if s["hist"] is not None:
            went = torch.where(walking, 1.0, 0.0)[:, None]
            at = best.clamp(min=0)[:, None]
            seen.scatter_add_(1, at, went)
            count.scatter_add_(1, at, went)
    return tuple(t.to(torch.int32) for t in (accept, cur, nxt, path))


def _plain_commit(s):
    n1 = s["path"].shape[1]
    page = s["k_cache"].shape[2]
    dev = s["path"].device
    taken = torch.arange(n1, device=dev) <= s["accept"][:, None]
    b, j = torch.nonzero(taken, as_tuple=True)
    node, slot = s["path"][b, j].long(), s["slots"][b, j]
    for cache, tree in ((s["k_cache"], s["k"]), (s["v_cache"], s["v"])):
        cache[:, slot // page, slot % page] = tree[:, b, node]
    return s["k_cache"], s["v_cache"], s["len"] + s["accept"] + 1


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(c):
    B = c["B"]
    if c["op"] == "plan":
        K, n, T = c["K"], len(_topk(c)), c["T"]
        return {"bytes": 4.0 * B * (K * n + 2 + 3 * T + T * ((T + 31) // 32) + K * (n + 1) + 1), "flops": 0.0}
    if c["op"] == "tables":
        new = c["max_new"] * (1.0 if c["new"] == "all" else 0.5)
        return {"bytes": B * (16.0 + 8.0 * c["max_new"] + 8.0 * math.ceil(new / c["page"])), "flops": 0.0}
    if c["op"] == "attention":
        nodes = c["T"] * (0.75 if c["ragged"] and c["T"] > 1 else 1.0)
        keys = 0.5 * (c["min_len"] + c["max_len"])
        sees = 0.5 * (nodes + 1) if c["tree"] == 0 else min(nodes, 0.5 * c["tree"] + 1)
        kv = 4.0 * c["Hkv"] * c["D"] * (keys + nodes)
        io = nodes * c["Hq"] * (4.0 * c["D"] + 4.0)
        mask = nodes * 4.0 * ((c["T"] + 31) // 32) if c["tree"] else 0.0
        return {"bytes": B * (kv + io + mask + 4.0 * keys / c["page"] + 8.0),
                "flops": 4.0 * B * nodes * c["Hq"] * c["D"] * (keys + sees)}
    if c["op"] == "verify":
        rows = 1.0 + 0.5 * len(_topk(c))
        row = c["V"] * (4.0 if c["dtype"] == "f32" else 2.0) + (c["V"] / 8.0 if c["grammar"] else 0.0)
        lists = 2.0 * c["history"] + 4.0 * c["biases"]
        return {"bytes": B * (rows * row + lists + 8.0 * c["T"] + 4.0 * (len(_topk(c)) + 8)), "flops": 0.0}
    rows = 1.0 + 0.5 * min(c["n"], c["T"] - 1)
    return {"bytes": B * (rows * c["L"] * c["H"] * c["D"] * 8.0 + 12.0 * (c["n"] + 1) + 12.0), "flops": 0.0}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _exact_plan(c, s):
    cand, last, lens, T = s["cand"].cpu().numpy(), s["last"].cpu().numpy(), s["len"].cpu().numpy(), s["T"]
    B, K, n = cand.shape
    tok, parent, count = _trie(cand, last, T)
    pos, mask = np.repeat(lens[:, None], T, 1), np.zeros((B, T, (T + 31) // 32), np.uint32)
    node_of = np.zeros((B, K, n + 1), np.int32)
    for b in range(B):
        down = {(int(parent[b, i]), int(tok[b, i])): i for i in range(1, count[b])}
        for i in range(count[b]):
            at = i
            while at >= 0:
                mask[b, i, at // 32] |= np.uint32(1 << (at % 32))
                pos[b, i] += at != 0
                at = parent[b, at]
        for k in range(K):
            for j in range(n):
                up = int(node_of[b, k, j])
                node_of[b, k, j + 1] = down.get((up, int(cand[b, k, j])), -1) if up >= 0 else -1
    return tuple(_gpu(a, torch.int32) for a in (tok, pos, parent, mask.view(np.int32), node_of, count))


def _exact_tables(c, s):
    table, held, page = s["table"].cpu().numpy().copy(), s["held"].cpu().numpy().copy(), s["page"]
    stack = s["free"].cpu().tolist()
    slots = np.full(tuple(s["out"][0].shape), -1, np.int64)
    for b, (length, new) in enumerate(zip(s["len"].tolist(), s["new"].tolist())):
        while held[b] * page < length + new:
            table[b, held[b]] = stack.pop()
            held[b] += 1
        at = np.arange(length, length + new)
        slots[b, :new] = table[b, at // page].astype(np.int64) * page + at % page
    return _gpu(slots), _gpu(table), _gpu(held), _gpu(np.array([len(stack)], np.int32))


def _exact_attention(c, s):
    B, T, Hq, D = s["q"].shape
    Hkv, page = s["k"].shape[2], s["k_cache"].shape[1]
    G, dev = Hq // Hkv, s["q"].device
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=dev)
    lse = torch.zeros((B, T, Hq), dtype=torch.float64, device=dev)
    if work(c)["flops"] > 3e12:
        return None
    masks = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    for b in range(B):
        L, N = int(s["len"][b]), int(s["nodes"][b])
        at = torch.arange(L, device=dev)
        ids = s["table"][b].long()[at // page]
        hidden = torch.ones((N, N), dtype=torch.bool)
        for i in range(N):
            for t in range(N):
                hidden[i, t] = t > i if masks is None else not (int(masks[b, i, t // 32]) >> (t % 32)) & 1
        hidden = hidden.to(dev)
        for h in range(Hkv):
            keys = torch.cat([s["k_cache"][ids, at % page, h], s["k"][b, :N, h]]).double()
            vals = torch.cat([s["v_cache"][ids, at % page, h], s["v"][b, :N, h]]).double()
            for g in range(h * G, h * G + G):
                score = s["scale"] * (s["q"][b, :N, g].double() @ keys.T)
                score[:, L:].masked_fill_(hidden, -math.inf)
                norm = torch.logsumexp(score, 1)
                out[b, :N, g] = torch.exp(score - norm[:, None]) @ vals
                lse[b, :N, g] = norm
    return out, lse


def _exact_verify(c, s):
    B, T, V = s["logits"].shape
    n = s["n"]
    tok, parent, nodes = s["tok"].cpu().numpy(), s["parent"].cpu().numpy(), s["nodes"].cpu().numpy()
    accept, last, nxt = np.zeros(B, np.int32), np.zeros(B, np.int32), np.zeros(B, np.int32)
    path = np.full((B, n + 1), -1, np.int32)
    lists = {k: None if s[k] is None else [t.cpu().numpy() for t in s[k]] for k in ("hist", "bias")}
    for b in range(B):
        at, went = 0, []
        for step in range(n + 1):
            path[b, step] = last[b] = at
            x = s["logits"][b, at].cpu().double().numpy()
            if lists["hist"] is not None:
                hist, size, prompt, rep, freq, pres = (a[b] for a in lists["hist"])
                text = hist[:size].tolist() + went
                for t in set(text):
                    x[t] = x[t] / float(rep) if x[t] > 0 else x[t] * float(rep)
                written = text[int(prompt):]
                for t, times in zip(*np.unique(np.array(written, np.int64), return_counts=True)):
                    x[t] -= float(freq) * times + float(pres)
            if lists["bias"] is not None:
                where, value, size = (a[b] for a in lists["bias"])
                for t, v in dict(zip(where[:size].tolist(), value[:size].tolist())).items():
                    x[t] += v
            choices = np.arange(V)
            if s["allow"] is not None:
                words = s["allow"][b, at].cpu().numpy().view(np.uint32)
                choices = choices[(words[choices // 32] >> (choices % 32).astype(np.uint32)) & 1 == 1]
            nxt[b] = choices[np.argmax(x[choices])] if len(choices) else -1
            down = [i for i in range(1, nodes[b]) if parent[b, i] == at and tok[b, i] == nxt[b]]
            if step == n or not down:
                break
            at, accept[b] = down[0], accept[b] + 1
            went.append(int(nxt[b]))
    return tuple(_gpu(a) for a in (accept, last, nxt, path))


def _exact_commit(c, s):
    page = s["k_cache"].shape[2]
    for b, (accept, path, slots) in enumerate(zip(s["accept"].tolist(), s["path"].tolist(), s["slots"].tolist())):
        for node, slot in zip(path[:accept + 1], slots):
            s["k_cache"][:, slot // page, slot % page] = s["k"][:, b, node]
            s["v_cache"][:, slot // page, slot % page] = s["v"][:, b, node]
    return s["k_cache"], s["v_cache"], s["len"] + s["accept"] + 1
