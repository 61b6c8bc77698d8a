"""What the speed of the operators around a paged cache is measured on: its pages, attention with other scores and masks, joins.

  attend   attention of new tokens over a paged cache (16 bits, or 8 with a scale for each block and head) where
             - scores are capped:  cap * tanh(score / cap)
             - scores get a bias that falls with distance:  - slope[head] * |p - t|
             - a prefix is seen by every query, and what follows it only backwards
             - a request holds several documents, and a query sees its own (and the prefix)
  join     results of attention over different keys, each with the logarithm of its sum, put together
  fork     sequences are forked, each fork grows by a few tokens, blocks that they share are copied before, and the forks go again
  compact  the blocks in use move to the front of a pool, all layers of it, and the tables follow

Sizes are given by the case alone; contents come from the seed.  `own` says which form `run` takes: elementary torch operations, or
the framework's operators.
"""
import heapq
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _attend(name, requests, hit, new, bs=64, heads=(32, 8), dim=128, dtype="bf16", cache="16", window=0, sinks=0, keys="all",
            lse=False, cap=0.0, slopes=False, prefix=(0, 0), documents=(0, 0)):
    return {"name": name, "op": "attend", "requests": requests, "hit_lo": hit[0], "hit_hi": hit[1], "new_lo": new[0], "new_hi": new[1],
            "block_tokens": bs, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim, "dtype": dtype, "cache": cache,
            "window": window, "sinks": sinks, "keys": keys, "lse": lse, "cap": cap, "slopes": slopes,
            "prefix_lo": prefix[0], "prefix_hi": prefix[1], "document_lo": documents[0], "document_hi": documents[1]}


def _join(name, tokens, heads, dim, parts, dtype="bf16", lse=False):
    return {"name": name, "op": "join", "tokens": tokens, "q_heads": heads, "head_dim": dim, "parts": parts, "dtype": dtype, "lse": lse}


def _pages(name, op, sequences, tokens, layers, bs, planes, scales=0, forks=0, grow=1, blocks=0):
    """planes: bytes of a token's row in each of them; scales: bytes of a block in each of two more planes."""
    return {"name": name, "op": op, "sequences": sequences, "tokens_lo": tokens[0], "tokens_hi": tokens[1], "layers": layers,
            "block_tokens": bs, "planes": len(planes), "row_bytes": planes[0], "scale_bytes": scales, "forks": forks, "grow": grow,
            "pool_blocks": blocks}


def listed():
    return [
        # a decode step of four short chats with capped scores, 16-token blocks: launches are all there is
        _attend("capped_step_small", 4, (1000, 1000), (1, 1), bs=16, cap=50.0),
        # a decode step of many long chats of a model that knows positions by a bias alone, 8-bit cache: the largest in bytes
        _attend("sloped_step_8bit", 64, (8192, 32768), (1, 1), cache="8", slopes=True, lse=True),
        # a draft's tokens checked, in requests of several documents behind a common prefix: a few queries each, a group of seven heads
        _attend("capped_documents_verify", 32, (700, 9000), (3, 6), bs=16, heads=(28, 4), lse=True, cap=30.0, prefix=(100, 400),
                documents=(600, 3000)),
        # appended tails with capped scores under a window, heads of 64, pages that end inside a tile
        _attend("capped_window_prefill", 8, (300, 6000), (400, 2000), bs=24, heads=(24, 8), dim=64, dtype="f16", window=1024, cap=50.0),
        # prompts whose first part (an image, instructions) is seen both ways
        _attend("prefix_prefill", 16, (0, 500), (300, 2500), prefix=(256, 2000)),
        # documents packed into a few long requests, a short prefix in common; an 8-bit cache
        _attend("documents_prefill_8bit", 4, (0, 3000), (3000, 6000), cache="8", lse=True, prefix=(0, 200), documents=(40, 1500)),
        # the largest in operations: appended tails over long cached prefixes, with the bias
        _attend("sloped_prefill", 4, (8192, 32768), (256, 1024), slopes=True),
        # the cached prefix's result and the tail's, in a decode step
        _join("join_step_small", 4, 32, 128, 2),
        # the same for a long prompt whose keys came in four parts, some of which some rows do not see
        _join("join_prefill", 8000, 64, 128, 4, dtype="f16", lse=True),
        # four chats are forked once each: a block a layer and fork is copied
        _pages("fork_step_small", "fork", 4, (900, 1100), 4, 16, (2048, 2048), forks=1),
        # a step of a search with eight ways on from each of 32 prompts, 8-bit cache
        _pages("fork_beams_8bit", "fork", 32, (300, 2000), 16, 64, (1024, 1024), scales=32, forks=8, grow=3),
        # a fragmented pool of latent rows, two in five blocks in use: most of these are copied
        _pages("compact_latent", "compact", 24, (200, 2400), 24, 64, (1152,), blocks=1200),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of these ranges."""
    op = rng.choice(["attend", "attend", "attend", "join", "fork", "compact"])
    if op == "attend":
        c = _draw_attend(rng)
    elif op == "join":
        dim, heads, parts = rng.choice([64, 128]), rng.choice([1, 4, 7, 16, 28, 32, 64]), rng.randint(2, 6)
        most = 8000 * 64 * 128 * 4 // (dim * heads * parts)
        c = _join("", _spread(rng, 1, min(most, 20000)), heads, dim, parts, rng.choice(["bf16", "f16"]), rng.random() < 0.5)
    else:
        planes, row = rng.choice([(2, 256), (2, 1024), (2, 2048), (1, 1152), (1, 656), (2, 80)])
        bs, layers = rng.choice([8, 16, 24, 64, 100]), _spread(rng, 1, 60)
        scales = rng.choice([0, 4, 32]) if planes == 2 else 0
        blocks = max(16, min(6000, (2 << 30) // (bs * row * planes * layers)))      # of the pool, about
        if op == "fork":
            n = _spread(rng, 1, max(1, min(64, blocks // 8)))
            forks, grow = rng.randint(1, max(1, min(8, blocks // (4 * n)))), rng.choice([1, 1, 2, 5, bs + 1])
            hi = _spread(rng, 1, max(2, min(blocks * bs // (2 * n), 8000)))
            c = _pages("", op, n, (rng.randint(1, hi), hi), layers, bs, (row,) * planes, scales, forks, grow)
        else:
            n = _spread(rng, 1, max(1, min(64, blocks // 4)))
            hi = _spread(rng, bs, max(bs + 1, min(blocks * bs // (3 * n), 8000)))
            need = n * ((hi + bs - 1) // bs)
            c = _pages("", op, n, (rng.randint(1, hi), hi), layers, bs, (row,) * planes, scales, blocks=int(need * rng.uniform(1.1, 2.5)) + 1)
    del c["name"]
    return c


def _draw_attend(rng):
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8])
    q = kv * rng.choice([1, 2, 3, 4, 5, 7, 8])
    cache = rng.choice(["16", "8"])
    bs = rng.choice([8, 16, 24, 32, 64, 64, 100, 128])
    form = rng.choice(["step", "few", "prefill"])
    requests = _spread(rng, 1, {"step": 128, "few": 64, "prefill": 16}[form])
    new = {"step": (1, 1), "few": (1, rng.randint(2, 9)), "prefill": (rng.randint(1, 200), _spread(rng, 200, 1024))}[form]
    most = min(131072, {"step": 1_000_000, "few": 500_000, "prefill": 40_000}[form] // requests)
    hi = _spread(rng, 60, most)
    total = hi + new[1]
    what = rng.choice(["cap", "slopes", "both", "prefix", "documents", "all"])
    prefix = (0, 0)
    if what == "prefix" or (what in ("documents", "all") and rng.random() < 0.5):
        prefix = (0, _spread(rng, 1, total))
    documents = (0, 0)
    if what in ("documents", "all"):
        longest = _spread(rng, 20, max(21, total))
        documents = (rng.randint(1, longest), longest)
    return _attend("", requests, (rng.randint(0, hi // 2), hi), new, bs, (q, kv), dim, rng.choice(["bf16", "bf16", "f16"]), cache,
                   window=_spread(rng, 16, 8192) if rng.random() < 0.3 else 0, sinks=rng.choice([0, 0, 1, 4, 70]),
                   keys=rng.choice(["all", "all", "all", "hit", "append"]), lse=rng.random() < 0.5,
                   cap=rng.choice([15.0, 30.0, 50.0]) if what in ("cap", "both", "all") else 0.0,
                   slopes=what in ("slopes", "both", "all"), prefix=prefix, documents=documents)


# Lengths, masks and tables: of the case alone ------------------------------------------------------------------------------------------

def _numbers(case):
    return np.random.Generator(np.random.PCG64([20260307, *(int(v) for v in case.values() if isinstance(v, int))]))


def _batch(case):
    """Of every request: cached and new tokens, the prefix's length, and the first tokens of the documents (int64)."""
    rng, n = _numbers(case), case["requests"]
    hit = rng.integers(case["hit_lo"], case["hit_hi"] + 1, size=n)
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=n)
    prefix = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, size=n)
    starts = []
    for total in (hit + new).tolist():
        at, some = 0, []
        while case["document_hi"] and at < total:
            some.append(at)
            at += int(rng.integers(case["document_lo"], case["document_hi"] + 1))
        starts.append(np.array(some, dtype=np.int64))
    return hit, new, prefix, starts


def _key_range(case, hit, new):
    """[first, last) of the keys that the case's plan holds, for each request."""
    return {"all": (0 * hit, hit + new), "hit": (0 * hit, hit), "append": (hit, hit + new)}[case["keys"]]


def _bounds(case, h, n, prefix, starts):
    """Of each query of a request: it sees the tokens in [lo, hi), and those before `first` and `hi`."""
    p = np.arange(h, h + n, dtype=np.int64)
    lo = np.maximum(p + 1 - case["window"], 0) if case["window"] else 0 * p
    if starts.size:
        lo = np.maximum(lo, starts[np.searchsorted(starts, p, side="right") - 1])
    return lo, np.maximum(p + 1, prefix), max(case["sinks"], prefix)


def _sequences(case):
    """Lengths of the sequences, their tables, and the pool's blocks."""
    rng, n, bs = _numbers(case), case["sequences"], case["block_tokens"]
    tokens = rng.integers(case["tokens_lo"], case["tokens_hi"] + 1, size=n)
    need = (tokens + bs - 1) // bs
    more = case["sequences"] * case["forks"] * ((case["grow"] + bs - 1) // bs + 1)
    blocks = max(case["pool_blocks"], int(need.sum()) + more)
    order = rng.permutation(blocks).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    return tokens, [order[a:b].copy() for a, b in zip(at[:-1], at[1:])], blocks


def _block_bytes(case):
    return [case["row_bytes"] * case["block_tokens"]] * case["planes"] + [case["scale_bytes"]] * (2 if case["scale_bytes"] else 0)


def work(case):
    """Inputs once, outputs once; of the cache the rows that some query sees, of the pool the blocks that are copied."""
    if case["op"] == "join":
        rows = case["tokens"] * case["q_heads"]
        return {"bytes": rows * ((case["parts"] + 1) * 2 * case["head_dim"] + 4 * case["parts"] + (4 if case["lse"] else 0)),
                "flops": 2 * rows * case["parts"] * case["head_dim"]}
    if case["op"] in ("fork", "compact"):
        tokens, tables, _ = _sequences(case)
        if case["op"] == "fork":
            copies = int((tokens % case["block_tokens"] != 0).sum()) * case["forks"]
        else:
            used = np.concatenate(tables)
            copies = int((used >= used.size).sum())
        return {"bytes": 2 * copies * case["layers"] * sum(_block_bytes(case)), "flops": 0}
    hit, new, prefix, starts = _batch(case)
    first, last = _key_range(case, hit, new)
    rows = pairs = 0
    for h, n, a, b, x, s in zip(hit.tolist(), new.tolist(), first.tolist(), last.tolist(), prefix.tolist(), starts):
        lo, hi, front = _bounds(case, h, n, x, s)
        end = np.minimum(hi, b)
        near = np.maximum(lo, a)
        pairs += int((np.maximum(end - near, 0) + np.maximum(np.minimum(np.minimum(front, near), end) - a, 0)).sum())
        seen = np.zeros(h + n + 1, dtype=np.int64)
        some = end > near
        np.add.at(seen, near[some], 1)
        np.add.at(seen, end[some], -1)
        seen = np.cumsum(seen) > 0
        seen[a:max(a, min(front, int(end.max())))] = True
        rows += int(seen[a:b].sum())
    n, d, q, kv, e = int(new.sum()), case["head_dim"], case["q_heads"], case["kv_heads"], 1 if case["cache"] == "8" else 2
    scales = int(8 * kv * rows / case["block_tokens"]) if e == 1 else 0
    return {"bytes": 4 * n * q * d + 2 * rows * kv * d * e + scales + (4 * n * q if case["lse"] else 0), "flops": 4 * d * q * pairs}


# What a program has in hand ---------------------------------------------------------------------------------------------------------

def _quantised_pool(blocks, bs, kv, d, gen):
    """A plane of e4m3 codes and its scales, of normal values whose spread differs by block and head."""
    codes = torch.empty(blocks, bs, kv, d, dtype=torch.uint8, device="cuda")
    scales = torch.empty(blocks, kv, dtype=torch.float32, device="cuda")
    some = max(1, (1 << 26) // (bs * kv * d))
    for at in range(0, blocks, some):
        n = min(some, blocks - at)
        x = torch.randn(n, bs, kv, d, device="cuda", generator=gen)
        x *= torch.randn(n, 1, kv, 1, device="cuda", generator=gen).mul_(0.3).exp_()
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(dim=(1, 3)) / 448)))
        scales[at:at + n] = s
        codes[at:at + n] = (x / s[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if own:
        import paper_2602_21548_amd as K
        s["kvl"] = K
    return {"attend": _prepare_attend, "join": _prepare_join, "fork": _prepare_pages, "compact": _prepare_pages}[case["op"]](s, seed, gen)


def _prepare_attend(s, seed, gen):
    case = s["case"]
    hit, new, prefix, starts = _batch(case)
    bs, d, q, kv = case["block_tokens"], case["head_dim"], case["q_heads"], case["kv_heads"]
    dtype = DTYPES[case["dtype"]]
    need = (hit + new + bs - 1) // bs
    blocks = int(math.ceil(1.05 * int(need.sum()))) + 1
    order = np.random.Generator(np.random.PCG64([seed, 11])).permutation(blocks).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    tables = [order[a:b].copy() for a, b in zip(at[:-1], at[1:])]
    n = int(new.sum())
    s.update(hit=hit, new=new, tables=tables, tokens=n, prefix=prefix, starts=starts)
    if case["cache"] == "8":
        (k, ks), (v, vs) = (_quantised_pool(blocks, bs, kv, d, gen) for _ in range(2))
        s["planes"] = [k, v, ks, vs]
    else:
        s["planes"] = [torch.randn(blocks, bs, kv, d, device="cuda", dtype=dtype, generator=gen) for _ in range(2)]
    # (scores whose spread is about 8, so that a cap is felt)
    s["q"] = (torch.randn(n, q, d, device="cuda", generator=gen) * (8 if case["cap"] else 1)).to(dtype)
    s["out"] = torch.zeros(n, q, d, device="cuda", dtype=dtype)
    s["lse"] = torch.zeros(n, q, device="cuda") if case["lse"] else None
    s["scale"] = 1 / math.sqrt(d)
    s["slopes"] = torch.exp2(-8 * torch.arange(1, q + 1, device="cuda") / q) if case["slopes"] else None
    if own:
        K = s["kvl"]
        layout = K.make_attn_layout(block_tokens=bs, q_heads=q, kv_heads=kv, head_dim=d, pool_blocks=blocks, dtype=dtype,
                                    cache_dtype=torch.float8_e4m3fn if case["cache"] == "8" else dtype, window=case["window"],
                                    sinks=case["sinks"])
        keys = {"all": K.KVL_TOKENS_ALL, "hit": 0, "append": K.KVL_TOKENS_APPEND}[case["keys"]]
        s["plan"] = K.kvl_attn_plan(layout, hit, new, tables, keys | K.KVL_GATHER, prefix=prefix if case["prefix_hi"] else None,
                                    documents=starts if case["document_hi"] else None)
        s["workspace"] = torch.empty(s["plan"].workspace_bytes, dtype=torch.uint8, device="cuda")
        return s
    # the same batch as index tensors
    dev = dict(device="cuda")
    padded = np.zeros((len(tables), max(1, int(need.max()))), dtype=np.int64)
    for r, t in enumerate(tables):
        padded[r, :t.size] = t
    most = int(new.max())
    lo, hi = np.zeros((2, len(new), most), dtype=np.int64)
    front = np.zeros(len(new), dtype=np.int64)
    for r in range(len(new)):
        lo[r, :new[r]], hi[r, :new[r]], front[r] = _bounds(case, int(hit[r]), int(new[r]), int(prefix[r]), starts[r])
    s["table"] = torch.from_numpy(padded).to(**dev)
    s["lo"], s["hi"], s["front"] = (torch.from_numpy(x).to(**dev) for x in (lo, hi, front))
    s["request"] = torch.from_numpy(np.repeat(np.arange(len(new)), new)).to(**dev)
    s["number"] = torch.from_numpy(np.arange(n) - np.repeat(np.cumsum(new) - new, new)).to(**dev)
    s["hit_t"], s["new_t"] = torch.from_numpy(hit).to(**dev), torch.from_numpy(new).to(**dev)
    return s


def _prepare_join(s, seed, gen):
    case = s["case"]
    n, h, d, dtype = case["tokens"], case["q_heads"], case["head_dim"], DTYPES[case["dtype"]]
    s["parts"], s["lses"] = [], []
    for _ in range(case["parts"]):
        lse = torch.randn(n, h, device="cuda", generator=gen) * 3
        lse[torch.rand(n, device="cuda", generator=gen) < 0.1] = -math.inf     # tokens that see no key of this part
        part = torch.randn(n, h, d, device="cuda", dtype=dtype, generator=gen)
        s["parts"].append(part.masked_fill_((lse == -math.inf)[..., None], 0))
        s["lses"].append(lse)
    s["out"] = torch.zeros(n, h, d, device="cuda", dtype=dtype)
    s["lse"] = torch.zeros(n, h, device="cuda") if case["lse"] else None
    if own:
        K = s["kvl"]
        layout = K.make_attn_layout(block_tokens=64, q_heads=h, kv_heads=h, head_dim=d, pool_blocks=n // 64 + 1, dtype=dtype)
        s["plan"] = K.kvl_attn_plan(layout, [0], [n], [np.arange(n // 64 + 1, dtype=np.int32)], K.KVL_GATHER)
    return s


def _prepare_pages(s, seed, gen):
    case = s["case"]
    tokens, tables, blocks = _sequences(case)
    sizes = _block_bytes(case)
    s.update(tokens=tokens, tables=tables, blocks=blocks)
    s["planes"] = [torch.randint(0, 256, (case["layers"], blocks, b), device="cuda", dtype=torch.uint8, generator=gen) for b in sizes]
    s["pools"] = [[plane[layer] for plane in s["planes"]] for layer in range(case["layers"])]
    if own:
        K = s["kvl"]
        s["page_pools"] = K.kvl_page_pools(sizes, blocks, s["pools"])
    if case["op"] == "fork":
        if own:
            s["pages"] = s["kvl"].kvl_pages(case["block_tokens"], blocks)
            s["sequences"] = s["kvl"].kvl_pages_adopt(s["pages"], tables, tokens)
        else:
            s["pages"] = _Pages(case["block_tokens"], blocks)
            s["sequences"] = [s["pages"].adopt(t, n) for t, n in zip(tables, tokens)]
    return s


# The plain form ---------------------------------------------------------------------------------------------------------------------

class _Pages:
    """Which blocks of a pool are whose: the lowest free block is taken first, a block goes when its last sequence does."""

    def __init__(self, block_tokens, blocks):
        self.bs, self.users, self.sequences, self.number = block_tokens, [0] * blocks, {}, 0
        self.free = list(range(blocks))

    def _put(self, table, tokens):
        self.number += 1
        self.sequences[self.number] = [table, tokens]
        return self.number

    def adopt(self, table, tokens):
        table = [int(b) for b in table]
        taken = set(table)
        for b in table:
            self.users[b] += 1
        self.free = [b for b in self.free if b not in taken]
        return self._put(table, int(tokens))

    def fork(self, sequence):
        table, tokens = self.sequences[sequence]
        for b in table:
            self.users[b] += 1
        return self._put(list(table), tokens)

    def _take(self):
        b = heapq.heappop(self.free)
        self.users[b] = 1
        return b

    def extend(self, sequence, n):
        table, tokens = s = self.sequences[sequence]
        copies = []
        if tokens % self.bs and self.users[table[-1]] > 1:
            self.users[table[-1]] -= 1
            copies.append((table[-1], self._take()))
            table[-1] = copies[0][1]
        while len(table) * self.bs < tokens + n:
            table.append(self._take())
        s[1] = tokens + n
        return copies

    def drop(self, sequence):
        for b in self.sequences.pop(sequence)[0]:
            self.users[b] -= 1
            if self.users[b] == 0:
                heapq.heappush(self.free, b)

    def compact(self):
        """The last block in use goes to the first free one, until there is none behind."""
        used = [b for b, n in enumerate(self.users) if n]
        copies = list(zip(reversed(used), sorted(b for b in self.free if b < len(used))))
        to = dict(copies)
        for s in self.sequences.values():
            s[0] = [to.get(b, b) for b in s[0]]
        for a, b in copies:
            self.users[a], self.users[b] = 0, self.users[a]
        self.free = list(range(len(used), len(self.users)))
        return copies


def _plain_copy(s, copies):
    if copies:
        pairs = torch.tensor(copies, device="cuda")
        for layer in s["pools"]:
            for plane in layer:
                plane[pairs[:, 1]] = plane[pairs[:, 0]]


def _plain_fork(s):
    pages, case = s["pages"], s["case"]
    forks = [pages.fork(x) for x in s["sequences"] for _ in range(case["forks"])]
    copies = [c for f in forks for c in pages.extend(f, case["grow"])]
    _plain_copy(s, copies)
    tables = np.concatenate([np.array(pages.sequences[f][0], dtype=np.int32) for f in forks])
    for f in forks:
        pages.drop(f)
    return [tables, *s["planes"]]


def _plain_compact(s):
    pages = _Pages(s["case"]["block_tokens"], s["blocks"])
    sequences = [pages.adopt(t, n) for t, n in zip(s["tables"], s["tokens"])]
    _plain_copy(s, pages.compact())
    tables = np.concatenate([np.array(pages.sequences[x][0], dtype=np.int32) for x in sequences])
    return [tables, *s["planes"]]


def _plain_join(s):
    lses = torch.stack(s["lses"])
    most = lses.amax(0)
    weights = (lses - most.masked_fill(most == -math.inf, 0)).exp_()
    total = weights.sum(0)
    out = sum(w[..., None] * x.float() for w, x in zip(weights, s["parts"])) / total.masked_fill(total == 0, 1)[..., None]
    s["out"].copy_(out)
    if s["lse"] is None:
        return [s["out"]]
    s["lse"].copy_(total.log() + most)
    return [s["out"], s["lse"]]


def _plain_attend(s):
    case = s["case"]
    bs, q_heads, kv, d = case["block_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    group = q_heads // kv
    first, last = _key_range(case, s["hit_t"], s["new_t"])
    n_new, n_keys = int(s["new"].max()), max(1, int((s["hit"] + s["new"]).max()))
    t = torch.arange(n_keys, device="cuda")
    scales = s["planes"][2:] or (None, None)
    queries = torch.zeros(len(s["hit"]), n_new, q_heads, d, device="cuda")
    queries[s["request"], s["number"]] = s["q"].float()
    outs, lses = [], []
    # as many requests at once as leave their scores some room
    some = max(1, (1 << 32) // (n_new * n_keys * q_heads))
    for a in range(0, len(s["hit"]), some):
        at = slice(a, a + some)
        block = s["table"][at][:, t // bs]
        row = block * bs + t % bs
        held = (t >= first[at, None]) & (t < last[at, None])
        requests = row.shape[0]

        def keys(plane, scales):
            x = plane.view(-1, kv, d)[row]
            x = x.float() if scales is None else x.view(torch.float8_e4m3fn).float() * scales[block][..., None]
            return x.masked_fill_(~held[..., None, None], 0).permute(0, 2, 1, 3).contiguous()

        q = queries[at].view(requests, n_new, kv, group, d).permute(0, 2, 1, 3, 4).reshape(requests, kv, n_new * group, d)
        score = torch.matmul(q, keys(s["planes"][0], scales[0]).transpose(-1, -2).contiguous()).mul_(s["scale"])
        by_head = score.view(requests, kv, n_new, group, n_keys)
        if case["cap"]:
            score.div_(case["cap"]).tanh_().mul_(case["cap"])
        p = s["hit_t"][at, None] + torch.arange(n_new, device="cuda")
        if s["slopes"] is not None:
            far = (p[..., None] - t).abs_().float()
            by_head.addcmul_(far[:, None, :, None], s["slopes"].view(1, kv, 1, group, 1), value=-1)
        see = held[:, None] & (t < s["hi"][at, :, None]) & ((t >= s["lo"][at, :, None]) | (t < s["front"][at, None, None]))
        by_head.masked_fill_(~see[:, None, :, None], -math.inf)
        most = score.amax(-1, keepdim=True)
        score.sub_(most.masked_fill(most == -math.inf, 0)).exp_()
        total = score.sum(-1, keepdim=True)
        out = torch.matmul(score, keys(s["planes"][1], scales[1])) / total.masked_fill(total == 0, 1)
        lses.append((total.log() + most).view(requests, kv, n_new, group).permute(0, 2, 1, 3).reshape(requests, n_new, q_heads))
        outs.append(out.view(requests, kv, n_new, group, d).permute(0, 2, 1, 3, 4).reshape(requests, n_new, q_heads, d))
    s["out"].copy_(torch.cat(outs)[s["request"], s["number"]])
    if s["lse"] is None:
        return [s["out"]]
    s["lse"].copy_(torch.cat(lses)[s["request"], s["number"]])
    return [s["out"], s["lse"]]


# The framework's form ---------------------------------------------------------------------------------------------------------------

def _own_attend(s):
    case = s["case"]
    s["kvl"].kvl_attn_layer(s["plan"], s["q"], s["planes"], s["out"], s["workspace"], scale=s["scale"], lse=s["lse"],
                            cap=case["cap"] or None, slopes=s["slopes"])
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


def _own_join(s):
    s["kvl"].kvl_attn_join(s["plan"], s["parts"], s["lses"], s["out"], lse=s["lse"])
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


def _own_fork(s):
    K, pages, case = s["kvl"], s["pages"], s["case"]
    forks = K.kvl_pages_fork(pages, np.repeat(s["sequences"], case["forks"]))
    K.kvl_copy_blocks(s["page_pools"], K.kvl_pages_extend(pages, forks, case["grow"]))
    tables = np.concatenate(K.kvl_pages_tables(pages, forks))
    K.kvl_pages_free(pages, forks)
    return [tables, *s["planes"]]


def _own_compact(s):
    K = s["kvl"]
    pages = K.kvl_pages(s["case"]["block_tokens"], s["blocks"])
    sequences = K.kvl_pages_adopt(pages, s["tables"], s["tokens"])
    K.kvl_copy_blocks(s["page_pools"], K.kvl_pages_compact(pages))
    tables = np.concatenate(K.kvl_pages_tables(pages, sequences))
    return [tables, *s["planes"]]


def run(s):
    form = {"attend": (_plain_attend, _own_attend), "join": (_plain_join, _own_join), "fork": (_plain_fork, _own_fork),
            "compact": (_plain_compact, _own_compact)}[s["case"]["op"]]
    return form[1 if own else 0](s)


# The definition, in 64 bits ---------------------------------------------------------------------------------------------------------

def _exact_attend(s):
    case = s["case"]
    bs, q_heads, kv, d = case["block_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    group, eight = q_heads // kv, case["cache"] == "8"
    out = torch.zeros(s["tokens"], q_heads, d, dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], q_heads), -math.inf, dtype=torch.float64, device="cuda")
    begin, end = _key_range(case, s["hit"], s["new"])
    done = 0
    for r, (h, n) in enumerate(zip(s["hit"].tolist(), s["new"].tolist())):
        t = np.arange(int(begin[r]), int(end[r]))
        document = lambda x: torch.from_numpy(np.searchsorted(s["starts"][r], x, side="right")).cuda()
        if t.size:
            block = torch.from_numpy(s["tables"][r][t // bs].astype(np.int64)).cuda()
            of_key, t = document(t), torch.from_numpy(t).cuda()
            both = []
            for x in range(2):
                rows = s["planes"][x][block, t % bs]
                both.append(rows.view(torch.float8_e4m3fn).double() * s["planes"][2 + x][block].double()[..., None] if eight else rows.double())
            k, v = (x.transpose(0, 1).contiguous() for x in both)
            some = max(1, (1 << 27) // (q_heads * t.shape[0]))
            for a in range(0, n, some):
                b = min(n, a + some)
                p = torch.arange(h + a, h + b, device="cuda")[:, None]
                near = of_key == document(np.arange(h + a, h + b))[:, None]
                if case["window"]:
                    near &= t > p - case["window"]
                see = (t < int(s["prefix"][r])) | ((t <= p) & (near | (t < case["sinks"])))
                q = s["q"][done + a:done + b].double().view(b - a, kv, group, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
                score = (q @ k.transpose(1, 2).contiguous() * s["scale"]).view(kv, group, b - a, -1)
                if case["cap"]:
                    score = case["cap"] * torch.tanh(score / case["cap"])
                if s["slopes"] is not None:
                    score = score - s["slopes"].double().view(kv, group, 1, 1) * (p - t).abs().double()
                score = torch.where(see, score, -math.inf)
                l = torch.logsumexp(score, dim=-1)
                weight = torch.where(see, torch.exp(score - l[..., None].nan_to_num(neginf=0.0)), 0.0)
                o = weight.view(kv, -1, t.shape[0]) @ v
                out[done + a:done + b] = o.view(kv, group, b - a, d).permute(2, 0, 1, 3).reshape(b - a, q_heads, d)
                lse[done + a:done + b] = l.permute(2, 0, 1).reshape(b - a, q_heads)
        done += n
    return [out, lse] if case["lse"] else [out]


def _exact_join(s):
    lses = torch.stack([x.double() for x in s["lses"]], dim=-1)
    lse = torch.logsumexp(lses, dim=-1)
    out = torch.zeros_like(s["parts"][0], dtype=torch.float64)
    for i, x in enumerate(s["parts"]):
        share = torch.exp(lses[..., i] - lse).nan_to_num(nan=0.0)
        out += share[..., None] * x.double()
    return [out, lse] if s["case"]["lse"] else [out]


def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None                 # (blocks and tables are whole numbers)
    s = prepare(case, seed)
    return _exact_attend(s) if case["op"] == "attend" else _exact_join(s)
