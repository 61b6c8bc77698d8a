"""What the speed of the attention operators over a paged cache is measured on.

Three operators, on one layer of a batch of requests (a cached prefix of `hit` tokens and `new` appended ones each):

  append   the new tokens' keys are rotated by their positions and written with their values into the paged cache, in 16 bits
           or in 8 bits with a scale for each block and head; their queries are rotated on the way
  attend   attention of the new tokens over the paged cache
             - held in 8 bits with a scale for each block of tokens and head
             - with a sliding window and a few first tokens that stay visible

Sizes are given by the case alone; block tables and contents come from the seed.  `own` says which form `run` takes: elementary
torch operations, or the framework's kernels.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, requests, hit, new, bs=64, heads=(32, 8), dim=128, dtype="bf16", cache="16", window=0, sinks=0,
          rope_dim=0, pairs="halves", keys="all", lse=False):
    return {"name": name, "op": op, "requests": requests, "hit_lo": hit[0], "hit_hi": hit[1], "new_lo": new[0], "new_hi": new[1],
            "block_tokens": bs, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim, "dtype": dtype, "cache": cache,
            "window": window, "sinks": sinks, "rope_dim": rope_dim, "pairs": pairs, "keys": keys, "lse": lse}


def listed():
    return [
        # a decode step of four short chats, 16-token blocks: launches are all there is
        _case("append_step_small", "append", 4, (1000, 1000), (1, 1), bs=16, rope_dim=128),
        # a decode step of a full batch into an 8-bit cache: the scale of the block that each token joins may grow
        _case("append_step_8bit", "append", 256, (256, 4096), (1, 1), cache="8", rope_dim=128),
        # prompts' tails of odd lengths, rotation of neighbouring elements over half of each head
        _case("append_prefill_f16", "append", 16, (100, 3000), (129, 1025), bs=24, heads=(16, 4), dtype="f16", rope_dim=64,
              pairs="neighbours"),
        # the appended tails of 64 agents' turns into an 8-bit cache
        _case("append_prefill_8bit", "append", 64, (500, 4000), (256, 1024), cache="8", rope_dim=128),
        # a decode step of four short chats under a window
        _case("window_step_small", "attend", 4, (1000, 1000), (1, 1), bs=16, window=512, sinks=4),
        # a decode step of a full batch: long chats, of which the window and the first tokens are left
        _case("window_step", "attend", 128, (2000, 12000), (1, 1), heads=(64, 8), window=4096, sinks=4, lse=True),
        # appended tails under a window, heads of 64, pages that end inside a tile, prefixes shorter than the window among them
        _case("window_prefill", "attend", 8, (300, 6000), (400, 2000), bs=24, heads=(24, 8), dim=64, dtype="f16", window=1024, sinks=4),
        # one long document, one token at a time: the keys have to be shared out
        _case("fp8_step_one", "attend", 1, (131000, 131000), (1, 1), cache="8"),
        # the largest in bytes: a decode step of 64 requests of 16-64 K tokens
        _case("fp8_step_batch", "attend", 64, (16384, 65536), (1, 1), heads=(64, 8), cache="8"),
        # a draft's tokens checked: a few queries a request, a group of seven heads, 16-token blocks
        _case("fp8_verify", "attend", 32, (700, 9000), (3, 6), bs=16, heads=(28, 4), cache="8", lse=True),
        # the largest in operations: appended tails over long cached prefixes
        _case("fp8_prefill", "attend", 4, (8192, 32768), (256, 1024), cache="8"),
        # the cached prefix alone, while the tail's own keys are still to come: some requests have none, and the window leaves rows empty
        _case("fp8_prefix_only", "attend", 24, (0, 1500), (1, 700), heads=(16, 2), dim=64, cache="8", window=512, sinks=0, keys="hit", lse=True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of these ranges: one to many requests, one to a thousand or so new tokens each, any block size and group of heads."""
    op = rng.choice(["append", "attend", "attend"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8])
    q = kv * rng.choice([1, 2, 3, 4, 5, 7, 8])
    cache = rng.choice(["16", "8"])
    bs = rng.choice([1, 8, 16, 24, 32, 64, 64, 100, 128])
    if cache == "8":
        bs = max(bs, 8)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    form = rng.choice(["step", "few", "prefill"])
    requests = _spread(rng, 1, {"step": 192, "few": 64, "prefill": 16}[form])
    new = {"step": (1, 1), "few": (1, rng.randint(2, 9)), "prefill": (rng.randint(1, 200), _spread(rng, 200, 1024))}[form]
    if op == "append":
        most = min(8000, 400_000 // requests)
        hi = _spread(rng, 40, most)
        c = _case("", op, requests, (rng.randint(0, hi // 2), hi), new, bs, (q, kv), dim, dtype, cache,
                  rope_dim=rng.choice([dim, dim, dim // 2, 0]), pairs=rng.choice(["halves", "neighbours"]))
    else:
        most = min(131072, {"step": 3_000_000, "few": 600_000, "prefill": 60_000}[form] // requests)
        hi = _spread(rng, 60, most)
        window = 0 if cache == "8" and rng.random() < 0.6 else _spread(rng, 16, 8192)
        c = _case("", op, requests, (rng.randint(0, hi // 2), hi), new, bs, (q, kv), dim, dtype, cache, window=window,
                  sinks=rng.choice([0, 1, 4, 16, 70]) if window else 0, keys=rng.choice(["all", "all", "all", "hit", "append"]),
                  lse=rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(case):
    """(hit, new) of every request, int64: drawn from the case's ranges, the same for every seed."""
    rng = np.random.Generator(np.random.PCG64([20260221, case["requests"], case["hit_hi"], case["new_hi"]]))
    n = case["requests"]
    return rng.integers(case["hit_lo"], case["hit_hi"] + 1, size=n), rng.integers(case["new_lo"], case["new_hi"] + 1, size=n)


def _key_range(case, hit, new):
    """[first, last) of the keys that the case's plan holds, for each request."""
    return {"all": (0 * hit, hit + new), "hit": (0 * hit, hit), "append": (hit, hit + new)}[case["keys"]]


def _visible(case):
    """(rows of keys that some query sees, visible pairs of query and key), over all requests."""
    hit, new = _lengths(case)
    first, last = _key_range(case, hit, new)
    w, sinks = case["window"] or 1 << 60, case["sinks"]
    rows = pairs = 0
    for h, n, a, b in zip(hit.tolist(), new.tolist(), first.tolist(), last.tolist()):
        p = np.arange(h, h + n, dtype=np.int64)
        end = np.minimum(p + 1, b)
        lo = np.maximum(p + 1 - w, a)
        near = np.maximum(end - lo, 0)
        far = np.maximum(np.minimum(np.minimum(sinks, lo), end) - a, 0)
        pairs += int((near + far).sum())
        lo0, end0 = max(h + 1 - w, a), min(h + n, b)
        rows += max(end0 - lo0, 0) + max(min(sinks, lo0, end0) - a, 0)
    return rows, pairs


def work(case):
    """Inputs once, outputs once; of the cache the rows that are written or that some query sees."""
    hit, new = _lengths(case)
    n, d, q, kv = int(new.sum()), case["head_dim"], case["q_heads"], case["kv_heads"]
    e = 1 if case["cache"] == "8" else 2
    if case["op"] == "append":
        bs = case["block_tokens"]
        touched = int(((hit + new + bs - 1) // bs - hit // bs).sum())
        return {"bytes": n * (2 * (2 * q + 2 * kv) * d + 2 * kv * d * e + 4 * case["rope_dim"]) + (16 * touched * kv if e == 1 else 0),
                "flops": 3 * n * (q + kv) * case["rope_dim"]}
    rows, pairs = _visible(case)
    scales = 8 * kv * rows / case["block_tokens"] if e == 1 else 0
    return {"bytes": 4 * n * q * d + 2 * rows * kv * d * e + int(scales) + (4 * n * q if case["lse"] else 0), "flops": 4 * d * q * pairs}


# What a program has in hand ---------------------------------------------------------------------------------------------------------

def _least_exponent(most):
    """The least e in [-32, 63] with most <= 448 * 2**e (doubles in, doubles out)."""
    m, e = torch.frexp(most / 448.0)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(most > 0, e, -32).clamp(-32, 63).double()


def _quantised_pool(blocks, bs, kv, d, gen):
    """A plane of e4m3 codes and its scales, of normal values whose spread differs by block and head."""
    codes = torch.empty(blocks, bs, kv, d, dtype=torch.uint8, device="cuda")
    scales = torch.empty(blocks, kv, dtype=torch.float32, device="cuda")
    some = max(1, (1 << 26) // (bs * kv * d))
    for at in range(0, blocks, some):
        n = min(some, blocks - at)
        x = torch.randn(n, bs, kv, d, device="cuda", generator=gen)
        x *= torch.randn(n, 1, kv, 1, device="cuda", generator=gen).mul_(0.3).exp_()
        s = torch.exp2(_least_exponent(x.abs().amax(dim=(1, 3)).double())).float()
        scales[at:at + n] = s
        codes[at:at + n] = (x / s[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scales


def _rope_table(positions, rope_dim):
    """(cos, sin) of position * 10000 ** (-2 j / rope_dim), angles in 64 bits."""
    j = torch.arange(rope_dim // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * torch.exp(-2 * j / rope_dim * math.log(10000.0))
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hit, new = _lengths(case)
    bs, d, q, kv = case["block_tokens"], case["head_dim"], case["q_heads"], case["kv_heads"]
    dtype = DTYPES[case["dtype"]]
    need = (hit + new + bs - 1) // bs
    blocks = int(math.ceil(1.05 * int(need.sum()))) + 1
    order = np.random.Generator(np.random.PCG64([seed, 7])).permutation(blocks).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    tables = [order[a:b].copy() for a, b in zip(at[:-1], at[1:])]
    n = int(new.sum())
    s = {"case": case, "hit": hit, "new": new, "tables": tables, "blocks": blocks, "tokens": n}
    if case["cache"] == "8":
        (k, ks), (v, vs) = (_quantised_pool(blocks, bs, kv, d, gen) for _ in range(2))
        s["planes"] = [k, v, ks, vs]
    else:
        s["planes"] = [torch.randn(blocks, bs, kv, d, device="cuda", dtype=dtype, generator=gen) for _ in range(2)]
    if case["op"] == "append":
        # queries, keys and values as a model has them: parts of one projection's output
        qkv = torch.randn(n, q + 2 * kv, d, device="cuda", dtype=dtype, generator=gen)
        s["q"], s["k"], s["v"] = qkv[:, :q], qkv[:, q:q + kv], qkv[:, q + kv:]
        s["rope"] = _rope_table(int((hit + new).max()) + 1, case["rope_dim"]) if case["rope_dim"] else None
        s["q_out"] = torch.zeros(n, q, d, device="cuda", dtype=dtype)
    else:
        s["q"] = torch.randn(n, q, d, device="cuda", dtype=dtype, generator=gen)
        s["out"] = torch.zeros(n, q, d, device="cuda", dtype=dtype)
        s["lse"] = torch.zeros(n, q, device="cuda") if case["lse"] else None
        s["scale"] = 1 / math.sqrt(d)
    if own:
        import paper_2602_21548_amd as K
        layout = K.make_attn_layout(block_tokens=bs, q_heads=q, kv_heads=kv, head_dim=d, pool_blocks=blocks, dtype=dtype,
                                    cache_dtype=torch.float8_e4m3fn if case["cache"] == "8" else dtype, window=case["window"],
                                    sinks=case["sinks"], rope_dim=case["rope_dim"],
                                    rope_pairs=K.KVL_ROPE_HALVES if case["pairs"] == "halves" else K.KVL_ROPE_NEIGHBOURS)
        keys = {"all": K.KVL_TOKENS_ALL, "hit": 0, "append": K.KVL_TOKENS_APPEND}[case["keys"]]
        s["plan"] = K.kvl_attn_plan(layout, hit, new, tables, keys | (K.KVL_SCATTER if case["op"] == "append" else K.KVL_GATHER))
        s["workspace"] = torch.empty(s["plan"].workspace_bytes, dtype=torch.uint8, device="cuda") if case["op"] == "attend" else None
        s["kvl"] = K
        return s
    # the same batch as index tensors
    dev = dict(device="cuda")
    padded = np.zeros((len(tables), max(1, int(need.max()))), dtype=np.int64)
    for r, t in enumerate(tables):
        padded[r, :t.size] = t
    request = np.repeat(np.arange(len(new)), new)
    number = np.arange(n) - np.repeat(np.cumsum(new) - new, new)
    s["table"] = torch.from_numpy(padded).to(**dev)
    s["request"], s["number"] = torch.from_numpy(request).to(**dev), torch.from_numpy(number).to(**dev)
    s["hit_t"], s["new_t"] = torch.from_numpy(hit).to(**dev), torch.from_numpy(new).to(**dev)
    s["position"] = s["hit_t"][s["request"]] + s["number"]
    if case["op"] == "append":
        # blocks that get rows, and which of them hold cached rows already
        first = hit // bs
        count = need - first
        base = np.cumsum(count) - count
        s["touched"] = torch.from_numpy(np.concatenate([t[f:] for t, f in zip(tables, first)]).astype(np.int64)).to(**dev)
        s["slot"] = torch.from_numpy(base[request] + (hit[request] + number) // bs - first[request]).to(**dev)
        s["held"] = torch.zeros(int(count.sum()), dtype=torch.int64, device="cuda")
        s["held"][torch.from_numpy(base).to(**dev)] = torch.from_numpy(hit % bs).to(**dev)
    return s


# The plain form ---------------------------------------------------------------------------------------------------------------------

def _rotate(x, rope, position, pairs, wide):
    """x [tokens, heads, dim] rotated, in 32 bits or, for what is rounded to 8 afterwards, in 64."""
    x = x.to(wide)
    if rope is None:
        return x
    half = rope.shape[1]
    c, s = rope[position].to(wide)[:, None].unbind(-1)
    r = x[..., :2 * half]
    a, b = (r[..., :half], r[..., half:]) if pairs == "halves" else (r[..., 0::2], r[..., 1::2])
    turned = [a * c - b * s, b * c + a * s]
    turned = torch.cat(turned, dim=-1) if pairs == "halves" else torch.stack(turned, dim=-1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], dim=-1)


def _e4m3(x):
    """Doubles rounded to the nearest value of e4m3, ties to the even one."""
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)
    return ((x / step).round() * step).clamp(-448, 448).float().to(torch.float8_e4m3fn)


def _plain_append(s):
    case = s["case"]
    bs, kv, d = case["block_tokens"], case["kv_heads"], case["head_dim"]
    dtype = DTYPES[case["dtype"]]
    s["q_out"].copy_(_rotate(s["q"], s["rope"], s["position"], case["pairs"], torch.float32))
    block = s["table"][s["request"], s["position"] // bs]
    row = block * bs + s["position"] % bs
    if case["cache"] == "16":
        k, v = s["planes"]
        k.view(-1, kv, d)[row] = _rotate(s["k"], s["rope"], s["position"], case["pairs"], torch.float32).to(dtype)
        v.view(-1, kv, d)[row] = s["v"]
        return [s["q_out"], k, v]
    held = s["held"] > 0
    rows_held = torch.arange(bs, device="cuda") < s["held"][held][:, None]
    blocks_held = s["touched"][held]

    def put(codes, scales, x):
        most = torch.zeros(held.shape[0], kv, dtype=torch.float64, device="cuda")
        most.index_reduce_(0, s["slot"], x.abs().amax(-1), "amax")
        fresh = torch.exp2(_least_exponent(most))
        old = scales[s["touched"]].double()
        to = torch.where(held[:, None], torch.maximum(old, fresh), fresh)
        was = codes[blocks_held].view(torch.float8_e4m3fn).double()
        again = _e4m3(was * (old[held] / to[held])[:, None, :, None]).view(torch.uint8)
        codes[blocks_held] = torch.where(rows_held[..., None, None], again, codes[blocks_held])
        codes.view(-1, kv, d)[row] = _e4m3(x / to[s["slot"]][..., None]).view(torch.uint8)
        scales[s["touched"]] = to.float()

    k, v, ks, vs = s["planes"]
    put(k, ks, _rotate(s["k"], s["rope"], s["position"], case["pairs"], torch.float64))
    put(v, vs, s["v"].double())
    return [s["q_out"], k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ks, vs]


def _plain_attend(s):
    case = s["case"]
    bs, q_heads, kv, d = case["block_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    group = q_heads // kv
    first, last = _key_range(case, s["hit_t"], s["new_t"])
    requests = s["hit_t"].shape[0]
    n_new, n_keys = int(s["new"].max()), max(1, int((s["hit"] + s["new"]).max()))
    t = torch.arange(n_keys, device="cuda")
    block = s["table"][:, t // bs]
    row = block * bs + t % bs
    held = (t >= first[:, None]) & (t < last[:, None])

    def keys(plane, scales):
        x = plane.view(-1, kv, d)[row]
        x = x.float() if scales is None else x.view(torch.float8_e4m3fn).float() * scales[block][..., None]
        return x.masked_fill_(~held[..., None, None], 0).permute(0, 2, 1, 3).contiguous()

    scales = s["planes"][2:] or (None, None)
    q = torch.zeros(requests, n_new, q_heads, d, device="cuda")
    q[s["request"], s["number"]] = s["q"].float()
    q = q.view(requests, n_new, kv, group, d).permute(0, 2, 1, 3, 4).reshape(requests, kv, n_new * group, d)
    score = torch.matmul(q, keys(s["planes"][0], scales[0]).transpose(-1, -2)).mul_(s["scale"])
    p = s["hit_t"][:, None] + torch.arange(n_new, device="cuda")
    see = held[:, None] & (t <= p[..., None])
    if case["window"]:
        see &= (p[..., None] - t < case["window"]) | (t < case["sinks"])
    score.view(requests, kv, n_new, group, n_keys).masked_fill_(~see[:, None, :, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    score.sub_(most.masked_fill(most == -math.inf, 0)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, keys(s["planes"][1], scales[1])) / total.masked_fill(total == 0, 1)
    lse = (total.log() + most).view(requests, kv, n_new, group).permute(0, 2, 1, 3).reshape(requests, n_new, q_heads)
    out = out.view(requests, kv, n_new, group, d).permute(0, 2, 1, 3, 4).reshape(requests, n_new, q_heads, d)
    s["out"].copy_(out[s["request"], s["number"]])
    if s["lse"] is None:
        return [s["out"]]
    s["lse"].copy_(lse[s["request"], s["number"]])
    return [s["out"], s["lse"]]


def run(s):
    op = s["case"]["op"]
    if not own:
        return _plain_append(s) if op == "append" else _plain_attend(s)
    if op == "attend":
        s["kvl"].kvl_attn_layer(s["plan"], s["q"], s["planes"], s["out"], s["workspace"], scale=s["scale"], lse=s["lse"])
        return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]
    s["kvl"].kvl_append_layer(s["plan"], s["k"], s["v"], s["planes"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
    k, v, *scales = s["planes"]
    return [s["q_out"], k, v] if not scales else [s["q_out"], k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), *scales]


# The definition, in 64 bits ---------------------------------------------------------------------------------------------------------

def _exact_turned(x, rope, position, pairs):
    """Each pair as a complex number, times that of its angle."""
    x = x.double()
    if rope is None:
        return x
    n = rope.shape[1]
    unit = torch.view_as_complex(rope.double())[position][:, None]
    i = torch.arange(n, device="cuda")
    a, b = (i, i + n) if pairs == "halves" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., a], x[..., b]) * unit
    y = x.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_codes():
    """Every value of e4m3 from 0 to 448, in order (so that a value's place is its code, and even codes are even values)."""
    return torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device="cuda")


def _exact_nearest(x, values):
    size = x.abs().clamp(max=448)
    up = torch.searchsorted(values, size).clamp(max=126)
    down = (up - 1).clamp(min=0)
    over, under = values[up] - size, size - values[down]
    near = torch.where((over < under) | ((over == under) & (up % 2 == 0)), values[up], values[down])
    return torch.where(x < 0, -near, near)


def _exact_append(s):
    case = s["case"]
    bs, eight = case["block_tokens"], case["cache"] == "8"
    position = torch.from_numpy(np.concatenate([np.arange(h, h + n) for h, n in zip(s["hit"], s["new"])])).cuda()
    q = _exact_turned(s["q"], s["rope"], position, case["pairs"])
    rows = [_exact_turned(s["k"], s["rope"], position, case["pairs"]), s["v"].double()]
    planes = [(p.view(torch.float8_e4m3fn) if eight else p).double() for p in s["planes"][:2]]
    scales = [p.double() for p in s["planes"][2:]]
    values = _exact_codes()
    done = 0
    for h, n, table in zip(s["hit"].tolist(), s["new"].tolist(), s["tables"]):
        for j in range(h // bs, (h + n + bs - 1) // bs):
            lo, hi = max(h, j * bs), min(h + n, (j + 1) * bs)
            b, at, span = int(table[j]), lo - j * bs, hi - lo
            for x in range(2):
                new = rows[x][done + lo - h:done + hi - h]
                if eight:
                    most = new.abs().amax(dim=(0, 2))
                    need = torch.pow(2.0, torch.ceil(torch.log2((most / 448).clamp(min=2.0 ** -32))))
                    need = torch.where(need / 2 * 448 >= most, need / 2, need).clamp(2.0 ** -32, 2.0 ** 63)
                    if at > 0:
                        old = scales[x][b]
                        need = torch.maximum(need, old)
                        planes[x][b, :at] = _exact_nearest(planes[x][b, :at] * (old / need)[:, None], values)
                    scales[x][b] = need
                    new = _exact_nearest(new / need[:, None], values)
                planes[x][b, at:at + span] = new
        done += n
    return [q, *planes, *scales]


def _exact_attend(s):
    case = s["case"]
    bs, q_heads, kv, d = case["block_tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    group, eight = q_heads // kv, case["cache"] == "8"
    out = torch.zeros(s["tokens"], q_heads, d, dtype=torch.float64, device="cuda")
    lse = torch.full((s["tokens"], q_heads), -math.inf, dtype=torch.float64, device="cuda")
    first, last = _key_range(case, s["hit"], s["new"])
    done = 0
    for r, (h, n) in enumerate(zip(s["hit"].tolist(), s["new"].tolist())):
        lo, hi = int(first[r]), int(last[r])
        near = max(lo, h + 1 - case["window"]) if case["window"] else lo
        t = np.unique(np.concatenate([np.arange(lo, min(hi, max(lo, case["sinks"]))), np.arange(near, hi)])).astype(np.int64)
        if t.size:
            block = torch.from_numpy(s["tables"][r][t // bs].astype(np.int64)).cuda()
            t = torch.from_numpy(t).cuda()
            both = []
            for x in range(2):
                rows = s["planes"][x][block, t % bs]
                both.append(rows.view(torch.float8_e4m3fn).double() * s["planes"][2 + x][block].double()[..., None] if eight else rows.double())
            k, v = (x.transpose(0, 1).contiguous() for x in both)
            some = max(1, (1 << 27) // (q_heads * t.shape[0]))
            for a in range(0, n, some):
                b = min(n, a + some)
                p = torch.arange(h + a, h + b, device="cuda")[:, None]
                unseen = t > p
                if case["window"]:
                    unseen |= (t <= p - case["window"]) & (t >= case["sinks"])
                q = s["q"][done + a:done + b].double().view(b - a, kv, group, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
                score = (q @ k.transpose(1, 2).contiguous() * s["scale"]).view(kv, group, b - a, -1)
                score = torch.where(unseen, -math.inf, score)
                l = torch.logsumexp(score, dim=-1)
                weight = torch.where(unseen, 0.0, torch.exp(score - l[..., None].nan_to_num(neginf=0.0)))
                o = weight.view(kv, -1, t.shape[0]) @ v
                out[done + a:done + b] = o.view(kv, group, b - a, d).permute(2, 0, 1, 3).reshape(b - a, q_heads, d)
                lse[done + a:done + b] = l.permute(2, 0, 1).reshape(b - a, q_heads)
        done += n
    return [out, lse] if case["lse"] else [out]


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)
