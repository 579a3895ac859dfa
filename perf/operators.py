"""The cache operators of token generation, as cases that can be timed and compared.

A serving program that drafts tokens keeps, per sequence, a cache of keys and values and goes round one loop: attention of
the drafted tree over the cache (`attn`), the accepted path's keys and values appended (`append`), the attention weight that
every cached row received added up (`weights`), and the rows of least weight evicted when the cache is over its budget:
in place after every step (`step`: append and evict), or once into a smaller cache behind the prompt (`prompt`).

Sizes are those of the attention shard this repository measures (12 heads of 128, 2048 tokens) and generic ones with
shared key and value heads.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _attn(name, B, T, Hq, Hk, D, least, most, dtype="bf16", shape="tree", ragged=False):
    """Attention of T drafted tokens per sequence over caches of `least` to `most` rows."""
    return dict(name=name, kind="attn", B=B, T=T, Hq=Hq, Hk=Hk, D=D, least=least, most=most, dtype=dtype, shape=shape, ragged=ragged)


def _weights(name, B, T, A, Hq, Hk, D, least, most, dtype="bf16"):
    """Up to A accepted of T drafted tokens; A = T: a prompt, accepted whole."""
    return dict(name=name, kind="weights", B=B, T=T, A=A, Hq=Hq, Hk=Hk, D=D, least=least, most=most, dtype=dtype)


def _append(name, B, T, A, Hk, D, least, most, dtype="bf16"):
    return dict(name=name, kind="append", B=B, T=T, A=A, Hk=Hk, D=D, least=least, most=most, dtype=dtype)


def _step(name, B, A, Hk, D, budget, recent, dtype="bf16"):
    return dict(name=name, kind="step", B=B, A=A, Hk=Hk, D=D, budget=budget, recent=recent, dtype=dtype)


def _prompt(name, B, Hk, D, least, most, budget, recent, dtype="bf16"):
    return dict(name=name, kind="prompt", B=B, Hk=Hk, D=D, least=least, most=most, budget=budget, recent=recent, dtype=dtype)


def listed():
    return [
        # one new token of one short conversation: latency
        _attn("attn_token_1x500", 1, 1, 12, 12, 128, 500, 500),
        # one new token for each of four sequences, the attention shard's own sizes, in fp16
        _attn("attn_token_4x2048_fp16", 4, 1, 12, 12, 128, 1500, 2048, dtype="fp16"),
        # a large serving batch, one token each, long caches of uneven length, shared key heads: HBM bandwidth
        _attn("attn_token_32x8192", 32, 1, 64, 8, 128, 2000, 8192),
        # a tree of 63 drafted tokens for each of eight requests; some drafted fewer
        _attn("attn_tree_8x63", 8, 63, 32, 8, 128, 500, 4096, ragged=True),
        # a small tree over one very long document, fp16, heads of 64
        _attn("attn_tree_long_fp16", 1, 13, 32, 8, 64, 120001, 120001, dtype="fp16"),
        # a wide tree search over long caches: the matrix cores' work
        _attn("attn_tree_4x256", 4, 256, 64, 8, 128, 9000, 16384),
        # weights after a step: one to five accepted of a tree of 16
        _weights("weights_step_16x4096", 16, 16, 5, 32, 8, 128, 2500, 4096),
        # weights of a whole prompt of the attention shard, every token against all before it
        _weights("weights_prompt_2048", 1, 2048, 2048, 12, 12, 128, 2048, 2048),
        # one to six accepted of a tree of 32, for 32 requests
        _append("append_tree_32x32", 32, 32, 6, 8, 128, 1000, 4000),
        # a chunk of a prompt, accepted whole, fp16
        _append("append_prompt_4x1024_fp16", 4, 1024, 1024, 8, 128, 0, 3000, dtype="fp16"),
        # steady generation at a budget of 2048 rows: append what was accepted, evict as many
        _step("evict_step_32x2048", 32, 5, 8, 128, 2048, 256),
        # behind long prompts: 2000 of up to 16384 rows go into the cache that generation uses
        _prompt("evict_prompt_4x16384", 4, 8, 128, 11000, 16384, 2000, 250),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["attn", "attn", "attn", "weights", "weights", "append", "step", "prompt"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    D = rng.choice([128, 128, 64])
    Hk = rng.choice([1, 2, 4, 8, 8, 12, 16])
    Hq = Hk * rng.choice([1, 1, 2, 4, 5, 8])
    B = _log(rng, 1, 48)
    if kind == "attn":
        most = _log(rng, 16, 100000)
        least = rng.choice([most, rng.randint(0, most)])
        return _attn("", B, rng.choice([1, _log(rng, 1, 256)]), Hq, Hk, D, least, most, dtype, rng.choice(["tree", "tree", "chain"]), rng.random() < 0.5)
    if kind == "weights":
        T = rng.choice([_log(rng, 1, 64), _log(rng, 1, 2048)])
        A = T if T > 64 else rng.randint(1, min(T, 8))
        least = _log(rng, max(A, 16), 40000)
        return _weights("", B, T, A, Hq, Hk, D, least, rng.randint(least, 2 * least), dtype)
    if kind == "append":
        T = rng.choice([_log(rng, 1, 64), _log(rng, 1, 1024)])
        A = T if T > 64 else rng.randint(1, min(T, 8))
        least = rng.choice([0, _log(rng, 1, 8000)])
        return _append("", B, T, A, Hk, D, least, least + rng.randint(0, 1000), dtype)
    budget = _log(rng, 64, 4096)
    recent = rng.randint(0, budget // 2)
    if kind == "step":
        return _step("", B, rng.randint(1, 8), Hk, D, budget, recent, dtype)
    most = _log(rng, budget, 32768)
    return _prompt("", B, Hk, D, rng.randint(budget // 2, most), most, budget, recent, dtype)


def draw(rng):
    """One more case of those ranges, no dearer than the largest listed: at most 4.5e11 flops, 1.2e9 bytes, a cache of 2e9 bytes, 1.1e9 scores."""
    while True:
        c = _draw_once(rng)
        del c["name"]
        w = work(c)
        rows = c["B"] * c.get("Hq", 1) * (c["A"] if c["kind"] == "weights" else c.get("T", 1)) * c.get("most", 1)
        cap = 2 * c["B"] * c["Hk"] * c["D"] * 2 * (c.get("most") or c["budget"])
        if w["flops"] <= 4.5e11 and w["bytes"] <= 1.2e9 and cap <= 2e9 and rows <= 1.1e9:
            return c


def _spread(lo, hi, n):
    """n lengths evenly from lo to hi, the same for every seed (their order is drawn)."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _counts(c):
    """(cached rows, new rows) of each sequence, as prepare() lays them out before their order is drawn."""
    B = c["B"]
    if c["kind"] == "attn":
        return _spread(c["least"], c["most"], B), [c["T"] - (c["T"] // 3) * (i % 3) // 2 if c["ragged"] else c["T"] for i in range(B)]
    if c["kind"] == "weights" or c["kind"] == "append":
        return _spread(c["least"], c["most"], B), [c["A"] if c["A"] == c["T"] else 1 + i % c["A"] for i in range(B)]
    if c["kind"] == "step":
        return [c["budget"]] * B, [1 + i % c["A"] for i in range(B)]
    return _spread(c["least"], c["most"], B), [0] * B


def work(c):
    cached, new = _counts(c)
    D, Hk, B = c["D"], c["Hk"], c["B"]
    row = 2 * 2 * D * Hk                              # a cached row: key and value of every head, 16 bits each
    if c["kind"] == "attn":
        Hq, T = c["Hq"], c["T"]
        pairs = sum(n * m + n * (n + 1) / 2 if c["shape"] == "chain" else n * m + n for m, n in zip(cached, new))
        return {"bytes": sum(cached) * row + sum(new) * (row + Hq * (2 * 2 * D + 4)) + B * (4 + 8 * T * -(-T // 64)), "flops": 4 * D * Hq * pairs}
    if c["kind"] == "weights":
        pairs = sum(n * (m - n) + n * (n + 1) / 2 for m, n in zip(cached, new))
        return {"bytes": sum(cached) * Hk * (2 * D + 8) + sum(new) * c["Hq"] * (2 * D + 4), "flops": 2 * D * c["Hq"] * pairs}
    if c["kind"] == "append":
        return {"bytes": sum(new) * (2 * row + 8 * Hk + 4), "flops": 0}
    if c["kind"] == "step":                           # every appended row evicts one: read its weight and position, move one row
        return {"bytes": sum(new) * (2 * row + 8 * Hk + 4) + sum(m + n for m, n in zip(cached, new)) * 8 * Hk + sum(new) * 2 * (row + 8 * Hk), "flops": 0}
    kept = sum(min(m, c["budget"]) for m in cached)
    return {"bytes": sum(cached) * 8 * Hk + kept * 2 * row + kept * 8 * Hk, "flops": 0}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _ints(v, order):
    return torch.tensor(v, dtype=torch.int32, device="cuda")[order].contiguous()


def _words(seen):
    """The bits of [.., T] truth values in 64-bit words: bit j of word w is column 64 w + j."""
    B, T, _ = seen.shape
    W = -(-T // 64)
    bits = torch.zeros((B, T, W * 64), dtype=torch.int64, device="cuda")
    bits[:, :, :T] = seen
    return (bits.view(B, T, W, 64) << torch.arange(64, device="cuda")).sum(-1)


def prepare(c, seed):
    g = _generator(seed)
    dt, B, Hk, D = DTYPES[c["dtype"]], c["B"], c["Hk"], c["D"]
    order = torch.randperm(B, generator=g, device="cuda")
    cached, new = _counts(c)
    s = {"c": c, "cached": _ints(cached, order), "new": _ints(new, order)}
    if c["kind"] == "attn":
        T, Hq, cap = c["T"], c["Hq"], max(c["most"], 1)
        qkv = _normal(g, (B, T, (Hq + 2 * Hk) * D), dt)            # one row per drafted token, as the QKV product leaves it
        qkv[:, :, : Hq * D] *= 2                                   # scores of deviation 2: some keys matter more than others
        s["q"] = qkv[:, :, : Hq * D].view(B, T, Hq, D)
        s["kn"] = qkv[:, :, Hq * D: (Hq + Hk) * D].view(B, T, Hk, D)
        s["vn"] = qkv[:, :, (Hq + Hk) * D:].view(B, T, Hk, D)
        s["kc"], s["vc"] = _normal(g, (B, cap, Hk, D), dt), _normal(g, (B, cap, Hk, D), dt)
        s["tree"] = None                                           # a chain: every drafted token sees those before it
        if c["shape"] == "tree":                                   # each sees itself and its ancestors in a random tree
            parent = (torch.rand((B, T), generator=g, device="cuda") * torch.arange(T, device="cuda")).long()   # (0 is the root, its own parent)
            seen = torch.eye(T, device="cuda").expand(B, T, T).clone()
            seen.scatter_(2, parent[:, :, None], 1.0)
            for _ in range(max(1, math.ceil(math.log2(max(T, 2))))):
                seen = (torch.matmul(seen, seen) > 0).float()
            s["tree"] = _words(seen > 0)
        s["out"] = torch.zeros((B, T, Hq, D), dtype=dt, device="cuda")
        s["lse"] = torch.zeros((B, T, Hq), dtype=torch.float32, device="cuda")
        if not c["ragged"]:
            s["new"] = None
        return s
    if c["kind"] == "weights":
        T, A, Hq, cap = c["T"], c["A"], c["Hq"], c["most"]
        s["q"] = _normal(g, (B, T, Hq, D), dt, 2.0)
        s["kc"] = _normal(g, (B, cap, Hk, D), dt)
        # the log-sums of these scores, near enough: ln(keys) + variance / 2
        s["lse"] = s["cached"].float().log()[:, None, None] + 2.0 + 0.1 * torch.randn((B, T, Hq), generator=g, device="cuda")
        s["accepted"] = None if A == T else torch.rand((B, T), generator=g, device="cuda").argsort(1)[:, :A].sort(1)[0].int().contiguous()
        s["weights"] = torch.rand((B, Hk, cap), generator=g, device="cuda")
        return s
    # append, step, prompt: a cache with its rows' weights and positions
    A = c.get("A", 0)
    cap = (c["budget"] if c["kind"] == "step" else c["most"]) + A
    s["kc"], s["vc"] = _normal(g, (B, cap, Hk, D), dt), _normal(g, (B, cap, Hk, D), dt)
    s["weights"] = torch.rand((B, Hk, cap), generator=g, device="cuda").square() * 8
    s["weights"][torch.rand((B, Hk, cap), generator=g, device="cuda") < 0.2] = 0.0   # rows that nothing attended to: equal weights
    s["pos"] = torch.arange(cap, device="cuda", dtype=torch.int32).expand(B, Hk, cap).contiguous()
    s["start"] = s["cached"].clone()
    s["cached_mid"], s["cached_out"] = torch.zeros_like(s["cached"]), torch.zeros_like(s["cached"])
    if A:
        T = c.get("T", 16)
        s["kn"], s["vn"] = _normal(g, (B, T, Hk, D), dt), _normal(g, (B, T, Hk, D), dt)
        s["accepted"] = None if A == T else torch.rand((B, T), generator=g, device="cuda").argsort(1)[:, :A].sort(1)[0].int().contiguous()
    if c["kind"] == "prompt":
        n = c["budget"]
        s["ko"], s["vo"] = torch.zeros((B, n, Hk, D), dtype=dt, device="cuda"), torch.zeros((B, n, Hk, D), dtype=dt, device="cuda")
        s["wo"], s["po"] = torch.zeros((B, Hk, n), device="cuda"), torch.zeros((B, Hk, n), dtype=torch.int32, device="cuda")
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _plain_attn(s):
    c, q = s["c"], s["q"].float()
    B, T, Hq, D = q.shape
    Hk, cap = c["Hk"], s["kc"].shape[1]
    G = Hq // Hk
    drafted = s["new"] if s["new"] is not None else torch.full((B,), T, device="cuda")
    at, row = torch.arange(cap, device="cuda"), torch.arange(T, device="cuda")
    if s["tree"] is None:
        seen = (row[None, :] <= row[:, None]).expand(B, T, T)
    else:
        seen = ((s["tree"][:, :, :, None] >> torch.arange(64, device="cuda")) & 1).bool().reshape(B, T, -1)[:, :, :T]
    live = row[None, :] < drafted[:, None]                                                         # [B, T]
    seen = torch.cat([(at[None, :] < s["cached"][:, None])[:, None, :].expand(B, T, cap), seen & live[:, None, :]], 2)
    k = torch.cat([s["kc"], s["kn"]], 1).float().permute(0, 2, 3, 1).contiguous()                  # [B, Hk, D, keys]
    v = torch.cat([s["vc"], s["vn"]], 1).float().permute(0, 2, 1, 3).contiguous()
    q = q.reshape(B, T, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * T, D)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(D)).view(B, Hk, G, T, -1).masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = x.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hk, G * T, -1), v).view(B, Hk, G, T, D) / torch.where(l == 0, 1.0, l)
    keep = live[:, :, None]
    s["out"] = torch.where(keep[..., None], o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D).to(s["out"].dtype), s["out"])
    s["lse"] = torch.where(keep, (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(B, T, Hq), s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _accepted_rows(x, accepted):
    """x[b, accepted[b, i]] for tensors [B, T, ..]."""
    if accepted is None:
        return x
    return x[torch.arange(x.shape[0], device="cuda")[:, None], accepted.long()]


def _plain_weights(s):
    q, lse = _accepted_rows(s["q"], s["accepted"]).float(), _accepted_rows(s["lse"], s["accepted"])
    B, A, Hq, D = q.shape
    Hk, cap = s["c"]["Hk"], s["kc"].shape[1]
    G = Hq // Hk
    i = torch.arange(A, device="cuda")
    last = s["cached"][:, None] - s["new"][:, None] + i                                            # the row's own key, [B, A]
    seen = (torch.arange(cap, device="cuda") <= last[:, :, None]) & (i[None, :] < s["new"][:, None])[:, :, None]
    k = s["kc"].float().permute(0, 2, 3, 1).contiguous()
    q = q.reshape(B, A, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * A, D)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(D)).view(B, Hk, G, A, cap)
    x = x.sub_(lse.view(B, A, Hk, G).permute(0, 2, 3, 1)[..., None]).exp_().masked_fill_(~seen[:, None, None], 0.0)
    s["weights"] += x.sum((2, 3))
    return {"weights": s["weights"]}


def _plain_append(s, cached_out):
    """The accepted rows behind the cached ones; rows that a sequence did not accept are left as they were."""
    kn, vn = _accepted_rows(s["kn"], s["accepted"]), _accepted_rows(s["vn"], s["accepted"])
    B, A = kn.shape[:2]
    i = torch.arange(A, device="cuda")
    mine = i[None, :] < s["new"][:, None]                                                          # [B, A]
    at = (s["cached"][:, None] + i).long()
    b = torch.arange(B, device="cuda")[:, None]
    s["kc"][b, at] = torch.where(mine[:, :, None, None], kn, s["kc"][b, at])
    s["vc"][b, at] = torch.where(mine[:, :, None, None], vn, s["vc"][b, at])
    h, b, at, mine = torch.arange(s["pos"].shape[1], device="cuda")[:, None], b[:, None], at[:, None], mine[:, None]
    s["weights"][b, h, at] = torch.where(mine, 0.0, s["weights"][b, h, at])
    s["pos"][b, h, at] = torch.where(mine, (s["start"][:, None] + i)[:, None].int(), s["pos"][b, h, at])
    cached_out.copy_(s["cached"] + s["new"])


def _kept(s, cached, budget, recent):
    """Truth values [B, Hk, cap]: the rows that stay, `budget` at most: the newest, then the heaviest, equal ones by lowest row."""
    w, pos = s["weights"], s["pos"]
    live = (torch.arange(w.shape[2], device="cuda") < cached[:, None])[:, None, :]
    newest = pos.masked_fill(~live, -1).amax(-1, keepdim=True)
    key = torch.where(w.isnan(), -math.inf, w).masked_fill(live & (pos > newest - recent), math.inf)
    # rows that hold nothing come last: by an order of two keys, both stable
    first = key.sort(stable=True, dim=-1, descending=True)[1]
    first = first.gather(-1, live.expand_as(w).gather(-1, first).int().sort(stable=True, dim=-1, descending=True)[1])
    keep = torch.zeros_like(live.expand_as(w)).clone()
    keep.scatter_(-1, first[:, :, :budget], True)
    return keep & live


def _rows(x, index):
    """x[b, index[b, h, j], h] of a cache [B, cap, Hk, D], as [B, n, Hk, D]."""
    return x.gather(1, index.permute(0, 2, 1)[..., None].expand(-1, -1, -1, x.shape[3]))


def _plain_evict(s, cached):
    """In place: the kept rows behind the budget fill, in order, the rows before it that are not kept."""
    n, cap = s["c"]["budget"], s["weights"].shape[2]
    keep = _kept(s, cached, n, s["c"]["recent"])
    over = (cached > n)[:, None, None]
    row = torch.arange(cap, device="cuda").expand_as(keep)
    hole, source = ~keep[:, :, :n] & over, keep[:, :, n:] & over
    # the j-th source, j-th in ascending order
    sources = torch.where(source, row[:, :, n:], cap).sort(-1)[0]
    sources = torch.cat([sources, torch.zeros_like(sources[:, :, :1])], -1)
    take = torch.where(hole, sources.gather(-1, (hole.int().cumsum(-1) - 1).clamp(0, sources.shape[2] - 1)), row[:, :, :n])
    s["kc"][:, :n], s["vc"][:, :n] = _rows(s["kc"], take), _rows(s["vc"], take)
    s["weights"][:, :, :n], s["pos"][:, :, :n] = s["weights"].gather(-1, take), s["pos"].gather(-1, take)
    s["cached_out"].copy_(cached.clamp(max=n))


def _plain_prompt(s):
    """Into another cache: the kept rows in order; rows of it that stay free are left as they were."""
    n = s["c"]["budget"]
    keep = _kept(s, s["cached"], n, s["c"]["recent"])
    cap = keep.shape[2]
    row = torch.arange(cap, device="cuda").expand_as(keep)
    take = torch.where(keep, row, cap).sort(-1)[0][:, :, :n]
    free = take == cap
    take = take.masked_fill(free, 0)
    gone = free.permute(0, 2, 1)[..., None]
    s["ko"], s["vo"] = torch.where(gone, s["ko"], _rows(s["kc"], take)), torch.where(gone, s["vo"], _rows(s["vc"], take))
    s["wo"], s["po"] = torch.where(free, s["wo"], s["weights"].gather(-1, take)), torch.where(free, s["po"], s["pos"].gather(-1, take))
    s["cached_out"].copy_(s["cached"].clamp(max=n))


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        import paper_2305_13450_amd as ds
    if kind == "attn":
        if not own:
            return _plain_attn(s)
        ds.dep_tree_attn(s["q"], s["kn"], s["vn"], s["kc"], s["vc"], s["cached"], s["out"], lse=s["lse"], tree=s["tree"], drafted=s["new"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "weights":
        if not own:
            return _plain_weights(s)
        ds.dep_cache_weights(s["q"], s["lse"], s["kc"], s["cached"], s["weights"], accepted=s["accepted"], n_accepted=s["new"])
        return {"weights": s["weights"]}
    if kind == "append":
        if not own:
            _plain_append(s, s["cached_out"])
        else:
            ds.dep_cache_append(s["kn"], s["vn"], s["kc"], s["vc"], s["cached"], s["cached_out"], accepted=s["accepted"], n_accepted=s["new"],
                                weights=s["weights"], pos=s["pos"], start=s["start"])
        return {"k": s["kc"], "v": s["vc"], "weights": s["weights"], "pos": s["pos"], "cached": s["cached_out"]}
    if kind == "step":
        # the cache is back at its budget after the step, and the next pass appends behind it again
        if not own:
            _plain_append(s, s["cached_mid"])
            _plain_evict(s, s["cached_mid"])
        else:
            ds.dep_cache_append(s["kn"], s["vn"], s["kc"], s["vc"], s["cached"], s["cached_mid"], accepted=s["accepted"], n_accepted=s["new"],
                                weights=s["weights"], pos=s["pos"], start=s["start"])
            ds.dep_cache_evict(s["kc"], s["vc"], s["weights"], s["pos"], s["cached_mid"], s["cached_out"], c["budget"], c["recent"])
        s["start"] += s["new"]
        n = c["budget"]
        return {"k": s["kc"][:, :n], "v": s["vc"][:, :n], "weights": s["weights"][:, :, :n], "pos": s["pos"][:, :, :n], "cached": s["cached_out"]}
    if not own:
        _plain_prompt(s)
    else:
        ds.dep_cache_evict(s["kc"], s["vc"], s["weights"], s["pos"], s["cached"], s["cached_out"], c["budget"], c["recent"],
                           k_out=s["ko"], v_out=s["vo"], weights_out=s["wo"], pos_out=s["po"])
    return {"k": s["ko"], "v": s["vo"], "weights": s["wo"], "pos": s["po"], "cached": s["cached_out"]}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    B, Hk, D, kind = c["B"], c["Hk"], c["D"], c["kind"]
    if kind == "attn":
        T, Hq = c["T"], c["Hq"]
        out, lse = s["out"].double(), s["lse"].double()
        for b in range(B):
            n, m = int(s["cached"][b]), T if s["new"] is None else int(s["new"][b])
            sees = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
            if s["tree"] is not None:
                for j in range(T):
                    sees[:, j] = (s["tree"][b, :, j // 64] >> (j % 64)) & 1 == 1
            for h in range(Hq):
                k = torch.cat([s["kc"][b, :n, h // (Hq // Hk)], s["kn"][b, :m, h // (Hq // Hk)]]).double()
                v = torch.cat([s["vc"][b, :n, h // (Hq // Hk)], s["vn"][b, :m, h // (Hq // Hk)]]).double()
                x = s["q"][b, :m, h].double() @ k.T / math.sqrt(D)
                x[:, n:][~sees[:m, :m]] = -math.inf
                lse[b, :m, h] = torch.logsumexp(x, 1)
                out[b, :m, h] = torch.softmax(x, 1) @ v
        return {"out": out, "lse": lse}
    if kind == "weights":
        w = s["weights"].double()
        for b in range(B):
            n, m = int(s["cached"][b]), int(s["new"][b])
            rows = list(range(m)) if s["accepted"] is None else s["accepted"][b, :m].tolist()
            for h in range(c["Hq"]):
                x = s["q"][b, rows, h].double() @ s["kc"][b, :n, h // (c["Hq"] // Hk)].double().T / math.sqrt(D)
                x = (x - s["lse"][b, rows, h].double()[:, None]).exp().tril(n - m)
                w[b, h // (c["Hq"] // Hk), :n] += x.sum(0)
        return {"weights": w}
    if kind != "append" and B * Hk * c.get("most", c.get("budget")) > 2e6:
        return None                                   # sorting that many rows one by one takes over 20 seconds
    # append, step, prompt: every value is one that the inputs hold, and is found again row by row
    k, v, w, pos = s["kc"].clone(), s["vc"].clone(), s["weights"].clone(), s["pos"].clone()
    cached, new = s["cached"].tolist(), s["new"].tolist()
    for b in range(B):
        for i in range(new[b]):
            a, at = i if s["accepted"] is None else int(s["accepted"][b, i]), cached[b] + i
            k[b, at], v[b, at], w[b, :, at], pos[b, :, at] = s["kn"][b, a], s["vn"][b, a], 0.0, int(s["start"][b]) + i
    if kind == "append":
        return {"k": k.double(), "v": v.double(), "weights": w.double(), "pos": pos, "cached": s["cached"] + s["new"]}
    budget, recent = c["budget"], c["recent"]
    ko, vo, wo, po = (k[:, :budget].clone(), v[:, :budget].clone(), w[:, :, :budget].clone(), pos[:, :, :budget].clone()) if kind == "step" else (s["ko"], s["vo"], s["wo"], s["po"])
    kept = []
    for b in range(B):
        n = cached[b] + new[b]
        for h in range(Hk):
            ws, ps = w[b, h, :n].tolist(), pos[b, h, :n].tolist()
            newest = max(ps, default=0)
            best = sorted(range(n), key=lambda r: (ps[r] <= newest - recent, 0.0 if ps[r] > newest - recent else -ws[r], r))[:budget]
            if kind == "prompt":
                rows = sorted(best)
            else:
                stay, come = set(best), sorted(r for r in best if r >= budget)
                rows = [r if r in stay else come.pop(0) for r in range(min(n, budget))]
            r = torch.tensor(rows, dtype=torch.long, device="cuda")
            ko[b, : len(rows), h], vo[b, : len(rows), h] = k[b, r, h], v[b, r, h]
            wo[b, h, : len(rows)], po[b, h, : len(rows)] = w[b, h, r], pos[b, h, r]
        kept.append(min(n, budget))
    return {"k": ko.double(), "v": vo.double(), "weights": wo.double(), "pos": po, "cached": torch.tensor(kept, dtype=torch.int32, device="cuda")}
