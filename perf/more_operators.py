"""One round of token generation from drafts over a cache of 8 bits, as cases that can be timed and compared.

A serving program that drafts tokens goes round one loop: the drafted tokens' queries and keys are normalised for each head and
rotated by their positions (`norm`), they attend to a cache held as 8-bit floating point numbers with a scale for each block of
tokens and head (`attn`), the target's probabilities decide which path of the drafted tree stays and which token comes next
(`verify`), and the path's keys and values go behind the cached ones (`append`).

The last rows of a sequence, those that do not fill a block, are held in 16 bits until they do: a block's scale is its own.

Sizes are those of the attention shard this repository measures (12 heads of 128, 2048 tokens) and generic ones with
shared key and value heads.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn


def _attn(name, B, T, Hq, Hk, D, least, most, block=64, dtype="bf16", shape="tree", ragged=False):
    """Attention of T drafted tokens per sequence over caches of `least` to `most` rows."""
    return dict(name=name, kind="attn", B=B, T=T, Hq=Hq, Hk=Hk, D=D, least=least, most=most, block=block, dtype=dtype, shape=shape, ragged=ragged)


def _append(name, B, T, A, Hk, D, least, most, block=64, dtype="bf16"):
    """Up to A accepted of T drafted tokens; A = T: a prompt, accepted whole."""
    return dict(name=name, kind="append", B=B, T=T, A=A, Hk=Hk, D=D, least=least, most=most, block=block, dtype=dtype)


def _norm(name, B, T, Hq, Hk, D, R, dtype="bf16", interleaved=False, shape="chain", ragged=False):
    """Norm and rotation of R of D dimensions."""
    return dict(name=name, kind="norm", B=B, T=T, Hq=Hq, Hk=Hk, D=D, R=R, dtype=dtype, interleaved=interleaved, shape=shape, ragged=ragged)


def _verify(name, B, T, V, drawn, shape="tree", ragged=False):
    """T tokens per sequence, the first known; drawn: from the draft's probabilities, else its most likely ones."""
    return dict(name=name, kind="verify", B=B, T=T, V=V, drawn=drawn, shape=shape, ragged=ragged)


def listed():
    return [
        # one new token of one short conversation: latency
        _attn("attn8_token_1x500", 1, 1, 12, 12, 128, 500, 500),
        # a large serving batch, one token each, long caches of uneven length, shared key heads: HBM bandwidth
        _attn("attn8_token_32x8192", 32, 1, 64, 8, 128, 2000, 8192),
        # a tree of 63 drafted tokens for each of eight requests; some drafted fewer
        _attn("attn8_tree_8x63", 8, 63, 32, 8, 128, 500, 4096, ragged=True),
        # a small tree over one very long document, fp16, heads of 64
        _attn("attn8_tree_long_fp16", 1, 13, 32, 8, 64, 120001, 120001, block=128, dtype="fp16"),
        # a wide tree search over long caches: the matrix cores' work
        _attn("attn8_tree_4x256", 4, 256, 64, 8, 128, 9000, 16384),
        # one to six accepted of a tree of 32, for 32 requests
        _append("append8_tree_32x32", 32, 32, 6, 8, 128, 1000, 4000),
        # a chunk of a prompt, accepted whole, fp16
        _append("append8_prompt_4x1024_fp16", 4, 1024, 1024, 8, 128, 0, 3000, block=32, dtype="fp16"),
        # one new token for each of 32 requests
        _norm("norm_token_32", 32, 1, 64, 8, 128, 128),
        # four prompts of 2048 tokens, as the attention shard's, with more heads
        _norm("norm_prompt_4x2048", 4, 2048, 64, 8, 128, 128),
        # a chain of five drafts behind the last token, drawn from the draft's probabilities
        _verify("verify_chain_32x6", 32, 6, 50257, True, shape="chain"),
        # a tree of the draft's most likely tokens
        _verify("verify_tree_16x32", 16, 32, 32000, False),
        # a wide tree of drawn tokens over a large vocabulary; some drafted fewer
        _verify("verify_tree_8x64_drawn", 8, 64, 128000, True, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["attn", "attn", "attn", "append", "norm", "norm", "verify", "verify"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    D = rng.choice([128, 128, 64])
    Hk = rng.choice([1, 2, 4, 8, 8, 12, 16])
    Hq = Hk * rng.choice([1, 1, 2, 4, 5, 8])
    B = _log(rng, 1, 48)
    block = rng.choice([32, 64, 64, 128])
    if kind == "attn":
        most = _log(rng, 16, 100000)
        least = rng.choice([most, rng.randint(0, most)])
        return _attn("", B, rng.choice([1, _log(rng, 1, 256)]), Hq, Hk, D, least, most, block, dtype, rng.choice(["tree", "tree", "chain"]), rng.random() < 0.5)
    if kind == "append":
        T = rng.choice([_log(rng, 1, 64), _log(rng, 1, 1024)])
        A = T if T > 64 else rng.randint(1, min(T, 8))
        least = rng.choice([0, _log(rng, 1, 8000)])
        return _append("", B, T, A, Hk, D, least, least + rng.randint(0, 1000), block, dtype)
    if kind == "norm":
        T = rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 8192)])
        return _norm("", B, T, Hq, Hk, D, rng.choice([D, D, D // 2, 16]), dtype, rng.random() < 0.3, "tree" if T <= 64 and rng.random() < 0.5 else "chain", rng.random() < 0.5)
    return _verify("", B, _log(rng, 1, 64), _log(rng, 100, 200000), rng.random() < 0.5, rng.choice(["tree", "chain"]), rng.random() < 0.5)


def draw(rng):
    """One more case of those ranges, no dearer than the largest listed: at most 4.5e11 flops, 3.3e8 bytes, a cache of 1e9 bytes, 1.1e9 scores, 6.6e7 probabilities."""
    while True:
        c = _draw_once(rng)
        del c["name"]
        w = work(c)
        rows = c["B"] * c.get("Hq", 1) * c["T"] * c.get("most", 1)
        cap = 2 * c["B"] * c.get("Hk", 0) * c.get("D", 0) * c.get("most", 0)
        if w["flops"] <= 4.5e11 and w["bytes"] <= 3.3e8 and cap <= 1e9 and rows <= 1.1e9 and c["B"] * c["T"] * c.get("V", 0) <= 6.6e7:
            return c


def _spread(lo, hi, n):
    """n lengths evenly from lo to hi, the same for every seed (their order is drawn)."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _counts(c):
    """(cached rows, new rows) of each sequence, as prepare() lays them out before their order is drawn."""
    B, T = c["B"], c["T"]
    if c["kind"] == "append":
        return _spread(c["least"], c["most"], B), [c["A"] if c["A"] == T else 1 + i % c["A"] for i in range(B)]
    new = [T - (T // 3) * (i % 3) // 2 if c["ragged"] else T for i in range(B)]
    return (_spread(c["least"], c["most"], B) if c["kind"] == "attn" else [0] * B), new


def work(c):
    cached, new = _counts(c)
    if c["kind"] == "verify":
        # the row that the next token is drawn from, target's and (where tokens were drawn) draft's; the rest is a few numbers a token
        rows = 2 if c["drawn"] else 1
        return {"bytes": c["B"] * (4 * rows * c["V"] + 8) + sum(new) * (4 * 5 + 4 * rows), "flops": 2 * rows * c["B"] * c["V"]}
    D, Hk, B = c["D"], c["Hk"], c["B"]
    if c["kind"] == "norm":
        n = sum(new) * (c["Hq"] + Hk) * D
        return {"bytes": 2 * 2 * n + 8 * D + 4 * c["R"] + 4 * B, "flops": 8 * n}
    row, block = 2 * 2 * D * Hk, c["block"]           # a row in 16 bits: key and value of every head; half of it in 8
    if c["kind"] == "attn":
        Hq, T = c["Hq"], c["T"]
        pairs = sum(n * m + n * (n + 1) / 2 if c["shape"] == "chain" else n * m + n for m, n in zip(cached, new))
        held = sum((m // block) * (block * row // 2 + 8 * Hk) + (m % block) * row for m in cached)
        return {"bytes": held + sum(new) * (row + Hq * (2 * 2 * D + 4)) + B * (4 + 8 * T * -(-T // 64)), "flops": 4 * D * Hq * pairs}
    moved = 0
    for m, n in zip(cached, new):
        full, left = divmod(m % block + n, block)
        moved += n * row + 4 * n                                          # the new rows
        if full:                                                         # blocks that are full now: the rows held in 16 bits read, the block written
            moved += (m % block) * row + full * (block * row // 2 + 8 * Hk) + left * row
        else:
            moved += n * row
    return {"bytes": moved + 12 * B, "flops": 0}


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


def _tree(g, B, T):
    """Parents [B, T] of a random tree, -1 for the root, and who sees whom [B, T, T]: each itself and its ancestors."""
    parent = (torch.rand((B, T), generator=g, device="cuda") * torch.arange(T, device="cuda")).long()
    seen = torch.eye(T, device="cuda").expand(B, T, T).clone()
    seen.scatter_(2, parent[:, :, None], 1.0)
    for _ in range(max(1, math.ceil(math.log2(max(T, 2))))):
        seen = (torch.matmul(seen, seen) > 0).float()
    parent[:, 0] = -1
    return parent, seen > 0


def _quantise(x):
    """x [.., rows, D] in 32 bits as (8-bit numbers, scale [..]): the scale is the smallest power of two, not below 2^-126, by which the largest
    finite magnitude is at most 448; 0 where that magnitude is 0.  Infinities become +-448."""
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax((-2, -1))
    m, e = torch.frexp(top)                                              # m in [1/2, 1)
    e = (e - 9 + (m > 0.875).int()).clamp(min=-126)                      # 448 = 0.875 * 2^9
    scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), 0.0)
    y = x / torch.where(top > 0, scale, 1.0)[..., None, None]
    return y.clamp(-448.0, 448.0).to(E4M3), scale


def _cache(g, B, cap, Hk, D, block):
    """A cache's rows of normal numbers in 8 bits [B, cap, Hk, D] and their blocks' scales [B, Hk, cap / block]."""
    # (heads differ in size as keys' and values' do)
    x = torch.randn((B, cap // block, Hk, block, D), generator=g, device="cuda") * (0.5 + torch.rand((Hk, 1, 1), generator=g, device="cuda"))
    y, scale = _quantise(x)
    return y.view(torch.uint8).permute(0, 1, 3, 2, 4).reshape(B, cap, Hk, D).view(E4M3), scale.permute(0, 2, 1).contiguous()


def prepare(c, seed):
    g = _generator(seed)
    B, T = c["B"], c["T"]
    order = torch.randperm(B, generator=g, device="cuda")
    cached, new = _counts(c)
    s = {"c": c, "cached": _ints(cached, order), "new": _ints(new, order)}
    if c["kind"] == "verify":
        V = c["V"]
        logits = torch.randn((B, T, V), generator=g, device="cuda") * 4                                # a few likely tokens, a long tail
        s["p"] = torch.softmax(logits, -1)
        logits += torch.randn((B, T, V), generator=g, device="cuda")                                   # the draft is near the target
        parent = torch.arange(T, device="cuda").expand(B, T) - 1
        if c["shape"] == "tree":
            parent = _tree(g, B, T)[0]
        s["parents"] = None if c["shape"] == "chain" else parent.int().contiguous()
        b = torch.arange(B, device="cuda")[:, None]
        at = parent.clamp(min=0)
        if c["drawn"]:
            s["q"] = torch.softmax(logits, -1)
            edges = s["q"].double().cumsum(-1)[b, at]                                                  # each child is drawn from its parent's row
            r = torch.rand((B, T, 1), generator=g, device="cuda", dtype=torch.float64) * edges[..., -1:]
            s["ids"] = torch.searchsorted(edges.contiguous(), r, right=True)[..., 0].clamp(max=V - 1).int()
        else:
            s["q"] = None
            t = torch.arange(T, device="cuda")
            rank = ((parent[:, :, None] == parent[:, None, :]) & (t[None, :] < t[:, None])).sum(-1)     # siblings before it
            best = logits.topk(min(V, T), -1)[1]
            s["ids"] = best[b, at, rank.clamp(max=best.shape[-1] - 1)].int().contiguous()
        s["u"] = torch.rand((B, T), generator=g, device="cuda")
        s["accepted"] = torch.full((B, T), -1, dtype=torch.int32, device="cuda")
        s["n"], s["next"] = (torch.full((B,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
        if not c["ragged"]:
            s["new"] = None
        return s
    dt, Hk, D = DTYPES[c["dtype"]], c["Hk"], c["D"]
    if c["kind"] == "norm":
        Hq = c["Hq"]
        s["qkv"] = _normal(g, (B, T, (Hq + 2 * Hk) * D), dt, 2.0)          # one row per token, as the QKV product leaves it
        s["q_gain"], s["k_gain"] = (1 + 0.2 * torch.randn((D,), generator=g, device="cuda") for _ in range(2))
        s["start"] = torch.randint(0, 100000, (B,), generator=g, device="cuda").int()
        s["depth"] = None
        if c["shape"] == "tree":
            s["depth"] = (_tree(g, B, T)[1].sum(-1) - 1).int().contiguous()
        s["q_out"], s["k_out"] = (torch.zeros((B, T, h, D), dtype=dt, device="cuda") for h in (Hq, Hk))
        s["angle"] = 10000.0 ** (-2 * torch.arange(c["R"] // 2, device="cuda", dtype=torch.float64) / c["R"])   # a position's turn, in radians
        if own:
            import paper_2305_13450_amd as ds
            s["freq"] = ds.rope_frequencies(s["angle"])
        if not c["ragged"]:
            s["new"] = None
        return s
    block = c["block"]
    cap = -(-max(c["most"] + c.get("A", 0), 1) // block) * block
    s["kc"], s["ks"] = _cache(g, B, cap, Hk, D, block)
    s["vc"], s["vs"] = _cache(g, B, cap, Hk, D, block)
    s["kt"], s["vt"] = _normal(g, (B, block, Hk, D), dt), _normal(g, (B, block, Hk, D), dt)
    if c["kind"] == "append":
        s["kn"], s["vn"] = _normal(g, (B, T, Hk, D), dt), _normal(g, (B, T, Hk, D), dt)
        s["accepted"] = None if c["A"] == T else torch.rand((B, T), generator=g, device="cuda").argsort(1)[:, :c["A"]].sort(1)[0].int().contiguous()
        s["cached_out"] = torch.zeros_like(s["cached"])
        return s
    Hq = c["Hq"]
    qkv = _normal(g, (B, T, (Hq + 2 * Hk) * D), dt)
    qkv[:, :, : Hq * D] *= 2                                               # scores of deviation 2: some keys matter more than others
    s["q"] = qkv[:, :, : Hq * D].view(B, T, Hq, D)
    s["kn"] = qkv[:, :, Hq * D: (Hq + Hk) * D].view(B, T, Hk, D)
    s["vn"] = qkv[:, :, (Hq + Hk) * D:].view(B, T, Hk, D)
    s["tree"] = None if c["shape"] == "chain" else _words(_tree(g, B, T)[1])   # (a chain: every drafted token sees those before it)
    s["out"] = torch.zeros((B, T, Hq, D), dtype=dt, device="cuda")
    s["lse"] = torch.zeros((B, T, Hq), dtype=torch.float32, device="cuda")
    if not c["ragged"]:
        s["new"] = None
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------------

def _values(x, scale, block):
    """The numbers that a cache of 8 bits stands for, [B, cap, Hk, D] in 32 bits."""
    return x.float() * scale.permute(0, 2, 1).repeat_interleave(block, 1)[..., None]


def _plain_attn(s):
    c, q = s["c"], s["q"].float()
    B, T, Hq, D = q.shape
    Hk, cap, block = c["Hk"], s["kc"].shape[1], c["block"]
    G = Hq // Hk
    drafted = s["new"] if s["new"] is not None else torch.full((B,), T, device="cuda")
    row = torch.arange(T, device="cuda")
    if s["tree"] is None:
        seen = (row[None, :] <= row[:, None]).expand(B, T, T)
    else:
        seen = ((s["tree"][:, :, :, None] >> torch.arange(64, device="cuda")) & 1).bool().reshape(B, T, -1)[:, :, :T]
    live = row[None, :] < drafted[:, None]                                                         # [B, T]
    left = s["cached"] % block
    held = torch.cat([torch.arange(cap, device="cuda")[None, :] < (s["cached"] - left)[:, None],
                      torch.arange(block, device="cuda")[None, :] < left[:, None]], 1)             # rows in 8 bits, rows in 16
    seen = torch.cat([held[:, None, :].expand(B, T, cap + block), seen & live[:, None, :]], 2)
    k = torch.cat([_values(s["kc"], s["ks"], block), s["kt"].float(), s["kn"].float()], 1).permute(0, 2, 3, 1).contiguous()   # [B, Hk, D, keys]
    v = torch.cat([_values(s["vc"], s["vs"], block), s["vt"].float(), s["vn"].float()], 1).permute(0, 2, 1, 3).contiguous()
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


def _plain_append(s):
    """The rows from the first block that is not full, those held in 16 bits and the accepted ones: full blocks go into 8 bits, the others stay."""
    c, kt = s["c"], s["kt"]
    B, block, Hk, D = kt.shape
    cached, n = s["cached"].long(), s["new"].long()
    first = cached // block
    blocks = (block - 1 + c["A"]) // block
    i = torch.arange((blocks + 1) * block, device="cuda")                                          # rows from the first block on
    left = (cached % block)[:, None]
    from_tail, from_new = i < left, (i >= left) & (i < left + n[:, None])
    b = torch.arange(B, device="cuda")[:, None]
    at = (i - left).clamp(0, c["A"] - 1)
    if s["accepted"] is not None:
        at = s["accepted"].long()[b, at]
    full = (left[:, 0] + n) // block                                                               # blocks that are full now
    now = (i // block == full[:, None]) & (from_tail | from_new)                                   # rows that are left
    for cache, scales, tail, new in (("kc", "ks", "kt", "kn"), ("vc", "vs", "vt", "vn")):
        rows = torch.where(from_tail[..., None, None], s[tail][b, i % block], s[new][b, at])
        rows = torch.where((from_tail | from_new)[..., None, None], rows, torch.zeros_like(rows))
        y, scale = _quantise(rows.float().view(B, blocks + 1, block, Hk, D).transpose(2, 3))
        for j in range(blocks):
            # (a block that is not full puts back what stands there)
            is_full = j < full
            to = (first + j).clamp(max=s["ks"].shape[2] - 1)
            there = to[:, None] * block + torch.arange(block, device="cuda")
            bits = s[cache].view(torch.uint8)
            bits[b, there] = torch.where(is_full[:, None, None, None], y[:, j].view(torch.uint8).transpose(1, 2), bits[b, there])
            k = torch.arange(Hk, device="cuda")
            s[scales][b, k, to[:, None]] = torch.where(is_full[:, None], scale[:, j], s[scales][b, k, to[:, None]])
        slot = torch.arange(block, device="cuda")
        take = full[:, None] * block + slot
        s[tail] = torch.where(now.gather(1, take)[..., None, None], rows[b, take], s[tail])
    s["cached_out"].copy_(cached + n)


def _plain_norm(s):
    c = s["c"]
    B, T, Hq, Hk, D, R = c["B"], c["T"], c["Hq"], c["Hk"], c["D"], c["R"]
    t = torch.arange(T, device="cuda")
    pos = s["start"][:, None] + (t if s["depth"] is None else s["depth"])
    live = None if s["new"] is None else (t[None, :] < s["new"][:, None])[..., None, None]
    angle = pos.double()[..., None] * s["angle"]                           # far positions: in 64 bits
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    for name, gain, lo, h in (("q_out", "q_gain", 0, Hq), ("k_out", "k_gain", Hq * D, Hk)):
        x = s["qkv"][:, :, lo: lo + h * D].view(B, T, h, D).float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * s[gain]
        a, b = (x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., : R // 2], x[..., R // 2: R])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
        y = torch.cat([y, x[..., R:]], -1).to(s[name].dtype)
        s[name] = y if live is None else torch.where(live, y, s[name])


def _plain_verify(s):
    """The tokens in order, all sequences at once: one is looked at where its parent is the last accepted one.  Probabilities stand for what is left of
    them: the weights max(p - C q, 0), or p without the tokens refused, of which there are R; in 64 bits, as borders are compared."""
    p, q, ids = s["p"], s["q"], s["ids"].long()
    B, T, V = p.shape
    b = torch.arange(B, device="cuda")
    last = torch.zeros(B, dtype=torch.long, device="cuda")
    n = torch.ones(B, dtype=torch.long, device="cuda")
    C, R = torch.zeros(B, dtype=torch.float64, device="cuda"), torch.ones(B, dtype=torch.float64, device="cuda")
    gone = torch.zeros((B, V), dtype=torch.bool, device="cuda")
    s["accepted"][:, 0] = 0

    def left():
        w = p[b, last].double()
        return w.masked_fill(gone, 0.0) if q is None else (w - C[:, None] * q[b, last].double()).clamp(min=0.0)
    for t in range(1, T):
        parent = torch.full((B,), t - 1, device="cuda") if s["parents"] is None else s["parents"][:, t]
        mine = parent == last
        if s["new"] is not None:
            mine = mine & (t < s["new"])
        x = ids[:, t]
        u = s["u"][:, t].double()
        px = p[b, last, x].double()
        if q is None:
            w = torch.where(gone[b, x], 0.0, px)
            yes = mine & (u * R < w)
        else:
            qx = q[b, last, x].double()
            w = (px - C * qx).clamp(min=0.0)
            yes = mine & (u * qx * R < w)
        no = mine & ~yes
        if q is None:
            gone[b, x] |= no
            R = torch.where(no, (R - w).clamp(min=0.0), R)
        else:
            C = torch.where(no, C + R, C)
            R = torch.where(no, left().sum(1), R)
        s["accepted"][b, n.clamp(max=T - 1)] = torch.where(yes, t, s["accepted"][b, n.clamp(max=T - 1)]).int()
        n, last = torch.where(yes, n + 1, n), torch.where(yes, t, last)
        C, R = torch.where(yes, 0.0, C), torch.where(yes, 1.0, R)
        gone &= ~yes[:, None]
    w = left()
    w = torch.where((w.sum(1) > 0)[:, None], w, p[b, last].double())
    edges = w.cumsum(1)
    s["next"].copy_((edges > s["u"][:, :1].double() * edges[:, -1:]).int().argmax(1))
    s["n"].copy_(n)


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        import paper_2305_13450_amd as ds
    if kind == "attn":
        if not own:
            _plain_attn(s)
        else:
            ds.dep_tree_attn8(s["q"], s["kn"], s["vn"], s["kc"], s["vc"], s["ks"], s["vs"], s["kt"], s["vt"], s["cached"], s["out"], lse=s["lse"],
                              tree=s["tree"], drafted=s["new"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "append":
        if not own:
            _plain_append(s)
        else:
            ds.dep_cache_append8(s["kn"], s["vn"], s["kc"], s["vc"], s["ks"], s["vs"], s["kt"], s["vt"], s["cached"], s["cached_out"],
                                 accepted=s["accepted"], n_accepted=s["new"])
        return {"k": s["kc"], "v": s["vc"], "k_scale": s["ks"], "v_scale": s["vs"], "k_tail": s["kt"], "v_tail": s["vt"], "cached": s["cached_out"]}
    if kind == "norm":
        if not own:
            _plain_norm(s)
        else:
            B, T, Hq, Hk, D = c["B"], c["T"], c["Hq"], c["Hk"], c["D"]
            q, k = s["qkv"][:, :, : Hq * D].view(B, T, Hq, D), s["qkv"][:, :, Hq * D: (Hq + Hk) * D].view(B, T, Hk, D)
            ds.dep_qk_norm_rope(q, k, s["freq"], s["q_gain"], s["k_gain"], q_out=s["q_out"], k_out=s["k_out"], start=s["start"], depth=s["depth"],
                                drafted=s["new"], eps=1e-6, interleaved=c["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if not own:
        _plain_verify(s)
    else:
        ds.dep_verify_drafts(s["p"], s["ids"], s["u"], s["accepted"], s["n"], s["next"], q=s["q"], parents=s["parents"], drafted=s["new"])
    return {"accepted": s["accepted"], "n": s["n"], "next": s["next"]}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    B, T, kind = c["B"], c["T"], c["kind"]
    new = [T] * B if s["new"] is None else s["new"].tolist()
    cached = s["cached"].tolist()
    if kind == "verify":
        accepted, n, following = s["accepted"].clone(), s["n"].clone(), s["next"].clone()
        for b in range(B):
            parents = list(range(-1, T - 1)) if s["parents"] is None else s["parents"][b].tolist()
            ids, u = s["ids"][b].tolist(), s["u"][b].double().tolist()
            path = [0]
            while True:
                w = s["p"][b, path[-1]].double()
                mass = 1.0
                for t in [t for t in range(1, new[b]) if parents[t] == path[-1]]:
                    wx = float(w[ids[t]])
                    if s["q"] is None:
                        if u[t] * mass < wx:
                            path.append(t)
                            break
                        w[ids[t]] = 0.0
                        mass = max(mass - wx, 0.0)
                    else:
                        q = s["q"][b, path[-1]].double()
                        if u[t] * float(q[ids[t]]) * mass < wx:
                            path.append(t)
                            break
                        w = (w - mass * q).clamp(min=0.0)
                        mass = float(w.sum())
                else:
                    break
            if float(w.sum()) == 0.0:
                w = s["p"][b, path[-1]].double()
            edges = w.cumsum(0)
            following[b] = int((edges > u[0] * edges[-1]).nonzero()[0])
            accepted[b, : len(path)] = torch.tensor(path, dtype=torch.int32, device="cuda")
            n[b] = len(path)
        return {"accepted": accepted, "n": n, "next": following}
    Hk, D = c["Hk"], c["D"]
    if kind == "norm":
        R = c["R"]
        res = {}
        angle = 10000.0 ** (torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / -R)
        for name, lo, h in (("q", 0, c["Hq"]), ("k", c["Hq"] * D, Hk)):
            out = torch.zeros((B, T, h, D), dtype=torch.float64, device="cuda")
            for b in range(B):
                m = new[b]
                x = s["qkv"][b, :m, lo: lo + h * D].double().reshape(m, h, D)
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * s[name + "_gain"].double()
                pos = int(s["start"][b]) + (torch.arange(m, device="cuda") if s["depth"] is None else s["depth"][b, :m]).double()
                turn = torch.polar(torch.ones((m, 1, R // 2), dtype=torch.float64, device="cuda"), pos[:, None, None] * angle)
                lower = slice(0, R, 2) if c["interleaved"] else slice(0, R // 2)
                upper = slice(1, R, 2) if c["interleaved"] else slice(R // 2, R)
                z = torch.complex(x[..., lower].contiguous(), x[..., upper].contiguous()) * turn
                x[..., lower], x[..., upper] = z.real, z.imag
                out[b, :m] = x
            res[name] = out
        return res
    block = c["block"]
    if kind == "append":
        k, v, ks, vs, kt, vt = (s[x].clone() for x in ("kc", "vc", "ks", "vs", "kt", "vt"))
        k, v = k.double(), v.double()
        for b in range(B):
            rows = [i if s["accepted"] is None else int(s["accepted"][b, i]) for i in range(new[b])]
            held = cached[b] % block
            for cache, scales, tail, fresh in ((k, ks, kt, s["kn"]), (v, vs, vt, s["vn"])):
                all_rows = torch.cat([tail[b, :held], fresh[b, rows]])
                at, full = cached[b] // block, all_rows.shape[0] // block
                for j in range(full):
                    x = all_rows[j * block: (j + 1) * block].double()
                    for h in range(Hk):
                        top = float(x[:, h].abs().max())
                        if top == 0:
                            cache[b, (at + j) * block: (at + j + 1) * block, h], scales[b, h, at + j] = 0.0, 0.0
                            continue
                        e = -126
                        while math.ldexp(top, -e) > 448:
                            e += 1
                        y = x[:, h] * 2.0 ** -e
                        # to the nearest number of three bits behind the leading one, ties to the even one; below 2^-6 steps of 2^-9
                        step = torch.exp2(y.abs().clamp(min=2.0 ** -6).log2().floor() - 3)
                        cache[b, (at + j) * block: (at + j + 1) * block, h] = (y / step).round() * step
                        scales[b, h, at + j] = 2.0 ** e
                rest = all_rows[full * block:]
                tail[b, : rest.shape[0]] = rest
        return {"k": k, "v": v, "k_scale": ks.double(), "v_scale": vs.double(), "k_tail": kt.double(), "v_tail": vt.double(),
                "cached": torch.tensor([m + n for m, n in zip(cached, new)], dtype=torch.int32, device="cuda")}
    Hq = c["Hq"]
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(B):
        m, left = new[b], cached[b] % block
        n = cached[b] - left
        sees = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
        if s["tree"] is not None:
            for j in range(T):
                sees[:, j] = (s["tree"][b, :, j // 64] >> (j % 64)) & 1 == 1
        for h in range(Hq):
            g = h // (Hq // Hk)
            rows = []
            for cache, scales, tail, fresh in (("kc", "ks", "kt", "kn"), ("vc", "vs", "vt", "vn")):
                held = s[cache][b, :n, g].double().view(-1, block, D) * s[scales][b, g, : n // block].double()[:, None, None]
                rows.append(torch.cat([held.reshape(n, D), s[tail][b, :left, g].double(), s[fresh][b, :m, g].double()]))
            x = s["q"][b, :m, h].double() @ rows[0].T / math.sqrt(D)
            x[:, cached[b]:][~sees[:m, :m]] = -math.inf
            lse[b, :m, h] = torch.logsumexp(x, 1)
            out[b, :m, h] = torch.softmax(x, 1) @ rows[1]
    return {"out": out, "lse": lse}
