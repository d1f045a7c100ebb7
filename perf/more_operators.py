"""What a serving loop does around the paged key-value cache, as measurable cases: heads that are normed before they are turned, batches that
share a long prefix, and caches that are kept short by throwing out what little attention went to.

  append   norm_rope_kv_append: the queries and keys of a Q | K | V product are normed head by head (root of the mean square, a gain for each dim)
           and turned by their positions, keys and values go into the cache.  Positions may run ahead of the cache's by a shift for each
           sequence: the tokens that were evicted from it.
  shared   attention_decode_shared: one new token of each sequence, where runs of sequences have their first tokens in common
  decode   attention_decode_weights: one new token of each sequence, and what weight each cached token got, added up
  prompt   attention_prefill_weights: the same for runs of new tokens, causal
  evict    kv_evict: of each sequence and key-value head the last tokens and those with the most weight stay, in order, on other pages

Sizes are those of the 700M ... 13B LLaMA-family layers of paper_2402_17764_amd.synth.CONFIGS (24 heads of 64, 32 of 100, 32 of 128, 40 of 128),
and grouped heads, 64 over 8, as at hidden 8192.

The cache.  Pages of `page` tokens (a multiple of 32) hold blocks of 32 tokens for each of the key-value heads; bf16.
  k_cache  [pages][kv heads][page / 32][Dp / 8][32][8]: 8 consecutive dims of a token together; token t of a block at slot
           16 ((t >> 2) & 1) + 4 (t >> 3) + (t & 3).  Dp: the head's dims rounded up to 8, zeros behind them.
  v_cache  [pages][kv heads][page / 32][4][Dp][8]: 8 consecutive tokens of a dim together
Position p of sequence b lies on page page_table[b][p // page]; kv_len[b] counts the cached tokens, the new ones included;
q_start[b] ... q_start[b + 1] are the rows of sequence b's new tokens, its last ones.  Sequences prefix_start[i] ... prefix_start[i + 1] - 1 share
their first prefix_len[i] tokens, which lie on the pages of the first of them (what their own tables name for these is not read).
weights [B][kv heads][capacity] are the sums of the softmax weights that a cached token has had, over rows and the heads of its key-value head.
"""
import math

import torch

own = False

THETA = 10000.0
EPS = 1e-6


def listed():
    return [
        # the smallest call: one token of a 700M-class model into its cache, fp32 activations
        dict(name="append_norm_700m_t1", kind="append", x="f32", hq=24, hkv=24, d=64, page=64, B=1, lo=511, hi=511, one=True, pairs=False, shifted=False),
        # chunks of prompts behind caches that have been cut short: heads of 100, neighbouring pairs, positions ahead of the cache's
        dict(name="append_norm_3b_ragged", kind="append", x="bf16", hq=32, hkv=32, d=100, page=32, B=5, lo=0, hi=300, n_lo=1, n_hi=400, one=False, pairs=True, shifted=True),
        # two long prompts, grouped heads
        dict(name="append_norm_gqa_prompts", kind="append", x="bf16", hq=64, hkv=8, d=128, page=256, B=2, lo=0, hi=0, n_lo=1900, n_hi=2300, one=False, pairs=False, shifted=False),
        # an odd number of requests behind one system prompt, a key-value head for each head
        dict(name="shared_7b_b13", kind="shared", y="bf16", hq=32, hkv=32, d=128, page=128, B=13, groups=1, p_lo=1500, p_hi=1500, lo=1, hi=300),
        # two system prompts that end inside pages, heads of 100, fp32 results
        dict(name="shared_3b_two_prefixes", kind="shared", y="f32", hq=32, hkv=32, d=100, page=32, B=7, groups=2, p_lo=333, p_hi=1111, lo=1, hi=90),
        # many requests on one long document, grouped heads
        dict(name="shared_gqa_b48", kind="shared", y="bf16", hq=64, hkv=8, d=128, page=256, B=48, groups=1, p_lo=24000, p_hi=24000, lo=10, hi=2000),
        # one request, a few hundred tokens in: latency alone
        dict(name="weights_700m_b1", kind="decode", y="f32", hq=24, hkv=24, d=64, page=64, B=1, lo=700, hi=700),
        # three long contexts, grouped heads
        dict(name="weights_gqa_long", kind="decode", y="bf16", hq=64, hkv=8, d=128, page=256, B=3, lo=20000, hi=49152),
        # chunks of several requests' prompts together, ragged, heads of 100
        dict(name="prompt_weights_3b_ragged", kind="prompt", y="bf16", hq=32, hkv=32, d=100, page=32, B=6, lo=0, hi=500, n_lo=1, n_hi=900),
        # the largest: a prompt of 2048 tokens of a 13B-class model
        dict(name="prompt_weights_13b_t2048", kind="prompt", y="bf16", hq=40, hkv=40, d=128, page=128, B=1, lo=0, hi=0, n_lo=2048, n_hi=2048),
        # three requests on heads of 100 cut to 512 tokens, some of which have not that many
        dict(name="evict_3b_b3", kind="evict", hkv=32, d=100, page=32, B=3, lo=400, hi=2047, keep=512, recent=128),
        # long contexts cut to a quarter
        dict(name="evict_gqa_long", kind="evict", hkv=8, d=128, page=256, B=5, lo=20000, hi=40000, keep=8000, recent=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["append", "shared", "shared", "decode", "prompt", "evict"])
    d = rng.choice([64, 80, 96, 100, 128, 128, 128])
    hkv, g = rng.choice([(24, 1), (32, 1), (40, 1), (8, 8), (8, 4), (4, 7), (16, 2), (1, 12)])
    c = dict(kind=kind, hq=hkv * g, hkv=hkv, d=d, page=rng.choice([32, 64, 96, 128, 256]))
    dt = rng.choice(["bf16", "bf16", "f32"])
    if kind == "decode":
        B = _log(rng, 1, 64)
        hi = _log(rng, 1, max(64, min(49152, 400_000_000 // (B * hkv * d * 4))))
        return dict(c, y=dt, B=B, lo=rng.randint(1, hi), hi=hi)
    if kind == "shared":
        B = _log(rng, 2, 64)
        groups = min(B, rng.choice([1, 1, 2, 3]))
        p_hi = _log(rng, 16, min(24000, 60_000_000 // (groups * hkv * d), 1_300_000_000 // (B * hkv * d)))
        hi = _log(rng, 1, max(2, min(2000, 40_000_000 // (B * hkv * d))))
        return dict(c, y=dt, B=B, groups=groups, p_lo=rng.randint(p_hi // 2, p_hi), p_hi=p_hi, lo=rng.randint(1, hi), hi=hi)
    if kind == "evict":
        del c["hq"]
        B = _log(rng, 1, 48)
        hi = _log(rng, 40, max(64, min(49152, 280_000_000 // (B * hkv * d * 4))))
        keep = _log(rng, 1, max(2, hi * 3 // 4))
        return dict(c, B=B, lo=rng.randint(1, hi), hi=hi, keep=keep, recent=rng.choice([0, keep // 8, keep // 2, keep]))
    if kind == "append" and rng.random() < 0.5:
        return dict(c, x=dt, B=_log(rng, 1, 64), lo=0, hi=_log(rng, 8, 500), one=True, pairs=rng.random() < 0.3, shifted=rng.random() < 0.5)
    B = rng.randint(1, 6)
    n_hi = _log(rng, 1, 4096 // B)
    n_lo = rng.randint(1, n_hi)
    hi = rng.choice([0, _log(rng, 1, 2000)])
    if kind == "append":
        return dict(c, x=dt, B=B, lo=rng.randint(0, hi), hi=hi, n_lo=n_lo, n_hi=n_hi, one=False, pairs=rng.random() < 0.3, shifted=rng.random() < 0.5)
    while B * n_hi * (n_hi / 2 + hi) * hkv * g > 2048 * 1024 * 40:
        n_hi = n_hi // 2 + 1
    return dict(c, y=dt, B=B, lo=rng.randint(0, hi), hi=hi, n_lo=min(n_lo, n_hi), n_hi=n_hi)


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, spread evenly over the range in a shuffled order."""
    return [lo + int((0.5 + b * 0.6180339887498949) % 1.0 * (hi - lo + 1)) for b in range(n)]


def _groups(c):
    """Of a batch with shared prefixes: the first sequence of each group and the end, and the lengths of the prefixes."""
    G, B = c["groups"], c["B"]
    return [(i * B + i) // G if i < G else B for i in range(G + 1)], _spread(G, c["p_lo"], c["p_hi"])


def _sizes(c):
    """(cached tokens before the call, new tokens) of each sequence; a decoded token is in the cache already."""
    lens = _spread(c["B"], c["lo"], c["hi"])
    if c["kind"] == "shared":
        start, prefix = _groups(c)
        return [(prefix[max(i for i in range(len(prefix)) if start[i] <= b)] + n - 1, 1) for b, n in enumerate(lens)]
    if c["kind"] in ("decode", "evict"):
        return [(n - 1, 1) for n in lens]
    return list(zip(lens, [1] * c["B"] if c.get("one") else _spread(c["B"], c["n_lo"], c["n_hi"])))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _gen(seed, tensor):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 64 + tensor) % (1 << 62))


def _dt(s):
    return torch.bfloat16 if s == "bf16" else torch.float32


def _normal(seed, tensor, shape, dt, std=1.0):
    return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=_gen(seed, tensor))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c, sizes = case, _sizes(case)
    B, D, P = c["B"], c["d"], c["page"]
    Dp = (D + 7) // 8 * 8
    per = max(-(-(old + new) // P) for old, new in sizes)
    T = sum(new for _, new in sizes)
    s = {"case": dict(c)}
    numbers, used = torch.randperm(B * per + B * -(-c.get("keep", 0) // P) + 2, device="cuda", generator=_gen(seed, 0)).to(torch.int32), B * per
    s["table"] = numbers[:used].reshape(B, per).contiguous()
    pages = len(numbers)
    if c["kind"] == "shared":                                  # the whole pages of a prefix are named by all; they are renumbered to few
        start, prefix = _groups(c)
        for i, n in enumerate(prefix):
            s["table"][start[i]:start[i + 1], : n // P] = s["table"][start[i], : n // P].clone()
        alive, s["table"] = torch.unique(s["table"], return_inverse=True)
        s["table"], pages = s["table"].to(torch.int32).reshape(B, per).contiguous(), len(alive) + 2
        s["prefix_start"], s["prefix_len"] = _ints(start), _ints(prefix)
    s["kv_len"] = _ints([old + new for old, new in sizes])
    starts = [0]
    for _, new in sizes:
        starts.append(starts[-1] + new)
    s["q_start"] = _ints(starts)
    s["k"] = _normal(seed, 1, (pages, c["hkv"], P // 32, Dp // 8, 32, 8), torch.bfloat16)
    s["k"][:, :, :, -1, :, 8 - (Dp - D):] = 0
    s["v"] = _normal(seed, 2, (pages, c["hkv"], P // 32, 4, Dp, 8), torch.bfloat16)
    if c["kind"] == "append":
        s["qkv"] = _normal(seed, 3, (T, (c["hq"] + 2 * c["hkv"]) * D), _dt(c["x"]), 3.0)
        s["q_gain"], s["k_gain"] = (_normal(seed, i, (D,), torch.float32, 0.2) + 1.0 for i in (5, 6))
        s["freq"] = (THETA ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).to(device="cuda", dtype=torch.float32)
        s["shift"] = torch.randint(0, 100000, (B,), device="cuda", dtype=torch.int32, generator=_gen(seed, 7)) if c["shifted"] else None
        return s
    if c["kind"] != "evict":
        s["q"] = _normal(seed, 4, (T, c["hq"], D), torch.bfloat16, 1.5)
    if c["kind"] in ("decode", "prompt", "evict"):             # few tokens have most of the weight, some have had none
        w = _normal(seed, 8, (B, c["hkv"], per * P), torch.float32, 2.0).exp_()
        s["weights"] = w * (torch.rand(w.shape, device="cuda", generator=_gen(seed, 9)) > 0.1)
    if c["kind"] == "evict":
        out = -(-c["keep"] // P)
        s["table_out"] = numbers[used: used + B * out].reshape(B, out).contiguous()
        s["len_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["weights_out"] = torch.zeros((B, c["hkv"], out * P), dtype=torch.float32, device="cuda")
        s["kept"] = torch.full((B, c["hkv"], c["keep"]), -1, dtype=torch.int32, device="cuda")
    return s


# ---- the plain form -------------------------------------------------------------------------------------------------------
def _slot(t):
    """Where a block's token t stands in the key cache."""
    return 16 * (t // 4 % 2) + 4 * (t // 8) + t % 4


def _rows(s):
    """The sequence and the position in the cache of each new token."""
    t = torch.arange(s["qkv"].shape[0], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    return seq, (s["kv_len"][seq] - s["q_start"][seq + 1] + t).long()


def _rope(x, pos, freq, pairs):
    """x [T, heads, D] in 32 bits, turned; the angles in 64."""
    angle = (pos.double()[:, None] * freq.double())[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    if pairs:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _normed(x, gain):
    return x * (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt() * gain


def _plain_append(s):
    c, k, v = s["case"], s["k"], s["v"]
    hq, hkv, D, P = c["hq"], c["hkv"], c["d"], c["page"]
    T = s["qkv"].shape[0]
    seq, pos = _rows(s)
    x = s["qkv"].float().reshape(T, hq + 2 * hkv, D)
    normed = torch.cat([_normed(x[:, :hq], s["q_gain"]), _normed(x[:, hq:hq + hkv], s["k_gain"])], dim=1)
    turned = _rope(normed, pos if s["shift"] is None else pos + s["shift"][seq], s["freq"], c["pairs"]).to(torch.bfloat16)
    page, block, t = s["table"][seq, pos // P].long(), pos % P // 32, pos % 32
    keys = torch.nn.functional.pad(turned[:, hq:], (0, k.shape[3] * 8 - D)).reshape(T, hkv, -1, 8)
    k[page, :, block, :, _slot(t), :] = keys
    v.permute(0, 1, 2, 3, 5, 4)[page, :, block, t // 8, t % 8, :D] = x[:, hq + hkv:].to(torch.bfloat16)
    return [turned[:, :hq].contiguous(), k, v]


def _gathered(s):
    """Keys and values of all sequences in 32 bits, [B, kv heads, capacity, D]."""
    c, table = s["case"], s["table"].long()
    B, hkv, D, P = c["B"], c["hkv"], c["d"], c["page"]
    pos = torch.arange(table.shape[1] * P, device="cuda")
    page = table[:, pos // P]                                  # [B, capacity]
    if c["kind"] == "shared":                                  # a prefix lies on the pages of the first of its sequences
        group = torch.searchsorted(s["prefix_start"].long(), torch.arange(B, device="cuda"), right=True) - 1
        page = torch.where(pos < s["prefix_len"].long()[group][:, None], page[s["prefix_start"].long()[group]], page)
    block, t = pos % P // 32, pos % 32
    k = s["k"][page, :, block, :, _slot(t), :]                 # [B, capacity, kv heads, Dp / 8, 8]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, hkv, len(pos), -1)
    v = s["v"].permute(0, 1, 2, 3, 5, 4)[page, :, block, t // 8, t % 8, :]
    return k[..., :D].float(), v.permute(0, 2, 1, 3)[..., :D].float().contiguous()


def _plain_attention(s):
    c, q = s["case"], s["q"]
    B, hq, hkv, D = c["B"], c["hq"], c["hkv"], c["d"]
    k, v = _gathered(s)
    start, n = s["q_start"][:-1].long(), s["q_start"].diff().long()
    most = 1 if c["kind"] != "prompt" else max(new for _, new in _sizes(c))
    i = torch.arange(most, device="cuda")
    row = start[:, None] + i.minimum(n[:, None] - 1)           # [B, most]; behind a sequence's last token that one again
    there = i < n[:, None]
    qs = q[row].float().reshape(B, most, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D)
    pos = (s["kv_len"].long() - n)[:, None] + i
    j = torch.arange(k.shape[2], device="cuda")
    seen = (j <= pos[..., None])[:, None, None]                # [B, 1, 1, most, capacity]
    held = j < s["kv_len"].long()[:, None]                     # [B, capacity]
    p = qs @ k.transpose(2, 3).contiguous()
    del k
    p = p.mul_(D ** -0.5).reshape(B, hkv, -1, most, len(j)).masked_fill_(~seen, -math.inf)
    p = p.sub_(p.amax(dim=-1, keepdim=True)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = p.reshape(B, hkv, -1, len(j)) @ v.masked_fill_(~held[:, None, :, None], 0.0)
    o = (o.reshape(B, hkv, -1, most, D) / total).permute(0, 3, 1, 2, 4).reshape(B, most, hq * D)
    o = o[there].to(_dt(c["y"]))
    if c["kind"] == "shared":
        return o
    got = (p / total).masked_fill_(~there[:, None, None, :, None], 0.0).sum(dim=(2, 3))
    old = s["weights"].masked_fill(j >= (s["kv_len"].long() - n)[:, None, None], 0.0)      # new tokens begin with nothing
    s["weights"].copy_(torch.where(held[:, None], old + got, s["weights"]))
    return [o, s["weights"]]


def _plain_evict(s):
    c, k, v, w = s["case"], s["k"], s["v"], s["weights"]
    P, keep = c["page"], c["keep"]
    length = s["kv_len"].long()[:, None, None]
    j = torch.arange(w.shape[2], device="cuda")
    key = w.masked_fill(j >= length - c["recent"], math.inf).masked_fill(j >= length, -1.0)
    first = torch.sort(key, dim=2, descending=True, stable=True).indices[..., :keep]       # of equal ones the lower position
    i = torch.arange(first.shape[2], device="cuda")
    there = i < length.clamp(max=keep)
    at = torch.where(there, first, len(j)).sort(dim=2).values
    b, h, i = torch.nonzero(there.expand_as(at), as_tuple=True)
    p = at[b, h, i]
    s["kept"][b, h, i] = p.to(torch.int32)
    s["len_out"].copy_(s["kv_len"].clamp(max=keep))
    s["weights_out"][b, h, i] = w[b, h, p]
    page, to = s["table"].long()[b, p // P], s["table_out"].long()[b, i // P]
    k[to, h, i % P // 32, :, _slot(i % 32), :] = k[page, h, p % P // 32, :, _slot(p % 32), :]
    u = v.permute(0, 1, 2, 3, 5, 4)
    u[to, h, i % P // 32, i % 32 // 8, i % 8, :] = u[page, h, p % P // 32, p % 32 // 8, p % 8, :]
    return [k, v, s["len_out"], s["weights_out"], s["kept"]]


def run(s):
    c = s["case"]
    if not own:
        return _plain_append(s) if c["kind"] == "append" else _plain_evict(s) if c["kind"] == "evict" else _plain_attention(s)
    from paper_2402_17764_amd import binding as bitnet

    if c["kind"] == "append":
        q = bitnet.norm_rope_kv_append(s["qkv"], s["freq"], s["k"], s["v"], s["table"], s["kv_len"], c["hq"], s["q_gain"], s["k_gain"], EPS,
                                       q_start=None if c["one"] else s["q_start"], pairs=c["pairs"], shift=s["shift"])
        return [q, s["k"], s["v"]]
    if c["kind"] == "evict":
        bitnet.kv_evict(s["k"], s["v"], s["table"], s["kv_len"], s["weights"], c["keep"], c["recent"], s["table_out"], kv_len_out=s["len_out"],
                        weights_out=s["weights_out"], kept=s["kept"])
        return [s["k"], s["v"], s["len_out"], s["weights_out"], s["kept"]]
    y = bitnet.F32 if c["y"] == "f32" else bitnet.BF16
    if c["kind"] == "shared":
        return bitnet.attention_decode_shared(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["prefix_start"], s["prefix_len"], y_dtype=y)
    if c["kind"] == "decode":
        return [bitnet.attention_decode_weights(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["weights"], y_dtype=y), s["weights"]]
    return [bitnet.attention_prefill_weights(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["q_start"], s["weights"], y_dtype=y), s["weights"]]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    c, sizes = case, _sizes(case)
    hkv, D = c["hkv"], c["d"]
    cached = [old + new for old, new in sizes]
    if c["kind"] == "evict":
        kept = sum(min(n, c["keep"]) for n in cached)
        return {"bytes": hkv * (kept * (2 * D * 4 + 8) + sum(cached) * 4), "flops": 1.0 * hkv * sum(cached)}
    hq = c["hq"]
    T = sum(new for _, new in sizes)
    if c["kind"] == "append":
        width = (hq + 2 * hkv) * D
        return {"bytes": T * width * ((2 if c["x"] == "bf16" else 4) + 2), "flops": 7.0 * T * (hq + hkv) * D}
    pairs = sum(new * old + new * (new + 1) // 2 for old, new in sizes)
    read = sum(cached)
    if c["kind"] == "shared":
        start, prefix = _groups(c)
        read -= sum((start[i + 1] - start[i] - 1) * n for i, n in enumerate(prefix))
    rest = 0 if c["kind"] == "shared" else sum(cached) * hkv * 8
    return {"bytes": read * hkv * D * 4 + T * hq * D * (2 + (2 if c["y"] == "bf16" else 4)) + rest, "flops": 4.0 * pairs * hq * D}


# ---- the same in 64 bits, sequence by sequence ------------------------------------------------------------------------------
def _places(s, row, positions, head, values, D):
    """Indexes into the flat cache of the elements [positions, D] on the pages of the table's row."""
    c = s["case"]
    P, hkv = c["page"], c["hkv"]
    Dp = (c["d"] + 7) // 8 * 8
    d = torch.arange(D, device="cuda")[None, :]
    p = positions[:, None]
    block = (row.long()[p // P] * hkv + head) * (P // 32) + p % P // 32
    t = p % 32
    if values:
        return block * (32 * Dp) + (t // 8 * Dp + d) * 8 + t % 8
    return block * (32 * Dp) + (d // 8 * 32 + (t & 4) * 4 + (t >> 3) * 4 + (t & 3)) * 8 + d % 8


def _exact_append(s, sizes):
    c = s["case"]
    hq, hkv, D = c["hq"], c["hkv"], c["d"]
    x = s["qkv"].double().reshape(-1, hq + 2 * hkv, D)
    q, k, v = x[:, :hq].clone(), s["k"].double(), s["v"].double()
    first, second = (slice(0, D, 2), slice(1, D, 2)) if c["pairs"] else (slice(0, D // 2), slice(D // 2, D))
    row = 0
    for b, (old, new) in enumerate(sizes):
        pos = torch.arange(old, old + new, device="cuda")
        turned = pos if s["shift"] is None else pos + int(s["shift"][b])
        z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), turned.double()[:, None] * s["freq"].double())
        for h in range(hq + hkv):
            y = x[row:row + new, h]
            y = y / torch.sqrt((y * y).sum(dim=1, keepdim=True) / D + EPS) * s["q_gain" if h < hq else "k_gain"].double()
            w = torch.view_as_real(torch.complex(y[:, first].contiguous(), y[:, second].contiguous()) * z)
            out = torch.empty_like(y)
            out[:, first], out[:, second] = w[..., 0], w[..., 1]
            if h < hq:
                q[row:row + new, h] = out
            else:
                k.view(-1)[_places(s, s["table"][b], pos, h - hq, False, D)] = out
                v.view(-1)[_places(s, s["table"][b], pos, h - hq, True, D)] = x[row:row + new, h + hkv]
        row += new
    return [q, k, v]


def _exact_evict(s, sizes):
    c = s["case"]
    Dp = (c["d"] + 7) // 8 * 8
    k, v, w, kept = s["k"].double(), s["v"].double(), s["weights_out"].double(), s["kept"].clone()
    kf, vf = k.clone().view(-1), v.clone().view(-1)
    for b, (old, _) in enumerate(sizes):
        n = old + 1
        late = max(n - c["recent"], 0)
        for h in range(c["hkv"]):
            had = s["weights"][b, h, :late].tolist()
            chosen = sorted(range(late), key=lambda p: -had[p])[: max(c["keep"] - (n - late), 0)]
            at = torch.tensor(sorted(chosen) + list(range(late, n)), device="cuda")
            m = len(at)
            kept[b, h, :m] = at
            w[b, h, :m] = s["weights"][b, h, at].double()
            to = torch.arange(m, device="cuda")
            for flat, cache, values in ((kf, k, False), (vf, v, True)):
                flat[_places(s, s["table_out"][b], to, h, values, Dp)] = cache.view(-1)[_places(s, s["table"][b], at, h, values, Dp)]
    return [kf.view(k.shape), vf.view(v.shape), None, w, None]


def exact(case, seed):
    c, sizes = case, _sizes(case)
    s = prepare(case, seed)
    if c["kind"] == "append":
        return _exact_append(s, sizes)
    if c["kind"] == "evict":
        return _exact_evict(s, sizes)
    hq, hkv, D = c["hq"], c["hkv"], c["d"]
    o, row, g = [], 0, hq // hkv
    weights = s["weights"].double() if "weights" in s else None
    start, prefix = _groups(c) if c["kind"] == "shared" else ([], [])
    for b, (old, new) in enumerate(sizes):
        pos = torch.arange(old + new, device="cuda")
        out = torch.empty((new, hq, D), dtype=torch.float64, device="cuda")
        hidden = pos[None, :] > torch.arange(old, old + new, device="cuda")[:, None]
        i = max((i for i in range(len(prefix)) if start[i] <= b), default=None)
        for h in range(hkv):
            at = [_places(s, s["table"][b], pos, h, values, D) for values in (False, True)]
            if i is not None:
                n = prefix[i]
                at = [torch.cat([_places(s, s["table"][start[i]], pos[:n], h, values, D), at[values][n:]]) for values in (False, True)]
            k, v = s["k"].view(-1)[at[0]].double(), s["v"].view(-1)[at[1]].double()
            for e in range(h * g, h * g + g):
                p = (s["q"][row:row + new, e].double() @ k.t()) / math.sqrt(D)
                p = torch.softmax(p.masked_fill(hidden, -math.inf), dim=-1)
                out[:, e] = p @ v
                if weights is not None:
                    if e == h * g:
                        weights[b, h, old:old + new] = 0.0
                    weights[b, h, : old + new] += p.sum(dim=0)
        o.append(out.reshape(new, hq * D))
        row += new
    return torch.cat(o) if weights is None else [torch.cat(o), weights]
