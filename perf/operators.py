"""The attention half of a decoder layer as measurable cases: between the merged Q | K | V product and the output projection.

  append   rope_kv_append: the rows of a Q | K | V product are turned by their positions (rotary), q comes back, keys and values
           go into a paged cache.  One token for each sequence (decode), or a run of tokens for each (a prompt, or a chunk of one).
  decode   attention_decode: one new token of each sequence over its cached keys and values
  prompt   attention_prefill: runs of new tokens over their sequences' caches, causal (the new ones are in the cache already)

Sizes are those of the 700M ... 13B LLaMA-family layers of paper_2402_17764_amd.synth.CONFIGS (hidden 1536, 3200, 4096, 5120: 24 heads
of 64, 32 of 100, 32 of 128, 40 of 128), and grouped heads, 64 over 8, as at hidden 8192.

The cache.  Pages of `page` tokens (a multiple of 32) hold blocks of 32 tokens for each of the key-value heads; bf16.
  k_cache  [pages][kv heads][page / 32][Dp / 8][32][8]: 8 consecutive dims of a token together; token t of a block at slot
           16 ((t >> 2) & 1) + 4 (t >> 3) + (t & 3).  Dp: the head's dims rounded up to 8, zeros behind them.
  v_cache  [pages][kv heads][page / 32][4][Dp][8]: 8 consecutive tokens of a dim together
Position p of sequence b lies on page page_table[b][p // page]; kv_len[b] counts the cached tokens, the new ones included;
q_start[b] ... q_start[b + 1] are the rows of sequence b's new tokens, its last ones.
"""
import math

import torch

own = False

THETA = 10000.0


def listed():
    return [
        # the smallest call: one token of a 700M-class model into its cache, fp32 activations
        dict(name="append_700m_t1", kind="append", x="f32", hq=24, hkv=24, d=64, page=64, B=1, lo=511, hi=511, one=True, pairs=False),
        # an odd number of requests decoded together on a 7B-class model
        dict(name="append_7b_t29", kind="append", x="bf16", hq=32, hkv=32, d=128, page=128, B=29, lo=1, hi=500, one=True, pairs=False),
        # ragged chunks of prompts on a 3B-class model: heads of 100, chunks that start and end inside blocks, neighbouring pairs
        dict(name="append_3b_ragged", kind="append", x="bf16", hq=32, hkv=32, d=100, page=32, B=5, lo=0, hi=300, n_lo=1, n_hi=400, one=False, pairs=True),
        # two long prompts, grouped heads
        dict(name="append_gqa_prompts", kind="append", x="bf16", hq=64, hkv=8, d=128, page=256, B=2, lo=0, hi=0, n_lo=1900, n_hi=2300, one=False, pairs=False),
        # one request, a few hundred tokens in: latency alone
        dict(name="decode_700m_b1", kind="decode", y="f32", hq=24, hkv=24, d=64, page=64, B=1, lo=333, hi=333),
        # three requests on heads of 100, small pages
        dict(name="decode_3b_b3", kind="decode", y="bf16", hq=32, hkv=32, d=100, page=32, B=3, lo=700, hi=2047),
        # a batch of requests of very different lengths, a key-value head for each head: the bytes of the cache count
        dict(name="decode_7b_b29", kind="decode", y="bf16", hq=32, hkv=32, d=128, page=128, B=29, lo=1, hi=4096),
        # three long contexts, grouped heads: few rows, a long axis
        dict(name="decode_gqa_long", kind="decode", y="bf16", hq=64, hkv=8, d=128, page=256, B=3, lo=20000, hi=49152),
        # a short prompt of a 700M-class model
        dict(name="prompt_700m_t77", kind="prompt", y="f32", hq=24, hkv=24, d=64, page=64, B=1, lo=0, hi=0, n_lo=77, n_hi=77),
        # chunks of several requests' prompts together, ragged, heads of 100
        dict(name="prompt_3b_ragged", kind="prompt", y="bf16", hq=32, hkv=32, d=100, page=32, B=6, lo=0, hi=500, n_lo=1, n_hi=900),
        # a prompt of 2048 tokens of a 13B-class model
        dict(name="prompt_13b_t2048", kind="prompt", y="bf16", hq=40, hkv=40, d=128, page=128, B=1, lo=0, hi=0, n_lo=2048, n_hi=2048),
        # the largest: a chunk of 1024 tokens at the end of a long context, grouped heads
        dict(name="prompt_gqa_chunk", kind="prompt", y="bf16", hq=64, hkv=8, d=128, page=256, B=1, lo=15000, hi=15000, n_lo=1024, n_hi=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["append", "decode", "decode", "prompt", "prompt"])
    d = rng.choice([64, 80, 96, 100, 128, 128, 128])
    hkv, g = rng.choice([(24, 1), (32, 1), (40, 1), (8, 8), (8, 4), (4, 7), (16, 2), (1, 12)])
    c = dict(kind=kind, hq=hkv * g, hkv=hkv, d=d, page=rng.choice([32, 64, 96, 128, 256]))
    dt = rng.choice(["bf16", "bf16", "f32"])
    if kind == "decode":
        B = _log(rng, 1, 64)
        hi = _log(rng, 1, max(64, min(49152, 400_000_000 // (B * hkv * d * 4))))
        return dict(c, y=dt, B=B, lo=rng.randint(1, hi), hi=hi)
    if kind == "append" and rng.random() < 0.5:
        return dict(c, x=dt, B=_log(rng, 1, 64), lo=0, hi=_log(rng, 8, 500), one=True, pairs=rng.random() < 0.3)
    B = rng.randint(1, 6)
    n_hi = _log(rng, 1, 4096 // B)
    n_lo = rng.randint(1, n_hi)
    hi = rng.choice([0, _log(rng, 1, 2000)])
    if kind == "append":
        return dict(c, x=dt, B=B, lo=rng.randint(0, hi), hi=hi, n_lo=n_lo, n_hi=n_hi, one=False, pairs=rng.random() < 0.3)
    while B * n_hi * (n_hi + hi) * hkv * g > 1024 * 16024 * 64:
        n_hi = n_hi // 2 + 1
    return dict(c, y=dt, B=B, lo=rng.randint(0, hi), hi=hi, n_lo=min(n_lo, n_hi), n_hi=n_hi)


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, spread evenly over the range in a shuffled order."""
    return [lo + int((0.5 + b * 0.6180339887498949) % 1.0 * (hi - lo + 1)) for b in range(n)]


def _sizes(c):
    """(cached tokens before the call, new tokens) of each sequence; a decoded token is in the cache already."""
    if c["kind"] == "decode":
        return [(n - 1, 1) for n in _spread(c["B"], c["lo"], c["hi"])]
    old = _spread(c["B"], c["lo"], c["hi"])
    return list(zip(old, [1] * c["B"] if c.get("one") else _spread(c["B"], c["n_lo"], c["n_hi"])))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _gen(seed, tensor):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 64 + tensor) % (1 << 62))


def _dt(s):
    return torch.bfloat16 if s == "bf16" else torch.float32


def _normal(seed, tensor, shape, dt, std=1.0):
    return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, std, generator=_gen(seed, tensor))


def prepare(case, seed):
    c, sizes = case, _sizes(case)
    B, D, P = c["B"], c["d"], c["page"]
    Dp = (D + 7) // 8 * 8
    per = max(-(-(old + new) // P) for old, new in sizes)
    T = sum(new for _, new in sizes)
    s = {"case": dict(c)}
    pages = B * per + 2
    s["table"] = torch.randperm(pages, device="cuda", generator=_gen(seed, 0))[: B * per].reshape(B, per).to(torch.int32)
    s["kv_len"] = torch.tensor([old + new for old, new in sizes], dtype=torch.int32, device="cuda")
    starts = [0]
    for _, new in sizes:
        starts.append(starts[-1] + new)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["k"] = _normal(seed, 1, (pages, c["hkv"], P // 32, Dp // 8, 32, 8), torch.bfloat16)
    s["k"][:, :, :, -1, :, 8 - (Dp - D):] = 0
    s["v"] = _normal(seed, 2, (pages, c["hkv"], P // 32, 4, Dp, 8), torch.bfloat16)
    if c["kind"] == "append":
        s["qkv"] = _normal(seed, 3, (T, (c["hq"] + 2 * c["hkv"]) * D), _dt(c["x"]))
        s["freq"] = (THETA ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).to(device="cuda", dtype=torch.float32)
    else:
        s["q"] = _normal(seed, 4, (T, c["hq"], D), torch.bfloat16, 1.5)
    return s


# ---- the plain form -------------------------------------------------------------------------------------------------------
def _slot(t):
    """Where a block's token t stands in the key cache."""
    return 16 * (t // 4 % 2) + 4 * (t // 8) + t % 4


def _rows(s):
    """The sequence and the position of each new token."""
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


def _plain_append(s):
    c, k, v = s["case"], s["k"], s["v"]
    hq, hkv, D, P = c["hq"], c["hkv"], c["d"], c["page"]
    T = s["qkv"].shape[0]
    seq, pos = _rows(s)
    x = s["qkv"].float().reshape(T, hq + 2 * hkv, D)
    turned = _rope(x[:, : hq + hkv], pos, s["freq"], c["pairs"]).to(torch.bfloat16)
    page, block, t = s["table"][seq, pos // P].long(), pos % P // 32, pos % 32
    keys = torch.nn.functional.pad(turned[:, hq:], (0, k.shape[3] * 8 - D)).reshape(T, hkv, -1, 8)
    k[page, :, block, :, _slot(t), :] = keys
    v.permute(0, 1, 2, 3, 5, 4)[page, :, block, t // 8, t % 8, :D] = x[:, hq + hkv:].to(torch.bfloat16)
    return [turned[:, :hq].contiguous(), k, v]


def _gathered(s):
    """Keys and values of all sequences in 32 bits, [B, kv heads, capacity, D]."""
    c, table = s["case"], s["table"].long()
    B, hkv, D = c["B"], c["hkv"], c["d"]
    k = s["k"][table]                                        # [B, pages, kv heads, blocks, Dp / 8, slot, 8]
    k = k[..., _slot(torch.arange(32, device="cuda")), :].permute(0, 2, 1, 3, 5, 4, 6).reshape(B, hkv, -1, k.shape[4] * 8)
    v = s["v"][table]                                        # [B, pages, kv heads, blocks, 4, Dp, 8]
    v = v.permute(0, 2, 1, 3, 4, 6, 5).reshape(B, hkv, -1, v.shape[5])
    return k[..., :D].float(), v[..., :D].float()


def _plain_attention(s):
    c, q = s["case"], s["q"]
    B, hq, hkv, D = c["B"], c["hq"], c["hkv"], c["d"]
    k, v = _gathered(s)
    start, n = s["q_start"][:-1].long(), s["q_start"].diff().long()
    most = 1 if c["kind"] == "decode" else max(new for _, new in _sizes(c))
    i = torch.arange(most, device="cuda")
    row = start[:, None] + i.minimum(n[:, None] - 1)         # [B, most]; behind a sequence's last token that one again
    qs = q[row].float().reshape(B, most, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, D)
    pos = (s["kv_len"].long() - n)[:, None] + i
    j = torch.arange(k.shape[2], device="cuda")
    seen = (j <= pos[..., None])[:, None, None]              # [B, 1, 1, most, capacity]
    held = (j < s["kv_len"][:, None])[:, None, :, None]
    p = qs @ k.transpose(2, 3).contiguous()
    p = p.mul_(D ** -0.5).reshape(B, hkv, -1, most, k.shape[2]).masked_fill_(~seen, -math.inf)
    p = p.sub_(p.amax(dim=-1, keepdim=True)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = p.reshape(B, hkv, -1, k.shape[2]) @ v.masked_fill_(~held, 0.0)
    o = (o.reshape(B, hkv, -1, most, D) / total).permute(0, 3, 1, 2, 4).reshape(B, most, hq * D)
    return o[i < n[:, None]].to(_dt(c["y"]))


def run(s):
    c = s["case"]
    if not own:
        return _plain_append(s) if c["kind"] == "append" else _plain_attention(s)
    from paper_2402_17764_amd import binding as bitnet

    if c["kind"] == "append":
        q = bitnet.rope_kv_append(s["qkv"], s["freq"], s["k"], s["v"], s["table"], s["kv_len"], c["hq"],
                                  q_start=None if c["one"] else s["q_start"], pairs=c["pairs"])
        return [q, s["k"], s["v"]]
    y = bitnet.F32 if c["y"] == "f32" else bitnet.BF16
    if c["kind"] == "decode":
        return bitnet.attention_decode(s["q"], s["k"], s["v"], s["table"], s["kv_len"], y_dtype=y)
    return bitnet.attention_prefill(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["q_start"], y_dtype=y)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    c, sizes = case, _sizes(case)
    hq, hkv, D = c["hq"], c["hkv"], c["d"]
    T = sum(new for _, new in sizes)
    if c["kind"] == "append":
        width = (hq + 2 * hkv) * D
        return {"bytes": T * width * ((2 if c["x"] == "bf16" else 4) + 2), "flops": 3.0 * T * (hq + hkv) * D}
    pairs = sum(new * old + new * (new + 1) // 2 for old, new in sizes)
    cached = sum(old + new for old, new in sizes)
    return {"bytes": cached * hkv * D * 4 + T * hq * D * (2 + (2 if c["y"] == "bf16" else 4)), "flops": 4.0 * pairs * hq * D}


# ---- the same in 64 bits, sequence by sequence ------------------------------------------------------------------------------
def _places(s, b, positions, head, values):
    """Indexes into the flat cache of the elements [positions, D] of sequence b."""
    c = s["case"]
    D, P, hkv = c["d"], c["page"], c["hkv"]
    Dp = (D + 7) // 8 * 8
    d = torch.arange(D, device="cuda")[None, :]
    p = positions[:, None]
    block = (s["table"][b].long()[p // P] * hkv + head) * (P // 32) + p % P // 32
    t = p % 32
    if values:
        return block * (32 * Dp) + (t // 8 * Dp + d) * 8 + t % 8
    return block * (32 * Dp) + (d // 8 * 32 + (t & 4) * 4 + (t >> 3) * 4 + (t & 3)) * 8 + d % 8


def exact(case, seed):
    c, sizes = case, _sizes(case)
    s = prepare(case, seed)
    hq, hkv, D = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "append":
        x = s["qkv"].double().reshape(-1, hq + 2 * hkv, D)
        q, k, v = x[:, :hq].clone(), s["k"].double(), s["v"].double()
        first, second = (slice(0, D, 2), slice(1, D, 2)) if c["pairs"] else (slice(0, D // 2), slice(D // 2, D))
        row = 0
        for b, (old, new) in enumerate(sizes):
            pos = torch.arange(old, old + new, device="cuda")
            z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * s["freq"].double())
            for h in range(hq + hkv):
                y = x[row:row + new, h]
                w = torch.view_as_real(torch.complex(y[:, first].contiguous(), y[:, second].contiguous()) * z)
                out = torch.empty_like(y)
                out[:, first], out[:, second] = w[..., 0], w[..., 1]
                if h < hq:
                    q[row:row + new, h] = out
                else:
                    k.view(-1)[_places(s, b, pos, h - hq, False)] = out
                    v.view(-1)[_places(s, b, pos, h - hq, True)] = x[row:row + new, h + hkv]
            row += new
        return [q, k, v]
    o, row, g = [], 0, hq // hkv
    for b, (old, new) in enumerate(sizes):
        pos = torch.arange(old + new, device="cuda")
        out = torch.empty((new, hq, D), dtype=torch.float64, device="cuda")
        hidden = pos[None, :] > torch.arange(old, old + new, device="cuda")[:, None]
        for h in range(hkv):
            k, v = s["k"].view(-1)[_places(s, b, pos, h, False)].double(), s["v"].view(-1)[_places(s, b, pos, h, True)].double()
            for i in range(h * g, h * g + g):
                p = (s["q"][row:row + new, i].double() @ k.t()) / math.sqrt(D)
                out[:, i] = torch.softmax(p.masked_fill(hidden, -math.inf), dim=-1) @ v
        o.append(out.reshape(new, hq * D))
        row += new
    return torch.cat(o)
