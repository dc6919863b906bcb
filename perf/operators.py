"""Cases of the paged key/value cache: appending to it (with the position rotation on the way) and attention over it,
with a 16-bit cache and with an e4m3 cache that has a scale for each page and head.

A batch is packed: sequence b has the rows q_start[b] .. q_start[b+1]-1 of Q, K, V, which are its last ones, and
kv_lens[b] keys in the cache after they have been appended.  A cache is [pages, Hkv, page, D]; page_table[b] lists the
pages of sequence b."""
import random

import torch

own = False

E4M3_MAX = 448.0
MIN_EXPONENT = -100  # of a page's scale
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

COMMON = dict(Hq=32, Hkv=8, D=128, page=64, dtype="bf16", causal=True, chunk=0)


def listed():
    def c(name, op, **kw):
        return {"name": name, "op": op, **COMMON, **kw}
    return [
        # one new token for each of a few sequences: what a decoding step of one layer appends; latency
        c("append_decode", "append", cache="16", B=8, q_lo=1, q_hi=1, ctx_lo=100, ctx_hi=4096, lens=1),
        # a batch of prompts and continuations of odd lengths, fp16
        c("append_prompts", "append", cache="16", B=7, q_lo=300, q_hi=4096, ctx_lo=0, ctx_hi=1500, lens=2, dtype="fp16",
          page=16),
        # a decoding step of a large batch into the 8-bit cache: most tokens land in a page that has others
        c("append8_decode", "append", cache="e4m3", B=64, q_lo=1, q_hi=1, ctx_lo=10, ctx_hi=4096, lens=3),
        # prompts into the 8-bit cache
        c("append8_prompts", "append", cache="e4m3", B=5, q_lo=700, q_hi=6000, ctx_lo=0, ctx_hi=900, lens=4),
        # the smallest decoding call: two sequences, a few hundred keys; latency
        c("decode_small", "attention", cache="16", B=2, Hq=8, Hkv=2, D=64, q_lo=1, q_hi=1, ctx_lo=150, ctx_hi=299,
          lens=5, dtype="fp16", page=16),
        # one new token each against an 8K cache, grouped heads
        c("decode", "attention", cache="16", B=8, q_lo=1, q_hi=1, ctx_lo=8191, ctx_hi=8191, lens=6),
        # speculative decoding: four new tokens each, lengths of a running batch
        c("spec_decode", "attention", cache="16", B=16, q_lo=4, q_hi=4, ctx_lo=500, ctx_hi=16000, lens=7, page=32),
        # a chunk of a prompt after the cached ones
        c("prefill_chunk", "attention", cache="16", B=1, q_lo=512, q_hi=512, ctx_lo=3584, ctx_hi=3584, lens=8),
        # whole prompts of different lengths
        c("prompts", "attention", cache="16", B=6, q_lo=1000, q_hi=8000, ctx_lo=0, ctx_hi=0, lens=9),
        # a running batch of 64 sequences of very different lengths on the 8-bit cache
        c("decode8_ragged", "attention", cache="e4m3", B=64, q_lo=1, q_hi=1, ctx_lo=100, ctx_hi=16000, lens=10),
        # one long document: few rows, many keys
        c("decode8_long", "attention", cache="e4m3", B=1, Hq=64, q_lo=1, q_hi=1, ctx_lo=131071, ctx_hi=131071, lens=11),
        # a chunk of one sequence's prompt beside the decoding of the others
        c("mixed8", "attention", cache="e4m3", B=16, q_lo=1, q_hi=1, ctx_lo=200, ctx_hi=8000, lens=12, chunk=512),
    ]


def lengths(c):
    """(rows, keys after the call) of each sequence: by the case alone."""
    r = random.Random("lengths %d" % c["lens"])

    def spread(lo, hi):
        return lo if hi <= lo else min(hi, int((lo + 1) * ((hi + 1) / (lo + 1)) ** r.random()))
    n = [spread(c["q_lo"], c["q_hi"]) for _ in range(c["B"])]
    if c["chunk"]:
        n[r.randrange(c["B"])] = c["chunk"]
    return n, [spread(c["ctx_lo"], c["ctx_hi"]) + x for x in n]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))
    most = max(cost(c) for c in listed())
    while True:
        op = rng.choice(("append", "attention"))
        cache = rng.choice(("16", "e4m3"))
        hkv = rng.choice((1, 2, 4, 8))
        d = rng.choice((64, 80, 96, 128, 128, 192, 256) + ((72, 104, 200) if cache == "16" else ()))
        c = dict(COMMON, op=op, cache=cache, Hkv=hkv, Hq=hkv * rng.choice((1, 2, 4, 5, 8)), D=d,
                 page=rng.choice((16, 32, 64, 128)), dtype=rng.choice(("bf16", "fp16")),
                 causal=rng.random() < 0.85, lens=rng.randrange(1 << 30))
        kind = rng.choice(("one", "few", "chunks", "mixed"))
        c["B"] = log(1, 96) if kind in ("one", "mixed") else log(1, 24)
        c["q_lo"], c["q_hi"] = {"one": (1, 1), "few": (1, log(2, 9)), "chunks": (1, log(20, 3000)),
                                "mixed": (1, 1)}[kind]
        c["chunk"] = log(30, 1500) if kind == "mixed" else 0
        c["ctx_hi"] = log(100, 60000 if kind == "one" and op == "attention" and c["B"] < 8 else 12000)
        c["ctx_lo"] = rng.randrange(0, c["ctx_hi"] + 1) if rng.random() < 0.5 else 0
        n, kv = lengths(c)
        wide = c["B"] * max(kv) * (c["Hq"] * max(n) + 4 * hkv * d)  # values of the padded batch
        if (wide <= 3e9 or op == "append") and cost(c) <= most:
            return c


def cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def work(c):
    n, kv = lengths(c)
    t, hq, hkv, d = sum(n), c["Hq"], c["Hkv"], c["D"]
    size = 2 if c["cache"] == "16" else 1
    if c["op"] == "append":
        # the tokens in and out, and the rotation's two tables
        moved = t * (2 * hkv + hq) * d * 2 + t * (2 * hkv * size + hq * 2) * d + t * d * 4
        return {"bytes": moved, "flops": 3 * t * (hq + hkv) * d}
    pairs = sum(i * k - (i * (i - 1) // 2 if c["causal"] else 0) for i, k in zip(n, kv))
    moved = sum(kv) * 2 * hkv * d * size + t * hq * (2 * d * 2 + 4)
    return {"bytes": moved, "flops": 4 * pairs * hq * d}


def scale_of(amax):
    """The least power of two, 2^-100 at least, by which values of up to amax fit e4m3."""
    f, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (f > 0.875).to(e.dtype), e.new_full((), MIN_EXPONENT))
    return torch.ldexp(torch.ones_like(amax), e.clamp(min=MIN_EXPONENT))


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    n, kv = lengths(c)
    hq, hkv, d, page, dt = c["Hq"], c["Hkv"], c["D"], c["page"], TYPES[c["dtype"]]
    b, t = c["B"], sum(n)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=dev)
    width = max(-(-k // page) for k in kv)
    used = sum(-(-k // page) for k in kv)
    pages = used + used // 8 + 2
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((b, width), -1, dtype=torch.int32)
    order, at = order.cpu(), 0
    for i, k in enumerate(kv):
        m = -(-k // page)
        table[i, :m] = order[at:at + m]
        at += m
    s = {"op": c["op"], "cache": c["cache"], "causal": c["causal"], "scale": d ** -0.5, "page": page,
         "max_q": max(n), "max_kv": max(kv), "touched": sum((k - 1) // page - (k - m) // page + 1 for m, k in zip(n, kv)),
         "page_table": table.to(dev), "kv_lens": torch.tensor(kv, dtype=torch.int32, device=dev),
         "q_start": torch.tensor([0] + [sum(n[:i + 1]) for i in range(b)], dtype=torch.int32, device=dev),
         "q": randn(t, hq, d).to(dt), "k_scale": None, "v_scale": None}
    # what the cache holds: pages of different magnitudes, as tokens are
    for x in ("k", "v"):
        values = randn(pages, hkv, page, d)
        values *= torch.exp(0.4 * randn(pages, 1, 1, 1))
        if c["cache"] == "16":
            s[x + "_cache"] = values.to(dt)
        else:
            by = scale_of(values.abs().amax((2, 3)))
            s[x + "_cache"] = (values / by[:, :, None, None]).to(torch.float8_e4m3fn)
            s[x + "_scale"] = by
        del values
    if c["op"] == "append":
        gain = torch.exp(0.4 * randn(t, 1, 1))
        s["k"], s["v"] = (randn(t, hkv, d) * gain).to(dt), (randn(t, hkv, d) * gain).to(dt)
        angle = torch.arange(width * page, device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(d // 2, device=dev, dtype=torch.float64) * 2 / d)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    return s


def run(s):
    if own:
        import paper_2601_16238_amd as attn
        if s["op"] == "append":
            q = attn.attn_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["page_table"], s["q_start"],
                                       s["kv_lens"], cos=s["cos"], sin=s["sin"], Q=s["q"], k_scale=s["k_scale"],
                                       v_scale=s["v_scale"])
            return appended(s, q)
        o, lse = attn.attn_fwd_paged(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["q_start"], s["kv_lens"],
                                     s["scale"], s["causal"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                     max_q=s["max_q"])
        return {"o": o, "lse": lse}
    return plain_append(s) if s["op"] == "append" else plain_attention(s)


def appended(s, q):
    r = {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if s["cache"] != "16":
        r["k_scale"], r["v_scale"] = s["k_scale"], s["v_scale"]
    return r


def rows_of(s):
    """Sequence, row in the sequence and position of each packed row."""
    start = s["q_start"].long()
    t = torch.arange(s["q"].shape[0], device=start.device)
    seq = torch.searchsorted(start, t, right=True) - 1
    i = t - start[seq]
    return seq, i, s["kv_lens"].long()[seq] - (start[seq + 1] - start[seq]) + i


def rotated(x, cos, sin):
    half = x.shape[-1] // 2
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def plain_append(s):
    seq, _, pos = rows_of(s)
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    q = rotated(s["q"], cos, sin).to(s["q"].dtype)
    k, v = rotated(s["k"], cos, sin), s["v"].float()
    if s["cache"] == "16":
        page = s["page_table"].long()[seq, pos // s["page"]]
        s["k_cache"][page, :, pos % s["page"]] = k.to(s["k_cache"].dtype)
        s["v_cache"][page, :, pos % s["page"]] = v.to(s["v_cache"].dtype)
        return appended(s, q)
    # the pages that get tokens, one after the other
    P, dev = s["page"], q.device
    start, new_len = s["q_start"].long(), s["kv_lens"].long()
    old_len = new_len - (start[1:] - start[:-1])
    first = old_len // P
    count = torch.where(new_len > old_len, (new_len - 1) // P - first + 1, 0)
    of = torch.repeat_interleave(torch.arange(len(count), device=dev), count, output_size=s["touched"])
    slot = first[of] + torch.arange(s["touched"], device=dev) - (count.cumsum(0) - count)[of]
    page = s["page_table"].long()[of, slot]
    at = slot[:, None] * P + torch.arange(P, device=dev)  # positions, [pages, P]
    older = (at < old_len[of][:, None])[:, None, :, None]
    newer = ((at >= old_len[of][:, None]) & (at < new_len[of][:, None]))[:, None, :, None]
    row = (start[of][:, None] + at - old_len[of][:, None]).clamp(0, q.shape[0] - 1)
    has_older = (slot * P < old_len[of])[:, None]
    for x, cache, scales in ((k, s["k_cache"], s["k_scale"]), (v, s["v_cache"], s["v_scale"])):
        x = torch.where(newer, x[row].transpose(1, 2), 0.0)
        before, codes = scales[page], cache[page]
        by = scale_of(x.abs().amax((2, 3)))
        by = torch.where(has_older, torch.maximum(by, before), by)
        grown = codes.float() * (before / by)[:, :, None, None]
        moved = torch.where(newer, x / by[:, :, None, None], grown).clamp(-E4M3_MAX, E4M3_MAX).to(codes.dtype)
        bits = torch.where(newer | older, moved.view(torch.uint8), codes.view(torch.uint8))
        cache.view(torch.uint8)[page] = bits
        scales[page] = by
    return appended(s, q)


def plain_attention(s):
    dev, P, B = s["q"].device, s["page"], s["kv_lens"].shape[0]
    T, hq, d = s["q"].shape
    hkv = s["k_cache"].shape[1]
    start, length = s["q_start"].long(), s["kv_lens"].long()
    n = start[1:] - start[:-1]
    pages = -(-s["max_kv"] // P)
    table = s["page_table"].long()[:, :pages].clamp(min=0)
    key = torch.arange(pages * P, device=dev)
    there = key < length[:, None]  # [B, L]

    def gathered(cache, scales):
        x = cache[table].float()  # [B, pages, Hkv, P, D]
        if scales is not None:
            x *= scales[table][:, :, :, None, None]
        return x.transpose(1, 2).reshape(B, hkv, pages * P, d)
    i = torch.arange(s["max_q"], device=dev)
    q = s["q"][(start[:-1, None] + i).clamp(max=T - 1)].float()  # [B, max_q, Hq, D]
    q = q.view(B, -1, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, d)
    x = q @ gathered(s["k_cache"], s["k_scale"]).transpose(2, 3)
    x = x.mul_(s["scale"]).view(B, hkv, hq // hkv, s["max_q"], -1)
    seen = there[:, None].expand(-1, s["max_q"], -1)
    if s["causal"]:
        seen = seen & (key <= (length - n)[:, None, None] + i[:, None])
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    v = torch.where(there[:, None, :, None], gathered(s["v_cache"], s["v_scale"]), 0.0)
    o = (p.view(B, hkv, -1, pages * P) @ v).view(B, hkv, hq // hkv, -1, d)
    o = torch.where(total > 0, o / total, 0.0)
    seq, row, _ = rows_of(s)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, -1, hq, d)[seq, row]
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, -1, hq)[seq, row]
    return {"o": o.to(s["q"].dtype), "lse": lse}


def exact(case, seed):
    """Sequence by sequence in 64 bits.  Stored values are given as they are before they are rounded."""
    s, c = prepare(case, seed), case
    n, kv = lengths(c)
    P, eight = c["page"], c["cache"] != "16"
    if sum(k * m for k, m in zip(kv, n)) * c["Hq"] * c["D"] > 1e13 or sum(n) > 200000:
        return None
    table = s["page_table"].tolist()
    first = [sum(n[:b]) for b in range(c["B"])]
    if c["op"] == "attention":
        o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            ids = torch.tensor(table[b][:-(-kv[b] // P)], device="cuda")

            def dense(name):
                x = s[name + "_cache"][ids].double()
                if eight:
                    x = x * s[name + "_scale"][ids].double()[..., None, None]
                return x.transpose(0, 1).flatten(1, 2)[:, :kv[b]]
            keys, values = dense("k"), dense("v")
            rows = slice(first[b], first[b] + n[b])
            group = c["Hq"] // c["Hkv"]
            hidden = None
            if c["causal"]:
                hidden = torch.ones(n[b], kv[b], dtype=torch.bool, device="cuda").triu(kv[b] - n[b] + 1)
            for h in range(c["Hq"]):
                x = s["q"][rows, h].double() @ keys[h // group].T * s["scale"]
                if hidden is not None:
                    x = x.masked_fill(hidden, -torch.inf)
                total = torch.logsumexp(x, -1)
                lse[rows, h] = total
                o[rows, h] = torch.exp(x - total[:, None]) @ values[h // group]
        return {"o": o, "lse": lse}
    pos = torch.cat([torch.arange(k - m, k, device="cuda") for m, k in zip(n, kv)])
    turn = torch.complex(s["cos"].double(), s["sin"].double())[pos][:, None]

    def turned(x):
        half = x.shape[-1] // 2
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * turn
        return torch.cat((z.real, z.imag), -1)
    r = {"q": turned(s["q"])}
    for name, x in (("k", turned(s["k"])), ("v", s["v"].double())):
        cache = s[name + "_cache"].double()
        scales = s[name + "_scale"].double() if eight else None
        for b in range(c["B"]):
            lo = kv[b] - n[b]
            while lo < kv[b]:
                p, hi = lo // P, min(kv[b], (lo // P + 1) * P)
                at = first[b] + lo - (kv[b] - n[b])
                new, g = x[at:at + hi - lo].transpose(0, 1), table[b][p]  # [Hkv, tokens, D]
                if eight:
                    by = torch.exp2(torch.ceil(torch.log2(new.abs().amax((1, 2)) / E4M3_MAX)).clamp(min=MIN_EXPONENT))
                    if lo > p * P:
                        by = torch.maximum(by, scales[g])
                        cache[g, :, :lo - p * P] *= (scales[g] / by)[:, None, None]
                    scales[g] = by
                    new = new / by[:, None, None]
                cache[g, :, lo - p * P:hi - p * P] = new
                lo = hi
        r[name + "_cache"] = cache
        if eight:
            r[name + "_scale"] = scales
    return r
