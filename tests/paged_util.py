"""Batches over a paged cache, and comparisons with the 64-bit implementation."""
import random

import torch

import paper_2601_16238_amd as attn
from oracle import paged_oracle as po

E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


class Batch:
    """Sequences of n rows and a length each, over a cache whose unused places are all NaN: pages of nobody, slots
    behind a sequence's last key (from `filled` keys on), their scales, and rows of Q, K, V behind the last sequence."""

    def __init__(self, seqs, Hq, Hkv, D, P, dtype="bf16", e4m3=False, seed=0, layout="HND", behind=0, spare=3,
                 filled=None, table_pad=0, gain=1.0, scales="powers"):
        g = torch.Generator().manual_seed(seed)
        rnd = random.Random(seed)
        self.dt, self.e4m3, self.P = TYPES[dtype], e4m3, P
        self.n, self.len = [s[0] for s in seqs], [s[1] for s in seqs]
        self.T, B = sum(self.n) + behind, len(seqs)
        used = [-(-k // P) for k in self.len]
        width = max([1] + used) + table_pad
        pages = sum(used) + spare
        ids = list(range(pages))
        rnd.shuffle(ids)
        self.table = torch.full((B, width), -7, dtype=torch.int32)
        for b, m in enumerate(used):
            self.table[b, :m] = torch.tensor([ids.pop() for _ in range(m)], dtype=torch.int32)
        self.q_start = torch.tensor([sum(self.n[:b]) for b in range(B + 1)], dtype=torch.int32)
        self.kv_lens = torch.tensor(self.len, dtype=torch.int32)

        def rows(*shape):
            x = (torch.randn(*shape, generator=g) * gain).to(self.dt)
            x[sum(self.n):] = float("nan")
            return x
        self.q, self.k, self.v = rows(self.T, Hq, D), rows(self.T, Hkv, D), rows(self.T, Hkv, D)
        filled = self.len if filled is None else filled
        self.cache, self.scale = [], []
        for _ in range(2):
            nan = torch.full((pages, Hkv, P, D), float("nan"))
            scale = torch.full((pages, Hkv), float("nan"))
            for b, m in enumerate(used):
                for w in range(m):
                    page, there = int(self.table[b, w]), min(P, filled[b] - w * P)
                    if there <= 0:
                        continue
                    x = torch.randn(Hkv, there, D, generator=g) * gain * 2.0 ** rnd.uniform(-2, 2)
                    if e4m3:
                        amax = x.abs().amax((1, 2))
                        s = amax / 448 if scales == "any" else torch.tensor([po.e4m3_scale(a) for a in amax.double()])
                        scale[page] = s
                        x = x / s[:, None, None]
                    nan[page, :, :there] = x
            x = nan.to(E4M3 if e4m3 else self.dt)
            if layout == "NHD":
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
            elif layout == "padded":
                big = torch.full((pages, Hkv + 1, P + 2, D + 16), float("nan")).to(x.dtype)
                big[:, :Hkv, :P, :D] = x
                x = big[:, :Hkv, :P, :D]
            self.cache.append(x)
            self.scale.append(scale)

    def scales(self):
        return tuple(self.scale) if self.e4m3 else (None, None)

    def on_gpu(self):
        """The tensors of a call, each with its layout."""
        def to(x):
            big = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
            if x.untyped_storage().nbytes() != x.numel() * x.itemsize:  # a view: with what lies between
                base = torch.empty(0, dtype=x.dtype).set_(x.untyped_storage()).cuda()
                return base.as_strided(x.shape, x.stride(), x.storage_offset())
            big.view(torch.uint8).copy_(x.view(torch.uint8)) if x.dtype == E4M3 else big.copy_(x)
            return big
        ks, vs = self.scales()
        return dict(q=to(self.q), k=to(self.k), v=to(self.v), kc=to(self.cache[0]), vc=to(self.cache[1]),
                    table=to(self.table), q_start=to(self.q_start), kv_lens=to(self.kv_lens),
                    ks=None if ks is None else to(ks), vs=None if vs is None else to(vs))


def step(t):
    """Half a step of the type relative to the value."""
    return torch.finfo(t).eps / 2


def call(g, scale, causal, **kw):
    return attn.attn_fwd_paged(g["q"], g["kc"], g["vc"], g["table"], g["q_start"], g["kv_lens"], scale, causal,
                               k_scale=g["ks"], v_scale=g["vs"], **kw)


def check_attention(b, o, lse, causal, scale=None, **changed):
    """Every element.  With e the type's half step: e |o| for the last rounding; 2 e sum p |v| for the probabilities,
    each rounded once, and their sum, which is of the rounded or of the exact ones; fp16 probabilities below 2^-14 are
    multiples of 2^-24: half of one for each key, on a sum of at least one.  The scores: D + 2 additions of 2^-24 of
    the largest partial sum, and as much for exp2 of an argument of its size; the row sums: one more for every key."""
    scale = b.q.shape[-1] ** -0.5 if scale is None else scale
    a = dict(q=b.q, k_cache=b.cache[0].float(), v_cache=b.cache[1].float(), table=b.table, q_start=b.q_start,
             kv_lens=b.kv_lens)
    a.update(changed)
    ks, vs = b.scales()
    ro, rl, spread, size = po.attention(**a, scale=scale, causal=causal, k_scale=ks, v_scale=vs)
    rows = int(b.q_start[-1])
    D, e, ulp = b.q.shape[-1], step(b.dt), 2.0 ** -24
    ro, rl, spread, size = ro[:rows], rl[:rows], spread[:rows], size[:rows]
    o, lse = o[:rows].double().cpu(), lse[:rows].double().cpu()
    keys = max([1] + b.len)
    score = ulp * (2 * (D + 2) * size + 8)
    empty = rl == -torch.inf
    assert torch.equal(lse == -torch.inf, empty) and o.isfinite().all()
    assert not o[empty].abs().sum()
    tol = e * ro.abs() + (2 * e + 2 * score[..., None] + ulp * keys) * spread
    if b.dt == torch.float16:
        tol = tol + keys * 2.0 ** -25 * 2 * max(1.0, float(torch.nan_to_num(a["v_cache"]).abs().max() *
                                                (torch.nan_to_num(vs).max() if vs is not None else 1))) + 2.0 ** -25
    off = (o - ro).abs() - tol
    assert (off <= 0).all(), ("o", float(off.max()), float((o - ro).abs().max()))
    ltol = score + ulp * (keys + rl.abs() + 8)
    off = ((lse - rl).abs() - ltol)[~empty]
    assert (off <= 0).all(), ("lse", float(off.max()), float((lse - rl)[~empty].abs().max()))
