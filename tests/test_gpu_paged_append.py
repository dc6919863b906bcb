"""Appending to the paged cache against the 64-bit implementation; appending and attending together."""
import pytest
import torch

import paper_2601_16238_amd as attn
from oracle import paged_oracle as po
from paged_util import Batch, E4M3, call, check_attention, step

pytestmark = pytest.mark.gpu

CASES = {
    "decode": [(1, 1), (1, 16), (1, 17), (1, 64), (1, 500), (1, 33)],
    "few": [(3, 40), (0, 30), (2, 2), (5, 33), (17, 17)],
    "prompts": [(130, 130), (1, 1), (67, 400), (200, 203)],
    "missing": [(3, 0), (0, 0), (9, 4), (1, 20)],
}


def tables(positions, half, seed=0):
    g = torch.Generator().manual_seed(seed)
    angle = torch.rand(positions, half, generator=g, dtype=torch.float64) * 6.3
    return angle.cos().float(), angle.sin().float()


def bits(x):
    return x.cpu().contiguous().view(torch.uint8 if x.itemsize == 1 else torch.int16)


def check_append(b, rot=None, with_q=True, in_place=False, lens=None, **kw):
    """One call, everything compared.  Rotated values: a half step of the type on the result (16-bit), and three
    roundings of 2^-24 of either product.  e4m3: K's codes within a half step (2^-4 of the value, 2^-10 of the scale
    below the normal ones) of the value, V's, which nothing rounds before, and the older ones equal.  What no row
    went to keeps its bits."""
    D, width = b.q.shape[-1], b.table.shape[1]
    rot = D if rot is None else rot
    cos, sin = tables(width * b.P + 3, rot // 2) if rot else (None, None)
    g = b.on_gpu()
    ks, vs = b.scales()
    q_rot = None
    if with_q:
        q_rot = g["q"] if in_place else torch.full_like(g["q"], 5.0)
    got = attn.attn_paged_append(g["k"], g["v"], g["kc"], g["vc"], g["table"], g["q_start"], g["kv_lens"],
                                 cos=None if cos is None else cos.cuda(), sin=None if sin is None else sin.cuda(),
                                 Q=g["q"] if with_q else None, Q_rot=q_rot, k_scale=g["ks"], v_scale=g["vs"], **kw)
    torch.cuda.synchronize()
    before = [c.float().double() for c in b.cache]
    kc, vc, rks, rvs, rq = po.append(b.k, b.v, before[0], before[1], b.table, b.q_start, b.kv_lens, cos, sin,
                                     b.q if with_q else None, ks, vs)
    e, ulp = step(b.dt), 2.0 ** -24
    small = 2.0 ** -25 if b.dt == torch.float16 else 2.0 ** -134
    rows = [(first + i) for _, first, n, length in po.sequences(b.q_start, b.kv_lens) for i in range(n)
            if length - n + i >= 0]
    if with_q:
        assert got is not None and got.data_ptr() == q_rot.data_ptr()
        r, x = rq[rows], b.q[rows].double().abs()
        y = got.cpu()[rows].double()
        pair = x.clone()
        if rot:
            pair[..., :rot] = x[..., :rot] + torch.roll(x[..., :rot], rot // 2, -1)
        assert ((y - r).abs() <= e * r.abs() + 3 * ulp * pair + small).all()
        rest = [t for t in range(b.T) if t not in set(rows)]
        same = b.q if in_place else torch.full_like(b.q, 5.0)
        assert torch.equal(bits(got[rest]), bits(same[rest]))
    else:
        assert got is None
    pages, Hkv, P, _ = b.cache[0].shape
    new = torch.zeros(pages, P, dtype=torch.bool)
    older = torch.zeros(pages, P, dtype=torch.bool)
    for s, first, n, length in po.sequences(b.q_start, b.kv_lens):
        for p, page, i in po.slots(b.table, s, length, P, pages):
            (new if p >= length - n else older)[page, i] = True
    for name, x, ref, was, scale, rscale in (("k", g["kc"], kc, b.cache[0], g["ks"], rks),
                                             ("v", g["vc"], vc, b.cache[1], g["vs"], rvs)):
        x = x.cpu()
        at_new = new[:, None, :].expand(-1, Hkv, -1)
        if not b.e4m3:
            r, y = ref[at_new], x.double()[at_new]
            size = 0.0 if name == "v" else 3 * ulp * 2 * float(torch.nan_to_num(b.k.float()).abs().max())
            assert ((y - r).abs() <= (0 if name == "v" else e * r.abs() + size + small)).all(), name
            assert torch.equal(bits(x)[~at_new], bits(was)[~at_new]), name
            continue
        touched = new.any(1)
        assert torch.equal(scale.cpu()[touched].double(), rscale[touched]), name
        s = scale.cpu()
        assert torch.equal(s[~touched].view(torch.int32), b.scale[0 if name == "k" else 1][~touched].view(torch.int32))
        at_older = (older & touched[:, None])[:, None, :].expand(-1, Hkv, -1)
        codes = x.float().double()
        assert torch.equal(codes[at_older], ref[at_older]), name
        if name == "v":
            assert torch.equal(codes[at_new], ref[at_new])
        else:
            # (the reference's codes are rounded: a value beside a border may take either neighbour, a whole step off)
            r, y = ref[at_new], codes[at_new]
            assert ((y - r).abs() <= 2 * (2.0 ** -4 * r.abs()).clamp(min=2.0 ** -10)).all()
            assert (y != r).double().mean() <= 1e-3
        same = ~(at_new | at_older)
        assert torch.equal(bits(x)[same], bits(was)[same]), name
    return g


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lengths", list(CASES))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 64), (5, 5, 80, 32), (2, 2, 256, 16)])
def test_lengths(lengths, Hq, Hkv, D, P, dtype, e4m3):
    seqs = CASES[lengths]
    check_append(Batch(seqs, Hq, Hkv, D, P, dtype, e4m3, seed=D, behind=2, filled=[max(k - n, 0) for n, k in seqs]))


@pytest.mark.parametrize("rot", [0, 8, 24, 32, 64, 120, 128])
@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_rotated_columns(rot, e4m3):
    check_append(Batch([(1, 50), (20, 40)], 4, 2, 128, 16, e4m3=e4m3, seed=rot, filled=[49, 20]), rot=rot)


@pytest.mark.parametrize("D", [8, 24, 72, 104, 200])
def test_odd_head_dimensions(D):
    check_append(Batch([(1, 50), (20, 40)], 3, 1, D, 16, "f16", seed=D, filled=[49, 20]))


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_without_q_and_in_place(e4m3):
    seqs = [(1, 50), (20, 40)]
    for kw in (dict(with_q=False), dict(in_place=True), dict(in_place=True, rot=32)):
        check_append(Batch(seqs, 4, 2, 64, 16, e4m3=e4m3, seed=3, filled=[49, 20], behind=1), **kw)


@pytest.mark.parametrize("layout", ["NHD", "padded"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_layouts(layout, e4m3):
    b = Batch([(1, 300), (2, 45), (140, 170)], 8, 2, 128, 32, e4m3=e4m3, layout=layout, seed=5, table_pad=3,
              filled=[299, 43, 30])
    # rows that are slices of one [T, Hq + 2 Hkv, D] projection
    all_rows = torch.cat((b.q, b.k, b.v), 1)
    b.q, b.k, b.v = all_rows[:, :8], all_rows[:, 8:10], all_rows[:, 10:]
    check_append(b)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_pages_that_are_none(e4m3):
    b = Batch([(1, 40), (50, 100), (3, 7)], 4, 2, 64, 16, e4m3=e4m3, seed=7, filled=[39, 50, 4])
    b.table[0, 2], b.table[1, 4], b.table[2, 0] = -1, b.cache[0].shape[0], 2 ** 31 - 1
    check_append(b)


def test_positions_past_the_table_count_as_its_end():
    """A length past the table's end is its end: the batch's rows are the last ones in front of it."""
    b = Batch([(3, 64), (1, 10)], 2, 1, 64, 16, seed=9, filled=[61, 9])
    b.kv_lens[0] = 10 ** 9
    g = b.on_gpu()
    b.kv_lens[0] = 64
    attn.attn_paged_append(g["k"], g["v"], g["kc"], g["vc"], g["table"], g["q_start"], g["kv_lens"])
    kc, vc, *_ = po.append(b.k, b.v, b.cache[0].double(), b.cache[1].double(), b.table, b.q_start, b.kv_lens)
    assert torch.equal(bits(g["kc"]), bits(kc.to(b.dt))) and torch.equal(bits(g["vc"]), bits(vc.to(b.dt)))


def test_large_pages_and_growing_scales():
    for P in (512, 4096):
        b = Batch([(700, 1100), (1, 513)], 2, 1, 64, P, e4m3=True, seed=P, filled=[400, 512])
        b.k *= 16
        check_append(b)


def test_values_of_every_size():
    """Zeros, subnormal and largest values, alone in their page."""
    for fill in (0.0, 1e-30, 1e-7, 448.0, 449.0, 3e38):
        b = Batch([(2, 18), (16, 16)], 2, 1, 64, 16, e4m3=True, seed=11, filled=[16, 0])
        b.v.fill_(fill)
        check_append(b, rot=0)


def test_many_sequences():
    seqs = [(1 + i % 3, 3 + 7 * i % 90) if i % 5 else (0, 30) for i in range(300)]
    for e4m3 in (False, True):
        check_append(Batch(seqs, 2, 1, 64, 16, e4m3=e4m3, seed=13, filled=[k - n for n, k in seqs]))


def test_bits_of_the_rotary_kernel():
    """Rotated rows in a bf16 cache are the rotary kernel's."""
    from paper_2601_16238_amd import rowops
    S, H, D, P = 100, 4, 128, 16
    x = torch.randn(1, H, S, D, device="cuda").bfloat16()
    cos, sin = (t.cuda() for t in tables(112, D // 2))
    y = rowops.rotary_fwd(x, cos[:S], sin[:S])
    rows = x[0].transpose(0, 1)
    kc = torch.zeros(7, H, P, D, device="cuda", dtype=torch.bfloat16)
    vc = torch.zeros_like(kc)
    table = torch.arange(7, device="cuda", dtype=torch.int32)[None]
    q = attn.attn_paged_append(rows, rows, kc, vc, table, torch.tensor([0, S], device="cuda", dtype=torch.int32),
                               torch.tensor([S], device="cuda", dtype=torch.int32), cos=cos, sin=sin, Q=rows)
    k = kc.transpose(0, 1).reshape(H, 112, D)[:, :S]
    assert torch.equal(k, y[0]) and torch.equal(q.transpose(0, 1), y[0])
    assert torch.equal(vc.transpose(0, 1).reshape(H, 112, D)[:, :S], x[0])


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_cache_past_32_bit_offsets(e4m3):
    P, Hkv, D = 64, 8, 128
    pages = (5 << 30) // (P * Hkv * D * (1 if e4m3 else 2))
    k = torch.randn(70, Hkv, D).bfloat16()
    kc = torch.empty(pages, Hkv, P, D, device="cuda", dtype=E4M3 if e4m3 else torch.bfloat16)
    vc = torch.empty_like(kc)
    scales = torch.zeros(2, pages, Hkv, device="cuda") if e4m3 else (None, None)
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32)
    attn.attn_paged_append(k.cuda(), k.cuda(), kc, vc, table.cuda(), torch.tensor([0, 70], dtype=torch.int32).cuda(),
                           torch.tensor([70], dtype=torch.int32).cuda(), k_scale=scales[0], v_scale=scales[1])
    for c, s in ((kc, scales[0]), (vc, scales[1])):
        got = torch.cat((c[pages - 1].float(), c[pages - 3].float()), 1)[:, :70].cpu()
        if not e4m3:
            assert torch.equal(got.bfloat16(), k.transpose(0, 1))
        else:
            s = torch.cat((s[pages - 1, :, None].expand(-1, P), s[pages - 3, :, None].expand(-1, P)), 1)[:, :70].cpu()
            x = k.transpose(0, 1).float()
            assert ((got * s[..., None] - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * s[..., None]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_a_batch_that_is_served(e4m3, dtype):
    """Prompts, then steps of one and of a few tokens: append, attend, each against the 64-bit implementation on the
    cache as it is; with a 16-bit cache also against dense attention over everything that was appended."""
    Hq, Hkv, D, P, width = 8, 2, 64, 16, 9
    g = torch.Generator().manual_seed(17)
    cos, sin = tables(width * P, D // 2)
    B = 3
    b = Batch([(1, 1)] * B, Hq, Hkv, D, P, dtype, e4m3, filled=[0] * B, spare=B * width)
    pages = b.cache[0].shape[0]
    b.table = torch.randperm(pages, generator=g)[:B * width].view(B, width).int()
    gpu = b.on_gpu()
    length = [0] * B
    dense = [[] for _ in range(B)]
    for step_, rows in enumerate(([40, 7, 100], [1, 1, 1], [1, 0, 1], [4, 3, 1], [1, 1, 20], [1, 1, 1])):
        length = [x + n for x, n in zip(length, rows)]
        b.n, b.len, b.T = rows, length, sum(rows)
        b.q_start = torch.tensor([sum(rows[:i]) for i in range(B + 1)], dtype=torch.int32)
        b.kv_lens = torch.tensor(length, dtype=torch.int32)
        b.q, b.k, b.v = (torch.randn(b.T, h, D, generator=g).to(b.dt) for h in (Hq, Hkv, Hkv))
        for n in ("q", "k", "v", "q_start", "kv_lens"):
            gpu[n] = getattr(b, n).cuda()
        q = attn.attn_paged_append(gpu["k"], gpu["v"], gpu["kc"], gpu["vc"], gpu["table"], gpu["q_start"],
                                   gpu["kv_lens"], cos=cos.cuda(), sin=sin.cuda(), Q=gpu["q"], k_scale=gpu["ks"],
                                   v_scale=gpu["vs"])
        gpu["q"] = q
        o, lse = call(gpu, D ** -0.5, True, max_q=max(rows))
        b.q = q.cpu()
        b.cache = [gpu["kc"].cpu(), gpu["vc"].cpu()]
        if e4m3:
            b.scale = [gpu["ks"].cpu(), gpu["vs"].cpu()]
        check_attention(b, o, lse, True)
        for s in range(B):
            at = slice(int(b.q_start[s]), int(b.q_start[s + 1]))
            p = torch.arange(length[s] - rows[s], length[s])
            turned = po.rotate(b.k[at], cos[p][:, None], sin[p][:, None]).to(b.dt)
            dense[s].append((turned, b.v[at]))
        if not e4m3:
            for s in range(B):
                kk, vv = (torch.cat([x[i] for x in dense[s]]) for i in (0, 1))
                where = po.slots(b.table, s, length[s], P, pages)
                stored = torch.stack([b.cache[1][page, :, i] for _, page, i in where])
                assert torch.equal(stored, vv)
                stored = torch.stack([b.cache[0][page, :, i] for _, page, i in where]).double()
                assert ((stored - kk.double()).abs() <= 2 * step(b.dt) * kk.double().abs() + 1e-5).all()


def test_replayed_graph_follows_the_lengths():
    b = Batch([(1, 30), (1, 5)], 4, 2, 64, 16, e4m3=True, seed=19, filled=[29, 4])
    g = b.on_gpu()
    start = [g[n].clone() for n in ("kc", "vc", "ks", "vs")]

    def append():
        attn.attn_paged_append(g["k"], g["v"], g["kc"], g["vc"], g["table"], g["q_start"], g["kv_lens"],
                               k_scale=g["ks"], v_scale=g["vs"])

    def restore():
        for n, x in zip(("kc", "vc", "ks", "vs"), start):
            g[n].copy_(x)
    append()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        append()
    for lens in ([30, 5], [17, 1], [32, 16], [0, 3]):
        g["kv_lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        restore()
        graph.replay()
        torch.cuda.synchronize()
        after = [g[n].clone() for n in ("kc", "vc", "ks", "vs")]
        restore()
        append()
        for n, x in zip(("kc", "vc", "ks", "vs"), after):
            assert torch.equal(g[n].view(torch.uint8), x.view(torch.uint8))
