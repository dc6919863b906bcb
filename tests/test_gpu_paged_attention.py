"""Attention over the paged cache against the 64-bit implementation."""
import math

import pytest
import torch

import paper_2601_16238_amd as attn
from paged_util import Batch, E4M3, call, check_attention

pytestmark = pytest.mark.gpu

LENGTHS = {
    "one_key": [(1, 1)],
    "decode": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 64), (1, 129), (1, 500)],
    "few": [(3, 40), (1, 700), (2, 2), (4, 33)],
    "prompts": [(130, 130), (1, 1), (67, 67)],
    "chunks": [(150, 411), (40, 200), (1, 300)],
    "none": [(1, 70), (0, 50), (2, 0), (0, 0), (5, 3), (1, 20)],
}


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (8, 1, 128, 64), (5, 1, 80, 32), (2, 2, 256, 16)])
def test_lengths(lengths, Hq, Hkv, D, P, dtype, e4m3):
    b = Batch(LENGTHS[lengths], Hq, Hkv, D, P, dtype, e4m3, seed=len(lengths) + D, behind=2)
    g = b.on_gpu()
    for causal in (True, False):
        o, lse = call(g, D ** -0.5, causal)
        check_attention(b, o, lse, causal)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(16, 1, 128, 32), (17, 1, 64, 16), (33, 1, 128, 16), (48, 2, 192, 64),
                                        (130, 1, 64, 128), (12, 4, 96, 256)])
def test_groups(Hq, Hkv, D, P, e4m3):
    b = Batch([(1, 190), (3, 77), (9, 300)], Hq, Hkv, D, P, e4m3=e4m3, seed=Hq)
    g = b.on_gpu()
    for max_q in (9, None):
        o, lse = call(g, D ** -0.5, True, max_q=max_q)
        check_attention(b, o, lse, True)


@pytest.mark.parametrize("D", [8, 24, 72, 104, 136, 200, 248])
def test_odd_head_dimensions(D):
    b = Batch([(1, 90), (70, 133)], 4, 2, D, 16, "f16", seed=D)
    o, lse = call(b.on_gpu(), D ** -0.5, True)
    check_attention(b, o, lse, True)


@pytest.mark.parametrize("D", [16, 48, 112, 144, 240])
def test_odd_head_dimensions_e4m3(D):
    b = Batch([(1, 90), (70, 133)], 4, 2, D, 16, e4m3=True, seed=D, scales="any")
    o, lse = call(b.on_gpu(), D ** -0.5, True)
    check_attention(b, o, lse, True)


@pytest.mark.parametrize("layout", ["NHD", "padded"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_layouts(layout, e4m3):
    b = Batch([(1, 300), (2, 45), (140, 170)], 8, 2, 128, 32, e4m3=e4m3, layout=layout, seed=5, table_pad=3)
    g = b.on_gpu()
    T, Hq, D = b.q.shape
    # query rows in [Hq,T,D] storage, a slice of a wider page table
    g["q"] = g["q"].transpose(0, 1).contiguous().transpose(0, 1)
    g["table"] = g["table"][:, :-2]
    o, lse = call(g, D ** -0.5, True)
    check_attention(b, o, lse, True)
    O = torch.full((Hq, T, D + 8), 2.0, device="cuda", dtype=b.dt).transpose(0, 1)[..., :D]   # strides of its own
    call(g, D ** -0.5, True, O=O)
    assert torch.equal(O, o) and (O._base[..., D:] == 2).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scales", ["any", "powers"])
def test_scales_of_pages(scales, dtype):
    b = Batch([(1, 513), (3, 257), (200, 300)], 8, 2, 128, 16, dtype, e4m3=True, scales=scales, seed=9)
    o, lse = call(b.on_gpu(), 128 ** -0.5, True)
    check_attention(b, o, lse, True)
    # a page of zeros: scale 0
    b.scale[0][b.table[0, 1]] = 0.0
    b.scale[1][b.table[0, 2]] = 0.0
    o, lse = call(b.on_gpu(), 128 ** -0.5, True)
    check_attention(b, o, lse, True)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_pages_that_are_none_are_not_seen(e4m3):
    b = Batch([(1, 200), (2, 150), (130, 400), (1, 16)], 4, 1, 64, 16, e4m3=e4m3, seed=11)
    b.table[0, 3], b.table[0, 12] = -1, b.cache[0].shape[0]
    b.table[1, 0] = 2 ** 31 - 1
    b.table[2, 1:9] = -5
    b.table[3, 0] = -1
    g = b.on_gpu()
    for causal in (True, False):
        o, lse = call(g, 0.125, causal)
        check_attention(b, o, lse, causal)
        assert (lse[-1] == -math.inf).all()


def test_metadata_out_of_range_stays_inside():
    """Lengths past the table count as its end, negative ones as none; rows past T as T."""
    b = Batch([(1, 40), (2, 50), (3, 64)], 4, 2, 64, 16, seed=13)
    g = b.on_gpu()
    g["kv_lens"] = torch.tensor([-3, 50, 10 ** 9], dtype=torch.int32, device="cuda")
    g["q_start"] = torch.tensor([-4, 1, 3, 99], dtype=torch.int32, device="cuda")
    o, lse = call(g, 0.125, True)
    b.len = [0, 50, 64]
    check_attention(b, o, lse, True, kv_lens=torch.tensor(b.len))


def test_rows_behind_the_last_sequence_are_left():
    b = Batch([(1, 40), (130, 150)], 4, 2, 64, 16, seed=17, behind=5)
    g = b.on_gpu()
    O, LSE = torch.full_like(g["q"], 3.0), torch.full(g["q"].shape[:2], 3.0, device="cuda")
    o, lse = call(g, 0.125, True, O=O, LSE=LSE)
    assert o.data_ptr() == O.data_ptr() and lse.data_ptr() == LSE.data_ptr()
    check_attention(b, o, lse, True)
    assert (O[131:] == 3).all() and (LSE[131:] == 3).all()
    # rows in front of the first sequence too, and those of a sequence that has more than max_q
    g["q_start"] = torch.tensor([1, 2, 132], dtype=torch.int32, device="cuda")
    g["q"] = torch.roll(g["q"], 1, 0)
    O.fill_(3.0)
    LSE.fill_(3.0)
    call(g, 0.125, True, O=O, LSE=LSE)
    assert (O[0] == 3).all() and (LSE[0] == 3).all() and (O[132:] == 3).all()
    check_attention(b, O[1:], LSE[1:], True)


def test_nothing_to_do():
    b = Batch([(1, 40)], 4, 2, 64, 16)
    g = b.on_gpu()
    g["q"] = g["q"][:0]
    o, lse = call(g, 0.125, True)
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
    g = b.on_gpu()
    g.update(table=g["table"][:0], kv_lens=g["kv_lens"][:0], q_start=g["q_start"][:1])
    O, LSE = torch.full_like(g["q"], 3.0), torch.full(g["q"].shape[:2], 3.0, device="cuda")
    call(g, 0.125, True, O=O, LSE=LSE)
    assert (O == 3).all() and (LSE == 3).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_long_sequences_with_and_without_a_workspace(e4m3):
    b = Batch([(1, 5000), (2, 9001), (1, 3), (4, 700)], 8, 2, 128, 64, e4m3=e4m3, seed=19)
    g = b.on_gpu()
    for kw in (dict(max_q=4), dict(), dict(split=False, max_q=4), dict(split=False)):
        o, lse = call(g, 128 ** -0.5, True, **kw)
        check_attention(b, o, lse, True)
    need = attn.attn_fwd_paged_workspace_bytes(b.T, 4, 8, 2, 128, b.cache[0].shape[0], 64, b.table.shape[1], max_q=4)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")  # all NaN
    o, lse = call(g, 128 ** -0.5, True, max_q=4, workspace=ws)
    check_attention(b, o, lse, True)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_chunk_against_many_keys(e4m3):
    b = Batch([(33, 6000), (1, 200)], 8, 2, 128, 32, e4m3=e4m3, seed=23)
    g = b.on_gpu()
    for causal in (True, False):
        for split in (True, False):
            o, lse = call(g, 128 ** -0.5, causal, split=split)
            check_attention(b, o, lse, causal)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_scores_that_grow_along_the_keys(e4m3):
    """The running maximum moves in every tile, by much more than a factor of e."""
    b = Batch([(1, 900), (100, 400)], 4, 2, 64, 16, e4m3=e4m3, seed=29, gain=1.0)
    for s in range(2):
        for w in range(b.table.shape[1]):
            page = int(b.table[s, w])
            if page < 0:
                continue
            if e4m3:
                b.scale[0][page] *= 2.0 ** min(w // 4, 6)
            else:
                b.cache[0][page] *= 1.0 + w
    o, lse = call(b.on_gpu(), 0.125, True)
    check_attention(b, o, lse, True)


def test_many_sequences():
    b = Batch([(1 + i % 2, 1 + 7 * i % 90) if i % 5 else (0, 30) for i in range(300)], 4, 2, 64, 16, seed=31)
    o, lse = call(b.on_gpu(), 0.125, True)
    check_attention(b, o, lse, True)
    o, lse = call(b.on_gpu(), 0.125, True, max_q=2)
    check_attention(b, o, lse, True)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_cache_past_32_bit_offsets(e4m3):
    """Pages behind the first 4 GiB of the cache (and 2^31 elements)."""
    P, Hkv, D = 64, 8, 128
    pages = (5 << 30) // (P * Hkv * D * (1 if e4m3 else 2))
    b = Batch([(1, 130), (140, 300)], 16, Hkv, D, P, e4m3=e4m3, seed=37)
    g = b.on_gpu()
    old = b.table.clone()
    far = pages - 1 - torch.arange(pages, dtype=torch.int32)[:b.cache[0].shape[0]]
    for c in ("kc", "vc"):
        big = torch.empty(pages, Hkv, P, D, dtype=g[c].dtype, device="cuda")
        big.view(torch.uint8)[far.long().cuda()] = g[c].view(torch.uint8)
        g[c] = big
    if e4m3:
        for c in ("ks", "vs"):
            big = torch.full((pages, Hkv), float("nan"), device="cuda")
            big[far.long().cuda()] = g[c]
            g[c] = big
    g["table"] = torch.where(old >= 0, far[old.long().clamp(min=0)], old).cuda()
    o, lse = call(g, D ** -0.5, True)
    check_attention(b, o, lse, True)


def test_replayed_graph_follows_the_lengths():
    b = Batch([(1, 900), (1, 40), (1, 300)], 8, 2, 128, 32, e4m3=True, seed=41)
    g = b.on_gpu()
    O, LSE = torch.zeros_like(g["q"]), torch.zeros(g["q"].shape[:2], device="cuda")
    call(g, 0.1, True, max_q=1, O=O, LSE=LSE)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(g, 0.1, True, max_q=1, O=O, LSE=LSE)
    for lens in ([900, 40, 300], [1, 40, 0], [899, 3, 290], [900, 40, 300]):
        g["kv_lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        O.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        o, lse = O.clone(), LSE.clone()
        eager = call(g, 0.1, True, max_q=1)
        assert torch.equal(o, eager[0]) and torch.equal(lse, eager[1])
        b.len = lens
        check_attention(b, o, lse, True, scale=0.1, kv_lens=torch.tensor(lens))


def test_on_a_stream_of_its_own():
    b = Batch([(1, 3000), (2, 40)], 8, 2, 128, 32, seed=43)
    g = b.on_gpu()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, lse = call(g, 0.1, True, max_q=2, stream=side)
    side.synchronize()
    check_attention(b, o, lse, True, scale=0.1)


def test_the_same_bits_every_time():
    b = Batch([(1, 5000), (1, 70), (64, 2000)], 8, 2, 128, 64, e4m3=True, seed=47)
    g = b.on_gpu()
    first = call(g, 0.1, True)
    for _ in range(3):
        again = call(g, 0.1, True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_agrees_with_the_dense_forward():
    """The paged call on one page table in order is the rectangular call."""
    B, Hq, Hkv, Sq, Sk, D, P = 2, 8, 2, 5, 200, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(B, Hq, Sq, D, device="cuda", generator=gen, dtype=torch.bfloat16)
    kv = torch.randn(2, B, Hkv, Sk, D, device="cuda", generator=gen, dtype=torch.bfloat16)
    O, LSE = attn.attn_fwd_rect(q, kv[0], kv[1], D ** -0.5, True)
    w = -(-Sk // P)
    pages = torch.zeros(2, B, Hkv, w * P, D, device="cuda", dtype=torch.bfloat16)
    pages[:, :, :, :Sk] = kv
    pages = pages.view(2, B, Hkv, w, P, D).transpose(2, 3).reshape(2, B * w, Hkv, P, D).contiguous()
    table = torch.arange(B * w, device="cuda", dtype=torch.int32).view(B, w)
    o, lse = attn.attn_fwd_paged(q.transpose(1, 2).reshape(B * Sq, Hq, D), pages[0], pages[1], table,
                                 torch.tensor([0, Sq, 2 * Sq], device="cuda", dtype=torch.int32),
                                 torch.tensor([Sk, Sk], device="cuda", dtype=torch.int32), D ** -0.5, True)
    o = o.view(B, Sq, Hq, D).transpose(1, 2).float()
    lse = lse.view(B, Sq, Hq).transpose(1, 2)
    # either side is within 3 half steps of the probabilities' weighted mean of |v|, here below 4
    assert (o - O.float()).abs().max() <= 6 * 2.0 ** -8 * 4 and (lse - LSE).abs().max() < 1e-4
