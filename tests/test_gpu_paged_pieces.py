"""Attention over the paged cache where sequences are cut into pieces and joined, and calls that run beside each other."""
import pytest
import torch

import paper_2601_16238_amd as attn
from paged_util import Batch, call, check_attention

pytestmark = pytest.mark.gpu


def workspace_bytes(b, max_q):
    Hq, D = b.q.shape[1:]
    return attn.attn_fwd_paged_workspace_bytes(b.T, len(b.n), Hq, b.k.shape[1], D, b.cache[0].shape[0], b.P,
                                               b.table.shape[1], max_q=max_q)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Hq,Hkv,D,P,q", [(4, 2, 64, 16, 1), (17, 1, 64, 32, 1), (8, 1, 48, 64, 4), (32, 1, 128, 64, 1),
                                          (12, 3, 80, 128, 5), (16, 1, 256, 16, 1), (6, 2, 192, 32, 4), (8, 8, 128, 4096, 1)])
def test_few_rows(Hq, Hkv, D, P, q, dtype, e4m3):
    b = Batch([(q, 1200), (q, q), (0, 30), (1, 129), (q, 2500), (1, 1), (q, 640), (1, 0)], Hq, Hkv, D, P, dtype, e4m3,
              seed=Hq + D, table_pad=4096 // P, behind=1)
    g = b.on_gpu()
    assert workspace_bytes(b, q) > 0
    for causal in (True, False):
        o, lse = call(g, D ** -0.5, causal, max_q=q)
        check_attention(b, o, lse, causal)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,P", [(8, 2, 64, 16), (6, 2, 128, 32), (16, 2, 128, 64), (33, 1, 112, 16), (8, 4, 256, 64)])
def test_many_rows_beside_few(Hq, Hkv, D, P, e4m3):
    b = Batch([(1, 1300), (200, 1500), (1, 1), (3, 64), (0, 9), (1, 700), (70, 70), (300, 300), (1, 2000), (9, 0)], Hq, Hkv, D,
              P, e4m3=e4m3, seed=Hq * D, behind=3)
    g = b.on_gpu()
    for causal in (True, False):
        o, lse = call(g, D ** -0.5, causal)
        check_attention(b, o, lse, causal)


def test_two_calls_at_once():
    """On two streams, of both kernels, each with a workspace of its own."""
    calls = []
    for i, (seqs, max_q) in enumerate((([(1, 5000), (1, 300), (1, 2600)], 1), ([(150, 3000), (1, 900), (400, 400)], 400))):
        b = Batch(seqs, 8, 2, 128, 32, e4m3=i == 0, seed=i)
        calls.append((b, b.on_gpu(), max_q, torch.cuda.Stream()))
    alone = [call(g, 0.1, True, max_q=m) for _, g, m, _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [call(g, 0.1, True, max_q=m, stream=s) for _, g, m, s in calls]
        torch.cuda.synchronize()
        for x, y in zip(alone, got):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    for (b, *_), (o, lse) in zip(calls, alone):
        check_attention(b, o, lse, True, scale=0.1)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
def test_replayed_graph_of_append_and_attention(e4m3):
    """A chunk beside decoding, captured together; replayed with other lengths, with eager calls in between."""
    b = Batch([(1, 1500), (90, 600), (1, 40), (300, 300)], 8, 2, 128, 16, e4m3=e4m3, seed=3,
              filled=[1499, 510, 39, 0])
    g = b.on_gpu()
    start = {n: g[n].clone() for n in ("kc", "vc", "ks", "vs") if g[n] is not None}

    def run():
        attn.attn_paged_append(g["k"], g["v"], g["kc"], g["vc"], g["table"], g["q_start"], g["kv_lens"], k_scale=g["ks"],
                               v_scale=g["vs"])
        return call(g, 0.1, True, max_q=300)

    def restore():
        for n, x in start.items():
            g[n].copy_(x)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, LSE = run()
    for lens in ([1500, 600, 40, 300], [1500, 600, 40, 300], [1, 95, 0, 300], [1400, 600, 33, 300]):
        g["kv_lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        restore()
        O.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        o, lse = O.clone(), LSE.clone()
        restore()
        eager = run()
        assert torch.equal(o, eager[0]) and torch.equal(lse, eager[1])
        b.len, b.kv_lens = lens, torch.tensor(lens, dtype=torch.int32)
        b.cache = [g["kc"].cpu(), g["vc"].cpu()]
        if e4m3:
            b.scale = [g["ks"].cpu(), g["vs"].cpu()]
        check_attention(b, o, lse, True, scale=0.1)


@pytest.mark.parametrize("e4m3", [False, True], ids=["16", "e4m3"])
@pytest.mark.parametrize("B", [7, 600])
def test_row_ranges_that_overlap(B, e4m3):
    """An error of the caller's, which stays inside the buffers: rows of nobody keep what they hold."""
    b = Batch([(1, 30 + 13 * i % 700) for i in range(B)], 4, 2, 64, 16, e4m3=e4m3, seed=B, behind=4, table_pad=80)
    g = b.on_gpu()
    for q_start in ([i % 2 * B for i in range(B + 1)], [B] + [0] * B, [max(0, B - 3 * i) for i in range(B + 1)],
                    [-5] * B + [B]):
        g["q_start"] = torch.tensor(q_start, dtype=torch.int32, device="cuda")
        for max_q in (1, None):
            O, LSE = torch.full_like(g["q"], 3.0), torch.full(g["q"].shape[:2], 3.0, device="cuda")
            call(g, 0.1, True, max_q=max_q, O=O, LSE=LSE)
            torch.cuda.synchronize()
            assert (O[B:] == 3).all() and (LSE[B:] == 3).all()
    g["q_start"] = b.q_start.cuda()
    o, lse = call(g, 0.1, True, max_q=1)
    check_attention(b, o, lse, True, scale=0.1)
