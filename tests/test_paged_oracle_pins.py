"""The paged cache's 64-bit implementation against closed forms and torch's own types."""
import math

import pytest
import torch

from oracle import paged_oracle as po


def test_e4m3_rounding_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = codes[codes.isfinite()]
    assert torch.equal(po.e4m3_round(codes), codes)
    x = torch.cat((torch.linspace(-448, 448, 20011), torch.linspace(-0.03, 0.03, 20011),
                   (codes[1:] + codes[:-1]).float() / 2))
    assert torch.equal(po.e4m3_round(x), x.to(torch.float8_e4m3fn).double())
    assert float(po.e4m3_round(torch.tensor(1e9))) == 448


@pytest.mark.parametrize("amax,scale", [(0.0, 2.0 ** -100), (448.0, 1.0), (448.5, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8),
                                        (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (1e-40, 2.0 ** -100)])
def test_scales(amax, scale):
    assert po.e4m3_scale(torch.tensor(amax, dtype=torch.float64)) == scale


def test_rotation_turns_pairs():
    x = torch.tensor([1.0, 2.0, 0.0, 5.0, 7.0])
    y = po.rotate(x, torch.tensor([0.0, 1.0]), torch.tensor([1.0, 0.0]))
    assert y.tolist() == [0.0, 2.0, 1.0, 5.0, 7.0]


def test_attention_of_equal_keys_and_of_none():
    k = torch.zeros(3, 1, 4, 2)
    v = torch.zeros(3, 1, 4, 2)
    v[2, 0] = torch.tensor([[1.0, 0], [3.0, 0], [5.0, 0], [7.0, 0]])
    v[0, 0, 0, 0] = 9.0
    q = torch.ones(5, 2, 2)
    table = [[2, 0], [1, -1]]
    o, lse, spread, _ = po.attention(q, k, v, table, [0, 3, 4], [5, 0], 1.0, True)
    assert o[:3, 0, 0].tolist() == [3.0, 4.0, 5.0] and lse[2, 1].item() == pytest.approx(math.log(5))
    assert lse[3].tolist() == [-math.inf] * 2 and o[3].abs().sum() == 0 and o[4].isnan().all()
    o, lse, *_ = po.attention(q, k, v, [[2, 7], [1, -1]], [0, 3, 4], [5, 0], 1.0, False)   # page 7 does not exist
    assert o[0, 0, 0].item() == pytest.approx(4.0) and lse[0, 0].item() == pytest.approx(math.log(4))


def test_appending_moves_older_codes_to_a_larger_scale():
    kc = torch.zeros(2, 1, 16, 2, dtype=torch.float64)
    kc[1, 0, :2] = torch.tensor([[448.0, 3.0], [0.017578125, -8.0]])
    ks = torch.tensor([[1.0], [0.5]])
    new = torch.tensor([[[1.0, 900.0]]])
    k2, v2, s2, _, q2 = po.append(new, new, kc, kc, [[1]], [0, 1], [3], k_scale=ks, v_scale=ks, q=new)
    assert s2[1].item() == 4.0 and s2[0].item() == 1.0   # 900 <= 448 * 4
    assert k2[1, 0, 0].tolist() == [56.0, 0.375] and k2[1, 0, 1].tolist() == [0.001953125, -1.0]
    assert k2[1, 0, 2].tolist() == [0.25, 224.0]  # (900 / 4 = 225: nearest of 224 and 240)
    assert torch.equal(q2, new.double())
