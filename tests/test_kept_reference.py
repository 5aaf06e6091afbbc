"""The 8-bit reference against torch's own conversion, and its scales by hand."""
import torch

from kept_reference import F8, pack, round_e4m3, scale_bytes, unpack


def test_rounding_is_that_of_the_format():
    g = torch.Generator().manual_seed(1)
    v = torch.cat((torch.linspace(-448, 448, 20001), torch.randn(20000, generator=g) * 0.02,
                   torch.arange(256, dtype=torch.uint8).view(F8).float().nan_to_num(0.0)))
    assert torch.equal(round_e4m3(v.double()).float(), v.to(F8).float())


def test_scales_by_hand():
    for v, byte in ((0.0, 1), (448.0, 127), (448.5, 128), (224.0, 126), (224.1, 127), (1.0, 119), (2.0 ** -140, 1),
                    (float("inf"), 1), (float("nan"), 1)):
        assert int(scale_bytes(torch.tensor([[v]], dtype=torch.double))[0, 0]) == byte, v


def test_each_group_has_its_scale_and_comes_back():
    x = torch.tensor([[2.0 ** (j // 32) * (1 + j % 8 / 8) for j in range(70)]])
    q, s = pack(x)
    assert s.shape == (1, 3) and torch.equal(unpack(q, s), x.double())
