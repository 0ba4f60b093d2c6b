"""Gradient through a vocabulary projection with weights near the largest fp32 numbers and low temperatures, whose logits are nevertheless finite: nothing
that belongs to no row, such as the rows that fill a tile, may reach the results.

All values are powers of two, so logits are exact; they are `size`, minus that and 0, so the largest has all the probability: dz is g / temperature in the token's
place, minus that in the largest one's and 0 elsewhere, and everything that is added up is exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 70, 300])
@pytest.mark.parametrize("exponent,temperature,size", [(100, 2.0 ** -10, 2.0 ** 30), (126, 2.0 ** -16, 2.0 ** 30), (126, 2.0 ** -40, 2.0 ** 100),
                                                       (60, 2.0 ** -100, 2.0 ** 60)])
def test_large_weights_and_low_temperatures(exponent, temperature, size, rows, dtype, layout):
    import paper_2605_16154_amd as pcm
    w = torch.zeros(8, 20)
    w[0, 3], w[0, 5] = 2.0 ** exponent, -2.0 ** exponent
    w = w.to(dtype).cuda()
    w = w.t().contiguous().t() if layout == "out_in" else w
    hidden = torch.zeros((rows, 8), dtype=dtype, device="cuda")
    hidden[:, 0] = size * temperature / 2.0 ** exponent
    tokens = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    tokens[0], tokens[1], tokens[2] = 3, 5, 7
    forward = pcm.pcm_linear_logprobs(hidden, w, tokens, temperature=temperature)
    assert forward["lse"][:3].tolist() == [size] * 3 and forward["logp"][:3].tolist() == [0.0, -2 * size, -size]
    g = torch.zeros(rows, device="cuda")
    g[:3] = torch.tensor([1.0, 2.0, 4.0]) / 16 * temperature
    got = pcm.pcm_linear_logprobs_backward(hidden, w, tokens, forward["lse"], g, temperature=temperature)
    want = torch.zeros(8, 20, dtype=torch.float64)
    want[0, 5], want[0, 7], want[0, 3] = 2 / 16, 4 / 16, -6 / 16
    want = (want * float(hidden[0, 0])).to(dtype).cuda()
    assert torch.equal(got["dweight"], want)
    dh = torch.zeros((rows, 8), dtype=torch.float64)
    dh[1, 0] = dh[2, 0] = -4 / 16 * 2.0 ** exponent
    assert torch.equal(got["dhidden"], dh.to(dtype).cuda())
