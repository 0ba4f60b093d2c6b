"""NaN among the logits of the log-probabilities through a vocabulary projection, wherever the vocabulary ends: a call whose rows go through tiles gives NaN
as one whose rows are few does, in the row's own results and nowhere else.  Vocabularies that end inside a block of 64 or 128 columns, behind its first
column, in the middle and on its border; NaN is looked for as such, so there is no tolerance."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# (rows, d): streamed past, small tiles, large tiles (with V = 8193)
ROWS = {BF16: (5, 130), F32: (5, 1100)}


def _inputs(rows, d, V, dtype, layout):
    gen = torch.Generator().manual_seed(rows + 3 * d + 7 * V)
    hidden = torch.randn((rows, d), generator=gen).to(dtype).cuda()
    w = torch.randn((V, d) if layout == "out_in" else (d, V), generator=gen).to(dtype).cuda()
    tokens = torch.randint(0, V, (rows,), generator=gen).cuda()
    return hidden, w.t() if layout == "out_in" else w, tokens


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("V", [1, 3, 33, 63, 64, 65, 97, 129, 321])
def test_a_nan_in_the_last_column_makes_every_row_nan(V, layout, dtype):
    import paper_2605_16154_amd as pcm
    for rows in ROWS[dtype]:
        hidden, w, tokens = _inputs(rows, 40, V, dtype, layout)
        tokens[:] = 0                                       # the token's own logit is no NaN, but for V = 1
        tokens[1] = -1
        w[7, V - 1] = float("nan")
        got = pcm.pcm_linear_logprobs(hidden, w, tokens)
        live = tokens >= 0
        for k, x in got.items():
            assert bool(torch.isnan(x[live]).all()), (rows, k)
            assert not x[~live].any(), (rows, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
@pytest.mark.parametrize("V", [1, 3, 33, 63, 64, 65, 97, 129, 321])
def test_a_nan_in_a_row_makes_that_row_nan(V, layout, dtype):
    import paper_2605_16154_amd as pcm
    for rows in ROWS[dtype]:
        hidden, w, tokens = _inputs(rows, 40, V, dtype, layout)
        clean = pcm.pcm_linear_logprobs(hidden, w, tokens)
        hidden[2, 11] = float("nan")
        got = pcm.pcm_linear_logprobs(hidden, w, tokens)
        others = torch.arange(rows, device="cuda") != 2
        for k, x in got.items():
            assert bool(torch.isnan(x[2])) and torch.equal(x[others], clean[k][others]), (rows, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["in_out", "out_in"])
def test_nan_in_large_tiles(layout, dtype):
    """1100 rows and 8193 columns: tiles of 256 x 256, the last column alone in its block."""
    import paper_2605_16154_amd as pcm
    hidden, w, tokens = _inputs(1100, 40, 8193, dtype, layout)
    tokens[:] = 5
    clean = pcm.pcm_linear_logprobs(hidden, w, tokens)
    assert all(bool(torch.isfinite(x).all()) for x in clean.values())
    w[7, 8192] = float("nan")
    for k, x in pcm.pcm_linear_logprobs(hidden, w, tokens).items():
        assert bool(torch.isnan(x).all()), k
    w[7, 8192] = 1.0
    clean = pcm.pcm_linear_logprobs(hidden, w, tokens)
    hidden[1099, 39] = float("nan")
    for k, x in pcm.pcm_linear_logprobs(hidden, w, tokens).items():
        assert bool(torch.isnan(x[1099])) and torch.equal(x[:1099], clean[k][:1099]), k
