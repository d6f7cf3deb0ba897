"""The operators on token sequences where sums are long: many rows of one token, more rows than the sort's short blocks take."""
import pytest
import torch

from paper_2105_08810_amd import snn

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_one_token_in_a_million_rows(dtype):
    """A token's sum is off by what 128 rows in float32 can be, not by more the more rows it has. The rows are such that a
    float32 chain of sums of 128 rows drops the same part of each of them."""
    R, N, V = (1 << 20) + 5, 9, 3
    v = 1.0 + 0.75 * 2.0 ** -14 if dtype == torch.float32 else 1.0
    dout = torch.full((R, N), v, device="cuda", dtype=dtype)
    ids = torch.ones(R, dtype=torch.int32, device="cuda")
    ids[R // 2], ids[R - 1] = 2, -1
    half = torch.finfo(dtype).eps / 2
    scale = 2.0 ** -20  # float16's range
    for acc in (False, True):
        dE = torch.full((V, N), 1.0, device="cuda", dtype=dtype)
        snn.embed_grad(ids, dout, V, scale, dE=dE, accumulate=acc)
        start = 1.0 if acc else 0.0
        want = torch.tensor([start, start + (R - 2) * v * scale, start + v * scale], dtype=torch.float64)
        off = (dE.double().cpu() - want[:, None]).abs()
        # 128 sums in float32, the whole rounded to it, the result's own rounding
        assert bool((off <= ((128 + 2) * U + half) * want[:, None]).all()), (acc, (off / (want[:, None] + 1e-30)).max())


@pytest.mark.parametrize("R", [16384, 16385, (1 << 20) + 3])
def test_lookup_gradient_of_many_tokens(R):
    """Rows on both sides of the sort's lines, against float64."""
    g = torch.Generator(device="cuda").manual_seed(R)
    V, N = 5000, 12
    ids = (torch.rand(R, generator=g, device="cuda") ** 4 * (V + 1)).to(torch.int32) - 1
    dout = torch.randn((R, N), generator=g, device="cuda")
    dE = snn.embed_grad(ids, dout, V, 0.5)
    at = ids.long().clamp_min(0)
    live = (ids >= 0).double()[:, None]
    want, size = (torch.zeros((V, N), device="cuda", dtype=torch.float64) for _ in range(2))
    want.index_add_(0, at, dout.double() * live * 0.5)
    size.index_add_(0, at, dout.double().abs() * live * 0.5)
    assert bool(((dE.double() - want).abs() <= (128 + 3) * U * size + 1e-45).all())
    assert torch.equal(dE, snn.embed_grad(ids, dout, V, 0.5))
