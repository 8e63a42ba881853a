"""Scale bytes that no write gives, 0 and 255: 2^-127 and NaN, as in the format float8_e8m0fnu that the scales may have, for a read and for
attention alike (needs an MI355X)."""
import math

import pytest
import torch

from paper_2601_12698_amd import serving as S

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def cache(d, byte):
    """Two pages of one head with codes 448, -1.75, 1 and 2^-9 in turn; the scale byte of the second key is `byte`, the others' 127."""
    codes = torch.tensor([448.0, -1.75, 1.0, 2.0 ** -9]).to(torch.float8_e4m3fn).repeat(d // 4)
    pages = codes.view(torch.uint8).repeat(2, 1, 16, 1).cuda().view(torch.float8_e4m3fn)
    scale = torch.full((2, 1, 16), 127, dtype=torch.uint8)
    scale[0, 0, 1] = byte
    return pages, scale.cuda(), codes.double()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("as_e8m0", [False, True])
def test_read_back(dtype, as_e8m0):
    for byte in (0, 1, 254, 255):
        pages, scale, codes = cache(16, byte)
        if as_e8m0:
            scale = scale.view(torch.float8_e8m0fnu)
        k, v = (torch.empty(2, 1, 16, dtype=TYPES[dtype], device="cuda") for _ in range(2))
        S.kvcache_read(pages, pages, scale, scale, torch.tensor([0, 1], device="cuda"), k, v, dtype)
        want = torch.full((16,), math.nan, dtype=torch.float64) if byte == 255 else codes * 2.0 ** (byte - 127)
        for got in (k, v):
            assert torch.equal(got[0, 0].cpu().double(), codes.to(TYPES[dtype]).double())
            assert torch.equal(got[1, 0].cpu().nan_to_num(7.0), want.to(TYPES[dtype]).nan_to_num(7.0)) and torch.equal(got[1, 0].cpu().isnan(), want.isnan())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("q_len", [1, 12, 20, 40])             # 4, 48, 80 and 160 rows: the forms of few rows and of many
def test_attention_takes_them_alike(q_len, d):
    """One key: the output is its value.  Values of 2^-118 are far above what the sums lose."""
    q = torch.zeros(q_len, 4, d, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([0], dtype=torch.int32, device="cuda")
    for byte in (0, 1, 127, 200):
        pages, scale, codes = cache(d, byte)
        pages, scale = pages[:, :, 1:2].contiguous(), scale[:, :, 1:2].contiguous()          # the key with that byte alone
        out, lse = torch.empty_like(q), torch.empty(q_len, 4, device="cuda")
        S.prefixattn_run(q, pages, pages, scale, scale, table, 1, None, None, out, lse, 1.0, "bf16", q_len=q_len)
        want = (codes * 2.0 ** (byte - 127))
        big = codes.abs() >= 1                                  # 2^-136, smaller than any bf16, may be anything near 0
        assert torch.equal(out.cpu().double()[:, :, big], want[big].expand(q_len, 4, -1)), byte
        assert (out.cpu().double()[:, :, ~big].abs() <= want[~big].abs() + 2.0 ** -133).all()
        assert (lse == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("q_len", [1, 12, 20, 40])
def test_attention_makes_nan_of_255(q_len, d, dtype):
    q = torch.zeros(q_len, 4, d, dtype=TYPES[dtype], device="cuda")
    table = torch.tensor([0], dtype=torch.int32, device="cuda")
    pages, scale, codes = cache(d, 255)
    pages, scale = pages[:, :, 1:2].contiguous(), scale[:, :, 1:2].contiguous()
    fine = torch.full_like(scale, 127)
    out, lse = torch.empty_like(q), torch.empty(q_len, 4, device="cuda")
    S.prefixattn_run(q, pages, pages, fine, scale, table, 1, None, None, out, lse, 1.0, dtype, q_len=q_len)
    assert out.isnan().all() and (lse == 0).all()
    S.prefixattn_run(q, pages, pages, scale, fine, table, 1, None, None, out, lse, 1.0, dtype, q_len=q_len)
    assert out.isnan().all() and lse.isnan().all()
