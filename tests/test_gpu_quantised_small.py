"""What codes stand for at the ends of the scale bytes' range: fp32 holds every such number, bf16 all from byte 3 on and rounds below."""
import pytest
import torch

import plain_cache as pc
from paper_2510_26475_amd import binding
from plain_cache import ints

pytestmark = pytest.mark.gpu


def read_back(codes, bytes_, dtype):
    """codes [tokens, Hkv, D] and bytes [tokens, Hkv] through pools of one page of 256 tokens."""
    n, Hkv, D = codes.shape
    pool = torch.zeros((1, 256, Hkv, D), dtype=torch.uint8, device="cuda")
    scale = torch.ones((1, Hkv, 256), dtype=torch.uint8, device="cuda")
    pool[0, :n], scale[0, :, :n] = codes, bytes_.t()
    out = [torch.empty((n, Hkv, D), dtype=dtype, device="cuda") for _ in range(2)]
    binding.respec_read_paged_quantised(pool, pool.clone(), scale, scale.clone(), ints([0, 1]), ints([0]), ints([n]), ints([0, n], torch.int64), *out, n)
    assert torch.equal(out[0].view(torch.uint8), out[1].view(torch.uint8))
    return out[0].cpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_code_under_every_byte(dtype):
    """float32 is exact; bf16 is float32 rounded once to nearest even, its subnormals included, which changes nothing from byte 3 on."""
    byte = torch.arange(1, 248)
    codes = torch.arange(256).view(1, 2, 128).expand(247, 2, 128).to(torch.uint8)
    want = pc.values(codes, byte[:, None].expand(247, 2).to(torch.uint8))
    small = want.abs() < 2.0 ** 128                               # (codes past 240 under byte 247: infinite)
    assert torch.equal(want.float().double()[small], want[small]) and torch.isinf(want.float()[want.abs() >= 2.0 ** 128]).all()
    got = read_back(codes.cuda(), byte[:, None].expand(247, 2).to(torch.uint8).cuda(), dtype)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    rounded = want.float().to(dtype)
    assert torch.equal(got[~nan], rounded[~nan])
    if dtype == torch.bfloat16:
        assert torch.equal(rounded[2:].double()[small[2:]], want[2:][small[2:]])


@pytest.mark.parametrize("power", [-149, -148, -140, -133, -130, -127, -126, -120, -118])
def test_heads_of_tiny_numbers(power):
    """Written and read back: in float32 what the codes stand for, half a step of e4m3 from what was written (of the least scale's subnormals: 2^-136)."""
    v = torch.linspace(-1, 1, 2 * 128, dtype=torch.float64).view(1, 2, 128)
    v = torch.ldexp(v, torch.tensor(power)).float().cuda()
    pools = [torch.zeros((1, 16, 2, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((1, 2, 16), dtype=torch.uint8, device="cuda") for _ in range(2)]
    tables = ints([0, 1]), ints([0]), ints([1])
    binding.respec_norm_rope_append_paged(None, v, v, None, None, None, None, None, *pools, *scales, ints([0, 1]), *tables, 1, 0.0)
    code, byte = pc.quantise(v.cpu())
    assert torch.equal(pools[0][0, 0].cpu(), code[0]) and torch.equal(scales[0][0, :, 0].cpu(), byte[0])
    out = [torch.empty_like(v) for _ in range(2)]
    binding.respec_read_paged_quantised(*pools, *scales, *tables, ints([0, 1], torch.int64), *out, 1)
    for o in out:
        assert torch.equal(o.cpu().double(), pc.values(code, byte))
        ref = v.cpu().double()
        assert ((o.cpu().double() - ref).abs() <= torch.maximum(2.0 ** -4 * ref.abs(), torch.tensor(2.0 ** -136, dtype=torch.float64))).all()
