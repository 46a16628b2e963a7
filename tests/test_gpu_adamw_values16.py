"""GPU: what the codes of 8-bit states stand for, around the workgroups that take sixteen bytes per store (4096 elements of 16 bits, 2048 of
32), against a table of all codes in float64."""
import numpy as np
import pytest
import torch

from paper_1806_04090_amd import binding
from gpu_common import ctx

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
MOST = 3 * 4096 + 130


def at_odd_address(x):
    """A copy of x that starts one element behind an address of sixteen bytes."""
    big = torch.empty(x.numel() + 1, device="cuda", dtype=x.dtype)
    big[1:].copy_(x)
    return big[1:]


def table(which):
    """The 256 values of a code for a block exponent of zero."""
    bias = 7 if which == "m" else 15
    x = []
    for code in range(256):
        c = code & 127 if which == "m" else code
        value = (8 + c % 8) * 2.0 ** (c // 8 - bias - 3) if c >= 8 else c * 2.0 ** (1 - bias - 3)
        if c == (127 if which == "m" else 255):
            value = np.nan
        x.append(-value if c != code else value)
    return np.array(x) * 2.0 ** -bias


@pytest.mark.parametrize("which", ["m", "v"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n", [2047, 2048, 2049, 4095, 4096, 4097, 6144 + 1, 8192, 8192 + 128, MOST])
@pytest.mark.parametrize("odd", [False, True])
def test_values(which, dtype, n, odd):
    rng = np.random.default_rng(n)
    codes = rng.permutation(np.resize(np.arange(256), MOST))[:n].astype(np.uint8)
    scales = rng.permutation(np.resize([0, 1, 2, 20, 60, 105, 120, 127, 128, 140, 200, 254], 98))[:-(-n // 128)].astype(np.uint8)
    want = table(which)[codes] * np.repeat(2.0 ** (np.maximum(scales.astype(np.float64), 1) - 127), 128)[:n]
    with np.errstate(over="ignore"):
        ref = torch.from_numpy(want.astype(np.float32)).to(dtype)                # (what a type cannot hold is rounded, in float32 first)
    place = at_odd_address if odd else lambda x: x
    whole = torch.full((n + 64,), 3.0, device="cuda", dtype=dtype)
    out = whole[32 + odd:32 + odd + n]
    got = binding.atomo_state8_unpack(ctx(), which, place(torch.from_numpy(codes).cuda()), place(torch.from_numpy(scales).cuda()), out=out)
    assert got is out
    assert torch.equal(torch.isnan(out).cpu(), torch.isnan(ref))
    live = ~torch.isnan(ref)
    assert torch.equal(out.cpu()[live], ref[live])
    assert (whole[:32 + odd] == 3).all() and (whole[32 + odd + n:] == 3).all()   # nothing beside
