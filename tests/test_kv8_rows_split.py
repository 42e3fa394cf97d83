"""bf16 query rows as two 8-bit numbers (the kernels for many rows): what the split loses, for
every bf16 number of a row whose largest lies in [128, 256)."""
import torch


def test_rounding_to_e4m3_and_the_rest_in_e5m2():
    x = torch.arange(0x0080, 0x4380, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()   # 2^-126 .. 256
    top = x.to(torch.float8_e4m3fn).float()
    rest = (x - top).to(torch.float8_e5m2).float()
    err = (x - top - rest).abs()
    assert err[x >= 2.0 ** -6].max() == 0            # 2^-13 of a largest value above 2^7
    assert err.max() <= 2.0 ** -14                   # 2^-21 of it
