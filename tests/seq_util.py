"""Helpers of the sequence operators' tests: types, unit roundoffs and the
element-wise comparison."""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# largest relative error of one rounding to nearest
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# largest absolute error where the type is subnormal
FLOOR = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U32 = 2.0 ** -24


def normal(seed, *size, dtype=torch.float32, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(*size, generator=gen, dtype=torch.float64) * scale).to(dtype).cuda()


def check(got, want, bound, what):
    """|got - want| <= bound + the rounding of got's type, element by element;
    infinities and NaN in the same places."""
    want = want.to(got.device)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{what}: other elements are finite"
    odd = ~finite
    assert torch.equal(got[odd].double().nan_to_num(nan=7.0), want[odd].nan_to_num(nan=7.0)), what
    err = (got.double() - want).abs()
    room = bound + UNIT[got.dtype] * (want.abs() + bound) + FLOOR[got.dtype]
    bad = finite & ~(err <= room)
    if bad.any():
        worst = torch.where(bad, err / room, 0.0).max()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} elements out of bounds, "
                             f"worst {worst:.3g} times its bound")
