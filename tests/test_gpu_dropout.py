"""Dropout against a big-integer Philox4x32-10 and plain arithmetic: the mask is
exact, a kept value is x * scale rounded once to fp32 (plus the residual, which
may be contracted with it: one rounding less), then once to its type."""
import pytest
import torch

from tests.seq_util import TYPES, U32, check, normal

pytestmark = pytest.mark.gpu


def philox(counter, offset, seed):
    """Salmon, Moraes, Dror & Shaw (2011), with Python integers."""
    low = 2 ** 32 - 1
    c = [counter & low, counter >> 32, offset & low, offset >> 32]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def mask(n, p, seed, offset):
    t = round(p * 65536)
    got = []
    for g in range((n + 7) // 8):
        for word in philox(g, offset, seed):
            got += [(word & 0xFFFF) >= t, (word >> 16) >= t]
    return torch.tensor(got[:n], dtype=torch.bool)


def ops():
    from paper_2207_10731_gb300 import sequence
    return sequence


def test_the_generator_itself():
    # the published known answers of philox4x32-10
    assert philox(0, 0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 2 ** 64 - 1
    assert philox(ones, ones, ones) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,gap,shift", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0),
                                                 (64, 128, 0, 0), (127, 129, 0, 0), (127, 129, 31, 0),
                                                 (50, 64, 16, 0), (50, 64, 17, 0), (50, 64, 16, 1),
                                                 (1, 4001, 0, 0), (2000, 7, 0, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_against_the_definition(kind, rows, cols, gap, shift, residual):
    dtype, seed, offset, p = TYPES[kind], 0xFEDCBA9876543210, 2 ** 40 + 5, 0.3
    x = normal(1, rows, cols + gap + shift, dtype=dtype)[:, shift:shift + cols]
    add = normal(2, rows, cols + gap + shift, dtype=dtype)[:, shift:shift + cols]
    y = ops().dropout(x, p, seed, offset, residual=add if residual else None)
    keep = mask(rows * cols, p, seed, offset).view(rows, cols).cuda()
    scale = 65536 / (65536 - round(p * 65536))
    want = torch.where(keep, x.double() * scale, 0.0)
    bound = 2 * U32 * want.abs()
    if residual:
        want = want + add.double()
        bound = bound + U32 * want.abs()
    else:
        assert torch.equal(y[~keep], torch.zeros_like(y[~keep]))
    check(y, want, bound, "y")
    # the backward pass is the same mask
    assert torch.equal(ops().dropout(torch.ones_like(x), p, seed, offset) != 0, keep)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.5, 1 - 1e-6, 1.0])
def test_probabilities_at_the_ends(p):
    x = normal(3, 33, 40)
    y = ops().dropout(x, p, seed=1)
    if round(p * 65536) == 0:
        assert torch.equal(y, x)
    elif round(p * 65536) == 65536:
        assert torch.equal(y, torch.zeros_like(x))
    else:
        assert torch.equal(y == 0, ~mask(x.numel(), p, 1, 0).view(x.shape).cuda())


def test_dropped_places_are_zero_whatever_they_hold():
    x = torch.full((64, 64), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = ops().dropout(x, 0.5, seed=9, offset=4)
    keep = mask(x.numel(), 0.5, 9, 4).view(x.shape).cuda()
    assert torch.equal(y[~keep], torch.zeros_like(y[~keep]))
    assert not y[keep].isfinite().any()
    add = normal(4, 64, 64)
    y = ops().dropout(x, 0.5, seed=9, offset=4, residual=add)
    assert torch.equal(y[~keep], add[~keep])


def test_in_place_and_share_kept():
    x = normal(5, 3000, 1024, dtype=torch.bfloat16)
    want = ops().dropout(x, 0.1, seed=2)
    n, kept = x.numel(), int((want != 0).sum())
    # binomial: 6 standard deviations (about 1e-9), and no x is zero
    q = 1 - round(0.1 * 65536) / 65536
    assert (x != 0).all() and abs(kept - n * q) < 6 * (n * q * (1 - q)) ** 0.5
    add = normal(6, 3000, 1024, dtype=torch.bfloat16)
    both = ops().dropout(x, 0.1, seed=2, residual=add)
    assert torch.equal(ops().dropout(x, 0.1, seed=2, residual=add, out=add), both)
    assert torch.equal(ops().dropout(x, 0.1, seed=2, out=x), want)
    # another offset or seed is another mask: equal in about q^2 + (1 - q)^2 of the places
    ones = torch.ones(1 << 20, device="cuda")
    a = ops().dropout(ones, 0.5, seed=2)
    for b in (ops().dropout(ones, 0.5, seed=3), ops().dropout(ones, 0.5, seed=2, offset=1)):
        assert abs(float((a == b).float().mean()) - 0.5) < 6 * 0.5 / 2 ** 10


def test_positions_past_32_bits():
    # 2^32 + 24 elements of one run: the element index
    # does not fit 32 bits
    n = 2 ** 32 + 24
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = ops().dropout(x, 0.5, seed=77, offset=3, out=x)
    low, want = n - 64, []
    for g in range(low // 8, n // 8):
        for word in philox(g, 3, 77):
            want += [(word & 0xFFFF) >= 32768, (word >> 16) >= 32768]
    assert (y[low:] != 0).cpu().tolist() == want


def test_empty_and_refusals():
    from paper_2207_10731_gb300 import binding
    x = normal(7, 4, 32)
    drop = ops().dropout
    assert drop(x[:0], 0.5, seed=0).shape == (0, 32)
    assert drop(x[:, :0], 0.5, seed=0).shape == (4, 0)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(binding.PSSError) as e:
            drop(x, p, seed=0)
        assert e.value.status == binding.PSS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        drop(x, 0.5, seed=2 ** 64)
    with pytest.raises(ValueError):
        drop(x, 0.5, seed=0, offset=-1)
    with pytest.raises(TypeError):
        drop(x, 0.5, seed=0, residual=x.half())
    with pytest.raises(ValueError):
        drop(x, 0.5, seed=0, residual=x[:2])
    with pytest.raises(ValueError):
        drop(x.cpu(), 0.5, seed=0)
    with pytest.raises(TypeError):
        drop(x.long(), 0.5, seed=0)
    with pytest.raises(ValueError):
        drop(x[:, ::2], 0.5, seed=0)
