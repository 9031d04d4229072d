"""sssd_op_rope against 64 bits.  Bound: cos and sin are off by 3 * 2^-25 at most (the rest of the angle after its quarter turns, rounded to 24 bits, its
square and the ends of two polynomials) and multiplied by the magnitude (one more rounding), products and sum round three times: (|a| + |b|) * magnitude *
8 * 2^-24 covers all; bf16 results are rounded once more, by half a step."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from kv8_reference import frequencies, rotate
from paper_2411_05894_amd import kv8

DEV = "cuda:0"
BANDS = dict(scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192)


def check(x, positions, got, rotary, interleaved, magnitude=1.0, **scaling):
    base = scaling.pop("base", 500000.0)
    want = rotate(x, positions, frequencies(rotary, base, **scaling), interleaved, magnitude)
    half = rotary // 2
    a = x.double().abs()
    pair = a.clone()
    if interleaved:
        pair[..., 0:rotary:2] = pair[..., 1:rotary:2] = a[..., 0:rotary:2] + a[..., 1:rotary:2]
    else:
        pair[..., :half] = pair[..., half:rotary] = a[..., :half] + a[..., half:rotary]
    bound = pair * abs(magnitude) * 8 * 2.0 ** -24
    bound[..., rotary:] = 0
    if x.dtype == torch.bfloat16:
        bound[..., :rotary] += (want[..., :rotary].abs() + bound[..., :rotary]) * torch.finfo(torch.bfloat16).eps / 2
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(128, 128), (64, 64), (128, 64), (128, 32), (64, 6), (80, 80), (96, 50), (64, 2), (50, 48), (7, 4), (1024, 1024), (600, 514)])
def test_rotation(dtype, interleaved, d, rotary):
    g = torch.Generator(device=DEV).manual_seed(d + rotary)
    rows, heads = 37, 5
    x = torch.randn(rows, heads, d, generator=g, device=DEV).to(dtype)
    positions = torch.randint(0, 1 << 20, (rows,), generator=g, device=DEV, dtype=torch.int32)
    positions[:4] = torch.tensor([0, 1, (1 << 31) - 1, -3], dtype=torch.int32)
    scaling = BANDS if d == 128 else dict(scaling="linear", factor=4.0) if d == 64 else {}
    rope = kv8.Rope(rotary, 500000.0, interleaved=interleaved, magnitude=1.25, device=DEV, **scaling)
    print(f"rope d={d} rotary={rotary} {dtype} interleaved={interleaved}", flush=True)
    check(x, positions, kv8.sssd_op_rope(x, positions, rope), rotary, interleaved, 1.25, **scaling)
    y = x.clone()
    assert kv8.sssd_op_rope(y, positions, rope, out=y) is y          # in place
    assert torch.equal(y, kv8.sssd_op_rope(x, positions, rope))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_batches(dtype):
    """Queries in the middle of a fused product's rows, at addresses that are and are not multiples of 16 bytes; what lies beside them stays."""
    g = torch.Generator(device=DEV).manual_seed(3)
    rope = kv8.Rope(128, 10000.0, device=DEV)
    for shift in (0, 1, 3):
        flat = torch.randn(3 * 7 * 9 * 128 + shift, generator=g, device=DEV).to(dtype)
        whole = flat[shift:].view(3, 7, 9, 128)
        x = whole[:, :, 2:7]
        positions = torch.randint(0, 4096, (3, 7), generator=g, device=DEV, dtype=torch.int32)
        keep = whole.clone()
        got = kv8.sssd_op_rope(x, positions, rope)
        check(x, positions, got, 128, False, base=10000.0)
        kv8.sssd_op_rope(x, positions, rope, out=x)
        assert torch.equal(x, got)
        assert torch.equal(whole[:, :, :2], keep[:, :, :2]) and torch.equal(whole[:, :, 7:], keep[:, :, 7:])
    t = torch.randn(7, 3, 5, 128, generator=g, device=DEV).to(dtype).transpose(0, 1)     # batches beside each other in memory
    positions = torch.arange(21, device=DEV, dtype=torch.int32).view(3, 7)
    check(t, positions, kv8.sssd_op_rope(t, positions, rope), 128, False, base=10000.0)


def test_one_row_and_many():
    rope = kv8.Rope(64, 10000.0, interleaved=True, device=DEV)
    for rows, heads in ((1, 1), (1, 72), (9001, 3), (257, 40)):
        x = torch.randn(rows, heads, 64, device=DEV)
        positions = torch.arange(rows, device=DEV, dtype=torch.int32) * 13
        check(x, positions, kv8.sssd_op_rope(x, positions, rope), 64, True, base=10000.0)


def test_numbers_that_are_none_stay_in_their_pair():
    x = torch.ones(2, 1, 64, device=DEV)
    x[0, 0, 3], x[1, 0, 40] = float("nan"), float("inf")
    y = kv8.sssd_op_rope(x, torch.tensor([5, 6], dtype=torch.int32, device=DEV), kv8.Rope(64, 10000.0, device=DEV))
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[0, 0, [3, 35]] = bad[1, 0, [8, 40]] = True
    assert torch.equal(~y.isfinite(), bad)


def test_angles():
    """(1, 0) turned: cos and sin themselves, at angles of every quarter and next to their ends."""
    rope = kv8.Rope(128, 10000.0, device=DEV)
    rope.turns[0], rope.turns[1], rope.turns[2], rope.turns[3] = 0.125, 0.25, 1 / 3, 0.125 + 2.0 ** -40
    x = torch.zeros(5000, 1, 128, device=DEV)
    x[..., :64] = 1
    positions = torch.arange(5000, device=DEV, dtype=torch.int32) - 2000
    positions[-100:] = torch.randint(0, 1 << 20, (100,), device=DEV, dtype=torch.int32)
    y = kv8.sssd_op_rope(x, positions, rope).double()
    t = positions.double()[:, None] * rope.turns
    angle = (t - t.round()) * 2 * torch.pi
    err = torch.stack([y[:, 0, :64] - angle.cos(), y[:, 0, 64:] - angle.sin()]).abs()
    assert err.max() <= 3 * 2.0 ** -25
    assert torch.equal(y[positions % 8 == 0][:, 0, 0], torch.ones_like(y[positions % 8 == 0][:, 0, 0]))
