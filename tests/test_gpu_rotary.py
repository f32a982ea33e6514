"""Rotary positions on the GPU against the definition in 64 bits.

Tolerance: a result is rounded once to bf16 (half a step: 2^-8 of it), from sines and cosines that are
off by at most 2^-20 (their approximations' 2^-21.4 over [-pi, pi], the angle's own rounding and the
gain's product) on two inputs, and two 32-bit roundings: 2^-8 |y| + 2^-19 gain (|u| + |v|)."""
import pytest
import torch

import paper_2609_32046_gb300 as cb
import packed_reference as ref

pytestmark = pytest.mark.gpu


def _rx(d):
    return cb.Receiver(1, 1, 1, d, 1, 1, 1)


def _x(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def _check(y, x, pos, f, gain, style, inverse=False):
    want = ref.rotary(x, pos, f, gain, style, inverse)
    size = ref.rotary(x.abs(), torch.zeros_like(pos), f, gain, style)
    r = 2 * len(f)
    first = torch.arange(r // 2, device=x.device) * (1 if style == "halves" else 2)
    second = first + (r // 2 if style == "halves" else 1)
    both = torch.zeros_like(size)
    both[..., first] = both[..., second] = size[..., first] + size[..., second]
    err = (y.double() - want).abs()
    assert (err <= want.abs() * 2.0 ** -8 + both * 2.0 ** -19).all(), float((err - want.abs() * 2.0 ** -8).max())
    assert torch.equal(ref.bf16_bits(y[..., r:]), ref.bf16_bits(x[..., r:]))       # behind the rotary part: as they were


@pytest.mark.parametrize("style", ["halves", "pairs"])
@pytest.mark.parametrize("d,dims", [(64, 0), (64, 16), (64, 48), (128, 0), (128, 32), (128, 64), (128, 112)])
@pytest.mark.parametrize("inverse", [False, True])
def test_layouts_and_parts(style, d, dims, inverse):
    q, k = _x((2, 37, 5, d), 1), _x((2, 37, 1, d), 2)
    rope = cb.Rotary(1e4, style, dims)
    y = _rx(d).rotary([q, k], rope, [torch.empty_like(q), torch.empty_like(k)], pos0=1000, inverse=inverse)
    f, gain = ref.frequencies(dims or d, 1e4)
    pos = torch.arange(37, device="cuda") + 1000
    for a, b in zip(y, (q, k)):
        _check(a, b, pos, f, gain, style, inverse)


@pytest.mark.parametrize("scaling,factor,original,base", [
    ("linear", 4.0, 0, 1e4), ("yarn", 4.0, 32768, 1e6), ("yarn", 16.0, 4096, 1e4), ("yarn", 1.0, 8, 1e4),
    ("yarn", 2.0, 1 << 40, 1e4)])
@pytest.mark.parametrize("d,dims", [(128, 0), (64, 32)])
def test_scaled_positions(scaling, factor, original, base, d, dims):
    x = _x((1, 50, 3, d), 3)
    pos = torch.randint(0, 1 << 20, (50,), dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    _rx(d).rotary([x], cb.Rotary(base, "halves", dims, scaling, factor, original), [y], pos=pos)
    f, gain = ref.frequencies(dims or d, base, scaling, factor, original)
    _check(y, x, pos, f, gain, "halves")
    _rx(d).rotary([x], cb.Rotary(base, "halves", dims, scaling, factor, original, attention=0.5), [y], pos=pos)
    _check(y, x, pos, f, 0.5, "halves")


def test_far_negative_and_equal_positions():
    x = _x((1, 6, 2, 128), 4)
    pos = torch.tensor([-(1 << 31), -1, 0, 5, 5, (1 << 31) - 1], dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    rx = _rx(128)
    rx.rotary([x], cb.Rotary(1e6), [y], pos=pos)
    f, gain = ref.frequencies(128, 1e6)
    _check(y, x, pos.long(), f, gain, "halves")
    assert torch.equal(ref.bf16_bits(y[:, 2]), ref.bf16_bits(x[:, 2]))                # position 0: as it was
    rx.rotary([x], cb.Rotary(1e6), [y], pos0=1 << 31)
    _check(y, x, torch.arange(6, device="cuda") + (1 << 31), f, gain, "halves")


@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_in_place_inside_a_wider_tensor(style):
    """Queries and keys inside a fused [tokens][heads + 2 kv heads][d] tensor; what lies beside them stays."""
    qkv = _x((70, 4 + 2 * 2, 64), 5)
    before = qkv.clone()
    q, k = qkv[:, :4], qkv[:, 4:6]
    rx = _rx(64)
    rope = cb.Rotary(1e4, style, 32)
    rx.rotary([q, k], rope, pos0=9)
    f, gain = ref.frequencies(32, 1e4)
    pos = torch.arange(70, device="cuda") + 9
    _check(q, before[:, :4], pos, f, gain, style)
    _check(k, before[:, 4:6], pos, f, gain, style)
    assert torch.equal(ref.bf16_bits(qkv[:, 6:]), ref.bf16_bits(before[:, 6:]))
    # head-major output, layers last but one
    x = _x((3, 40, 4, 64), 6)
    y = torch.empty((4, 40, 3, 64), dtype=torch.bfloat16, device="cuda")
    rx.rotary([x], rope, [y.permute(2, 1, 0, 3)])
    _check(y.permute(2, 1, 0, 3), x, torch.arange(40, device="cuda"), f, gain, style)


def test_transposed_turn_is_the_gradient():
    """<g, R x> = <R^T g, x>, the forward turn's differences against the transposed one (64-bit sums of
    bf16 results: within the sum of both sides' tolerances)."""
    x, g = _x((1, 20, 2, 128), 7), _x((1, 20, 2, 128), 8)
    rx, rope = _rx(128), cb.Rotary(1e4, "pairs", 64, "yarn", 4.0, 4096)
    y, back = (torch.empty_like(x) for _ in range(2))
    rx.rotary([x], rope, [y], pos0=50)
    rx.rotary([g], rope, [back], pos0=50, inverse=True)
    left, right = (g.double() * y.double()).sum(), (back.double() * x.double()).sum()
    bound = 2.0 ** -8 * ((g.double() * y.double()).abs().sum() + (back.double() * x.double()).abs().sum())
    assert abs(left - right) <= bound
    # a difference of the forward turn along one element is a column of R
    e = torch.zeros_like(x)
    e[..., 6] = 1.0
    col, row = torch.empty_like(x), torch.empty_like(x)
    rx.rotary([e], rope, [col], pos0=50)
    rx.rotary([e], rope, [row], pos0=50, inverse=True)
    assert torch.equal(ref.bf16_bits(col[..., 6]), ref.bf16_bits(row[..., 6]))
    assert torch.equal(col[..., 7], -row[..., 7])


def test_many_sets_and_empty_ones():
    xs = [_x((1, i % 5, 2, 64), i) for i in range(70)]
    ys = _rx(64).rotary(xs, cb.Rotary(1e4), [torch.empty_like(x) for x in xs], pos0=3)
    f, gain = ref.frequencies(64, 1e4)
    for x, y in zip(xs, ys):
        if x.numel():
            _check(y, x, torch.arange(x.shape[1], device="cuda") + 3, f, gain, "halves")


def test_refusals():
    x = _x((1, 8, 2, 64), 1)
    rx = _rx(64)
    for rope in (cb.Rotary(1.0), cb.Rotary(float("nan")), cb.Rotary(1e4, dims=8), cb.Rotary(1e4, dims=80),
                 cb.Rotary(1e4, scaling="linear", factor=0.5), cb.Rotary(1e4, scaling="yarn", factor=2.0),
                 cb.Rotary(1e4, scaling="yarn", factor=2.0, original=100, beta_fast=1.0, beta_slow=2.0),
                 cb.Rotary(1e4, attention=-1.0)):
        with pytest.raises(cb.CBError, match="CB_EINVAL"):
            rx.rotary([x], rope)
    ok = cb.Rotary(1e4)
    for call in (lambda: rx.rotary([x.cpu()], ok),
                 lambda: rx.rotary([x[:, 1:]], ok, [x[:, :7]]),                     # overlapping, not in place
                 lambda: rx.rotary([x], ok, pos0=1 << 41),
                 lambda: rx.rotary([x], ok, pos=torch.zeros(8, dtype=torch.int32)),
                 lambda: rx.rotary([x], ok, [torch.empty(64, dtype=torch.bfloat16, device="cuda").expand(1, 8, 2, 64)])):
        with pytest.raises(cb.CBError, match="CB_EINVAL"):
            call()
    with pytest.raises(cb.CBError, match="CB_ESHAPE"):
        rx.rotary([], ok)
    with pytest.raises(ValueError):
        rx.rotary([x], ok, pos=torch.zeros(7, dtype=torch.int32, device="cuda"))
    before = x.clone()
    rx.sync_status()
    assert torch.equal(x, before)


def test_lists_and_types_that_do_not_fit_are_refused():
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    rx, rope = cb.Receiver(1, 2, 2, 64, 8, 64), cb.Rotary(1e4)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in (lambda: rx.rotary([x, x], rope, [x]), lambda: rx.rotary([x, x], rope, pos=[pos]),
                 lambda: rx.rotary([x.half()], rope), lambda: rx.rotary([x], rope, pos=pos.float())):
        with pytest.raises(ValueError):
            call()
