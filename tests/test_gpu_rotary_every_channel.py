"""Rotary positions, each channel by itself against 64 bits: a comparison that a channel
left out, or one that is no number, fails.

The angle has the product's rounding in fp64 (2^-52 of it with the turn's), its rest
within an eighth of a turn one of 2^-24, sine and cosine at most 4 steps of 2^-24, and
magnitude, products and sum one each: 10 steps of 2^-24 of m (|u| + |v|) together, and
half a step of the output."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

BF, F32 = torch.bfloat16, torch.float32


def within(got, x, angle, layout, m):
    """Whether every channel of got is x turned by angle [B, L, pairs] (64 bits)."""
    n, xd = angle.shape[-1], x.double()
    at_u = torch.arange(n) if layout == "half" else 2 * torch.arange(n)
    at_v = at_u + (n if layout == "half" else 1)
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    u, v = xd[..., at_u], xd[..., at_v]
    want, err = xd.clone(), torch.zeros_like(xd)
    want[..., at_u], want[..., at_v] = m * (u * c - v * s), m * (u * s + v * c)
    size = abs(m) * (u.abs() + v.abs())
    e = 10 * 2.0 ** -24 * size + size * (angle.abs() * 2.0 ** -51)[:, :, None] + 1e-38
    err[..., at_u], err[..., at_v] = e, e
    err[..., : 2 * n] += torch.finfo(x.dtype).eps / 2 * want[..., : 2 * n].abs()
    return bool(((got.double() - want).abs() <= err).all())    # (no comparison with NaN holds)


def _case(g, B, L, H, dh, dims, layout, dtype):
    x = torch.randn(B, L, H, dh, generator=g).to(dtype)
    f = 10000.0 ** (-2 * torch.arange(dims // 2).double() / dims)
    pos = torch.randint(0, 10 ** 6, (B, L), generator=g, dtype=torch.int32)
    return x, f, pos, pos.double()[:, :, None] * f


def test_the_comparison_sees_every_channel():
    """On the host: the formula in 64 bits passes; one channel off, not a number or
    another's does not."""
    g = torch.Generator().manual_seed(1)
    for layout in ("half", "interleaved"):
        x, _, _, angle = _case(g, 2, 3, 2, 10, 6, layout, F32)
        z = torch.complex(*x.double()[..., :6].chunk(2, -1)) if layout == "half" else torch.view_as_complex(
            x.double()[..., :6].unflatten(-1, (-1, 2)).contiguous())
        z = z * torch.polar(torch.ones_like(angle), angle)[:, :, None]
        y = x.clone()
        y[..., :6] = torch.cat((z.real, z.imag), -1) if layout == "half" else torch.view_as_real(z).flatten(-2)
        assert within(y, x, angle, layout, 1.0)
        assert not within(torch.full_like(y, float("nan")), x, angle, layout, 1.0)
        for c in range(10):
            for v in (float("nan"), float("inf"), y[1, 2, 1, c] + 0.01):
                t = y.clone()
                t[1, 2, 1, c] = v
                assert not within(t, x, angle, layout, 1.0), (layout, c, v)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("B,L,H,Hk,dh,dims", [(1, 1, 1, 0, 2, 2), (2, 3, 2, 1, 7, 4), (1, 5, 3, 3, 10, 10), (3, 17, 4, 2, 64, 64),
                                              (2, 301, 3, 3, 64, 32), (32, 1, 40, 8, 128, 128), (1, 700, 5, 1, 80, 40),
                                              (1, 66, 2, 2, 80, 20), (2, 9, 7, 0, 96, 90), (1, 40, 2, 1, 512, 512),
                                              (1, 33, 3, 1, 511, 510), (1, 5000, 12, 4, 128, 64), (4, 2, 257, 3, 16, 16)])
def test_sizes_and_layouts(B, L, H, Hk, dh, dims, layout, dtype):
    """Into new tensors and in place, queries and keys."""
    g = torch.Generator().manual_seed(B * L + H + dh)
    say(f"rotary {B}x{L}x{H}+{Hk}x{dh} ({dims}) {layout} {dtype}")
    x, f, pos, angle = _case(g, B, L, H + Hk, dh, dims, layout, dtype)
    rot, on = api.Rotary(f.to(device()), layout), x.to(device())
    q, k = api.rotary(on[:, :, :H], rot, on[:, :, H:] if Hk else None, positions=pos.to(device()))
    assert within(q.cpu(), x[:, :, :H], angle, layout, 1.0)
    assert k is None if Hk == 0 else within(k.cpu(), x[:, :, H:], angle, layout, 1.0)
    q, k = on[:, :, :H], on[:, :, H:] if Hk else None
    api.rotary(q, rot, k, positions=pos.to(device()), out=q, k_out=k)
    assert within(on.cpu(), x, angle, layout, 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", {}), ("base", {}), ("ramp", {}), ("bands", dict(low=1.0, high=4.0))])
def test_scaled_contexts_far_positions(scaling, kw):
    g = torch.Generator().manual_seed(2)
    x = torch.randn(2, 9, 3, 128, generator=g)
    pos = torch.tensor([0, 1, -1, 4095, 131071, 10 ** 7, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32)
    rot = api.Rotary.make(128, device(), "half", base=500000.0, scaling=scaling, factor=8.0, original_length=4096, **kw)
    y, _ = api.rotary(x.to(device()), rot, positions=pos.to(device()))
    assert within(y.cpu(), x, (pos.double()[:, None] * rot.freq.cpu()).expand(2, -1, -1), "half", rot.magnitude)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("grid,pairs,dh", [((30, 52), (22, 21, 21), 128), ((3, 5), (2, 5, 1), 16), ((1, 1), (8, 0, 0), 20),
                                           ((7, 2), (0, 3, 5), 16)])
def test_grid(grid, pairs, dh, layout, dtype):
    g = torch.Generator().manual_seed(dh)
    rot = api.Rotary.make(2 * sum(pairs), device(), layout, grid=grid, pairs=pairs)
    x = torch.randn(2, 50, 3, dh, generator=g).to(dtype)
    tok = torch.randint(0, 21 * grid[0] * grid[1], (50,), generator=g, dtype=torch.int32)
    for given, p in ((tok.to(device()), tok.long()), (None, torch.arange(50))):
        axes = (p // (grid[0] * grid[1]), p // grid[1] % grid[0], p % grid[1])
        angle = torch.cat([a.double()[:, None] * v for a, v in zip(axes, rot.freq.cpu().split(list(pairs)))], 1)
        y, _ = api.rotary(x.to(device()), rot, positions=given)
        assert within(y.cpu(), x, angle.expand(2, -1, -1), layout, 1.0)
