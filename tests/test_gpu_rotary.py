"""GPU parity of the rotary positions against complex numbers in 64 bits.

The angle has the product's rounding in fp64 (2^-52 of it with the turn's), its rest
within an eighth of a turn one of 2^-24, sine and cosine at most 4 steps of 2^-24, and
magnitude, products and sum one each: 10 steps of 2^-24 of m (|u| + |v|) together, and
half a step of the output."""
import math

import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _pairs(x, n, layout):
    p = x[..., : 2 * n]
    return torch.complex(*p.chunk(2, -1)) if layout == "half" else torch.complex(p[..., ::2], p[..., 1::2])


def check(got, x, angle, layout, m, what):
    """angle [B, L, pairs] in 64 bits."""
    n = angle.shape[-1]
    xd = x.double()
    z = _pairs(xd, n, layout)
    want = z * torch.polar(torch.full_like(angle, m), angle)[:, :, None]
    out = _pairs(got.double(), n, layout)
    size = abs(m) * (z.real.abs() + z.imag.abs())
    err = 10 * U32 * size + size * (angle.abs() * 2.0 ** -51)[:, :, None] + 1e-38
    worst = 0.0
    for a, b in ((out.real, want.real), (out.imag, want.imag)):
        worst = max(worst, float(((a - b).abs() / (err + HALF_STEP[x.dtype] * b.abs())).max()))
    say(f"  {what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0
    assert torch.equal(got[..., 2 * n:], x[..., 2 * n:])            # the other channels pass as they are


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("B,L,H,Hk,dh,dims", [(1, 1, 1, 0, 2, 2), (2, 3, 2, 1, 7, 4), (1, 5, 3, 3, 10, 10), (3, 17, 4, 2, 64, 64),
                                              (2, 301, 3, 3, 64, 32), (32, 1, 40, 8, 128, 128), (1, 700, 5, 1, 80, 40),
                                              (1, 66, 2, 2, 80, 20), (2, 9, 7, 0, 96, 90), (1, 40, 2, 1, 512, 512),
                                              (1, 33, 3, 1, 511, 510), (1, 5000, 12, 4, 128, 64), (4, 2, 257, 3, 16, 16)])
def test_sizes_and_layouts(B, L, H, Hk, dh, dims, layout, dtype):
    g = _gen(B * L + H + dh)
    say(f"rotary {B}x{L}x{H}+{Hk}x{dh} ({dims}) {layout} {dtype}")
    qkv = torch.randn(B, L, H + 2 * Hk, dh, generator=g).to(dtype)      # queries, keys and values of one product
    on = qkv.to(device())
    rot = api.Rotary.make(dims, device(), layout)
    pos = torch.randint(0, 10 ** 6, (B, L), generator=g, dtype=torch.int32)
    q, k = api.rotary(on[:, :, :H], rot, on[:, :, H:H + Hk] if Hk else None, positions=pos.to(device()))
    torch.cuda.synchronize()
    f = 10000.0 ** (-2 * torch.arange(dims // 2).double() / dims)
    assert torch.allclose(rot.freq.cpu(), f, rtol=1e-14, atol=0) and rot.magnitude == 1.0
    angle = pos.double()[:, :, None] * rot.freq.cpu()
    assert torch.equal(on.cpu(), qkv)
    check(q.cpu(), qkv[:, :, :H], angle, layout, 1.0, "q")
    if Hk:
        check(k.cpu(), qkv[:, :, H:H + Hk], angle, layout, 1.0, "k")
    else:
        assert k is None


@pytest.mark.parametrize("scaling,kw", [("linear", {}), ("base", {}), ("ramp", {}), ("bands", dict(low=1.0, high=4.0))])
def test_scaled_contexts_far_positions(scaling, kw):
    """Positions to the last that 32 bits hold, below zero too, of one row for all
    elements, with a magnitude."""
    g = _gen(1)
    x = torch.randn(2, 9, 3, 128, generator=g)
    pos = torch.tensor([0, 1, -1, 4095, 131071, 10 ** 7, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32)
    rot = api.Rotary.make(128, device(), "half", base=500000.0, scaling=scaling, factor=8.0, original_length=4096, **kw)
    if scaling == "ramp":
        assert abs(rot.magnitude - (1 + 0.1 * math.log(8))) < 1e-6
    y, _ = api.rotary(x.to(device()), rot, positions=pos.to(device()))
    angle = (pos.double()[:, None] * rot.freq.cpu()).expand(2, -1, -1)
    check(y.cpu(), x, angle, "half", rot.magnitude, scaling)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("grid,pairs,dh", [((30, 52), None, 128), ((3, 5), (2, 5, 1), 16), ((1, 1), (8, 0, 0), 20), ((7, 2), (0, 3, 5), 16)])
def test_grid(grid, pairs, dh, layout, dtype):
    """Tokens of a grid, picked ones, turn by frame, row and column."""
    g = _gen(dh)
    dims = dh if pairs is None else 16
    rot = api.Rotary.make(dims, device(), layout, grid=grid, pairs=pairs)
    t, r, c = rot.pairs
    if pairs is None:
        assert (t, r, c) == (22, 21, 21)
    x = torch.randn(2, 50, 3, dh, generator=g).to(dtype)
    tok = torch.randint(0, 21 * grid[0] * grid[1], (50,), generator=g, dtype=torch.int32)
    p = tok.long()
    axes = (p // (grid[0] * grid[1]), p // grid[1] % grid[0], p % grid[1])
    f = [10000.0 ** (-torch.arange(n).double() / n) for n in (t, r, c)]
    assert torch.allclose(rot.freq.cpu(), torch.cat(f), rtol=1e-14, atol=0)
    angle = torch.cat([a.double()[:, None] * v for a, v in zip(axes, rot.freq.cpu().split([t, r, c]))], 1).expand(2, -1, -1)
    y, _ = api.rotary(x.to(device()), rot, positions=tok.to(device()))
    check(y.cpu(), x, angle, layout, 1.0, f"grid {grid}")
    y, _ = api.rotary(x.to(device()), rot)                             # without positions: the tokens in order
    p = torch.arange(50)
    axes = (p // (grid[0] * grid[1]), p // grid[1] % grid[0], p % grid[1])
    angle = torch.cat([a.double()[:, None] * v for a, v in zip(axes, rot.freq.cpu().split([t, r, c]))], 1).expand(2, -1, -1)
    check(y.cpu(), x, angle, layout, 1.0, "in order")


@pytest.mark.parametrize("grid", [(21, 30, 52), (5, 3, 4)])
def test_as_the_wan_style_block_turns(grid):
    """The positions of the Wan-style block, by its own oracle."""
    from oracle import wan_block as OW
    H, dh = 3, 128
    n = grid[0] * grid[1] * grid[2]
    g = _gen(7)
    rows = torch.randint(0, n, (60,), generator=g, dtype=torch.int32)
    x = torch.randn(1, 60, H, dh, generator=g)
    rot = api.Rotary.make(dh, device(), grid=grid[1:])
    got, _ = api.rotary(x.to(device()), rot, positions=rows.to(device()))
    want = torch.from_numpy(OW.apply_rope(x[0].reshape(60, H * dh).double().numpy(), rows.numpy(), grid[1:], H)).view(60, H, dh)
    err = 12 * U32 * x[0].abs().reshape(60, H, dh // 2, 2).sum(-1, keepdim=True).expand(-1, -1, -1, 2).reshape(60, H, dh)
    assert ((got.cpu().double()[0] - want).abs() <= err.double() + 1e-30).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dims", [128, 64, 36])
def test_in_place_strides_and_surroundings(dims, dtype):
    """In place, equal to the call into a new tensor bit for bit; heads first, an offset
    of one element, padded rows; what lies around the output stays."""
    g = _gen(dims)
    rot = api.Rotary.make(dims, device(), "half")
    x = torch.randn(2, 11, 6, 128, generator=g).to(dtype).to(device())
    want, _ = api.rotary(x, rot)
    for i in range(4):
        if i == 0:                                                     # [B, H, L, dh] held, heads first
            t = x.transpose(1, 2).contiguous().transpose(1, 2)
        elif i == 1:                                                   # one element off
            t = torch.zeros(x.numel() + 1, dtype=dtype, device=device())[1:].view(x.shape).copy_(x)
        elif i == 2:                                                   # rows apart
            t = torch.full((2, 11, 7, 131), 5.0, dtype=dtype, device=device())
            t[:, :, :6, :128] = x
        else:
            t = x.clone()
        v = t[:, :, :6, :128]
        new, _ = api.rotary(v, rot)
        assert torch.equal(new, want), i
        q, k = api.rotary(v[:, :, :4], rot, v[:, :, 4:], out=v[:, :, :4], k_out=v[:, :, 4:])
        assert torch.equal(v, want) and q.data_ptr() == v.data_ptr(), i
        if i == 2:
            assert (t[:, :, 6] == 5).all() and (t[..., 128:] == 5).all()
    # the same row for every element (a stride of 0), read only
    one = x[:1].expand(3, -1, -1, -1)
    y, _ = api.rotary(one, rot)
    assert torch.equal(y[2], want[0])
    assert api.rotary(x[:, :0], rot)[0].shape == (2, 0, 6, 128)


def test_values_that_are_not_finite_stay_in_their_pair():
    rot = api.Rotary.make(8, device(), "interleaved")
    x = torch.ones(1, 3, 2, 10, device=device())
    x[0, 1, 0, 2], x[0, 1, 1, 9] = float("nan"), float("inf")
    y = api.rotary(x, rot)[0].cpu()
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[0, 1, 0, 2:4], want[0, 1, 1, 9] = True, True
    assert torch.equal(bad, want)


def test_streams_and_graphs():
    g = _gen(9)
    rot = api.Rotary.make(64, device(), "half")
    x = torch.randn(4, 50, 8, 128, generator=g).bfloat16().to(device())
    pos = torch.arange(50, dtype=torch.int32, device=device())
    side = torch.cuda.Stream()
    want, _ = api.rotary(x, rot, positions=pos)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got, _ = api.rotary(x, rot, positions=pos)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = api.rotary(x, rot, positions=pos)
    for turn in range(3):
        x.mul_(-0.5)
        pos += 1000
        graph.replay()
        ref, _ = api.rotary(x, rot, positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(y, ref), turn
