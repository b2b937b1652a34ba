"""GPU parity of the norms on both sides of a sub-layer against 64 bits.

A norm in fp32 sums at most 16 terms a lane and joins them in 22 steps, so that a
normed value is within 256 steps of 2^-24 of the row's largest (mean, variance, root and
quotient among them).  The second norm divides what the first one left: an error of E
in y is one of at most 2 E / s (1 + |n|) in n = (y - mean) / s, mean(|n|) being below 1."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def norm64(x, kind, eps):
    """(normed, what it was divided by)"""
    if kind is None:
        return x, torch.ones(len(x), 1, dtype=torch.float64)
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    s = (x.square().mean(1, keepdim=True) + eps).sqrt()
    return x / s, s


def check(y, h, z, x, after, w1, gate, alpha, before, w2, scale, shift, eps, what):
    """gate, scale, shift: [M, D] or None, in 64 bits."""
    one = torch.ones(1, dtype=torch.float64)
    g = (one if gate is None else gate) * (one if w1 is None else w1.double())
    n1, _ = norm64(z.double(), after, eps)
    y64 = alpha * x.double() + g * n1
    e1 = 0 if after is None else 256 * U32 * n1.abs().amax(1, keepdim=True)
    e_y = (g.abs() * (e1 + 3 * U32 * n1.abs()) + 3 * U32 * (abs(alpha) * x.double().abs() + (g * n1).abs())) * 1.01 + 1e-38
    worst = float(((y.double() - y64).abs() / (e_y + HALF_STEP[y.dtype] * y64.abs())).max()) if y.numel() else 0.0
    worst_h = 0.0
    if before is not None:
        n2, s = norm64(y64, before, eps)
        e2 = 2 * e_y.amax(1, keepdim=True) / s * (1 + n2.abs()) + 256 * U32 * n2.abs().amax(1, keepdim=True)
        m = (one if w2 is None else w2.double()) * (one if scale is None else 1 + scale)
        t = torch.zeros(1, dtype=torch.float64) if shift is None else shift
        want = n2 * m + t
        e_h = (e2 * m.abs() + 4 * U32 * ((n2 * m).abs() + t.abs())) * 1.01 + 1e-38
        worst_h = float(((h.double() - want).abs() / (e_h + HALF_STEP[h.dtype] * want.abs())).max()) if h.numel() else 0.0
    say(f"  {what}: worst error {worst:.3f} and {worst_h:.3f} of the bounds")
    assert worst <= 1.0 and worst_h <= 1.0


SIZES = [(1, 1), (2, 7), (5, 8), (3, 33), (70, 64), (4, 250), (9, 512), (5, 513), (6, 1536), (3, 2047), (2, 2056), (11, 5120),
         (3, 6144), (2, 6145), (4, 8192), (2, 13824), (3, 16384), (2, 16383), (3000, 64), (2500, 520)]


@pytest.mark.parametrize("after,before", [("rms", "layer"), ("layer", "rms"), (None, "layer"), ("rms", None), (None, "rms")])
@pytest.mark.parametrize("M,D", SIZES)
def test_sizes_and_norms(M, D, after, before):
    g = _gen(M * 31 + D)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    zt, xt = (BF, F32) if D % 3 else (F32, BF)
    z, x = (r(M, D) * 3 + 1).to(zt), r(M, D).to(xt)
    w1, w2, gate, scale, shift = 1 + 0.1 * r(D), 1 + 0.1 * r(D), r(D), 0.1 * r(D), 0.1 * r(D)
    d = lambda t: t.to(device())  # noqa: E731
    kw = dict(before_weight=d(w2), scale=d(scale), shift=d(shift)) if before else {}
    y, h = api.gated_norm(d(z), d(x), after=after, after_weight=d(w1), gate=d(gate), residual_scale=0.7, before=before,
                          eps=1e-6, **kw)
    torch.cuda.synchronize()
    assert y.dtype == xt and (h is None) == (before is None) and (h is None or h.dtype == zt)
    check(y.cpu(), None if h is None else h.cpu(), z, x, after, w1, gate.double()[None], 0.7, before, w2,
          scale.double()[None], shift.double()[None], 1e-6, f"{M}x{D} {after} {before}")


@pytest.mark.parametrize("zt,xt,yt,ht", [(BF, BF, BF, BF), (BF, F32, F32, BF), (F32, F32, F32, F32), (F32, BF, F32, BF),
                                         (BF, BF, F32, F32), (BF, F32, BF, F32)])
@pytest.mark.parametrize("D", [40, 1536, 5125])
def test_types_nothing_optional(D, zt, xt, yt, ht):
    g = _gen(D)
    z, x = torch.randn(13, D, generator=g).to(zt), torch.randn(13, D, generator=g).to(xt)
    y, h = api.gated_norm(z.to(device()), x.to(device()), y_dtype=yt, h_dtype=ht)
    assert y.dtype == yt and h.dtype == ht
    check(y.cpu(), h.cpu(), z, x, "rms", None, None, 1.0, "layer", None, None, None, 1e-6, f"{zt} {xt}")


@pytest.mark.parametrize("D", [64, 250, 5120, 7000])
def test_groups_and_picked_rows(D):
    """A modulation for each of G groups: equal shares of the rows, or an index for each
    row; residual rows picked, the same one twice; rows and groups that are not there
    are NaN, alone; modulations of one row and of G together, their rows apart."""
    g = _gen(D + 5)
    M, G, n = 60, 3, 25
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    z, x, w = r(M, D), r(n, D), r(D)
    mod, shift = 0.3 * r(G, 4, D), 0.1 * r(1, D)
    rows = torch.randint(0, n, (M,), generator=g, dtype=torch.int32)
    groups = torch.randint(0, G, (M,), generator=g, dtype=torch.int32)
    rows[4], rows[40], groups[9], groups[41] = -1, n, G, -1
    m = mod.to(device())
    for given in (None, groups):
        y, h = api.gated_norm(z.to(device()), x.to(device()), after="layer", after_weight=w.to(device()), gate=m[:, 1],
                              residual_rows=rows.to(device()), scale=m[:, 3], shift=shift.to(device()),
                              groups=None if given is None else given.to(device()))
        y, h = y.cpu(), h.cpu()
        at = torch.arange(M) // (M // G) if given is None else given.long()
        ok = (rows >= 0) & (rows < n) & (at >= 0) & (at < G)
        assert torch.isnan(y[~ok]).all() and torch.isnan(h[~ok]).all() and int((~ok).sum()) == (2 if given is None else 4)
        at, md = at[ok], mod.double()
        check(y[ok], h[ok], z[ok], x[rows[ok].long()], "layer", w, md[at, 1], 1.0, "layer", None, md[at, 3],
              shift.double(), 1e-6, f"groups {D}")


@pytest.mark.parametrize("D", [128, 130, 1536, 6200])
def test_in_place_and_surroundings(D):
    """y in the residual's place and h in z's equal new tensors bit for bit; rows apart,
    what lies around them stays."""
    g = _gen(D)
    M = 37
    z, x, gate = (torch.randn(M, D, generator=g).bfloat16().to(device()), torch.randn(M, D, generator=g).to(device()),
                  torch.randn(D, generator=g).to(device()))
    y, h = api.gated_norm(z, x, gate=gate, residual_scale=0.5)
    z2, x2 = z.clone(), x.clone()
    a, b = api.gated_norm(z2, x2, gate=gate, residual_scale=0.5, y=x2, h=z2)
    assert a is x2 and b is z2 and torch.equal(x2, y) and torch.equal(z2, h)
    for off in (0, 8, 3):
        wy, wh = torch.full((M + 2, D + 24), 7.0, device=device()), torch.full((M + 2, D + 24), 7.0, dtype=BF, device=device())
        api.gated_norm(z, x, gate=gate, residual_scale=0.5, y=wy[1:-1, off:off + D], h=wh[1:-1, off:off + D])
        if off != 3 or D % 8:
            assert torch.equal(wy[1:-1, off:off + D], y) and torch.equal(wh[1:-1, off:off + D], h)
        for w in (wy, wh):
            w[1:-1, off:off + D] = 7
            assert (w == 7).all()


def test_edges():
    """Rows of zeros, of one value, not finite (alone), no rows, one column."""
    z = torch.randn(6, 96, generator=_gen(0))
    x = torch.zeros(6, 96)
    z[0], z[1], z[2, 5], z[3, 7], z[4] = 0, 3, float("nan"), float("inf"), 1e-30
    x[5, 3] = float("inf")
    y, h = (t.cpu() for t in api.gated_norm(z.to(device()), x.to(device()), after="layer"))
    assert (y[:2] == 0).all() and (h[:2] == 0).all()
    assert torch.isnan(y[2]).all() and torch.isnan(h[2:4]).all() and torch.isfinite(y[4]).all()
    assert torch.isinf(y[5, 3]) and torch.isnan(h[5]).any()
    big = torch.full((2, 64), 1e4).bfloat16()
    y, h = api.gated_norm(big.to(device()), torch.zeros(2, 64, device=device()), before="rms")
    assert (y.cpu() == 1).all() and ((h.float().cpu() - 1).abs() < 2.0 ** -7).all()
    e = torch.zeros(0, 64, device=device())
    y, h = api.gated_norm(e, e)
    assert y.shape == h.shape == (0, 64)
    w = torch.randn(2, 64, device=device())
    assert api.gated_norm(e, e, gate=w)[0].shape == (0, 64)


def test_streams_and_graphs():
    g = _gen(9)
    z, x = torch.randn(500, 1536, generator=g).bfloat16().to(device()), torch.randn(500, 1536, generator=g).to(device())
    want = api.gated_norm(z, x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = api.gated_norm(z, x)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = api.gated_norm(z, x)
    for turn in range(3):
        z.mul_(-0.5)
        graph.replay()
        ref = api.gated_norm(z, x)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), turn
