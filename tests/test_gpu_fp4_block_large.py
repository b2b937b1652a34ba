"""The block on 4-bit rows at a width and at counts of tokens where its products run in
the largest tiles, from tile to tile, and split along the depth: three frames of the
14B-shaped block at 480p.  As in test_gpu_fp4_block.py each step is checked in 64 bits on
what the library's step before it gave, and the block against the steps bit for bit."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say
from test_gpu_fp4 import GRID, check_linear, _check_rows
from test_gpu_fp4_tiles import forms
from test_gpu_gated_norm import check as check_norm
from test_gpu_rotary_every_channel import within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
L, D, H, F, EPS = 3 * 30 * 52, 5120, 40, 13824, 1e-6


def _values(r):
    """The values of 4-bit rows in 64 bits, on the device."""
    table = torch.cat((GRID, -GRID)).to(device())
    v = table[torch.stack((r.codes & 15, r.codes >> 4), 2).flatten(1).int()][:, : r.cols]
    return v * torch.exp2(r.scales[:, : (r.cols + 31) // 32].double() - 127).repeat_interleave(32, 1)[:, : r.cols]


@pytest.fixture(scope="module")
def made():
    g = torch.Generator(device=device())
    g.manual_seed(17)

    def r(*s, std=1.0):
        return torch.randn(*s, device=device(), generator=g) * std
    shapes = dict(wq=(D, D), wk=(D, D), wv=(D, D), wo=(D, D), w1=(F, D), w2=(D, F))
    P = {n: r(*s, std=s[1] ** -0.5).bfloat16() for n, s in shapes.items()}
    P.update({n: r(F if n == "b1" else D, std=0.02).bfloat16() for n in ("bq", "bk", "bv", "bo", "b1", "b2")})
    P["mod"] = r(6, D, std=0.1)
    P["mod"][[2, 5]] += 0.25
    Q = api.quantize_block(P, bits=4)
    return {**Q, "after1": 1 + r(D, std=0.1), "after2": 1 + r(D, std=0.1)}, r(L, D).bfloat16()


@pytest.mark.parametrize("n,normed", [(1872, False), (1872, True), (L, False)])
def test_each_step_and_the_block(made, n, normed):
    Q, x = made
    if not normed:
        Q = {k: t for k, t in Q.items() if not k.startswith("after")}
    rot = api.Rotary.make(D // H, device(), grid=(30, 52))
    g = torch.Generator().manual_seed(n)
    idx = torch.randperm(L, generator=g)[:n].sort().values.to(torch.int32).to(device())
    m, at = Q["mod"], torch.randperm(n, generator=g)[:150]         # rows that are looked at where all would take minutes
    up = lambda t: t.cpu().double()  # noqa: E731
    seen = set()

    def linear(a, w, b, **kw):
        y, names = forms(lambda: api.linear_fp4(a, Q[w], Q[b], **kw))
        seen.update(names)
        kw["out_dtype"], kw["act"], res = kw.pop("dtype"), kw.pop("activation", None), kw.pop("residual", None)
        rows = kw.pop("residual_rows", None)
        if res is not None:
            kw["res"] = res if rows is None else res[rows.long()]
        check_linear(y, _values(a), _values(Q[w]), Q[b], what=w, **kw)
        return y

    a, s = api.quantize_rows_fp4(x, shift=m[0], scale=m[1]), api.quantize_rows_fp4(x, rows=idx, shift=m[0], scale=m[1])
    assert torch.equal(s.codes, a.codes[idx.long()]) and torch.equal(s.scales, a.scales[idx.long()])
    q, k, v = (linear(t, "w" + c, "b" + c, dtype=BF).view(1, -1, H, D // H) for t, c in ((s, "q"), (a, "k"), (a, "v")))
    q0, k0 = q.cpu(), k.cpu()
    q, k = api.rotary(q, rot, positions=idx)[0], api.rotary(k, rot)[0]
    for t, t0, p in ((q, q0, idx.cpu().long()), (k, k0, torch.arange(L))):
        p = p[at]
        axes = (p // 1560, p // 52 % 30, p % 52)
        angle = torch.cat([i.double()[:, None] * f for i, f in zip(axes, rot.freq.cpu().split(list(rot.pairs)))], 1)
        assert within(t.cpu()[:, at], t0[:, at], angle[None], "interleaved", 1.0)
    o = api.cross_attention(q, k, v).view(n, D)
    for h in (0, 17, H - 1):
        p = torch.softmax(q[0, :, h].double() @ k[0, :, h].double().T / (D // H) ** 0.5, 1)
        size = p @ v[0, :, h].double().abs()
        off = (o[:, h * 128:(h + 1) * 128].double() - p @ v[0, :, h].double()).abs()
        # each weight and its exponent a rounding of 2^-8 of it off, sums and output as well
        assert bool((off <= 4 * 2.0 ** -8 * size + 1e-6).all())
    so = api.quantize_rows_fp4(o)
    _check_rows(api.Fp4Rows(so.codes[at.to(device())], so.scales[at.to(device())], D), up(o[at.to(device())]))
    if normed:
        z = linear(so, "wo", "bo", dtype=BF)
        x1, c = api.gated_norm(z, x, after_weight=Q["after1"], gate=m[2], residual_rows=idx, scale=m[4], shift=m[3], eps=EPS,
                               y_dtype=F32)
        check_norm(x1.cpu(), c.cpu(), z.cpu(), x.cpu()[idx.cpu().long()], "rms", Q["after1"].cpu(), up(m[2])[None], 1.0,
                   "layer", None, up(m[4])[None], up(m[3])[None], EPS, "after attention")
        b = api.quantize_rows_fp4(c)
    else:
        x1 = linear(so, "wo", "bo", gate=m[2], residual=x, residual_rows=idx, dtype=F32)
        b = api.quantize_rows_fp4(x1, shift=m[3], scale=m[4])
    hid = linear(b, "w1", "b1", activation="gelu", dtype=BF)
    sh = api.quantize_rows_fp4(hid)
    _check_rows(api.Fp4Rows(sh.codes[at.to(device())], sh.scales[at.to(device())], F), up(hid[at.to(device())]))
    if normed:
        z = linear(sh, "w2", "b2", dtype=BF)
        y, _ = api.gated_norm(z, x1, after_weight=Q["after2"], gate=m[5], before=None, eps=EPS)
        check_norm(y.cpu(), None, z.cpu(), x1.cpu(), "rms", Q["after2"].cpu(), up(m[5])[None], 1.0, None, None, None, None,
                   EPS, "y")
    else:
        y = linear(sh, "w2", "b2", gate=m[5], residual=x1, dtype=F32)
    say(f"  products of {n} tokens: {sorted(seen)}")
    assert "gemm_fp4_256_stream" in seen and (normed or "gemm_fp4_reduce" in seen)
    ws = api.Workspace()
    for kw in ({}, dict(workspace=ws), dict(workspace=ws)):
        assert torch.equal(api.block_partial(Q, x, idx, n, H, rotary=rot, **kw), y), kw.keys()
