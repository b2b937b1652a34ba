"""The block on 4-bit and 8-bit rows with rotary positions and norms after its
sub-layers: the operators run together as block_partial runs them.

A token's value next to a border of two 4-bit codes takes the one or the other by its
last rounding, so an oracle of the whole block in 64 bits says little; each step is
therefore checked in 64 bits on what the library's step before it gave, and the block
against the steps bit for bit."""
import math

import pytest
import torch

import synth
from paper_2608_02474_amd import api

from gpu_util import device, say
from test_gpu_fp4 import check_linear, unpacked, values_of, _check_rows
from test_gpu_gated_norm import check as check_norm
from test_gpu_rotary import check as check_rotary

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24


def _make(dtype, bits, after=(), L=300, seed=31):
    w = synth.Workload("fp4_300tok", T=3, grid=(10, 10), D=256, H=2, F=512, n_samples=4000, ratio=0.37,
                       dtype=dtype, audio="speech", seed=seed)
    dt = BF if dtype == "bf16" else F32
    P = {k: torch.from_numpy(v).to(F32 if k == "mod" else dt).to(device()) for k, v in synth.make_block_weights(w).items()}
    xref, x = (torch.from_numpy(t).to(dt).to(device()) for t in synth.make_latents(w))
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    Q = api.quantize_block(P, bits=bits)
    Q.update({n: (1 + 0.1 * torch.randn(w.D, generator=g)).to(device()) for n in after})
    return w, dt, P, Q, xref, x


def _values(r):
    code, byte = unpacked(r)
    return values_of(code.view(len(r), -1, 32), byte[:, : code.shape[1] // 32])[:, : r.cols]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("after", [(), ("after1", "after2"), ("after2",)])
@pytest.mark.parametrize("turned", [False, True])
def test_each_step_and_the_block(dtype, after, turned):
    w, dt, P, Q, xref, x = _make(dtype, 4, after)
    assert api.is_fp4_block(Q) and not api.is_int8_block(Q) and not api.is_fp4_block(P)
    L, D, H, dh, eps = w.L, w.D, w.H, w.dh, 1e-6
    rot = api.Rotary.make(dh, device(), grid=w.grid) if turned else None
    idx = torch.arange(0, L, 3, dtype=torch.int32, device=device())[:90]
    n, m = len(idx), Q["mod"]
    up = lambda t: t.cpu().double()  # noqa: E731
    W = {name: _values(Q[name]) for name in ("wq", "wk", "wv", "wo", "w1", "w2")}
    for name in W:
        _check_rows(Q[name], up(P[name]), name)

    a, s = api.quantize_rows_fp4(x, shift=m[0], scale=m[1]), api.quantize_rows_fp4(x, rows=idx, shift=m[0], scale=m[1])
    assert torch.equal(s.codes, a.codes[idx.long()]) and torch.equal(s.scales, a.scales[idx.long()])
    q, k, v = (api.linear_fp4(t, Q["w" + c], P["b" + c], dtype=dt) for t, c in ((s, "q"), (a, "k"), (a, "v")))
    for t, r, c in ((q, s, "q"), (k, a, "k"), (v, a, "v")):
        check_linear(t.cpu(), _values(r), W["w" + c], P["b" + c].cpu(), dt, what=c)
    q, k, v = (t.view(1, -1, H, dh) for t in (q, k, v))
    if turned:
        q0, k0 = q.cpu(), k.cpu()
        q, k = api.rotary(q, rot, positions=idx)[0], api.rotary(k, rot)[0]
        for t, t0, p in ((q, q0, idx.cpu().long()), (k, k0, torch.arange(L))):
            axes = (p // 100, p // 10 % 10, p % 10)
            angle = torch.cat([i.double()[:, None] * f for i, f in zip(axes, rot.freq.cpu().split(list(rot.pairs)))], 1)
            check_rotary(t.cpu(), t0, angle[None], "interleaved", 1.0, "turned")
    o = api.cross_attention(q, k, v).view(n, D)
    for h in range(H):
        p = torch.softmax(up(q)[0, :, h] @ up(k)[0, :, h].T / math.sqrt(dh), 1)
        want = p @ up(v)[0, :, h]
        # each weight and its exponent a rounding of the type's (2^-8 or 2^-24 of it) off, sums and output as well
        e = 2.0 ** -8 if dt == BF else 64 * U32
        assert ((up(o)[:, h * dh:(h + 1) * dh] - want).abs() <= 4 * e * (p @ up(v)[0, :, h].abs()) + 1e-6).all()
    so = api.quantize_rows_fp4(o)
    _check_rows(so, up(o))
    if "after1" in after:
        z = api.linear_fp4(so, Q["wo"], P["bo"], dtype=dt)
        check_linear(z.cpu(), _values(so), W["wo"], P["bo"].cpu(), dt, what="o")
        x1, c = api.gated_norm(z, x, after_weight=Q["after1"], gate=m[2], residual_rows=idx, scale=m[4], shift=m[3], eps=eps,
                               y_dtype=F32)
        check_norm(x1.cpu(), c.cpu(), z.cpu(), x.cpu()[idx.cpu().long()], "rms", Q["after1"].cpu(), up(m[2])[None], 1.0,
                   "layer", None, up(m[4])[None], up(m[3])[None], eps, "after attention")
        b = api.quantize_rows_fp4(c)
        _check_rows(b, up(c))
    else:
        x1 = api.linear_fp4(so, Q["wo"], P["bo"], gate=m[2], residual=x, residual_rows=idx, dtype=F32)
        check_linear(x1.cpu(), _values(so), W["wo"], P["bo"].cpu(), F32, gate=m[2].cpu(), res=x.cpu()[idx.cpu().long()], what="x1")
        b = api.quantize_rows_fp4(x1, shift=m[3], scale=m[4])
    hid = api.linear_fp4(b, Q["w1"], P["b1"], activation="gelu", dtype=dt)
    check_linear(hid.cpu(), _values(b), W["w1"], P["b1"].cpu(), dt, act="gelu", what="hidden")
    sh = api.quantize_rows_fp4(hid)
    if "after2" in after:
        z = api.linear_fp4(sh, Q["w2"], P["b2"], dtype=dt)
        y, _ = api.gated_norm(z, x1, after_weight=Q["after2"], gate=m[5], before=None, eps=eps)
        check_norm(y.cpu(), None, z.cpu(), x1.cpu(), "rms", Q["after2"].cpu(), up(m[5])[None], 1.0, None, None, None, None, eps, "y")
    else:
        y = api.linear_fp4(sh, Q["w2"], P["b2"], gate=m[5], residual=x1, dtype=F32)
        check_linear(y.cpu(), _values(sh), W["w2"], P["b2"].cpu(), F32, gate=m[5].cpu(), res=x1.cpu(), what="y")
    ws = api.Workspace()
    for kw in ({}, dict(workspace=ws), dict(workspace=ws), dict(y_sel=torch.empty(L, D, device=device()), workspace=ws)):
        assert torch.equal(api.block_partial(Q, x, idx, n, H, rotary=rot, **kw), y), kw.keys()
    assert api.block_partial(Q, x, idx, 0, H, rotary=rot).shape == (0, D)
    if not after and not turned:
        ref = api.block_partial(P, x, idx, n, H).double() - x[idx.long()].double()
        off = float(((y.double() - x[idx.long()].double()) - ref).norm() / ref.norm())
        say(f"  the update differs from the {dtype} block's by {off:.3f}")
        assert off < 0.5


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_block_and_stack(bits, dtype):
    """With positions and norms, through the cache: fresh rows are the block's own."""
    w, dt, P, Q, xref, x = _make(dtype, bits, ("after1", "after2"))
    rot = api.Rotary.make(w.dh, device(), grid=w.grid)
    fw = torch.ones(w.T, device=device())
    blk = api.CachedBlock(Q, w.H, w.L, w.D, device(), dt, rotary=rot)
    blk.init(xref)
    y = blk.step(x, fw, w.N, k=w.K)
    sel = blk.sel.idx[: w.K]
    fresh = api.block_partial(Q, x, sel, w.K, w.H, rotary=rot)
    assert torch.equal(y[sel.long()], fresh.to(dt)) and torch.isfinite(y.float()).all()
    plain = api.block_partial({n: t for n, t in Q.items() if not n.startswith("after")}, x, sel, w.K, w.H)
    assert not torch.equal(plain, fresh)
    st = api.BlockStack([Q, Q], w.H, w.L, w.D, device(), dt, api.Scheduler.latent_only(1, 0.3), rotary=rot)
    st.step(xref, fw, w.N)
    out = st.step(x, fw, w.N)
    assert torch.isfinite(out.float()).all() and st.history[1][0] == api.topk_count(0.3, w.L)
    for kw in (dict(rotary=rot), dict()):
        R = P if kw else {**P, "after2": Q["after2"]}
        with pytest.raises(ValueError, match="8 or 4 bits"):
            api.block_partial(R, x, sel, w.K, w.H, **kw)
    with pytest.raises(ValueError, match="pairs"):
        api.block_partial(Q, x, sel, w.K, w.H, rotary=api.Rotary.make(2 * w.dh, device()))
    with pytest.raises(ValueError, match="after1"):
        api.block_partial({**Q, "after1": Q["after1"][:-1]}, x, sel, w.K, w.H)


def _block(seed, given=False):
    w, dt, P, Q, xref, x = _make("bf16", 4, ("after1", "after2"), seed=seed)
    rot = api.Rotary.make(w.dh, device(), grid=w.grid)
    idx = torch.arange(0, w.L, 2, dtype=torch.int32, device=device())
    ws = api.Workspace() if given else None
    return lambda: api.block_partial(Q, x, idx, len(idx), w.H, workspace=ws, rotary=rot)


def _linear(seed):
    """A product whose tiles are split along the depth."""
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    a = api.quantize_rows_fp4(torch.randn(200, 13824, device=device(), generator=g, dtype=BF))
    w = api.quantize_rows_fp4(torch.randn(512, 13824, device=device(), generator=g))
    seen, own = [], api._scratch
    api._scratch = lambda need, ws, like: seen.append(need) or own(need, ws, like)
    try:
        api.linear_fp4(a, w)
    finally:
        api._scratch = own
    assert seen[0] > 0
    return lambda: api.linear_fp4(a, w)


@pytest.mark.parametrize("make", [_linear, _block, lambda s: _block(s, True)], ids=["linear", "block", "block, workspaces"])
def test_two_streams_and_two_graphs_at_once(make):
    calls = [make(seed) for seed in (1, 2)]
    want = [call() for call in calls]
    torch.cuda.synchronize()
    want = [t.clone() for t in want]
    streams, got = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(8):
        for i, (call, stream) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(stream):
                got[i].append(call())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(t, want[i]) for t in got[i])
    graphs = []
    for call in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, call()))
    for turn in range(3):
        for _, y in graphs:
            y.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(6):
            for (graph, _), stream in zip(graphs, streams):
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, t) for (_, y), t in zip(graphs, want)), turn
