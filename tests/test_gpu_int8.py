"""GPU parity of the rows in 8 bits, the linear layer on them and the block in
8 bits, against plain 64-bit computations on the CPU.

Codes and scales are exact by definition, and so are the integer sums; what is
left are fp32 roundings (half a step each, 2^-24 of the value) and the rounding
of the output (half a step of its type: bf16 2^-8, fp32 2^-24)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import synth
from paper_2608_02474_amd import _lib, api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g).to(dtype)


def codes_of(a):
    """Codes and unit of each row of float64 values: the quotient 127 a / amax,
    rounded with its halves told in exact arithmetic (254 a against odd
    multiples of amax: products of at most 24 + 8 bits)."""
    top = a.abs().amax(1, keepdim=True)
    safe = torch.where(top > 0, top, torch.ones_like(top))
    low = torch.floor(a * 127 / safe)
    for _ in range(2):      # the floor itself may be one off after its division
        low = torch.where(127 * a < low * safe, low - 1, torch.where(127 * a >= (low + 1) * safe, low + 1, low))
    side = 254 * a - (2 * low + 1) * safe
    even = 2 * torch.floor((low + 1) / 2)
    n = torch.where(side > 0, low + 1, torch.where(side < 0, low, even))
    return torch.where(top > 0, n, torch.zeros_like(n)), top


# ------------------------------------------------------------ quantize_rows

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,D,ld", [(1, 1, 1), (3, 7, 7), (5, 8, 8), (4, 127, 127), (2, 128, 130), (7, 129, 200),
                                    (33, 250, 250), (6, 512, 520), (3, 513, 513), (9, 2048, 2048), (2, 2056, 2063),
                                    (5, 5120, 10240), (3, 6144, 6144), (2, 13824, 13824), (2, 16385, 16385),
                                    (1, 65535, 65535), (2, 65536, 65536)])
def test_quantize_rows_exact(M, D, ld, dtype):
    say(f"quantize {M} x {D} (ld {ld}) {dtype}")
    g = _gen(M * 100003 + D)
    wide = _rand(g, M, ld, dtype=dtype)
    wide[:, : D // 2] *= 0.01                                   # small codes among large
    x = wide[:, :D]
    if D > 4:
        x[:, 3] = x.float().abs().amax(1).to(dtype) / 2         # 63.5: a half, to the even code
    want, top = codes_of(x.double())
    buf = torch.full((M + 2, ld), float("nan"), dtype=dtype)     # rows apart, NaN around them
    buf[:M, :D] = x
    r = api.quantize_rows(buf.to(device())[:M, :D])
    torch.cuda.synchronize()
    codes = r.codes.cpu()
    assert codes.shape == (M, (D + 127) // 128 * 128) and r.cols == D
    assert torch.equal(codes[:, :D].double(), want)
    assert (codes[:, D:] == 0).all()
    assert torch.equal(r.scale.cpu(), (top[:, 0].float() / 127.0))
    back = api.dequantize_rows(r, dtype)
    value = (codes[:, :D].float() * r.scale.cpu()[:, None]).to(dtype)
    assert torch.equal(back.cpu(), value)


def test_quantize_rows_unaligned_and_into_given_rows():
    """An element offset (no vector loads), outputs of a wider pitch, rows behind the last left as they were."""
    g = _gen(3)
    x = _rand(g, 6, 200, dtype=torch.bfloat16)
    want, _ = codes_of(x[:, 3:].double())
    out = api.Int8Rows(torch.full((8, 384), 99, dtype=torch.int8, device=device()),
                       torch.full((8,), 5.0, device=device()), 197)
    view = api.Int8Rows(out.codes[1:7], out.scale[1:7], 197)
    r = api.quantize_rows(x.to(device())[:, 3:], out=view)
    torch.cuda.synchronize()
    c = out.codes.cpu()
    assert r is view
    assert torch.equal(c[1:7, :197].double(), want) and (c[1:7, 197:] == 0).all()
    assert (c[0] == 99).all() and (c[7] == 99).all()
    assert float(out.scale[0]) == 5.0 and float(out.scale[7]) == 5.0
    y = torch.full((8, 220), 7.0, dtype=torch.bfloat16, device=device())
    api.dequantize_rows(r, out=y[1:7, 5:202])
    y = y.cpu()
    assert torch.equal(y[1:7, 5:202], (c[1:7, :197].float() * r.scale.cpu()[:, None]).bfloat16())
    assert (y[0] == 7).all() and (y[7] == 7).all() and (y[:, :5] == 7).all() and (y[:, 202:] == 7).all()


def test_quantize_rows_edge_values():
    """Zeros, the smallest and the largest numbers, infinities and NaN: a row that is
    not finite is NaN as a whole, and alone."""
    t = 1e-45                                                    # the smallest fp32
    rows = [[0.0] * 9, [-0.0] * 9, [t, -t, 0, 3 * t, t, 0, 0, 0, 2 * t],
            [1e-38, 5e-39, -1e-38, 2.4e-40, 0, 0, 0, 0, 1e-38], [3.4028235e38, -1e38, 1.0, 0, 0, 0, 0, 0, 1e30],
            [1.0, float("inf"), 0, 0, 0, 0, 0, 0, 0], [1.0, 0, 0, 0, 0, 0, 0, float("nan"), 2.0],
            [-float("inf"), float("nan"), 0, 0, 0, 0, 0, 0, 0], [1.0, 0.5, 0.25, -0.5, 127.0, 63.5, 0.0, 1.5, 2.5]]
    x = torch.tensor(rows, dtype=torch.float32)
    r = api.quantize_rows(x.to(device()))
    torch.cuda.synchronize()
    codes, scale = r.codes.cpu()[:, :9].double(), r.scale.cpu()
    fine = torch.isfinite(x).all(1)
    want, top = codes_of(x[fine].double())
    assert torch.equal(codes[fine], want)
    assert torch.equal(scale[fine], top[:, 0].float() / 127.0)
    assert torch.isnan(scale[~fine]).all() and (codes[~fine] == 0).all()
    assert torch.isnan(api.dequantize_rows(r, torch.float32).cpu()[~fine]).all()


@pytest.mark.parametrize("D", [64, 130, 5120])
def test_quantize_rows_picks_rows(D):
    g = _gen(D)
    x = _rand(g, 50, D, dtype=torch.bfloat16)
    rows = torch.tensor([49, 0, 7, 7, 3, -1, 50, 2 ** 31 - 1, 12], dtype=torch.int32)
    r = api.quantize_rows(x.to(device()), rows=rows.to(device()))
    torch.cuda.synchronize()
    ok = (rows >= 0) & (rows < 50)
    want, top = codes_of(x[rows[ok].long()].double())
    assert torch.equal(r.codes.cpu()[ok][:, :D].double(), want)
    assert torch.equal(r.scale.cpu()[ok], top[:, 0].float() / 127.0)
    assert torch.isnan(r.scale.cpu()[~ok]).all() and (r.codes.cpu()[~ok] == 0).all()   # no such row


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,D", [(1, 8), (5, 64), (4, 250), (3, 1536), (7, 5120), (2, 13824), (2, 20001)])
def test_quantize_rows_layernorm(M, D, dtype):
    """LayerNorm in fp32 in front: sums of at most 80 terms a lane and 10 joining
    steps, so the mean, the variance and with them a value are within 256 steps of
    2^-24 of the row's largest value; a code may then lie beside the 64-bit one
    where the quotient is that near to a half."""
    g = _gen(D + 1)
    x = (_rand(g, M, D) * 2 + 0.5).to(dtype)
    sh, sc = _rand(g, D) * 0.1, _rand(g, D) * 0.1
    r = api.quantize_rows(x.to(device()), shift=sh.to(device()), scale=sc.to(device()), ln_eps=1e-6)
    torch.cuda.synchronize()
    xd = x.double()
    z = (xd - xd.mean(1, keepdim=True)) / (xd.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    z = z * (1 + sc.double()) + sh.double()
    top = z.abs().amax(1, keepdim=True)
    tol = 256 * U32
    assert ((r.scale.cpu().double()[:, None] * 127 - top).abs() <= (tol + U32) * top).all()
    q = z * 127 / top
    assert ((r.codes.cpu()[:, :D].double() - q).abs() <= 0.5 + 2 * 127 * tol).all()
    assert (r.codes.cpu()[:, D:] == 0).all()
    # picked rows are the rows themselves, bit for bit
    pick = torch.arange(M - 1, -1, -1, dtype=torch.int32)
    r2 = api.quantize_rows(x.to(device()), rows=pick.to(device()), shift=sh.to(device()), scale=sc.to(device()))
    assert torch.equal(r2.codes.cpu().flip(0), r.codes.cpu()) and torch.equal(r2.scale.cpu().flip(0), r.scale.cpu())


def test_quantize_rows_empty():
    r = api.quantize_rows(torch.zeros(0, 64, device=device()))
    assert r.codes.shape == (0, 128) and r.scale.shape == (0,)
    assert api.dequantize_rows(r).shape == (0, 64)
    w = api.quantize_rows(torch.ones(8, 64, device=device()))
    assert api.linear_int8(r, w).shape == (0, 8)


# -------------------------------------------------------------- linear_int8

def _gelu(z):
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def _random_rows(g, n, K, std=1.0):
    """Rows of codes over the whole range with scales of their own."""
    pitch = (K + 127) // 128 * 128
    codes = torch.zeros(n, pitch, dtype=torch.int8)
    codes[:, :K] = torch.randint(-127, 128, (n, K), generator=g, dtype=torch.int8)
    scale = (torch.rand(n, generator=g) + 0.5) * std / 73
    return codes, scale


def _on(codes, scale, K):
    return api.Int8Rows(codes.to(device()), scale.to(device()), K)


def _check_linear(got, a, w, K, bias, out_dtype, act=None, gate=None, res=None, what=""):
    """z = sum sa sw + b: the sum's rounding, two products and one addition (fused),
    4 steps of 2^-24 of |sum sa sw| + |b| at most; GELU (slope below 1.13, its own
    exponent's argument, exponential and quotient) at most 16 in all; gate and
    residual one more step of the result each."""
    acc = (a[0][:, :K].double() @ w[0][:, :K].double().T)
    z0 = acc * a[1].double()[:, None] * w[1].double()
    b = torch.zeros(w[0].shape[0], dtype=torch.float64) if bias is None else bias.double()
    z = z0 + b
    err = 16 * U32 * (z0.abs() + b.abs())
    if act == "gelu":
        want = _gelu(z)
    elif gate is not None:
        want = res.double() + gate.double() * z
        err = err * gate.double().abs() + 2 * U32 * (res.double().abs() + want.abs())
    else:
        want = z
    err = err * 1.01 + HALF_STEP[out_dtype] * want.abs() + 1e-40
    off = (got.double() - want).abs()
    worst = float((off / err).max()) if off.numel() else 0.0
    say(f"  {what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0


SIZES = [(1, 1, 1), (1, 16, 64), (1, 300, 5120), (2, 77, 129), (5, 1000, 700), (16, 64, 128), (17, 129, 640),
         (32, 48, 256), (33, 100, 100), (64, 512, 1024), (65, 65, 65), (100, 200, 300), (128, 128, 128),
         (130, 70, 13824), (257, 255, 200), (300, 512, 256), (500, 1030, 384), (1000, 96, 4000), (1111, 2049, 130),
         (2100, 2304, 256), (4100, 4100, 128)]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_int8_sizes(M, N, K, out_dtype):
    g = _gen(M * 7 + N * 3 + K)
    say(f"linear {M} x {N} x {K} -> {out_dtype}")
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    bias = (_rand(g, N) * 0.1).to(out_dtype)
    got = api.linear_int8(_on(*a, K), _on(*w, K), bias.to(device()), dtype=out_dtype)
    torch.cuda.synchronize()
    _check_linear(got.cpu(), a, w, K, bias, out_dtype, what=f"{M}x{N}x{K}")


@pytest.mark.parametrize("M,N,K", [(1, 200, 300), (20, 77, 130), (60, 64, 512), (140, 260, 260), (700, 1000, 200),
                                   (4096, 4100, 128), (90, 256, 8000)])
@pytest.mark.parametrize("epi", ["none", "gelu", "gate_bf16", "gate_f32_rows"])
def test_linear_int8_epilogues(M, N, K, epi):
    g = _gen(M + N + K)
    say(f"linear {M} x {N} x {K} {epi}")
    a, w = _random_rows(g, M, K, 3.0), _random_rows(g, N, K, 0.05)
    A, W = _on(*a, K), _on(*w, K)
    if epi == "none":
        got = api.linear_int8(A, W)
        _check_linear(got.cpu(), a, w, K, None, torch.bfloat16, what=epi)
    elif epi == "gelu":
        bias = _rand(g, N)
        got = api.linear_int8(A, W, bias.to(device()), activation="gelu", dtype=torch.float32)
        _check_linear(got.cpu(), a, w, K, bias, torch.float32, act="gelu", what=epi)
    else:
        rdt = torch.bfloat16 if epi == "gate_bf16" else torch.float32
        gate, bias = _rand(g, N), _rand(g, N, dtype=rdt)
        n = M if epi == "gate_bf16" else M + 9
        res = _rand(g, n, N + 3, dtype=rdt)[:, :N] if N % 2 else _rand(g, n, N, dtype=rdt)
        rows = None if epi == "gate_bf16" else torch.randint(0, n, (M,), generator=g, dtype=torch.int32)
        got = api.linear_int8(A, W, bias.to(device()), gate=gate.to(device()), residual=res.to(device()),
                              residual_rows=None if rows is None else rows.to(device()), dtype=torch.float32)
        _check_linear(got.cpu(), a, w, K, bias, torch.float32, gate=gate,
                      res=res if rows is None else res[rows.long()], what=epi)


def test_linear_int8_largest_sums():
    """Every product 127 * 127 over the longest depth: the sum stays in 32 bits."""
    K = 65536
    for M in (3, 70):
        a = torch.full((M, K), 127, dtype=torch.int8)
        w = torch.full((65, K), -127, dtype=torch.int8)
        one = torch.ones(M), torch.ones(65)
        got = api.linear_int8(_on(a, one[0], K), _on(w, one[1], K), dtype=torch.float32)
        assert (got.cpu().double() == float(np.float32(-127 * 127 * K))).all()


@pytest.mark.parametrize("M,N,K", [(3, 40, 128), (12, 100, 256), (100, 200, 4096), (600, 516, 256), (300, 203, 128)])
def test_linear_int8_onto_its_residual(M, N, K):
    g = _gen(M)
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    gate, res = _rand(g, N).to(device()), _rand(g, M, N).to(device())
    want = api.linear_int8(_on(*a, K), _on(*w, K), gate=gate, residual=res, dtype=torch.float32)
    got = api.linear_int8(_on(*a, K), _on(*w, K), gate=gate, residual=res, out=res)
    assert got is res and torch.equal(got, want)


def test_linear_int8_rows_are_independent_and_behind_is_left():
    """A row's result does not depend on how many rows come with it, NaN rows stay
    alone, missing residual rows are NaN, and the output's surroundings stay."""
    g = _gen(77)
    M, N, K = 300, 200, 260
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    a[1][5] = float("nan")
    a[0][5] = 0
    A, W = _on(*a, K), _on(*w, K)
    buf = torch.full((M + 2, N + 5), 3.0, device=device())
    whole = api.linear_int8(A, W, dtype=torch.float32, out=buf[1:M + 1, 2:N + 2])
    b = buf.cpu()
    assert (b[0] == 3).all() and (b[-1] == 3).all() and (b[:, :2] == 3).all() and (b[:, N + 2:] == 3).all()
    nan = torch.isnan(whole.cpu())
    assert nan[5].all() and not nan[torch.arange(M) != 5].any()
    for lo, hi in ((6, 7), (6, 30), (10, 110), (0, 5)):
        part = api.linear_int8(api.Int8Rows(A.codes[lo:hi], A.scale[lo:hi], K), W, dtype=torch.float32)
        assert torch.equal(part.cpu(), whole.cpu()[lo:hi])
    gate, res = torch.ones(N, device=device()), torch.zeros(4, N, device=device())
    rows = torch.zeros(M, dtype=torch.int32, device=device())
    rows[7], rows[8] = 4, -1
    y = api.linear_int8(A, W, gate=gate, residual=res, residual_rows=rows, dtype=torch.float32).cpu()
    bad = torch.isnan(y).all(1)
    assert bad[[5, 7, 8]].all() and int(bad.sum()) == 3


def test_linear_int8_streams_and_graphs():
    """Two captured graphs and eager calls in between, on a side stream: each replay
    equals the eager result (split products have a workspace of their own)."""
    g = _gen(5)
    shapes = [(130, 200, 8192), (1, 4000, 1024), (600, 700, 512)]
    made = []
    for M, N, K in shapes:
        x = _rand(g, M, K, dtype=torch.bfloat16).to(device())
        w = api.quantize_rows((_rand(g, N, K) * 0.05).to(device()))
        made.append((x, w, api.linear_int8(api.quantize_rows(x), w)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = [api.linear_int8(api.quantize_rows(x), w) for x, w, _ in made]
    side.synchronize()
    for e, (_, _, ref) in zip(eager, made):
        assert torch.equal(e, ref)
    graphs = []
    for x, w, ref in made:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            y = api.linear_int8(api.quantize_rows(x), w)
        graphs.append((gr, y))
    for turn in range(3):
        for (gr, y), (x, w, _) in zip(graphs, made):
            x.mul_(-0.5)
            gr.replay()
            ref = api.linear_int8(api.quantize_rows(x), w)
            torch.cuda.synchronize()
            assert torch.equal(y, ref), turn


# ------------------------------------------------------------ the whole block

def _block_oracle(P, Q, x, idx, H):
    """The block in 64 bits on the same 8-bit weights, its tokens quantised in front
    of every product and its intermediates rounded where the library holds them in
    bf16."""
    def q8(a):
        top = a.abs().amax(1, keepdim=True)
        top = torch.where(top > 0, top, torch.ones_like(top))
        return torch.round(a * 127 / top) * (top / 127)

    def lin(a, n, b):
        W = Q[n].codes.cpu()[:, : Q[n].cols].double() * Q[n].scale.cpu().double()[:, None]
        return q8(a) @ W.T + P[b].cpu().double()

    def ln(z):
        return (z - z.mean(1, keepdim=True)) / (z.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    bf = (lambda t: t.bfloat16().double()) if x.dtype == torch.bfloat16 else (lambda t: t.float().double())
    m = P["mod"].cpu().double()
    xd = x.cpu().double()
    a = ln(xd) * (1 + m[1]) + m[0]
    D = xd.shape[1]
    dh = D // H
    q, k, v = bf(lin(a[idx], "wq", "bq")), bf(lin(a, "wk", "bk")), bf(lin(a, "wv", "bv"))
    o = torch.empty(len(idx), D, dtype=torch.float64)
    for h in range(H):
        s = slice(h * dh, (h + 1) * dh)
        o[:, s] = torch.softmax(q[:, s] @ k[:, s].T / math.sqrt(dh), 1) @ v[:, s]
    x1 = xd[idx] + m[2] * lin(bf(o), "wo", "bo")
    hid = bf(_gelu(lin(ln(x1) * (1 + m[4]) + m[3], "w1", "b1")))
    return x1 + m[5] * lin(hid, "w2", "b2")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_in_8_bits(dtype):
    """The operators run together as the block does: against the 64-bit block on the
    same 8-bit weights, by the block's own tolerance in bf16 (2e-2, 1e-2 of the
    norm).  An fp32 block is held to it too: a token value next to a half takes the
    code beside, and one code is 1/127 of the row's largest value."""
    w = synth.Workload("int8_300tok", T=3, grid=(10, 10), D=256, H=2, F=512, n_samples=4000, ratio=0.37,
                       dtype=dtype, audio="speech", seed=31)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    P = {k: torch.from_numpy(v).to(torch.float32 if k == "mod" else dt).to(device())
         for k, v in synth.make_block_weights(w).items()}
    xref, x = (torch.from_numpy(t).to(dt).to(device()) for t in synth.make_latents(w))
    Q = api.quantize_block(P)
    assert api.is_int8_block(Q) and not api.is_int8_block(P)
    idx = torch.arange(0, w.L, 3, dtype=torch.int32, device=device())
    y = api.block_partial(Q, x, idx, 90, w.H)
    torch.cuda.synchronize()
    want = _block_oracle(P, Q, x, idx[:90].cpu().long(), w.H)
    off = y.cpu().double() - want
    say(f"  8-bit block {dtype}: max {float(off.abs().max()):.2e}, rel {float(off.norm() / want.norm()):.2e}")
    assert float(off.abs().max()) <= 2e-2 and float(off.norm() / want.norm()) <= 1e-2
    assert api.block_partial(Q, x, idx, 0, w.H).shape == (0, w.D)

    # through the cached block: the first step and a cached one
    fw = torch.ones(w.T, device=device())
    blk = api.CachedBlock(Q, w.H, w.L, w.D, device(), dt)
    blk.init(xref)
    y8 = blk.step(x, fw, w.N, k=w.K)
    sel = blk.sel.idx[: w.K]
    fresh = api.block_partial(Q, x, sel, w.K, w.H)
    torch.cuda.synchronize()
    assert torch.equal(y8[sel.long()], fresh.to(dt))            # fresh rows are the block's own
    assert torch.isfinite(y8.float()).all()
    st = api.BlockStack([Q, Q], w.H, w.L, w.D, device(), dt, api.Scheduler.latent_only(1, 0.3))
    st.step(xref, fw, w.N)
    out = st.step(x, fw, w.N)
    assert torch.isfinite(out.float()).all() and st.history[1][0] == api.topk_count(0.3, w.L)


# ------------------------------------------------- offsets of more than 32 bits

def test_rows_beyond_32_bit_offsets():
    """More than 2^31 codes, and with them the values read back (both loop over their
    launches), and products over them: the first and the last rows against the CPU."""
    M, D = 32800, 65536
    g = torch.Generator(device=device())
    g.manual_seed(1)
    x = torch.empty(M, D, dtype=torch.bfloat16, device=device())
    for i in range(0, M, 4100):
        x[i:i + 4100] = torch.randn(4100, D, device=device(), generator=g)
    r = api.quantize_rows(x)
    back = api.dequantize_rows(r)
    at = [0, 1, 16383, 32767, 32768, M - 1]
    want, top = codes_of(x[at].cpu().double())
    assert torch.equal(r.codes[at].cpu().double(), want)
    assert torch.equal(back[at].cpu(), (want.float() * (top.float() / 127)).bfloat16())
    del back
    w = _random_rows(_gen(2), 8, D, 0.05)
    y = api.linear_int8(r, _on(*w, D), dtype=torch.float32)         # tokens far apart
    _check_linear(y[at].cpu(), (r.codes[at].cpu(), r.scale[at].cpu()), w, D, None, torch.float32, what="tokens")
    a = _random_rows(_gen(3), 100, D)
    for m in (3, 12, 100):                                          # channels far apart
        y = api.linear_int8(api.Int8Rows(a[0][:m].to(device()), a[1][:m].to(device()), D), r, dtype=torch.float32)
        _check_linear(y[:, at].cpu(), (a[0][:m], a[1][:m]), (r.codes[at].cpu(), r.scale[at].cpu()), D, None,
                      torch.float32, what=f"channels, {m} tokens")


def test_linear_int8_output_beyond_32_bit_offsets():
    M, N, K = 70000, 32768, 128
    g = _gen(4)
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    y = api.linear_int8(_on(*a, K), _on(*w, K))
    at = [0, 255, 65535, 65536, M - 1]
    _check_linear(y[at].cpu(), (a[0][at], a[1][at]), w, K, None, torch.bfloat16, what="last rows")


def test_quantize_rows_more_than_a_launch_of_rows():
    M, D = 4 * 2 ** 20 + 37, 136                                    # 4 rows to each of at most 2^20 workgroups
    x = torch.randn(M, D, device=device()).bfloat16()
    r = api.quantize_rows(x)
    at = [0, 4 * 2 ** 20 - 1, 4 * 2 ** 20, M - 1]
    want, top = codes_of(x[at].cpu().double())
    assert torch.equal(r.codes[at].cpu()[:, :D].double(), want)
    assert torch.equal(r.scale[at].cpu(), top[:, 0].float() / 127)


# ------------------------------------------------------- plans and random shapes

@pytest.mark.parametrize("M,N,K,act", [(8813, 2304, 8320, None), (3276, 5120, 5120, "gelu"), (1950, 1536, 8960, "gate"),
                                       (771, 11072, 5504, None), (100, 5120, 5120, "gate"), (20, 5120, 13824, "gelu"),
                                       (4100, 4106, 4096, None), (700, 130, 9000, "gate")])
def test_linear_int8_split_products(M, N, K, act):
    """Deep products, whose tiles are split along the depth (all of them, those of the
    last round, or none): the join runs just where the plan asks for a workspace, and
    sampled rows and the last ones match."""
    g = _gen(M + K)
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    A, W, bias = _on(*a, K), _on(*w, K), _rand(g, N)
    kw, gate, res = {}, None, None
    if act == "gate":
        gate, res = _rand(g, N), _rand(g, M, N, dtype=torch.bfloat16)
        kw = dict(gate=gate.to(device()), residual=res.to(device()))
    elif act:
        kw = dict(activation=act)
    api.profile_enable(True)
    try:
        api.profile_read()
        y = api.linear_int8(A, W, bias.to(device()), dtype=torch.float32, **kw)
        names = set(api.profile_read())
    finally:
        api.profile_enable(False)
    cfg = _lib.LinearInt8Cfg(M=M, N=N, K=K, out_dtype=_lib.ECHO_F32, bias_dtype=_lib.ECHO_F32,
                             residual_dtype=_lib.ECHO_F32, lda=A.codes.stride(0), ldw=W.codes.stride(0), ldc=N)
    assert ("gemm_int8_reduce" in names) == (_lib.load().echo_linear_int8_workspace(ctypes.byref(cfg)) > 0), names
    at = torch.unique(torch.cat([torch.randint(0, M, (24,), generator=g), torch.tensor([0, M // 2, M - 1])]))
    _check_linear(y[at.to(device())].cpu(), (a[0][at], a[1][at]), w, K, bias, torch.float32, act=act if act == "gelu" else None,
                  gate=gate, res=None if res is None else res[at], what=f"{M}x{N}x{K}")


@pytest.mark.parametrize("seed", range(24))
def test_linear_int8_random_shapes(seed):
    """Any tokens, channels and depth, any epilogue and type, rows of the operands and
    of the output inside wider buffers."""
    rng = np.random.default_rng(seed)
    g = _gen(1000 + seed)
    M, N, K = (int(np.exp(rng.uniform(np.log(lo), np.log(hi)))) for lo, hi in ((1, 3000), (1, 3000), (1, 3000)))
    out_dtype = [torch.bfloat16, torch.float32][int(rng.integers(2))]
    a, w = _random_rows(g, M, K), _random_rows(g, N, K, 0.05)
    wide = torch.full((M, a[0].shape[1] + 256), 77, dtype=torch.int8)
    wide[:, 128:-128] = a[0]
    A = api.Int8Rows(wide.to(device())[:, 128:-128], a[1].to(device()), K)
    buf = torch.full((M, N + int(rng.integers(0, 9))), 5.0, dtype=out_dtype, device=device())
    bias = _rand(g, N, dtype=out_dtype) if rng.integers(2) else None
    kw, act, gate, res = {}, None, None, None
    kind = int(rng.integers(3))
    if kind == 1:
        act = "gelu"
        kw["activation"] = act
    elif kind == 2:
        gate, rows = _rand(g, N), torch.randint(0, M + 3, (M,), generator=g, dtype=torch.int32)
        full = _rand(g, M + 3, N + 5, dtype=[torch.bfloat16, torch.float32][int(rng.integers(2))])[:, :N]
        res = full[rows.long()]
        kw.update(gate=gate.to(device()), residual=full.to(device()), residual_rows=rows.to(device()))
    y = api.linear_int8(A, _on(*w, K), None if bias is None else bias.to(device()), out=buf[:, :N], **kw)
    torch.cuda.synchronize()
    assert (buf[:, N:] == 5).all()
    _check_linear(y.cpu(), a, w, K, bias, out_dtype, act=act, gate=gate, res=res, what=f"{M}x{N}x{K} kind {kind}")


# ------------------------------------------------ the block, its workspace and graphs

def _block_of(L, D, H, F, dt, seed):
    """Weights in dt and in 8 bits, tokens."""
    g = _gen(seed)
    P = {n: _rand(g, *s) * s[1] ** -0.5 for n, s in (("wq", (D, D)), ("wk", (D, D)), ("wv", (D, D)), ("wo", (D, D)),
                                                    ("w1", (F, D)), ("w2", (D, F)))}
    P.update({n: _rand(g, F if n == "b1" else D) * 0.02 for n in ("bq", "bk", "bv", "bo", "b1", "b2")})
    P = {n: t.to(dt).to(device()) for n, t in P.items()}
    mod = _rand(g, 6, D) * 0.1
    mod[2] += 0.25
    mod[5] += 0.25
    P["mod"] = mod.to(device())
    return P, api.quantize_block(P), _rand(g, L, D, dtype=dt).to(device())


@pytest.mark.parametrize("L,D,H,F,dt", [(300, 256, 2, 512, torch.bfloat16), (2101, 512, 4, 1300, torch.bfloat16),
                                        (333, 200, 5, 300, torch.float32)])
def test_block_in_8_bits_lives_in_its_workspace(L, D, H, F, dt):
    """With a workspace that has grown once the block allocates nothing, whatever ran in
    it in between, and its rows are those of a call without one."""
    _, Q, x = _block_of(L, D, H, F, dt, 3)
    idx = torch.randperm(L, generator=_gen(4)).to(torch.int32).to(device())
    ws = api.Workspace()
    counts = (L, 1, L // 3, 20)
    want = {n: api.block_partial(Q, x, idx, n, H) for n in counts}
    y = torch.empty(L, D, device=device())
    api.block_partial(Q, x, idx, L, H, y_sel=y, workspace=ws)
    assert ws.buf is not None
    for n in counts:
        api.block_partial(Q, x, idx, n, H, y_sel=y, workspace=ws)
    held = ws.buf.data_ptr()
    for n in counts + counts[::-1]:
        ws.buf.fill_(0x7f)
        y.fill_(5.0)
        torch.cuda.synchronize()
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        got = api.block_partial(Q, x, idx, n, H, y_sel=y, workspace=ws)
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before, n
        assert ws.buf.data_ptr() == held
        assert torch.equal(got, want[n]) and (y[n:] == 5).all(), n
    # another block's larger needs: the pieces follow the buffer
    ws.get(ws.buf.numel() + 1, device())
    assert torch.equal(api.block_partial(Q, x, idx, 20, H, workspace=ws), want[20])


def test_block_in_8_bits_and_in_16_share_a_workspace():
    L, D, H, F = 500, 256, 2, 512
    P, Q, x = _block_of(L, D, H, F, torch.bfloat16, 8)
    idx = torch.arange(0, L, 3, dtype=torch.int32, device=device())
    n, ws = len(idx), api.Workspace()
    want16, want8 = api.block_partial(P, x, idx, n, H), api.block_partial(Q, x, idx, n, H)
    for turn in range(3):
        assert torch.equal(api.block_partial(Q, x, idx, n, H, workspace=ws), want8), turn
        assert torch.equal(api.block_partial(P, x, idx, n, H, workspace=ws), want16), turn


@pytest.mark.parametrize("given", [False, True])
def test_block_in_8_bits_captured(given):
    """The whole block in a graph, replayed on changing tokens between eager calls of
    the same weights, with a workspace of its own or the call's."""
    L, D, H, F = 1200, 512, 4, 1024
    _, Q, x = _block_of(L, D, H, F, torch.bfloat16, 6)
    idx = torch.arange(0, L, 2, dtype=torch.int32, device=device())
    ws = api.Workspace() if given else None
    api.block_partial(Q, x, idx, len(idx), H, workspace=ws)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        y = api.block_partial(Q, x, idx, len(idx), H, workspace=ws)
    for turn in range(4):
        x.mul_(-0.7)
        idx.copy_((idx + 1) % L)
        gr.replay()
        want = api.block_partial(Q, x, idx, len(idx), H)
        torch.cuda.synchronize()
        assert torch.isfinite(y).all() and torch.equal(y, want), turn


@pytest.mark.parametrize("L,n,D,H,F,dt", [(2500, 901, 512, 4, 1300, torch.bfloat16), (1111, 1111, 640, 5, 2100, torch.bfloat16),
                                          (1500, 333, 264, 3, 1000, torch.float32)])
def test_block_in_8_bits_of_many_tokens(L, n, D, H, F, dt):
    """Tiles, splits and ragged ends together, some tokens more than once: against the
    64-bit block on the same weights, by the tolerance above."""
    P, Q, x = _block_of(L, D, H, F, dt, L)
    idx = torch.randint(0, L, (n,), generator=_gen(n), dtype=torch.int32)
    idx[1] = idx[0]
    y = api.block_partial(Q, x, idx.to(device()), n, H)
    torch.cuda.synchronize()
    want = _block_oracle(P, Q, x, idx.long(), H)
    off = y.cpu().double() - want
    say(f"  8-bit block {L} tokens, {n} of them, {dt}: max {float(off.abs().max()):.2e}, rel {float(off.norm() / want.norm()):.2e}")
    assert float(off.abs().max()) <= 2e-2 and float(off.norm() / want.norm()) <= 1e-2
    assert torch.equal(y[0], y[1])
