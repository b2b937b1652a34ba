"""GPU parity of the 4-bit product's largest tile, 256 x 256, which products of some
thousands of rows and channels take: the persistent form that goes from tile to tile and
stores from its accumulators, the form that goes through LDS (outputs off an alignment),
and tiles split along the depth with the kernel that joins them.  Each case asserts which
of them ran, so that another choice by estimated times does not take the cases away.

Inputs are such that every sum is exact in fp32, in any order: a product of codes is a
multiple of 1/4, scales are 2^-1 .. 2^1, so that sums are multiples of 2^-4, and below
2^20 in magnitude by the sum of magnitudes (asserted); bias, gate and residual are small
multiples of 1/8.  Outputs are compared bit for bit with the product in 64 bits."""
import math

import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24
GRID = (0, 0.5, 1, 1.5, 2, 3, 4, 6)


def _gen(seed):
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    return g


def _eighths(g, *shape, most=64, dtype=F32):
    """Multiples of 1/8 of at most most / 8 (64 and below: exact in bf16)."""
    return (torch.randint(-most, most + 1, shape, device=device(), generator=g) / 8.0).to(dtype)


def _rows(g, n, K):
    """Rows of random codes and scales of 2^-1 .. 2^1, and their values in 64 bits."""
    codes = torch.randint(0, 256, (n, (K + 255) // 256 * 128), device=device(), generator=g, dtype=torch.uint8)
    cols = torch.arange(codes.shape[1], device=device()) * 2
    codes &= ((cols < K) * 15 + (cols + 1 < K) * 240).to(torch.uint8)
    scales = torch.zeros(n, (K + 511) // 512 * 16, device=device(), dtype=torch.uint8)
    nb = (K + 31) // 32
    scales[:, :nb] = torch.randint(126, 129, (n, nb), device=device(), generator=g, dtype=torch.uint8)
    table = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device=device())
    v = table[torch.stack((codes & 15, codes >> 4), 2).flatten(1).int()][:, :K]
    return api.Fp4Rows(codes, scales, K), v * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :K]


def _product(g, M, N, K):
    (A, a), (W, w) = _rows(g, M, K), _rows(g, N, K)
    assert float((a.abs() @ w.abs().T).max()) * 16 < 2 ** 24
    return A, W, a @ w.T


def forms(run):
    """run(), and the names of the products' kernels that it launched."""
    api.profile_enable(True)
    try:
        api.profile_read()
        out = run()
        torch.cuda.synchronize()
        names = {n for n in api.profile_read() if n.startswith("gemm_fp4")}
    finally:
        api.profile_enable(False)
    return out, names


STREAM, STAGED, JOIN = "gemm_fp4_256_stream", "gemm_fp4_256", "gemm_fp4_reduce"


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K", [(2429, 3456, 1280),      # five k-steps, fewer tiles than the device has CUs
                                   (2561, 5136, 1100),      # the same with a ragged depth, one row in the last tiles
                                   (4100, 8704, 1280),      # some workgroups run three tiles of five k-steps, some two
                                   (5000, 9000, 2600)])     # the same, of eleven
def test_whole_tiles(M, N, K, out_dtype):
    say(f"whole tiles {M} x {N} x {K} {out_dtype}")
    g = _gen(M + N + K)
    A, W, z = _product(g, M, N, K)
    bias = _eighths(g, N, dtype=out_dtype)
    got, names = forms(lambda: api.linear_fp4(A, W, bias, dtype=out_dtype))
    assert names == {STREAM}, names
    assert torch.equal(got, (z + bias.double()).float().to(out_dtype))
    assert torch.equal(api.linear_fp4(A, W, dtype=out_dtype), z.float().to(out_dtype))


@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_gelu(out_dtype):
    """z is exact here, so that GELU (slope below 1.13; its argument, exponential and
    quotient) is at most 16 steps of 2^-24 of z off, and half a step of the output."""
    M, N, K = 1789, 7040, 1280
    say(f"GELU {out_dtype}")
    g = _gen(3)
    (A, a), (W, w) = _rows(g, M, K), _rows(g, N, K)
    A.scales[:, : K // 32] -= 4                                       # z of about 8 (2^-5 of it exact)
    W.scales[:, : K // 32] -= 3
    z = (a @ w.T) / 128
    got, names = forms(lambda: api.linear_fp4(A, W, activation="gelu", dtype=out_dtype))
    assert names == {STREAM}, names
    want = 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    err = 1.01 * 16 * U32 * z.abs() + torch.finfo(out_dtype).eps / 2 * want.abs() + 1e-38
    off = (got.double() - want).abs()
    say(f"  worst error {float((off / err).max()):.3f} of its bound")
    assert bool((off <= err).all())


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("res_dtype", [BF, F32])
@pytest.mark.parametrize("M,N,K,split", [(1789, 5376, 5120, False), (2173, 7296, 10240, True)])
def test_gate_and_residual(M, N, K, split, res_dtype, out_dtype):
    """Residuals by row and picked, the same one several times; rows that are not there
    are NaN, alone (in whole tiles and in the split ones at the end)."""
    say(f"gate and residual {M} x {N} x {K} {res_dtype} {out_dtype}")
    g = _gen(N)
    A, W, z = _product(g, M, N, K)
    gate, bias = _eighths(g, N, most=16), _eighths(g, N, most=16)
    n = M + 40
    res = _eighths(g, n, N, dtype=res_dtype)
    rows = torch.randint(0, n, (M,), device=device(), generator=g, dtype=torch.int32)
    # what is finite: |z + bias| < 2^20 in multiples of 2^-4, times at most 2 in multiples of 2^-3: may take more than
    # 24 bits, so once rounded; in 64 bits it is exact
    y = (z + bias.double()) * gate.double()
    for pick in (None, rows):
        if pick is not None:
            pick[5], pick[M // 2], pick[M - 1] = -1, n, 2 ** 31 - 1
        r = res[:M] if pick is None else res
        got, names = forms(lambda: api.linear_fp4(A, W, bias, gate=gate, residual=r, residual_rows=pick, dtype=out_dtype))
        assert names == ({STREAM, JOIN} if split else {STREAM}), names
        there = torch.ones(M, dtype=torch.bool, device=device()) if pick is None else (pick >= 0) & (pick < n)
        at = torch.arange(M, device=device()) if pick is None else pick.long().clamp(0, n - 1)
        want = (y + r[at].double()).float().to(out_dtype)
        assert torch.equal(got[there], want[there]) and int((~there).sum()) == (0 if pick is None else 3)
        assert bool(torch.isnan(got[~there]).all())


@pytest.mark.parametrize("M,N,K,split", [(1789, 5376, 5120, False), (2173, 7296, 10240, True)])
def test_onto_its_residual(M, N, K, split):
    g = _gen(K)
    A, W, _ = _product(g, M, N, K)
    for dtype in (F32, BF):
        gate, res = _eighths(g, N), _eighths(g, M, N, dtype=dtype)
        want = api.linear_fp4(A, W, gate=gate, residual=res, dtype=dtype)
        got, names = forms(lambda: api.linear_fp4(A, W, gate=gate, residual=res, out=res))
        assert names == ({STREAM, JOIN} if split else {STREAM}) and got is res and torch.equal(got, want)


@pytest.mark.parametrize("N", [5372, 5371])
def test_outputs_off_an_alignment(N):
    """Channels that are no multiple of a vector's, an output one element off, rows apart:
    the form that goes through LDS; what lies around the output stays."""
    M, K = 1789, 5100
    g = _gen(N)
    A, W, z = _product(g, M, N, K)
    bias, gate, res = _eighths(g, N, dtype=BF), _eighths(g, N), _eighths(g, M, N, dtype=BF)
    got, names = forms(lambda: api.linear_fp4(A, W, bias))
    assert names == {STAGED}, names
    assert torch.equal(got, (z + bias.double()).float().bfloat16())
    buf = torch.full((M + 2, N + 9), 3.0, device=device())
    got, names = forms(lambda: api.linear_fp4(A, W, bias, gate=gate, residual=res, out=buf[1:-1, 3:N + 3]))
    assert names == {STAGED}, names
    assert torch.equal(got, ((z + bias.double()) * gate.double() + res.double()).float())
    got.fill_(3.0)
    assert bool((buf == 3).all())


@pytest.mark.parametrize("M,N,K", [(2429, 3456, 1280), (5000, 9000, 2600), (2600, 4995, 1280)])
def test_nan_blocks(M, N, K):
    """Of an odd number of k-steps: a NaN block, of the last one too, makes its own row
    (its own channel) NaN and no other; every other output is what it was."""
    g = _gen(K)
    A, W, z = _product(g, M, N, K)
    row, col = [0, 300, M - 1], [7, 256, N - 1]
    for i, b in zip(row, (0, K // 32 - 1, K // 64)):
        A.scales[i, b] = 255
    for j, b in zip(col, (K // 32 - 1, 0, 1)):
        W.scales[j, b] = 255
    got, names = forms(lambda: api.linear_fp4(A, W, dtype=F32))
    assert names == {STAGED if N % 4 else STREAM}, names
    want = z.float()
    want[row], want[:, col] = float("nan"), float("nan")
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def test_repeats_itself():
    """With other work in between, on another stream, replayed: the same bits."""
    g = _gen(11)
    x = torch.randn(3000, 2600, device=device(), generator=g).bfloat16()
    w = api.quantize_rows_fp4(torch.randn(9000, 2600, device=device(), generator=g))
    m = torch.randn(2, 2600, device=device(), generator=g) * 0.1

    def run():
        return api.linear_fp4(api.quantize_rows_fp4(x, shift=m[0], scale=m[1]), w)
    want, names = forms(run)
    assert names == {STREAM}, names
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = run()
    side = torch.cuda.Stream()
    for turn in range(5):
        y.fill_(7.0)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = run()
        again = run()
        torch.cuda.synchronize()
        for t in (y, other, again):
            assert torch.equal(t, want), turn
