"""GPU parity of the rows in microscaled 4-bit floating point and the linear layer on
them, against plain 64-bit computations on the CPU.

Codes and scales are exact by definition.  A product of two codes is a multiple of
1/4 and at most 36, so the sum of a block of 32 is exact in fp32 too; what is left are
the additions of blocks in fp32 and the rounding of the output (half a step of its
type: bf16 2^-8, fp32 2^-24)."""
import math

import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _rand(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g).to(dtype)


def _blocks(a):
    return torch.nn.functional.pad(a, (0, -a.shape[1] % 32)).view(len(a), -1, 32)


def fp4_of(a):
    """Codes [M, blocks, 32] (0 .. 15) and scale bytes [M, blocks] of float64 values,
    by the exponents of the numbers themselves."""
    b = _blocks(a)
    top = b.abs().amax(2)
    fine = torch.isfinite(b).all(2)
    _, e = torch.frexp(torch.where(fine, top, torch.zeros_like(top)))     # top = f 2^e, f in [1/2, 1)
    e = torch.where(top > 0, (e - 3).clamp(min=-127), torch.full_like(e, -127))
    m = torch.where(fine[..., None], b, torch.zeros_like(b)).abs() * torch.exp2(-e.double())[..., None]
    code = torch.zeros(m.shape, dtype=torch.int64)
    for border, even_below in ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)):
        code += (m > border) if even_below else (m >= border)
    sign = torch.signbit(b) & fine[..., None]
    return code + 8 * sign, torch.where(fine, e + 127, torch.full_like(e, 255))


def values_of(code, byte):
    v = GRID[code & 7] * torch.where(code >= 8, -1.0, 1.0)
    return (v * torch.exp2(byte.double() - 127)[..., None]).flatten(1)


def unpacked(r):
    """Codes [M, pitch * 2] and scale bytes [M, scale pitch] of rows on the device."""
    c = r.codes.cpu().long()
    return torch.stack((c & 15, c >> 4), 2).flatten(1), r.scales.cpu().long()


def _check_rows(r, a, what=""):
    M, D = a.shape
    code, byte = fp4_of(a)
    got, scales = unpacked(r)
    nb = byte.shape[1]
    live = (byte != 255)[..., None].expand(-1, -1, 32).reshape(M, -1)[:, :D]
    same = got[:, :D] == code.flatten(1)[:, :D]
    zero = (got[:, :D] & 7 == 0) & (code.flatten(1)[:, :D] & 7 == 0)      # the sign of a zero says nothing
    assert (same | zero)[live].all(), what
    assert (got[:, :D][~live] == 0).all(), what
    assert torch.equal(scales[:, :nb], byte), what
    pitch, spitch = (D + 255) // 256 * 128, (D + 511) // 512 * 16
    assert (got[:, D: 2 * pitch] == 0).all() and (scales[:, nb:spitch][byte.amax(1) != 255] == 0).all(), what


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,D,ld", [(1, 1, 1), (3, 7, 7), (5, 32, 32), (4, 33, 40), (2, 255, 256), (7, 256, 256),
                                    (33, 250, 250), (6, 512, 520), (3, 513, 513), (9, 2048, 2048), (2, 2056, 2063),
                                    (5, 5120, 10240), (3, 6144, 6144), (2, 13824, 13824), (2, 16385, 16385),
                                    (1, 65535, 65535), (2, 65536, 65536)])
def test_quantize_exact(M, D, ld, dtype):
    say(f"quantize fp4 {M} x {D} (ld {ld}) {dtype}")
    g = _gen(M * 100003 + D)
    x = (_rand(g, M, D) * torch.exp2(torch.randint(-12, 12, (M, D), generator=g).float())).to(dtype)
    x[:, ::5] = (torch.randint(-16, 17, x[:, ::5].shape, generator=g) / 4.0).to(dtype)   # halves of small blocks
    if D >= 64:
        x[:, 32:64] = (torch.randint(-31, 32, (M, 32), generator=g) / 4.0).to(dtype)     # every border, 7.75 / 4 .. 8
        x[0, :32] = 0
    buf = torch.full((M + 2, ld), float("nan"), dtype=dtype)                             # rows apart, NaN around them
    buf[:M, :D] = x
    r = api.quantize_rows_fp4(buf.to(device())[:M, :D])
    torch.cuda.synchronize()
    assert r.codes.shape == (M, (D + 255) // 256 * 128) and r.scales.shape == (M, (D + 511) // 512 * 16) and r.cols == D
    _check_rows(r, x.double())
    back = api.dequantize_rows_fp4(r, dtype).cpu().double()
    assert torch.equal(back, values_of(*fp4_of(x.double()))[:, :D])


def test_quantize_unaligned_and_into_given_rows():
    """An element offset (no vector loads), outputs of wider pitches; what lies behind a
    row's own pitch and around the rows stays."""
    g = _gen(3)
    x = _rand(g, 6, 300, dtype=torch.bfloat16)
    codes = torch.full((8, 512), 99, dtype=torch.uint8, device=device())
    scales = torch.full((8, 64), 77, dtype=torch.uint8, device=device())
    view = api.Fp4Rows(codes[1:7], scales[1:7], 297)
    r = api.quantize_rows_fp4(x.to(device())[:, 3:], out=view)
    torch.cuda.synchronize()
    assert r is view
    _check_rows(r, x[:, 3:].double())
    c, s = codes.cpu(), scales.cpu()
    assert (c[[0, 7]] == 99).all() and (c[:, 256:] == 99).all() and (s[[0, 7]] == 77).all() and (s[:, 16:] == 77).all()
    y = torch.full((8, 320), 7.0, dtype=torch.bfloat16, device=device())
    api.dequantize_rows_fp4(r, out=y[1:7, 5:302])
    y = y.cpu()
    assert torch.equal(y[1:7, 5:302].double(), values_of(*fp4_of(x[:, 3:].double()))[:, :297])
    assert (y[[0, 7]] == 7).all() and (y[:, :5] == 7).all() and (y[:, 302:] == 7).all()


def test_quantize_edge_values():
    """Zeros, the smallest and the largest numbers, infinities and NaN: a block that is
    not finite is NaN as a whole, and alone."""
    t = 2.0 ** -149
    rows = [[0.0, -0.0, 0, 0], [t, -t, 3 * t, 0], [2.0 ** -126, 2.0 ** -127, -2.0 ** -128, 2.0 ** -129],
            [2.0 ** -125, -1.5 * 2.0 ** -126, 2.0 ** -127, 2.0 ** -130], [2.0 ** -124, 2.0 ** -127, 0, 2.0 ** -149],
            [7.9999995 * 2.0 ** -127, 5 * 2.0 ** -127, 2.5 * 2.0 ** -127, 0],
            [3.4028235e38, -2.0 ** 127, 2.0 ** 125, 1.0], [1.0, float("inf"), 0, 0], [1.0, 0, float("nan"), 2.0],
            [7.99, 8.0, -5.0, 6.0], [7.99, 5.0, -5.0, 2.5], [-float("inf"), float("nan"), 0, 0]]
    x = torch.zeros(len(rows), 70)
    x[:, :4] = torch.tensor(rows, dtype=torch.float64).float()
    x[:, 40] = 1.25                                             # the block beside
    r = api.quantize_rows_fp4(x.to(device()))
    torch.cuda.synchronize()
    _check_rows(r, x.double())
    back = api.dequantize_rows_fp4(r, torch.float32).cpu()
    fine = torch.isfinite(x[:, :32]).all(1)
    assert torch.equal(back[fine].double(), values_of(*fp4_of(x[fine].double()))[:, :70])
    assert torch.isnan(back[~fine][:, :32]).all() and (back[:, 40] == 1.0).all()


@pytest.mark.parametrize("D", [64, 130, 5120])
def test_quantize_picks_rows(D):
    g = _gen(D)
    x = _rand(g, 50, D, dtype=torch.bfloat16)
    rows = torch.tensor([49, 0, 7, 7, 3, -1, 50, 2 ** 31 - 1, 12], dtype=torch.int32)
    r = api.quantize_rows_fp4(x.to(device()), rows=rows.to(device()))
    torch.cuda.synchronize()
    ok = (rows >= 0) & (rows < 50)
    _check_rows(api.Fp4Rows(r.codes.cpu()[ok], r.scales.cpu()[ok], D), x[rows[ok].long()].double())
    assert (r.scales.cpu()[~ok][:, : (D + 31) // 32] == 255).all() and (r.codes.cpu()[~ok] == 0).all()   # no such row


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,D", [(1, 8), (5, 64), (70, 128), (4, 250), (33, 512), (9, 700), (5, 1024), (3, 1536), (4, 3000), (7, 5120), (3, 8192),
                                 (2, 13824), (2, 20001)])
def test_quantize_layernorm(M, D, dtype):
    """LayerNorm in fp32 in front: sums of at most 80 terms a lane and 10 joining
    steps, so a value is within 256 steps of 2^-24 of the row's largest; its code is
    that of a number so near to it, on a scale of one so near to the block's largest."""
    g = _gen(D + 1)
    x = (_rand(g, M, D) * 2 + 0.5).to(dtype)
    sh, sc = _rand(g, D) * 0.1, _rand(g, D) * 0.1
    r = api.quantize_rows_fp4(x.to(device()), shift=sh.to(device()), scale=sc.to(device()), ln_eps=1e-6)
    torch.cuda.synchronize()
    xd = x.double()
    z = (xd - xd.mean(1, keepdim=True)) / (xd.var(1, unbiased=False, keepdim=True) + 1e-6).sqrt()
    z = z * (1 + sc.double()) + sh.double()
    tol = 256 * U32 * z.abs().amax(1, keepdim=True)
    b, t = _blocks(z), tol[:, :, None]
    top = b.abs().amax(2, keepdim=True)
    got, scales = unpacked(r)
    nb = b.shape[1]
    byte = scales[:, :nb]
    low, high = (torch.frexp(v.clamp(min=2.0 ** -120))[1].squeeze(2) - 3 + 127 for v in (top - t, top + t))
    assert ((byte >= low) & (byte <= high)).all()
    unit = torch.exp2(byte.double() - 127)[..., None]
    code = got[:, : nb * 32].view(M, nb, 32)
    mag = lambda v: sum((v > e if even else v >= e).long() for e, even in  # noqa: E731
                        ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)))
    lo, hi = mag(((b.abs() - t) / unit).clamp(min=0)), mag((b.abs() + t) / unit)
    assert ((code & 7 >= lo) & (code & 7 <= hi)).all()
    assert ((code >= 8) == (b < 0))[(b.abs() > t) & (code & 7 > 0)].all()
    pick = torch.arange(M - 1, -1, -1, dtype=torch.int32)        # picked rows are the rows themselves, bit for bit
    r2 = api.quantize_rows_fp4(x.to(device()), rows=pick.to(device()), shift=sh.to(device()), scale=sc.to(device()))
    assert torch.equal(r2.codes.cpu().flip(0), r.codes.cpu()) and torch.equal(r2.scales.cpu().flip(0), r.scales.cpu())


@pytest.mark.parametrize("M,D", [(3, 37), (40, 260), (5, 1025), (4, 3003), (3, 7341), (2, 10001)])
def test_quantize_layernorm_with_vectors_at_any_element(M, D):
    """Rows of one modulation [2, D]: of an odd D the second starts off a vector's
    border.  The values are those of vectors of their own, bit for bit."""
    g = _gen(D + 2)
    x, m = _rand(g, M, D, dtype=torch.bfloat16).to(device()), (_rand(g, 2, D) * 0.1).to(device())
    r = api.quantize_rows_fp4(x, shift=m[0], scale=m[1])
    own = api.quantize_rows_fp4(x, shift=m[0].clone(), scale=m[1].clone())
    assert torch.equal(r.codes, own.codes) and torch.equal(r.scales, own.scales)


def test_quantize_empty():
    r = api.quantize_rows_fp4(torch.zeros(0, 64, device=device()))
    assert r.codes.shape == (0, 128) and r.scales.shape == (0, 16)
    assert api.dequantize_rows_fp4(r).shape == (0, 64)
    w = api.quantize_rows_fp4(torch.ones(8, 64, device=device()))
    assert api.linear_fp4(r, w).shape == (0, 8)


# --------------------------------------------------------------- linear_fp4

def _gelu(z):
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def random_rows(g, n, K, mid=127, spread=3):
    """Rows of codes over the whole range with scales of 2^-spread .. 2^spread around
    2^(mid - 127): as on the device, and their values."""
    nb = (K + 31) // 32
    code = torch.randint(0, 16, (n, nb, 32), generator=g)
    byte = torch.randint(mid - spread, mid + spread + 1, (n, nb), generator=g)
    flat = torch.zeros(n, (K + 255) // 256 * 256, dtype=torch.int64)
    flat[:, :K] = code.flatten(1)[:, :K]
    scales = torch.zeros(n, (K + 511) // 512 * 16, dtype=torch.uint8)
    scales[:, :nb] = byte.to(torch.uint8)
    codes = (flat[:, ::2] + 16 * flat[:, 1::2]).to(torch.uint8)
    return api.Fp4Rows(codes.to(device()), scales.to(device()), K), values_of(code, byte)[:, :K]


def check_linear(got, a, w, bias, out_dtype, act=None, gate=None, res=None, what=""):
    """The sum of K / 32 exact block sums, of parts joined (at most 16), and the bias:
    K / 32 + 20 additions, each within a step of 2^-23 of sum |a w| + |b| (the matrix
    instruction may cut where it does not round); GELU (slope below 1.13, its argument,
    exponential and quotient) at most 16 steps of 2^-24 more; gate and residual one
    more step of the result each."""
    K = a.shape[1]
    b = torch.zeros(w.shape[0], dtype=torch.float64) if bias is None else bias.double()
    z = a @ w.T + b
    err = (K / 32 + 20) * 2 * U32 * (a.abs() @ w.abs().T + b.abs())
    if act == "gelu":
        want = _gelu(z)
        err = 1.13 * err + 16 * U32 * z.abs()
    elif gate is not None:
        want = res.double() + gate.double() * z
        err = err * gate.double().abs() + 2 * U32 * (res.double().abs() + want.abs())
    else:
        want = z
    err = err * 1.01 + HALF_STEP[out_dtype] * want.abs() + 1e-38
    off = (got.double() - want).abs()
    worst = float((off / err).max()) if off.numel() else 0.0
    say(f"  {what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0


SIZES = [(1, 1, 1), (1, 16, 64), (1, 300, 5120), (2, 77, 129), (4, 33, 2049), (5, 1000, 700), (8, 64, 4100), (9, 40, 300),
         (16, 64, 128), (17, 129, 640), (32, 48, 256), (33, 100, 100), (48, 1000, 2600), (64, 512, 1024), (65, 65, 65),
         (100, 200, 300), (128, 128, 128), (130, 70, 13824), (257, 255, 200), (300, 512, 256), (500, 1030, 384),
         (1000, 96, 4000), (1111, 2049, 130), (2100, 2304, 768), (4100, 4100, 128), (70, 300, 40000), (4200, 4400, 1100),
         (3000, 6400, 1500), (5000, 5128, 300), (3, 5, 30), (3, 1536, 1536), (8, 1001, 1535), (15, 5130, 1500),
         (16, 2000, 5120), (7, 5131, 5000), (16, 5120, 5120), (18, 5121, 1537), (31, 2100, 515), (32, 1536, 1536),
         (32, 9000, 256), (12, 37, 33000), (25, 8300, 4097)]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_sizes(M, N, K, out_dtype):
    g = _gen(M * 7 + N * 3 + K)
    say(f"linear fp4 {M} x {N} x {K} -> {out_dtype}")
    (A, a), (W, w) = random_rows(g, M, K), random_rows(g, N, K, 121)
    bias = (_rand(g, N) * 0.1).to(out_dtype)
    got = api.linear_fp4(A, W, bias.to(device()), dtype=out_dtype)
    torch.cuda.synchronize()
    check_linear(got.cpu(), a, w, bias, out_dtype, what=f"{M}x{N}x{K}")


@pytest.mark.parametrize("M,N,K", [(1, 200, 300), (6, 60, 1500), (12, 96, 520), (13, 1500, 1536), (29, 5120, 1500), (20, 77, 130), (60, 64, 512),
                                   (140, 260, 260), (700, 1000, 200), (4096, 4100, 128), (90, 256, 8000), (4200, 4400, 1100),
                                   (5000, 5128, 300), (2600, 7000, 900)])
@pytest.mark.parametrize("epi", ["none", "gelu", "gate_bf16", "gate_f32_rows"])
def test_linear_epilogues(M, N, K, epi):
    g = _gen(M + N + K)
    say(f"linear fp4 {M} x {N} x {K} {epi}")
    (A, a), (W, w) = random_rows(g, M, K), random_rows(g, N, K, 121)
    if epi == "none":
        got = api.linear_fp4(A, W)
        check_linear(got.cpu(), a, w, None, torch.bfloat16, what=epi)
    elif epi == "gelu":
        bias = _rand(g, N)
        got = api.linear_fp4(A, W, bias.to(device()), activation="gelu", dtype=torch.float32)
        check_linear(got.cpu(), a, w, bias, torch.float32, act="gelu", what=epi)
    else:
        rdt = torch.bfloat16 if epi == "gate_bf16" else torch.float32
        gate, bias = _rand(g, N), _rand(g, N, dtype=rdt)
        n = M if epi == "gate_bf16" else M + 9
        res = _rand(g, n, N + 3, dtype=rdt)[:, :N] if N % 2 else _rand(g, n, N, dtype=rdt)
        rows = None if epi == "gate_bf16" else torch.randint(0, n, (M,), generator=g, dtype=torch.int32)
        got = api.linear_fp4(A, W, bias.to(device()), gate=gate.to(device()), residual=res.to(device()),
                             residual_rows=None if rows is None else rows.to(device()), dtype=torch.float32)
        check_linear(got.cpu(), a, w, bias, torch.float32, gate=gate,
                     res=res if rows is None else res[rows.long()], what=epi)


def test_linear_every_code_and_scale():
    """Each pair of codes in turn, at each place of a block, and scales over the whole
    range (2^-63 2^63 and the like): one product a sum, exact."""
    for M in (1, 16, 256):
        K = 512
        code_a = torch.zeros(M, K, dtype=torch.int64)
        code_w = torch.zeros(256, K, dtype=torch.int64)
        at = torch.arange(256) % K
        code_w[torch.arange(256), at] = torch.arange(256) // 16
        for m in range(M):
            code_a[m] = (torch.arange(K) + m) % 16
        sa = torch.full((M, 16), 64, dtype=torch.uint8) + (torch.arange(M)[:, None] % 120).to(torch.uint8)
        sw = torch.full((256, 16), 190, dtype=torch.uint8) - (torch.arange(256)[:, None] % 120).to(torch.uint8)
        pack = lambda c: (c[:, ::2] + 16 * c[:, 1::2]).to(torch.uint8).to(device())  # noqa: E731
        A, W = api.Fp4Rows(pack(code_a), sa.to(device()), K), api.Fp4Rows(pack(code_w), sw.to(device()), K)
        got = api.linear_fp4(A, W, dtype=torch.float32).cpu().double()
        a, w = values_of(code_a.view(M, 16, 32), sa.long()), values_of(code_w.view(256, 16, 32), sw.long())
        assert torch.equal(got, a @ w.T)


@pytest.mark.parametrize("M,N,K", [(3, 40, 128), (12, 100, 256), (100, 200, 4096), (600, 516, 256), (300, 203, 128)])
def test_linear_onto_its_residual(M, N, K):
    g = _gen(M)
    (A, _), (W, _) = random_rows(g, M, K), random_rows(g, N, K, 121)
    gate, res = _rand(g, N).to(device()), _rand(g, M, N).to(device())
    want = api.linear_fp4(A, W, gate=gate, residual=res, dtype=torch.float32)
    got = api.linear_fp4(A, W, gate=gate, residual=res, out=res)
    assert got is res and torch.equal(got, want)


@pytest.mark.parametrize("M", [1, 7, 14, 40, 300])
def test_linear_nan_rows_and_surroundings(M):
    """A NaN block makes its own row (its own channel) NaN and no other, missing
    residual rows are NaN, and the output's surroundings stay."""
    g = _gen(77)
    N, K = 200, 1060
    (A, _), (W, _) = random_rows(g, M, K), random_rows(g, N, K, 121)
    A.scales[M // 2, 30] = 255
    W.scales[3, 0] = 255
    buf = torch.full((M + 2, N + 5), 3.0, device=device())
    whole = api.linear_fp4(A, W, dtype=torch.float32, out=buf[1:M + 1, 2:N + 2])
    b = buf.cpu()
    assert (b[0] == 3).all() and (b[-1] == 3).all() and (b[:, :2] == 3).all() and (b[:, N + 2:] == 3).all()
    nan = torch.isnan(whole.cpu())
    want = torch.zeros(M, N, dtype=torch.bool)
    want[M // 2], want[:, 3] = True, True
    assert torch.equal(nan, want)
    (A, _), (W, _) = random_rows(g, M, K), random_rows(g, N, K, 121)
    gate, res = torch.ones(N, device=device()), torch.zeros(4, N, device=device())
    rows = torch.zeros(M, dtype=torch.int32, device=device())
    rows[0], rows[M - 1] = 4, -1
    y = api.linear_fp4(A, W, gate=gate, residual=res, residual_rows=rows, dtype=torch.float32).cpu()
    bad = torch.isnan(y).all(1)
    assert bad[[0, M - 1]].all() and int(bad.sum()) == min(M, 2) and int(torch.isnan(y).any(1).sum()) == min(M, 2)


@pytest.mark.parametrize("M,N,K,pa,pw", [(5, 70, 300, 512, 384), (20, 130, 600, 384, 1024), (200, 300, 1000, 640, 512),
                                         (600, 520, 200, 128, 256)])
def test_linear_pitches_and_codes_behind_the_depth(M, N, K, pa, pw):
    """Wider pitches than the depth needs: what lies behind them is not read, and codes
    behind the depth in one operand meet zeros in the other."""
    g = _gen(M + K)
    (A, a), (W, w) = random_rows(g, M, K), random_rows(g, N, K, 121)
    wide = lambda r, p, q: api.Fp4Rows(torch.full((len(r), p), 255, dtype=torch.uint8, device=device()),  # noqa: E731
                                       torch.full((len(r), q), 255, dtype=torch.uint8, device=device()), K)
    A2, W2 = wide(A, pa, 112), wide(W, pw, 48)
    for r, s in ((A, A2), (W, W2)):
        s.codes[:, : r.codes.shape[1]], s.scales[:, : r.scales.shape[1]] = r.codes, r.scales
    got = api.linear_fp4(A2, W2, dtype=torch.float32)
    check_linear(got.cpu(), a, w, None, torch.float32, what="wide pitches")
    if K % 256:
        W2.codes[:, (K + 1) // 2: W.codes.shape[1]] = 0x77                 # codes behind the depth, in one operand
        W2.scales[:, (K + 31) // 32: W.scales.shape[1]] = 130
        assert torch.equal(api.linear_fp4(A2, W2, dtype=torch.float32), got)


def test_linear_streams_and_graphs():
    """Captured graphs with eager calls in between, on a side stream: each replay equals
    the eager result (split products have a workspace of their own)."""
    g = _gen(5)
    shapes = [(130, 200, 8192), (1, 4000, 1024), (30, 1000, 5120), (600, 700, 512)]
    made = []
    for M, N, K in shapes:
        x = _rand(g, M, K, dtype=torch.bfloat16).to(device())
        w = api.quantize_rows_fp4((_rand(g, N, K) * 0.05).to(device()))
        made.append((x, w, api.linear_fp4(api.quantize_rows_fp4(x), w)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager = [api.linear_fp4(api.quantize_rows_fp4(x), w) for x, w, _ in made]
    side.synchronize()
    for e, (_, _, ref) in zip(eager, made):
        assert torch.equal(e, ref)
    graphs = []
    for x, w, ref in made:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            y = api.linear_fp4(api.quantize_rows_fp4(x), w)
        graphs.append((gr, y))
    for turn in range(3):
        for (gr, y), (x, w, _) in zip(graphs, made):
            x.mul_(-0.5)
            gr.replay()
            ref = api.linear_fp4(api.quantize_rows_fp4(x), w)
            torch.cuda.synchronize()
            assert torch.equal(y, ref), turn
