"""The 4-bit rows, the linear layer on them, the rotary positions and the gated norm past
offsets of 32 bits: rows at both ends of tensors of more than 2^31 bytes and elements,
against the same rows in small tensors, bit for bit."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device, say

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _fill(t, seed):
    """Normal values, some thousand rows at a time."""
    g = torch.Generator(device=device())
    g.manual_seed(seed)
    for part in t.split(4096):
        part.copy_(torch.randn(part.shape, device=device(), generator=g, dtype=t.dtype))
    return t


def test_rows_and_products():
    M, D, N = 66000, 65536, 70
    x = _fill(torch.empty(M, D, dtype=BF, device=device()), 1)
    r = api.quantize_rows_fp4(x)
    assert r.codes.numel() > 2 ** 31
    say("  quantized")
    ends = torch.cat((torch.arange(20), torch.arange(M - 20, M))).to(device())
    small = api.quantize_rows_fp4(x[ends])
    assert torch.equal(r.codes[ends], small.codes) and torch.equal(r.scales[ends], small.scales)
    picked = api.quantize_rows_fp4(x, rows=ends.to(torch.int32))
    assert torch.equal(picked.codes, small.codes)
    back = api.dequantize_rows_fp4(r, out=x)
    assert torch.equal(back[ends], api.dequantize_rows_fp4(small))
    say("  read back")
    del x, back
    w = api.quantize_rows_fp4(_fill(torch.empty(N, D, device=device()), 2) * 0.01)
    y = api.linear_fp4(r, w, dtype=torch.float32)
    # (whole tiles of 64 rows, so that the few rows take the same sums as the many)
    for lo, hi in ((0, 64), (M - M % 64 - 64, M - M % 64)):
        part = api.linear_fp4(api.Fp4Rows(r.codes[lo:hi], r.scales[lo:hi], D), w, dtype=torch.float32)
        off = (part - y[lo:hi]).abs().max()
        say(f"  rows {lo}..: {float(off):.2e}")
        # other splits of 2048 block sums: 2 (2048 + 20) steps of 2^-23 of sum |a w|, below 0.01 * 65536 here
        assert float(off) <= 2 * 2068 * 2.0 ** -23 * 0.01 * 65536
    wide = api.linear_fp4(w, r, dtype=torch.float32)              # the many rows as channels
    assert float((wide.T - y).abs().max()) <= 2 * 2068 * 2.0 ** -23 * 0.01 * 65536


def test_rotary_positions():
    L, H, dh = 140000, 128, 128
    x = _fill(torch.empty(L, H * dh, dtype=BF, device=device()), 3).view(1, L, H, dh)
    assert x.numel() > 2 ** 31
    rot = api.Rotary.make(dh, device(), "half")
    ends = torch.cat((torch.arange(9), torch.arange(L - 9, L))).to(device())
    want, _ = api.rotary(x[:, ends], rot, positions=ends.to(torch.int32))
    api.rotary(x, rot, out=x)
    assert torch.equal(x[:, ends], want)


def test_gated_norm():
    M, D = 140000, 16384
    z, x = (_fill(torch.empty(M, D, dtype=BF, device=device()), s) for s in (4, 5))
    assert z.numel() > 2 ** 31
    ends = torch.cat((torch.arange(9), torch.arange(M - 9, M))).to(device())
    gate = torch.randn(D, device=device())
    want = api.gated_norm(z[ends], x[ends], gate=gate)
    rows = torch.arange(M - 1, -1, -1, dtype=torch.int32, device=device())
    y, h = api.gated_norm(z, x, gate=gate)
    assert torch.equal(y[ends], want[0]) and torch.equal(h[ends], want[1])
    back = api.gated_norm(z, x, gate=gate, residual_rows=rows, before=None, y=h)[0]
    assert torch.equal(back[ends], api.gated_norm(z[ends], x[(M - 1 - ends)], gate=gate, before=None)[0])
