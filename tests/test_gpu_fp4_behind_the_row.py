"""What lies behind the last column of 4-bit rows: codes and scales of zero up to the
row's pitches, whatever the row holds, a row that is not there among them."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [1, 32, 40, 64, 127, 128, 129, 300, 520, 1100, 2049, 5150, 9000, 20001])
@pytest.mark.parametrize("ln", [False, True])
def test_zeros_behind_the_last_column(D, ln, dtype):
    g = torch.Generator().manual_seed(D)
    x = torch.randn(9, D, generator=g).to(dtype)
    x[1, D - 1], x[2, 0], x[3, D // 2], x[4] = float("inf"), float("nan"), -float("inf"), 0
    rows = torch.tensor([0, 1, 2, 3, 4, -1, 9, 8, 2 ** 31 - 1, 5], dtype=torch.int32)
    kw = {}
    if ln:
        kw = dict(shift=torch.randn(D, generator=g).to(device()), scale=torch.randn(D, generator=g).to(device()))
    nb = (D + 31) // 32
    for pick in (None, rows):
        n = 9 if pick is None else len(rows)
        out = api.Fp4Rows(torch.full((n, (D + 255) // 256 * 128), 99, dtype=torch.uint8, device=device()),
                          torch.full((n, (D + 511) // 512 * 16), 99, dtype=torch.uint8, device=device()), D)
        r = api.quantize_rows_fp4(x.to(device()), rows=None if pick is None else pick.to(device()), out=out, **kw)
        codes, scales = r.codes.cpu(), r.scales.cpu()
        assert (scales[:, nb:] == 0).all()
        assert (codes[:, (D + 1) // 2:] == 0).all() and (D % 2 == 0 or (codes[:, D // 2] >> 4 == 0).all())
        at = torch.arange(9) if pick is None else pick.long()
        there = (at >= 0) & (at < 9)
        assert (scales[~there][:, :nb] == 255).all() and (codes[~there] == 0).all()
        for i, row in zip(at[there], scales[there]):
            bad = torch.zeros(nb, dtype=torch.bool)
            fine = torch.isfinite(x[i].float())
            bad[(~fine).nonzero().flatten() // 32] = True
            if ln and not fine.all():
                bad[:] = True
            assert torch.equal(row[:nb] == 255, bad), int(i)
