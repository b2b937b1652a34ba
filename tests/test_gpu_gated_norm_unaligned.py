"""The gated norm's unaligned form at widths of whole vectors, where only an address or a
distance between rows is off: every tensor in turn one element off, and all of them,
against 64 bits by the bounds of test_gpu_gated_norm.py."""
import pytest
import torch

from paper_2608_02474_amd import api

from gpu_util import device
from test_gpu_gated_norm import check

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
VECTORS = ("w1", "w2", "gate", "scale", "shift")


def _off(t, by):
    """t on the device, `by` elements behind an aligned address, rows one vector and one
    element apart."""
    if t.dim() == 1:
        buf = torch.full((len(t) + by,), 9.0, dtype=t.dtype, device=device())
        buf[by:] = t.to(device())
        return buf[by:]
    buf = torch.full((len(t), t.shape[1] + 9), 9.0, dtype=t.dtype, device=device())
    buf[:, by: by + t.shape[1]] = t.to(device())
    return buf[:, by: by + t.shape[1]]


@pytest.mark.parametrize("D", [8, 128, 512, 1536, 4096, 6200, 8192, 13824])
@pytest.mark.parametrize("zt,xt", [(BF, F32), (F32, BF)])
def test_one_tensor_off_and_all(D, zt, xt):
    g = torch.Generator().manual_seed(D)
    M = 19
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    host = dict(z=(r(M, D) * 3 + 1).to(zt), x=r(M, D).to(xt), w1=1 + 0.1 * r(D), w2=1 + 0.1 * r(D), gate=r(D),
                scale=0.1 * r(D), shift=0.1 * r(D))
    names = ("z", "x", "y", "h") + VECTORS
    for which in (*[(n,) for n in names], names):
        on = {n: _off(t, 1) if n in which else t.to(device()) for n, t in host.items()}
        y, h = (torch.full((M + 2, D + 9), 7.0, dtype=t, device=device()) for t in (xt, zt))
        at = {n: slice(1, 1 + D) if n in which else slice(0, D) for n in ("y", "h")}
        yv = y[1:-1, at["y"]] if "y" in which else torch.empty(M, D, dtype=xt, device=device())
        hv = h[1:-1, at["h"]] if "h" in which else torch.empty(M, D, dtype=zt, device=device())
        api.gated_norm(on["z"], on["x"], after="rms", after_weight=on["w1"], gate=on["gate"], residual_scale=0.7,
                       before="layer", before_weight=on["w2"], scale=on["scale"], shift=on["shift"], y=yv, h=hv)
        check(yv.cpu(), hv.cpu(), host["z"], host["x"], "rms", host["w1"], host["gate"].double()[None], 0.7, "layer",
              host["w2"], host["scale"].double()[None], host["shift"].double()[None], 1e-6, f"{D} {which}")
        for t, v in ((y, yv), (h, hv)):          # what lies around an output stays
            v.fill_(7.0)
            assert bool((t == 7).all()), which
