"""Refusals of the 4-bit rows, the linear layer on them, the rotary positions and the
norms on both sides of a sub-layer, on the CPU: the C ABI rejects bad arguments before
any HIP call, sizes its workspaces as pure functions and takes empty calls as done; the
binding rejects what the ABI cannot see.  And the host function of the frequencies
against its formulas."""
import ctypes
import math

import pytest
import torch

from paper_2608_02474_amd import _lib, api

FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10001)
FAKE2 = ctypes.c_void_p(0x20000)
OFF4 = ctypes.c_void_p(0x10004)
BF, F32 = _lib.ECHO_BF16, _lib.ECHO_F32
OK, EINVAL, EUNSUP, EWS = _lib.ECHO_OK, _lib.ECHO_EINVAL, _lib.ECHO_EUNSUPPORTED, _lib.ECHO_EWORKSPACE


class _AsOnDevice(torch.Tensor):
    """A host tensor that says it is on the device: the checks of a call run as for
    one that is, and nothing is launched."""
    is_cuda = property(lambda self: True)


def on(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_AsOnDevice)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_packed_structures_are_the_structures():
    for cfg, pack in ((_lib.QuantizeFp4Cfg, _lib.PACK_QUANTIZE_FP4), (_lib.LinearFp4Cfg, _lib.PACK_LINEAR_FP4),
                      (_lib.RotaryCfg, _lib.PACK_ROTARY), (_lib.GatedNormCfg, _lib.PACK_GATED_NORM)):
        n = sum(3 if t is _lib.Strides else 1 for _, t in cfg._fields_)
        b = pack(*range(1, n + 1))
        got, want = cfg.from_buffer_copy(b.ljust(ctypes.sizeof(cfg), b"\0")), iter(range(1, n + 1))
        for name, t in cfg._fields_:
            v = getattr(got, name)
            for x in ((v.batch, v.row, v.head) if t is _lib.Strides else (v,)):
                assert x == next(want), (cfg, name)


def test_pitches(lib):
    assert [lib.echo_fp4_pitch(d) for d in (1, 256, 257, 5120, 65536)] == [128, 128, 256, 2560, 32768]
    assert [lib.echo_fp4_scale_pitch(d) for d in (1, 512, 513, 5120, 65536)] == [16, 16, 32, 160, 2048]
    assert [f(d) for f in (lib.echo_fp4_pitch, lib.echo_fp4_scale_pitch) for d in (0, -1, 65537)] == [0] * 6


def test_quantize_rejects_before_launch(lib):
    def run(M=4, D=64, dt=BF, nx=4, ldx=64, ldq=128, lds=16, eps=1e-6, x=FAKE, rows=None, sh=None, sc=None, q=FAKE, s=FAKE):
        cfg = _lib.QuantizeFp4Cfg(M, D, dt, nx, ldx, ldq, lds, eps)
        return lib.echo_quantize_rows_fp4(ctypes.byref(cfg), x, rows, sh, sc, q, s, None)
    for bad in (dict(M=-1), dict(D=0), dict(D=65537, ldx=65537, ldq=65536), dict(dt=2), dict(ldx=63), dict(ldq=64),
                dict(ldq=192), dict(ldq=65536 + 128), dict(lds=8), dict(lds=24), dict(lds=65552), dict(D=513, ldx=513, ldq=384),
                dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(x=ODD), dict(q=None), dict(q=OFF4),
                dict(s=None), dict(s=OFF4), dict(nx=3), dict(rows=FAKE, nx=0), dict(rows=ODD), dict(sh=FAKE),
                dict(sc=FAKE), dict(sh=ODD, sc=FAKE), dict(sh=OFF4, sc=ODD)):
        assert run(**bad) == EINVAL, bad
    assert lib.echo_quantize_rows_fp4(None, FAKE, None, None, None, FAKE, FAKE, None) == EINVAL
    assert run(M=0, x=None, q=None, s=None) == OK

    def back(M=4, D=64, dt=BF, ldx=64, ldq=128, lds=16, x=FAKE, q=FAKE, s=FAKE):
        cfg = _lib.QuantizeFp4Cfg(M, D, dt, 0, ldx, ldq, lds, 0.0)
        return lib.echo_dequantize_rows_fp4(ctypes.byref(cfg), q, s, x, None)
    for bad in (dict(M=-1), dict(D=0), dict(dt=-1), dict(ldx=63), dict(ldq=127), dict(lds=0), dict(x=None), dict(x=ODD),
                dict(q=OFF4), dict(s=None), dict(s=ODD)):
        assert back(**bad) == EINVAL, bad
    assert back(M=0, x=None, q=None, s=None) == OK


def _linear(M=100, N=70, K=64, epi=0, od=BF, bd=BF, rd=BF, nres=100, lda=128, ldsa=16, ldw=128, ldsw=16, ldc=70, ldr=70):
    return _lib.LinearFp4Cfg(M, N, K, epi, od, bd, rd, nres, lda, ldsa, ldw, ldsw, ldc, ldr)


def test_linear_rejects_before_launch(lib):
    def run(a=FAKE, sa=FAKE, w=FAKE, sw=FAKE, b=FAKE, g=None, r=None, rr=None, c=FAKE, ws=FAKE, n=1 << 40, **kw):
        return lib.echo_linear_fp4(ctypes.byref(_linear(**kw)), a, sa, w, sw, b, g, r, rr, c, ws, n, None)
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(K=65537, lda=1 << 16, ldw=1 << 16), dict(epi=3), dict(epi=-1),
                dict(od=2), dict(bd=2), dict(rd=2), dict(lda=64), dict(lda=192), dict(ldw=64), dict(ldsa=8), dict(ldsw=17),
                dict(ldc=69), dict(a=None), dict(a=OFF4), dict(sa=None), dict(sa=OFF4), dict(w=OFF4), dict(sw=OFF4),
                dict(b=ODD), dict(c=None), dict(c=ODD), dict(g=FAKE), dict(r=FAKE), dict(rr=FAKE), dict(epi=2),
                dict(epi=2, g=FAKE), dict(epi=2, g=FAKE, r=FAKE, ldr=69), dict(epi=2, g=FAKE, r=FAKE, nres=99),
                dict(epi=2, g=FAKE, r=FAKE, rr=FAKE, nres=0)):
        assert run(**bad) == EINVAL, bad
    assert lib.echo_linear_fp4(None, *[FAKE] * 9, FAKE, 0, None) == EINVAL
    assert run(N=(1 << 22) + 1, ldc=1 << 23) == EUNSUP
    assert run(M=1 << 30, N=1 << 22, ldc=1 << 22) == EUNSUP
    assert run(M=0, a=None, c=None, ws=None, n=0) == OK
    some = 0
    for kw in (dict(), dict(M=70, N=64, K=40000, lda=20096, ldsa=1264, ldw=20096, ldsw=1264),
               dict(M=20, N=5120, K=5120, lda=2560, ldsa=160, ldw=2560, ldsw=160, ldc=5120)):
        need = lib.echo_linear_fp4_workspace(ctypes.byref(_linear(**kw)))
        if need:
            some += 1
            assert run(ws=None, **kw) == EWS and run(n=need - 1, **kw) == EWS and run(ws=OFF4, **kw) == EWS
    assert some and lib.echo_linear_fp4_workspace(ctypes.byref(_linear(K=0))) == 0


def _rotary(B=2, L=5, H=4, Hk=2, dh=64, dims=64, layout=0, dt=BF, gh=0, gw=0, pt=0, pr=0, m=1.0, pb=0, q=(1280, 256, 64),
            k=(640, 128, 64), qo=(1280, 256, 64), ko=(640, 128, 64)):
    return _lib.RotaryCfg(B, L, H, Hk, dh, dims, layout, dt, gh, gw, pt, pr, m, pb, q, k, qo, ko)


def test_rotary_rejects_before_launch(lib):
    def run(q=FAKE, k=FAKE, p=None, f=FAKE, qo=FAKE2, ko=FAKE2, **kw):
        return lib.echo_rotary(ctypes.byref(_rotary(**kw)), q, k, p, f, qo, ko, None)
    nan = float("nan")
    for bad in ({"B": -1}, {"L": -1}, {"H": 0}, {"Hk": -1}, {"dims": 0}, {"dims": 63}, {"dims": 66}, {"layout": 2},
                {"dt": 2}, {"gh": 3}, {"gw": 3}, {"gh": -1, "gw": 2}, {"pt": -1}, {"pt": 20, "pr": 13}, {"m": nan},
                {"m": float("inf")}, {"pb": -1}):
        assert lib.echo_rotary(ctypes.byref(_rotary(**bad)), FAKE, FAKE, None, FAKE, FAKE2, FAKE2, None) == EINVAL, bad
    for t in ("q", "k", "qo", "ko"):
        bad = _rotary(**{t: (-1, 256, 64)})
        assert lib.echo_rotary(ctypes.byref(bad), FAKE, FAKE, None, FAKE, FAKE2, FAKE2, None) == EINVAL
    for bad in (dict(q=None), dict(q=ODD), dict(k=None), dict(qo=None), dict(ko=ODD), dict(f=None), dict(f=OFF4), dict(p=ODD)):
        assert run(**bad) == EINVAL, bad
    same = _rotary(qo=(1280, 512, 64))
    assert lib.echo_rotary(ctypes.byref(same), FAKE, FAKE, None, FAKE, FAKE, FAKE2, None) == EINVAL   # in place, other strides
    assert lib.echo_rotary(None, FAKE, FAKE, None, FAKE, FAKE2, FAKE2, None) == EINVAL
    for bad in (dict(dh=513), dict(H=65535), dict(B=1 << 12, L=1 << 12)):
        assert run(**bad) == EUNSUP, bad
    assert run(B=0, q=None, qo=None) == OK and run(L=0, f=None) == OK


def test_rotary_frequencies(lib):
    base, L0, s, n = 10000.0, 4096.0, 8.0, 64
    plain = [base ** (-j / n) for j in range(n)]
    get = lambda **kw: api.rotary_frequencies(128, **kw)  # noqa: E731
    near = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a, b)) and len(a) == len(b)  # noqa: E731
    f, m, p = get()
    assert near(f, plain) and m == 1.0 and p is None
    f, m, _ = get(scaling="linear", factor=s)
    assert near(f, [v / s for v in plain]) and m == 1.0
    f, m, _ = get(scaling="base", factor=s)
    assert near(f, [(base * s ** (128 / 126)) ** (-j / n) for j in range(n)]) and m == 1.0
    f, m, _ = get(scaling="ramp", factor=s, original_length=L0)
    at = lambda turns: n * math.log(L0 / (2 * math.pi * turns)) / math.log(base)  # noqa: E731
    lo, hi = math.floor(at(32.0)), math.ceil(at(1.0))
    keep = [1 - min(1.0, max(0.0, (j - lo) / (hi - lo))) for j in range(n)]
    assert near(f, [k * v + (1 - k) * v / s for k, v in zip(keep, plain)]) and abs(m - 1 - 0.1 * math.log(s)) < 1e-6
    assert f[0] == plain[0] and abs(f[-1] * s / plain[-1] - 1) < 1e-14
    f, m, _ = get(scaling="bands", factor=s, original_length=L0, low=1.0, high=4.0)
    keep = [min(1.0, max(0.0, (L0 * v / (2 * math.pi) - 1.0) / 3.0)) for v in plain]
    assert near(f, [k * v + (1 - k) * v / s for k, v in zip(keep, plain)]) and m == 1.0
    f, m, p = get(grid=(30, 52))
    assert p == (22, 21, 21) and near(f, [base ** (-j / k) for k in p for j in range(k)])
    f, m, p = get(grid=(3, 4), pairs=(0, 40, 24), scaling="linear", factor=2.0)
    assert near(f, [base ** (-j / k) / 2 for k in p[1:] for j in range(k)])
    nan, inf = float("nan"), float("inf")
    for bad in (dict(base=1.0), dict(base=nan), dict(scaling="linear", factor=0.5), dict(scaling="ramp", factor=inf, original_length=L0),
                dict(scaling="ramp", factor=2.0), dict(scaling="bands", factor=2.0, original_length=L0, low=4.0, high=4.0),
                dict(scaling="bands", factor=2.0, original_length=L0, low=0.0), dict(scaling="ramp", factor=2.0, original_length=L0, grid=(2, 2))):
        with pytest.raises(RuntimeError, match="echo_rotary_frequencies"):
            get(**bad)
    for dims in (0, 3, -2, 514):
        with pytest.raises(RuntimeError, match="echo_rotary_frequencies"):
            api.rotary_frequencies(dims)
    with pytest.raises(RuntimeError):
        api.rotary_frequencies(2, scaling="base", factor=2.0)
    for bad in (dict(scaling="x"), dict(pairs=(1, 2, 3)), dict(grid=(2, 2), pairs=(1, 2, 3)), dict(grid=(2, 2), pairs=(-1, 65, 0)),
                dict(grid=(2, 2), pairs=(0, 0, 64))):
        with pytest.raises(ValueError):
            get(**bad)
    cfg = _lib.RotaryFreqCfg(128, 0, 0, 0, base, 1.0, 0.0, 1.0, 32.0)
    assert lib.echo_rotary_frequencies(ctypes.byref(cfg), None, None) == EINVAL
    assert lib.echo_rotary_frequencies(None, (ctypes.c_double * 64)(), ctypes.byref(ctypes.c_float())) == EINVAL
    cfg.scaling = 5
    assert lib.echo_rotary_frequencies(ctypes.byref(cfg), (ctypes.c_double * 64)(), ctypes.byref(ctypes.c_float())) == EINVAL


def _norm(M=6, D=64, G=1, after=1, before=2, zd=BF, rd=F32, yd=F32, hd=BF, n=6, a=1.0, eps=1e-6, ldz=64, ldr=64, ldy=64, ldh=64,
          ldg=0, lds=0, ldt=0):
    return _lib.GatedNormCfg(M, D, G, after, before, zd, rd, yd, hd, n, a, eps, ldz, ldr, ldy, ldh, ldg, lds, ldt)


def test_norm_rejects_before_launch(lib):
    F3, F4 = ctypes.c_void_p(0x30000), ctypes.c_void_p(0x40000)
    def run(z=FAKE, x=FAKE2, rows=None, w1=None, g=None, w2=None, s=None, t=None, gr=None, y=F3, h=F4, **kw):
        return lib.echo_gated_norm(ctypes.byref(_norm(**kw)), z, x, rows, w1, g, w2, s, t, gr, y, h, None)
    inf, nan = float("inf"), float("nan")
    for bad in (dict(M=-1), dict(D=0), dict(G=0), dict(after=3), dict(before=-1), dict(zd=2), dict(rd=-1), dict(yd=2),
                dict(hd=2), dict(a=nan), dict(a=inf), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(ldz=63), dict(ldr=63),
                dict(ldy=63), dict(ldh=63), dict(ldg=63), dict(lds=-1), dict(ldt=1), dict(z=None), dict(z=ODD), dict(x=None),
                dict(x=ODD), dict(y=None), dict(y=ODD), dict(h=None), dict(h=ODD), dict(rows=ODD), dict(w1=ODD), dict(g=ODD),
                dict(w2=ODD), dict(s=ODD), dict(t=ODD), dict(gr=ODD), dict(n=5), dict(rows=FAKE, n=0), dict(G=4),
                dict(before=0), dict(before=0, h=None, w2=FAKE), dict(before=0, h=None, s=FAKE), dict(before=0, h=None, t=FAKE),
                dict(y=FAKE2, rows=FAKE), dict(y=FAKE2, yd=BF), dict(y=FAKE2, ldy=72), dict(h=FAKE, hd=F32), dict(h=FAKE, ldh=72)):
        assert run(**bad) == EINVAL, bad
    assert lib.echo_gated_norm(None, *[FAKE] * 12) == EINVAL
    assert run(D=16385, ldz=16385, ldr=16385, ldy=16385, ldh=16385) == EUNSUP
    assert run(M=0, n=0, z=None, x=None, y=None, h=None) == OK
    assert run(M=0, G=5, n=0) == OK


def test_binding_rejects_host_tensors_shapes_and_types():
    x = torch.zeros(4, 64)
    rot = api.Rotary(on(32, dtype=torch.float64))
    with pytest.raises(ValueError, match="device tensor"):
        api.quantize_rows_fp4(x)
    with pytest.raises(TypeError, match="Fp4Rows"):
        api.dequantize_rows_fp4(x)
    with pytest.raises(TypeError, match="Fp4Rows"):
        api.linear_fp4(x, x)
    with pytest.raises(TypeError, match="Fp4Rows"):
        api.linear_fp4(api.Int8Rows(on(4, 128, dtype=torch.int8), on(4, dtype=torch.float32), 64), None)
    for c, s, cols in ((on(4, 128), on(4, 16, dtype=torch.uint8), 64), (on(4, 64, dtype=torch.uint8), on(4, 16, dtype=torch.uint8), 64),
                       (on(4, 128, dtype=torch.uint8), on(4, 8, dtype=torch.uint8), 64), (on(4, 128, dtype=torch.uint8), on(3, 16, dtype=torch.uint8), 64),
                       (on(4, 128, dtype=torch.uint8), on(4, 16, dtype=torch.uint8), 257), (on(4, 128, dtype=torch.uint8), on(4, 16, dtype=torch.uint8), 0)):
        with pytest.raises((ValueError, TypeError), match="r.codes|r.scales|as many rows"):
            api.dequantize_rows_fp4(api.Fp4Rows(c, s, cols))
    q = on(1, 5, 2, 64)
    for kw in (dict(k=on(1, 4, 2, 64)), dict(k=on(1, 5, 2, 32)), dict(k=on(1, 5, 2, 64, dtype=torch.float32)), dict(k_out=q),
               dict(positions=on(4, dtype=torch.int32)), dict(positions=on(5, dtype=torch.int64)), dict(positions=on(2, 5, dtype=torch.int32)),
               dict(out=on(1, 5, 2, 32)), dict(out=on(1, 1, 2, 64).expand(1, 5, 2, 64))):
        with pytest.raises((ValueError, TypeError)):
            api.rotary(q, rot, **kw)
    with pytest.raises(TypeError, match="Rotary"):
        api.rotary(q, rot.freq)
    for bad in (api.Rotary(on(32, dtype=torch.float32)), api.Rotary(on(32, dtype=torch.float64), "other"), api.Rotary(on(257, dtype=torch.float64)),
                api.Rotary(on(32, dtype=torch.float64), grid=(2, 2), pairs=(10, 10, 11)), api.Rotary(on(32, dtype=torch.float64), grid=(0, 2), pairs=(12, 10, 10)),
                api.Rotary(on(32, dtype=torch.float64), pairs=(12, 10, 10))):
        with pytest.raises((ValueError, TypeError)):
            api.rotary(q, bad)
    z = on(6, 64)
    f = lambda *s: on(*s, dtype=torch.float32)  # noqa: E731
    for kw in (dict(after="x"), dict(before="none"), dict(after_weight=f(63)), dict(gate=on(64)), dict(gate=f(4, 64)), dict(gate=f(2, 64), scale=f(3, 64)),
               dict(residual_rows=on(5, dtype=torch.int32)), dict(groups=on(6, dtype=torch.int64)), dict(y=f(6, 63)), dict(h=f(5, 64)),
               dict(before=None, scale=f(64)), dict(before=None, h=z), dict(before_weight=f(1, 64)), dict(y=f(6, 64), y_dtype=torch.bfloat16),
               dict(residual=f(5, 64)), dict(residual=f(6, 63))):
        with pytest.raises((ValueError, TypeError)):
            api.gated_norm(z, kw.pop("residual", f(6, 64)), **kw)


def test_block_on_4_bit_rows_refuses_before_any_launch():
    """Codes of the other kind among the matrices, norms of another shape, positions of
    more channels than a head has; what goes with such rows alone, and what does not."""
    D, F, L = 256, 512, 6
    u8 = torch.uint8
    w = lambda n, k: api.Fp4Rows(on(n, (k + 255) // 256 * 128, dtype=u8), on(n, (k + 511) // 512 * 16, dtype=u8), k)  # noqa: E731
    w8 = api.Int8Rows(on(D, D, dtype=torch.int8), on(D, dtype=torch.float32), D)
    p = {"wq": w(D, D), "wk": w(D, D), "wv": w(D, D), "wo": w(D, D), "w1": w(F, D), "w2": w(D, F),
         "bq": on(D), "bk": on(D), "bv": on(D), "bo": on(D), "b1": on(F), "b2": on(D), "mod": on(6, D, dtype=torch.float32)}
    x, idx, y = on(L, D), on(L, dtype=torch.int32), on(L, D, dtype=torch.float32)
    f = lambda *s: on(*s, dtype=torch.float32)  # noqa: E731
    assert api.is_fp4_block(p) and not api.is_int8_block(p)
    for kw in (dict(y_sel=on(L, D)), dict(y_sel=y[:3]), dict(idx=idx[:3]), dict(wk=w8), dict(wk=on(D, D)), dict(w1=w(F, F)), dict(w2=w(D, D)),
               dict(after1=f(D - 1)), dict(after2=f(1, D)), dict(after2=on(D)), dict(mod=f(5, D)),
               dict(rotary=api.Rotary(on(D, dtype=torch.float64))), dict(rotary=1.0)):
        q = {**p, **{n: t for n, t in kw.items() if n in p or n.startswith("after")}}
        with pytest.raises((ValueError, TypeError), match=next(iter(kw))):
            api.block_partial(q, x, kw.get("idx", idx), 4, 2, y_sel=kw.get("y_sel", y), rotary=kw.get("rotary"))
    with pytest.raises(ValueError, match="batch_invariant"):
        api.block_partial(p, x, idx, 4, 2, batch_invariant=True)
    with pytest.raises(ValueError, match="4"):
        api.wan_block_partial(p, None, None, None, [0], 1, (1, 1, 1))
    for n_sel, H in ((-1, 2), (2, 0)):
        with pytest.raises(RuntimeError, match="echo_block_partial"):
            api.block_partial(p, x, idx, n_sel, H)
    with pytest.raises(ValueError, match="bits"):
        api.quantize_block({}, bits=2)
    bf = {n: on(2, 2) for n in p}
    for kw in (dict(rotary=api.Rotary(on(1, dtype=torch.float64))), dict()):
        with pytest.raises(ValueError, match="8 or 4 bits"):
            api.block_partial(bf if kw else {**bf, "after1": f(2)}, x, idx, 4, 2, **kw)
