"""Refusals of the 8-bit rows, the 8-bit linear layer and the cross attention,
on the CPU: the C ABI rejects bad arguments before any HIP call, sizes its
workspaces as pure functions and takes empty calls as done; the binding
rejects what the ABI cannot see (host tensors, shapes, types)."""
import ctypes

import pytest
import torch

from paper_2608_02474_amd import _lib, api

FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10001)
OFF4 = ctypes.c_void_p(0x10004)
BF, F32 = _lib.ECHO_BF16, _lib.ECHO_F32
OK, EINVAL, EUNSUP, EWS = _lib.ECHO_OK, _lib.ECHO_EINVAL, _lib.ECHO_EUNSUPPORTED, _lib.ECHO_EWORKSPACE


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_pitch(lib):
    assert [lib.echo_int8_pitch(d) for d in (1, 128, 129, 5120, 65536)] == [128, 128, 256, 5120, 65536]
    assert [lib.echo_int8_pitch(d) for d in (0, -1, 65537)] == [0, 0, 0]


def test_quantize_rejects_before_launch(lib):
    def run(M=4, D=64, dt=BF, nx=4, ldx=64, ldq=128, eps=1e-6, x=FAKE, rows=None, sh=None, sc=None, q=FAKE, s=FAKE):
        cfg = _lib.QuantizeCfg(M, D, dt, nx, ldx, ldq, eps)
        return lib.echo_quantize_rows(ctypes.byref(cfg), x, rows, sh, sc, q, s, None)
    for bad in (dict(M=-1), dict(D=0), dict(D=65537, ldx=65537), dict(dt=2), dict(ldx=63), dict(ldq=64),
                dict(ldq=192), dict(ldq=65536 + 128), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(x=ODD),
                dict(q=None), dict(q=OFF4), dict(s=None), dict(s=ODD), dict(nx=3), dict(rows=FAKE, nx=0),
                dict(rows=ODD), dict(sh=FAKE), dict(sc=FAKE), dict(sh=OFF4, sc=FAKE)):
        assert run(**bad) == EINVAL, bad
    assert lib.echo_quantize_rows(None, FAKE, None, None, None, FAKE, FAKE, None) == EINVAL
    assert run(M=0, x=None, q=None, s=None) == OK


def test_dequantize_rejects_before_launch(lib):
    def run(M=4, D=64, dt=BF, ldx=64, ldq=128, x=FAKE, q=FAKE, s=FAKE):
        cfg = _lib.QuantizeCfg(M, D, dt, 0, ldx, ldq, 0.0)
        return lib.echo_dequantize_rows(ctypes.byref(cfg), q, s, x, None)
    for bad in (dict(M=-1), dict(D=0), dict(dt=-1), dict(ldx=63), dict(ldq=127), dict(x=None), dict(x=ODD), dict(q=OFF4),
                dict(s=None)):
        assert run(**bad) == EINVAL, bad
    assert run(M=0, x=None, q=None, s=None) == OK


def _linear(M=100, N=70, K=64, epi=0, od=BF, bd=BF, rd=BF, nres=100, lda=128, ldw=128, ldc=70, ldr=70):
    return _lib.LinearInt8Cfg(M, N, K, epi, od, bd, rd, nres, lda, ldw, ldc, ldr)


def test_linear_rejects_before_launch(lib):
    def run(a=FAKE, sa=FAKE, w=FAKE, sw=FAKE, b=FAKE, g=None, r=None, rr=None, c=FAKE, ws=FAKE, n=1 << 40, **kw):
        return lib.echo_linear_int8(ctypes.byref(_linear(**kw)), a, sa, w, sw, b, g, r, rr, c, ws, n, None)
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(K=65537, lda=1 << 17, ldw=1 << 17), dict(epi=3), dict(epi=-1),
                dict(od=2), dict(bd=2), dict(rd=2), dict(lda=64), dict(lda=192), dict(ldw=64), dict(ldc=69),
                dict(a=None), dict(a=OFF4), dict(sa=None), dict(sa=ODD), dict(w=OFF4), dict(sw=None), dict(b=ODD),
                dict(c=None), dict(c=ODD), dict(g=FAKE), dict(r=FAKE), dict(rr=FAKE),
                dict(epi=2), dict(epi=2, g=FAKE), dict(epi=2, g=FAKE, r=FAKE, ldr=69),
                dict(epi=2, g=FAKE, r=FAKE, nres=99), dict(epi=2, g=FAKE, r=FAKE, rr=FAKE, nres=0)):
        assert run(**bad) == EINVAL, bad
    assert lib.echo_linear_int8(None, *[FAKE] * 9, FAKE, 0, None) == EINVAL
    assert run(N=(1 << 22) + 1, ldc=1 << 23) == EUNSUP
    assert run(M=1 << 30, N=1 << 22, ldc=1 << 22) == EUNSUP
    assert run(M=0, a=None, c=None, ws=None, n=0) == OK
    for kw in (dict(), dict(M=70, N=64, K=40000, lda=40064, ldw=40064), dict(M=2000, N=5120, K=5120, lda=5120, ldw=5120, ldc=5120)):
        need = lib.echo_linear_int8_workspace(ctypes.byref(_linear(**kw)))
        if need:
            assert run(ws=None, **kw) == EWS and run(n=need - 1, **kw) == EWS and run(ws=OFF4, **kw) == EWS
    assert lib.echo_linear_int8_workspace(ctypes.byref(_linear(K=0))) == 0


def _cross(B=2, Lq=8, Lk=16, H=4, Hkv=2, dh=64, dt=BF, scale=0.125, q=None, k=None, v=None, o=None):
    S = _lib.Strides
    return _lib.CrossAttentionCfg(B, Lq, Lk, H, Hkv, dh, dt, scale, q or S(Lq * H * dh, H * dh, dh),
                                  k or S(Lk * Hkv * dh, Hkv * dh, dh), v or S(Lk * Hkv * dh, Hkv * dh, dh),
                                  o or S(Lq * H * dh, H * dh, dh))


def test_cross_rejects_before_launch(lib):
    S = _lib.Strides
    def run(q=FAKE, k=FAKE, v=FAKE, n=None, m=None, o=FAKE, ws=FAKE, nb=1 << 40, **kw):
        return lib.echo_cross_attention(ctypes.byref(_cross(**kw)), q, k, v, n, m, o, ws, nb, None)
    bad_cfg = (dict(B=-1), dict(Lq=-1), dict(Lk=-1), dict(H=0), dict(Hkv=0), dict(H=3), dict(dh=0), dict(dt=2),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")))
    for bad in bad_cfg:
        assert lib.echo_cross_attention(ctypes.byref(_cross(**bad)), *[FAKE] * 6, FAKE, 1 << 40, None) == EINVAL, bad
        assert lib.echo_cross_attention_workspace(ctypes.byref(_cross(**bad)), 1) == 0
    for t in "qkvo":
        for s in (S(-8, 256, 64), S(2048, 252, 64), S(2048, 256, 63)):
            cfg = _cross(**{t: s})
            assert lib.echo_cross_attention(ctypes.byref(cfg), *[FAKE] * 6, FAKE, 1 << 40, None) == EINVAL
    assert lib.echo_cross_attention(None, *[FAKE] * 6, FAKE, 0, None) == EINVAL
    for bad in (dict(q=None), dict(q=OFF4), dict(k=None), dict(v=OFF4), dict(o=None), dict(n=ODD)):
        assert run(**bad) == EINVAL, bad
    for bad in (dict(dh=32), dict(dh=96), dict(dh=256), dict(dt=F32, dh=132), dict(scale=3e38),
                dict(B=1 << 24, Hkv=1, H=1), dict(Lq=1 << 30, H=4, Hkv=1)):
        assert run(**bad) == EUNSUP, bad
    for t in "kv":
        far = _cross(**{t: S(1 << 30, 1 << 24, 64)})
        assert lib.echo_cross_attention(ctypes.byref(far), *[FAKE] * 6, FAKE, 1 << 40, None) == EUNSUP
    odd = _cross(dt=F32, dh=6, q=S(192, 24, 8), k=S(192, 24, 8), v=S(192, 24, 8), o=S(192, 24, 8))
    assert lib.echo_cross_attention(ctypes.byref(odd), *[FAKE] * 6, FAKE, 1 << 40, None) == EUNSUP
    assert run(B=0, q=None, o=None, ws=None, nb=0) == OK
    assert run(Lq=0, q=None, o=None) == OK
    need = lib.echo_cross_attention_workspace(ctypes.byref(_cross()), 1)
    assert need >= 2 * 16 * 4 + 2 * 4
    assert run(m=FAKE, ws=None) == EWS and run(m=FAKE, nb=need - 1) == EWS and run(m=FAKE, ws=OFF4) == EWS


def test_binding_rejects_host_tensors_shapes_and_types():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device tensor"):
        api.quantize_rows(x)
    with pytest.raises(TypeError):
        api.quantize_rows("x")
    with pytest.raises(TypeError, match="Int8Rows"):
        api.dequantize_rows(x)
    with pytest.raises(TypeError, match="Int8Rows"):
        api.linear_int8(x, x)
    with pytest.raises(ValueError, match="device tensor"):
        api.linear_int8(api.Int8Rows(torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4), 64), None)
    q = torch.zeros(1, 2, 2, 64)
    with pytest.raises(ValueError, match="device tensor"):
        api.cross_attention(q, q, q)
    with pytest.raises(TypeError):
        api.cross_attention(None, q, q)


def test_int8_block_weights_are_told_from_others():
    w = api.Int8Rows(torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4), 64)
    assert api.is_int8_block({"wq": w}) and not api.is_int8_block({"wq": torch.zeros(4, 64)})
    with pytest.raises(ValueError, match="batch_invariant"):
        api.block_partial({"wq": w}, None, None, 0, 1, batch_invariant=True)
    with pytest.raises(ValueError, match="8 bits"):
        api.wan_block_partial({"wq": w}, None, None, None, [0], 1, (1, 1, 1))


@pytest.mark.parametrize("n_sel,H", [(-1, 1), (2, 0)])
def test_int8_block_refuses_counts_as_the_block_does(lib, n_sel, H):
    """A negative count is no slice that leaves the last tokens out."""
    w = api.Int8Rows(torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4), 64)
    with pytest.raises(RuntimeError, match="echo_block_partial"):
        api.block_partial({"wq": w}, None, None, n_sel, H)


@pytest.mark.parametrize("dt,dh", [(BF, 64), (BF, 128), (F32, 32)])
def test_cross_refuses_states_whose_numbers_overflow(lib, dt, dh):
    """Tiles are counted, and states past the last one numbered, in 32 bits: 2^31 - 128
    states are the most, with state strides of 0 no large tensor is needed for more."""
    S = _lib.Strides
    def cfg(Lk):
        return _cross(B=1, Lq=1, Lk=Lk, H=1, Hkv=1, dh=dh, dt=dt, k=S(0, 0, 0), v=S(0, 0, 0))
    most = 2 ** 31 - 128
    assert lib.echo_cross_attention_workspace(ctypes.byref(cfg(most)), 0) > 0      # split over the states
    assert lib.echo_cross_attention_workspace(ctypes.byref(cfg(most)), 1) > 4 * most
    for Lk in (most + 1, 2 ** 31 - 64, 2 ** 31 - 1):
        assert lib.echo_cross_attention_workspace(ctypes.byref(cfg(Lk)), 0) == 0
        assert lib.echo_cross_attention(ctypes.byref(cfg(Lk)), *[FAKE] * 6, FAKE, 1 << 40, None) == EUNSUP


class _AsOnDevice(torch.Tensor):
    """A host tensor that says it is on the device: the checks of a call run as for
    one that is, and nothing is launched."""
    is_cuda = property(lambda self: True)

    @staticmethod
    def of(*shape, dtype=torch.bfloat16):
        """Of any size, in the memory of one row."""
        return torch.zeros(shape[-1], dtype=dtype).expand(*shape).as_subclass(_AsOnDevice)


def test_binding_refuses_counts_that_32_bits_would_wrap():
    """2^32 + 5 states are not 5."""
    n = 2 ** 32 + 5
    q = _AsOnDevice.of(1, 2, 1, 64)
    few, many = _AsOnDevice.of(1, 5, 1, 64), _AsOnDevice.of(1, n, 1, 64)
    with pytest.raises(ValueError, match=r"2\^31"):
        api.cross_attention(q, many, many)
    with pytest.raises(ValueError, match=r"2\^31"):
        api.cross_attention(many, few, few)
    with pytest.raises(ValueError, match=r"2\^31"):
        api.cross_attention(_AsOnDevice.of(n, 1, 1, 64), _AsOnDevice.of(n, 5, 1, 64), _AsOnDevice.of(n, 5, 1, 64))
    # rows of one value each, `n` of them (a view of host memory that is never touched)
    x = torch.zeros(1, dtype=torch.bfloat16).as_strided((1, 1), (1, 1)).expand(n, 1).as_subclass(_AsOnDevice)
    with pytest.raises(ValueError, match=r"2\^31"):
        api.quantize_rows(x)
    with pytest.raises(ValueError, match=r"2\^31"):
        api.quantize_rows(x, rows=_AsOnDevice.of(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="2.31"):
        api.dequantize_rows(api.Int8Rows(_AsOnDevice.of(4, 128, dtype=torch.int8).contiguous().as_subclass(_AsOnDevice),
                                         torch.zeros(4).as_subclass(_AsOnDevice), 1), out=x)
    # as many 8-bit rows (the usual case of a pitch that is the width)
    rows = torch.empty((n, 128), dtype=torch.int8, device="meta").as_subclass(_AsOnDevice)
    wide = api.Int8Rows(rows, torch.empty(n, device="meta").as_subclass(_AsOnDevice), 64)
    with pytest.raises(ValueError, match="2.31"):
        api.linear_int8(wide, wide)


def test_int8_block_refuses_before_any_launch():
    """An output of another type, width or too few rows, too few indices, matrices that
    are no codes or of other shapes."""
    D, F, L = 128, 256, 6
    on = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt).as_subclass(_AsOnDevice)  # noqa: E731
    w = lambda n, k: api.Int8Rows(on(n, k, dt=torch.int8), on(n, dt=torch.float32), k)  # noqa: E731
    p = {"wq": w(D, D), "wk": w(D, D), "wv": w(D, D), "wo": w(D, D), "w1": w(F, D), "w2": w(D, F),
         "bq": on(D), "bk": on(D), "bv": on(D), "bo": on(D), "b1": on(F), "b2": on(D), "mod": on(6, D, dt=torch.float32)}
    x, idx = on(L, D), on(L, dt=torch.int32)
    y = on(L, D, dt=torch.float32)
    for kw in (dict(y_sel=on(L, D)), dict(y_sel=y[:, :64]), dict(y_sel=y[:3]), dict(idx=idx[:3]), dict(idx=on(L, 1, dt=torch.int32)),
               dict(idx=on(L, dt=torch.int64)), dict(wk=on(D, D)), dict(w1=w(F, F)), dict(w2=w(D, D)), dict(wo=w(F, D))):
        q = {**p, **{n: t for n, t in kw.items() if n in p}}
        with pytest.raises((ValueError, TypeError), match=next(iter(kw))):
            api.block_partial(q, x, kw.get("idx", idx), 4, 1, y_sel=kw.get("y_sel", y))


def test_workspace_pieces():
    """Pieces lie apart at multiples of 256 bytes, stay for the same key, and are laid
    out again for another one and where the buffer has grown under them."""
    ws, cpu = api.Workspace(), torch.device("cpu")
    specs = (((3, 5), torch.float32), ((7,), torch.int8), ((1, 2, 3), torch.bfloat16), ((300,), torch.uint8))
    calls = []
    lay = lambda key: ws.pieces(key, lambda: calls.append(key) or specs, cpu)  # noqa: E731
    one = lay("a")
    assert [(tuple(t.shape), t.dtype) for t in one] == list(specs)
    starts = [t.data_ptr() - ws.buf.data_ptr() for t in one]
    assert starts == [0, 256, 512, 768] and ws.buf.numel() == 768 + 512
    assert lay("a") is one and calls == ["a"]
    two = lay("b")
    assert two is not one and [t.data_ptr() for t in two] == [t.data_ptr() for t in one]   # the same buffer
    ws.get(1 << 20, cpu)
    three = lay("b")
    assert calls == ["a", "b", "b"] and three[0].data_ptr() == ws.buf.data_ptr()


def test_pitch_of_a_single_row_is_its_width():
    """One row of codes taken from far apart ones has a stride that no next row needs;
    of more rows it is their pitch, at most 65536."""
    codes = torch.zeros(400, 512, dtype=torch.int8).as_subclass(_AsOnDevice)
    scale = torch.zeros(400).as_subclass(_AsOnDevice)
    one, far = codes[7::300][:1], codes[::200]
    assert one.stride(0) == 300 * 512
    assert api._int8_rows(api.Int8Rows(one, scale[:1], 400), "a") == (1, 512)
    assert api._int8_rows(api.Int8Rows(codes[::2], scale[:200], 400), "a") == (200, 1024)
    with pytest.raises(ValueError, match="65536"):
        api._int8_rows(api.Int8Rows(far, scale[:2], 400), "a")
