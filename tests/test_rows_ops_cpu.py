"""Refusals of the entry points of the norm, dropout and the 8-bit integers, through the C ABI and the binding: every bad
argument is turned into a status before anything is enqueued (no GPU here).  And the tests' own generator against
the published answers."""
import ctypes

import pytest

from rows_reference import philox


def lib():
    from paper_2301_06284_amd import rgnn
    return rgnn, rgnn.lib()


P = 0x10000     # an address that no check dereferences


class Drop(ctypes.Structure):
    _fields_ = [("rng", ctypes.c_void_p), ("call", ctypes.c_int64), ("p", ctypes.c_double)]


def fields(pointers, sizes, tail, ints):
    """A structure's fields in the header's order."""
    return [(n, ctypes.c_void_p) for n in pointers.split()] + [(n, ctypes.c_int64) for n in sizes.split()] + tail + \
        [(n, ctypes.c_int32) for n in ints.split()]


class DropoutRows(ctypes.Structure):
    _fields_ = fields("X res Y", "rows ldx ldr ldy", [("drop", Drop)], "cols dtype y_dtype")


class Norm(ctypes.Structure):
    _fields_ = fields("X res sum w Y scales rstd", "rows ldx ldr lds ldy", [("eps", ctypes.c_double), ("drop", Drop)],
                      "cols dtype sum_dtype w_dtype y_dtype")


class NormBackward(ctypes.Structure):
    _fields_ = fields("dY sum rstd w dsum dres dX dW ws", "rows lddy lds ldds lddr lddx ws_bytes", [("drop", Drop)],
                      "cols dy_dtype sum_dtype w_dtype dx_dtype dw_dtype")


def drop(p=0.5, rng=P, call=0):
    return Drop(rng, call, p)


def call(function, structure, a, kw):
    assert set(kw) <= set(a)
    a.update(kw)
    a["drop"] = a["drop"] or Drop()
    return function(bytes(structure(**a)), None)


@pytest.mark.parametrize("counter,key,answer", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator(counter, key, answer):
    """The known answers that were published with the generator."""
    assert tuple(int(x) for x in philox(*counter, *key)) == answer


def norm(**kw):
    _, l = lib()
    a = dict(dtype=1, X=P, rows=10, ldx=64, cols=64, drop=None, sum_dtype=1, res=P, ldr=64, sum=P, lds=64, w_dtype=1, w=P,
             eps=1e-6, y_dtype=1, Y=P, ldy=64, scales=None, rstd=None)
    return call(l.rgnn_rms_norm, Norm, a, kw)


def dropout(**kw):
    _, l = lib()
    a = dict(dtype=1, X=P, rows=4, ldx=64, cols=64, drop=drop(), y_dtype=1, res=P, ldr=64, Y=P, ldy=64)
    return call(l.rgnn_dropout, DropoutRows, a, kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), -1), (dict(dtype=4), -1), (dict(sum_dtype=3), -1), (dict(w_dtype=5), -1), (dict(y_dtype=5), -1),
    (dict(y_dtype=-1), -1), (dict(dtype=2), -1), (dict(w_dtype=2), -1), (dict(y_dtype=2), -1), (dict(sum_dtype=2), -1),
    (dict(rows=-1), -1), (dict(cols=0), -1), (dict(cols=2 ** 24 + 1, ldx=2 ** 25), -2), (dict(rows=2 ** 31 - 1), -2),
    (dict(X=None), -1), (dict(Y=None), -1), (dict(X=P + 1), -1), (dict(Y=P + 1), -1), (dict(res=P + 1), -1),
    (dict(sum=P + 1), -1), (dict(sum_dtype=0, sum=P + 2), -1), (dict(w=P + 1), -1), (dict(rstd=P + 2), -1),
    (dict(ldx=63), -1), (dict(ldr=63), -1), (dict(lds=63), -1), (dict(ldy=63), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(y_dtype=3), -1), (dict(y_dtype=4), -1),
    (dict(y_dtype=3, scales=P, Y=P + 8), -1), (dict(y_dtype=4, scales=P + 2), -1),
])
def test_norm_refusals(kw, status):
    _, l = lib()
    assert norm(**kw) == status
    assert l.rgnn_last_error()


@pytest.mark.parametrize("kw", [dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(rng=P + 4)])
def test_dropout_arguments_are_refused(kw):
    assert norm(drop=drop(**kw)) == -1
    assert dropout(drop=drop(**kw)) == -1
    assert backward(drop=drop(**kw)) == -1


def test_no_rows_are_ok():
    _, l = lib()
    assert norm(rows=0, X=None, Y=None, res=None, sum=None) == 0
    assert dropout(rows=0, X=None, Y=None, res=None) == 0
    assert l.rgnn_int8_quantize_rows(1, None, 0, 64, 64, None, None, None) == 0
    assert backward(rows=0, dW=None, dY=None, sum=None, rstd=None) == 0
    assert backward(dW=None, dX=None, dres=None) == 0            # nothing wanted


def backward(**kw):
    rgnn, l = lib()
    a = dict(dy_dtype=1, dY=P, rows=10, lddy=64, cols=64, sum_dtype=1, sum=P, lds=64, rstd=P, w_dtype=1, w=P, dsum=P, ldds=64,
             drop=None, dres=P, lddr=64, dx_dtype=1, dX=P, lddx=64, dw_dtype=1, dW=P, ws=P, ws_bytes=1 << 20)
    return call(l.rgnn_rms_norm_backward, NormBackward, a, kw)


@pytest.mark.parametrize("kw,status", [
    (dict(dy_dtype=3), -1), (dict(sum_dtype=4), -1), (dict(w_dtype=7), -1), (dict(dx_dtype=3), -1), (dict(dw_dtype=-2), -1),
    (dict(dy_dtype=2), -1), (dict(dx_dtype=2), -1), (dict(dw_dtype=2), -1), (dict(rows=-1), -1), (dict(cols=0), -1),
    (dict(rows=2 ** 31 - 1), -2), (dict(cols=2 ** 24 + 1, lddy=2 ** 25), -2), (dict(dY=None), -1), (dict(sum=None), -1),
    (dict(rstd=None), -1), (dict(rstd=P + 2), -1), (dict(w=P + 1), -1), (dict(dsum=P + 1), -1), (dict(dres=P + 1), -1),
    (dict(dX=P + 1), -1), (dict(dW=P + 1), -1), (dict(dw_dtype=0, dW=P + 2), -1), (dict(lddy=63), -1), (dict(lds=63), -1),
    (dict(ldds=63), -1), (dict(lddr=63), -1), (dict(lddx=63), -1), (dict(ws=None), -1), (dict(ws_bytes=16), -1),
    (dict(ws=P + 4), -1),
])
def test_norm_backward_refusals(kw, status):
    assert backward(**kw) == status


def test_backward_workspace_size():
    """Grows with the rows, so that one sized for the most rows serves fewer."""
    rgnn, l = lib()
    rows = [0, 1, 3, 4, 5, 31, 32, 33, 1000, 4096, 10007, 32768, 100000, 10 ** 6, 2 ** 31 - 2]
    for cols in (1, 8, 64, 65, 333, 1024, 2048, 5000, 16384, 40000, 2 ** 24):
        sizes = [rgnn.rms_norm_backward_workspace_size(r, cols) for r in rows]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] >= 4 * cols
        assert sizes[-1] < 2 ** 36
    assert l.rgnn_rms_norm_backward_workspace_size(4, 4, None) == -1
    for bad in ((-1, 4), (4, 0), (2 ** 31 - 1, 4), (4, 2 ** 24 + 1)):
        with pytest.raises(rgnn.RgnnError):
            rgnn.rms_norm_backward_workspace_size(*bad)


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(y_dtype=4), dict(dtype=2), dict(rows=-1), dict(cols=0), dict(X=None),
                                dict(Y=None), dict(X=P + 1), dict(Y=P + 1), dict(res=P + 1), dict(ldx=63), dict(ldy=63),
                                dict(ldr=63)])
def test_dropout_refusals(kw):
    assert dropout(**kw) == -1


def test_no_arguments_are_refused():
    _, l = lib()
    assert l.rgnn_dropout(None, None) == l.rgnn_rms_norm(None, None) == l.rgnn_rms_norm_backward(None, None) == -1


def test_packed_arguments_are_the_structures():
    rgnn, _ = lib()
    assert rgnn._DROPOUT_PACK(*range(1, 9), -9, 0.5, 11, 12, 13) == bytes(DropoutRows(1, 2, 3, 4, 5, 6, 7, Drop(8, -9, 0.5), 11, 12, 13))
    assert rgnn._NORM_PACK(*range(1, 13), 0.25, 14, -15, 0.5, 17, 18, 19, 20, 21) == bytes(
        Norm(*range(1, 13), 0.25, Drop(14, -15, 0.5), 17, 18, 19, 20, 21))
    assert rgnn._NORM_BACKWARD_PACK(*range(1, 18), -18, 0.5, *range(20, 26)) == bytes(
        NormBackward(*range(1, 17), Drop(17, -18, 0.5), *range(20, 26)))


@pytest.mark.parametrize("args", [
    (3, P, 4, 64, 64, P, P, None), (4, P, 4, 64, 64, P, P, None), (1, None, 4, 64, 64, P, P, None), (1, P, 4, 63, 64, P, P, None),
    (1, P, 4, 64, 0, P, P, None), (1, P, -1, 64, 64, P, P, None), (1, P, 4, 64, 64, P + 8, P, None),
    (1, P, 4, 64, 64, P, P + 2, None), (1, P, 4, 64, 64, None, P, None), (1, P, 4, 64, 64, P, None, None),
    (1, P + 1, 4, 64, 64, P, P, None),
])
def test_int8_rows_refusals(args):
    _, l = lib()
    assert l.rgnn_int8_quantize_rows(*args) == -1


@pytest.mark.parametrize("args", [
    (3, P, 4, 64, 64, P, P, None), (1, None, 4, 64, 64, P, P, None), (1, P, 0, 64, 64, P, P, None), (1, P, 4, 0, 64, P, P, None),
    (1, P, 4, 64, 64, P + 8, P, None), (1, P, 4, 64, 64, P, None, None), (0, P + 2, 4, 64, 64, P, P, None),
    (1, P, 4, 64, 64, P, P + 2, None),
])
def test_int8_weights_refusals(args):
    _, l = lib()
    assert l.rgnn_int8_quantize_weights(*args) == -1


@pytest.mark.parametrize("kw,status", [
    (dict(X=P + 8), -1), (dict(xs=P + 2), -1), (dict(W=P + 8), -1), (dict(ws=P + 1), -1), (dict(xs=None), -1), (dict(ws=None), -1),
    (dict(W=None), -1), (dict(Y=None), -1), (dict(ptr=None), -1), (dict(y_dtype=3), -1), (dict(y_dtype=4), -1),
    (dict(x_rows=9), -1), (dict(ldy=31), -1), (dict(T=0), -1), (dict(K=0), -1), (dict(K=130945), -2), (dict(T=65536), -2),
])
def test_int8_linear_refusals(kw, status):
    _, l = lib()
    a = dict(X=P, xs=P, x_rows=10, gather=None, ptr=P, T=3, M=10, W=P, ws=P, K=64, N=32, y_dtype=1, Y=P, y_rows=10, ldy=32,
             scatter=None, stream=None)
    a.update(kw)
    assert l.rgnn_typed_linear_int8(*a.values()) == status


def test_wrappers_refuse_cpu_tensors_and_bad_shapes():
    import torch
    rgnn, _ = lib()
    x, w = torch.zeros(4, 64), torch.ones(64)
    rng = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        rgnn.rms_norm(x, w, torch.empty_like(x))
    with pytest.raises(ValueError):
        rgnn.rms_norm_backward(x, x, torch.ones(4), w, dX=torch.empty_like(x))
    with pytest.raises(ValueError):
        rgnn.dropout(x, torch.empty_like(x), rgnn.Dropout(0.5, rng))
    with pytest.raises(ValueError):
        rgnn.int8_quantize_rows(x)
    with pytest.raises(ValueError):
        rgnn.int8_quantize_weights(torch.zeros(1, 64, 64))
    for bad in (torch.zeros(2), torch.zeros(3, dtype=torch.int64), torch.zeros(2, 2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            rgnn.Dropout(0.5, bad)
    for p in (-0.5, 1.01, float("nan")):
        with pytest.raises(ValueError):
            rgnn.Dropout(p, rng)


@pytest.mark.parametrize("change", [
    dict(Y=(4, 63, "f")), dict(Y=(3, 64, "f")), dict(residual=(4, 65, "f")), dict(sum=(4, 64, "h"), residual=(4, 64, "f")),
    dict(weight=(63,)), dict(rstd=(5,)), dict(Y=(4, 64, "i")), dict(Y=(4, 128, "i"), scales=(5,)), dict(scales=(4,)),
    dict(Y=(4, 64, "8"), scales=(4,)),
])
def test_norm_wrapper_checks_shapes(change, monkeypatch):
    """Shapes, types and strides are checked before the library is called (devices apart, which a CPU tensor fails first)."""
    import torch
    rgnn, _ = lib()
    monkeypatch.setattr(rgnn, "_device_of", lambda t, _: t.get_device())
    monkeypatch.setattr(rgnn, "_stream_of", lambda *t: None)
    kinds = {"f": torch.float32, "h": torch.bfloat16, "i": torch.int8, "8": torch.float8_e4m3fn}

    def make(spec):
        return torch.zeros(spec[:-1], dtype=kinds[spec[-1]]) if isinstance(spec[-1], str) else torch.zeros(spec)
    args = dict(X=torch.zeros(4, 64), weight=torch.ones(64), Y=torch.zeros(4, 64))
    args.update({k: make(v) for k, v in change.items()})
    with pytest.raises((ValueError, rgnn.RgnnError)):
        rgnn.rms_norm(**args)


def test_other_devices_are_refused():
    """A stream of another device than the tensors', and tensors of another device than the current one."""
    rgnn, _ = lib()

    class Stream:
        device_index, cuda_stream = 1, 0

    class Tensor:
        device = 0

        def get_device(self):
            return self.device

    class Torch:
        raw_stream = None

        @staticmethod
        def current():
            return 0
    with pytest.raises(ValueError):
        rgnn._stream_of(Stream(), 0, Torch)
    x = Tensor()
    assert rgnn._device_of(x, Torch) == 0
    for x.device in (1, -1):
        with pytest.raises(ValueError):
            rgnn._device_of(x, Torch)


def test_tile_of_int8():
    """The 8-bit forms share their tiles."""
    rgnn, l = lib()
    for rows, types, K, N in ((16, 32, 2048, 1536), (8192, 1, 4096, 4096), (300, 4, 128, 64)):
        got = []
        for dtype in (rgnn.F8_E4M3, rgnn.I8):
            t = rgnn.Tile()
            assert l.rgnn_typed_linear_select_tile(dtype, P, rows, K, None, types, rows, P, K, N, 1, ctypes.byref(t)) == 0
            got.append((t.rows, t.cols, t.stages, t.any))
        assert got[0] == got[1]


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(sum_dtype=3)])
def test_messages_name_the_arguments_as_documented(kw):
    _, l = lib()
    assert norm(**kw) == -1
    assert l.rgnn_last_error() == b"X and sum must be fp32, bf16 or fp16"
