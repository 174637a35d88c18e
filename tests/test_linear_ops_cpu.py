"""Refusals of the typed linear's and AdamW's entry points, through the C ABI: every bad
argument is turned into a status before anything is enqueued (no GPU here)."""
import ctypes

import pytest


def lib():
    from paper_2301_06284_amd import rgnn
    return rgnn, rgnn.lib()


P = 0x10000     # an address that no check dereferences


def linear(**kw):
    rgnn, l = lib()
    a = dict(dtype=1, X=P, x_rows=10, ldx=64, gather=None, ptr=P, T=3, M=10, W=P, K=64, N=32, trans=0, y_dtype=1, Y=P,
             y_rows=10, ldy=32, scatter=None, stream=None)
    assert set(kw) <= set(a)
    a.update(kw)
    return l.rgnn_typed_linear(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(dtype=9), -1), (dict(y_dtype=2), -1), (dict(trans=2), -1),
    (dict(T=0), -1), (dict(T=65536), -2), (dict(M=-1), -1), (dict(K=0), -1), (dict(N=-4), -1),
    (dict(M=2 ** 31 - 1, x_rows=2 ** 31 - 2, gather=P, scatter=P), -2), (dict(K=2 ** 24 + 1, ldx=2 ** 25), -2),
    (dict(X=None), -1), (dict(W=None), -1), (dict(Y=None), -1), (dict(ptr=None), -1), (dict(X=P + 1), -1),
    (dict(W=P + 1), -1), (dict(Y=P + 1), -1), (dict(y_dtype=0, Y=P + 2), -1), (dict(ldx=63), -1), (dict(ldy=31), -1),
    (dict(x_rows=9), -1), (dict(y_rows=9), -1), (dict(x_rows=-1, gather=P), -2), (dict(y_rows=2 ** 31, scatter=P), -2),
])
def test_linear_refusals(kw, status):
    rgnn, l = lib()
    assert linear(**kw) == status
    assert l.rgnn_last_error()


def test_linear_without_positions_is_ok():
    assert linear(M=0, x_rows=0, y_rows=0, X=None, Y=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), -1), (dict(dw_dtype=2), -1), (dict(T=0), -1), (dict(K=0), -1), (dict(ldx=63), -1), (dict(lddy=31), -1),
    (dict(X=None), -1), (dict(dY=None), -1), (dict(dW=None), -1), (dict(ptr=None), -1), (dict(dW=P + 1), -1),
    (dict(x_rows=99999), -1), (dict(dy_rows=5), -1), (dict(ws=None), -1), (dict(ws_bytes=100), -1), (dict(ws=P + 4), -1),
])
def test_wgrad_refusals(kw, status):
    rgnn, l = lib()
    import torch
    need = rgnn.typed_linear_wgrad_workspace_size(torch.bfloat16, 100000, 3, 64, 32)
    assert need > 100
    a = dict(dtype=1, X=P, x_rows=100000, ldx=64, gather=None, dY=P, dy_rows=100000, lddy=32, dyg=None, ptr=P, T=3,
             M=100000, K=64, N=32, dw_dtype=1, dW=P, ws=P, ws_bytes=need, stream=None)
    a.update(kw)
    assert l.rgnn_typed_linear_wgrad(*a.values()) == status


def test_wgrad_workspace_size():
    """Grows with the rows, so that one sized for the most rows serves fewer."""
    rgnn, l = lib()
    import torch
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        for T, K, N in ((1, 64, 64), (96, 64, 128), (32, 2048, 1536), (7, 100, 77), (1, 300, 40)):
            rows = [0, 1, 63, 1000, 1024, 1025, 2047, 2048, 4096, 5000, 8191, 8192, 16384, 100000, 300007, 1000003, 5000000]
            sizes = [rgnn.typed_linear_wgrad_workspace_size(dt, m, T, K, N) for m in rows]
            assert sizes == sorted(sizes)
            assert sizes[0] == 0
    with pytest.raises(rgnn.RgnnError):
        rgnn.typed_linear_wgrad_workspace_size(torch.float32, -1, 1, 64, 64)


@pytest.mark.parametrize("args", [
    (3, P, 4, 64, 64, P, P, None), (1, None, 4, 64, 64, P, P, None), (1, P, 4, 63, 64, P, P, None), (1, P, 4, 64, 0, P, P, None),
    (1, P, -1, 64, 64, P, P, None), (1, P, 4, 64, 64, P + 8, P, None), (1, P, 4, 64, 64, P, P + 2, None),
    (1, P, 4, 64, 64, None, P, None), (1, P, 4, 64, 64, P, None, None),
])
def test_fp8_rows_refusals(args):
    _, l = lib()
    assert l.rgnn_fp8_quantize_rows(*args) == -1


@pytest.mark.parametrize("args", [
    (3, P, 4, 64, 64, P, P, None), (1, None, 4, 64, 64, P, P, None), (1, P, 0, 64, 64, P, P, None), (1, P, 4, 0, 64, P, P, None),
    (1, P, 4, 64, 64, P + 8, P, None), (1, P, 4, 64, 64, P, None, None), (0, P + 2, 4, 64, 64, P, P, None),
])
def test_fp8_weights_refusals(args):
    _, l = lib()
    assert l.rgnn_fp8_quantize_weights(*args) == -1


@pytest.mark.parametrize("kw", [dict(X=P + 8), dict(xs=P + 4), dict(W=P + 8), dict(ws=P + 8), dict(xs=None), dict(ws=None),
                                dict(W=None), dict(Y=None), dict(ptr=None), dict(y_dtype=3), dict(x_rows=9), dict(ldy=31),
                                dict(T=0), dict(K=0)])
def test_fp8_linear_refusals(kw):
    _, l = lib()
    a = dict(X=P, xs=P, x_rows=10, gather=None, ptr=P, T=3, M=10, W=P, ws=P, K=64, N=32, y_dtype=1, Y=P, y_rows=10, ldy=32,
             scatter=None, stream=None)
    a.update(kw)
    assert l.rgnn_typed_linear_fp8(*a.values()) == -1


def adamw(entries, hyper=None, step=1, step_dev=None, count=None, tensors=True):
    rgnn, l = lib()
    arr = (rgnn.AdamwTensor * max(1, len(entries)))()
    for at, kw in zip(arr, entries):
        e = dict(param=P, grad=P, m=P, v=P, m_scale=None, v_scale=None, copy=None, n=10, param_dtype=0, grad_dtype=0,
                 copy_dtype=0, state_bits=32)
        e.update(kw)
        for k, x in e.items():
            setattr(at, k, x)
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    h.update(hyper or {})
    return l.rgnn_adamw_step(arr if tensors else None, len(entries) if count is None else count,
                             ctypes.byref(rgnn.AdamwHyper(*h.values())), step, step_dev, None, None)


@pytest.mark.parametrize("entry,status", [
    (dict(n=-1), -1), (dict(n=2 ** 40), -2), (dict(param=None), -1), (dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1),
    (dict(param_dtype=3), -1), (dict(grad_dtype=-1), -1), (dict(copy=P, copy_dtype=7), -1), (dict(state_bits=16), -1),
    (dict(state_bits=8), -1), (dict(state_bits=8, m_scale=P, v_scale=P + 2), -1), (dict(param=P + 2), -1),
    (dict(m=P + 2), -1), (dict(copy=P + 1, copy_dtype=1), -1),
])
def test_adamw_refuses_tensors(entry, status):
    assert adamw([dict(param=P + 4096), entry]) == status


@pytest.mark.parametrize("hyper", [dict(lr=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(beta1=1.0), dict(beta2=-0.1),
                                   dict(beta2=float("nan")), dict(weight_decay=float("inf"))])
def test_adamw_refuses_hyper_parameters(hyper):
    assert adamw([{}], hyper) == -1


def test_adamw_refuses_steps_and_lists():
    assert adamw([{}], step=0) == -1
    assert adamw([{}], step_dev=P + 4) == -1
    assert adamw([], count=-1) == -1
    assert adamw([{}], tensors=False) == -1
    assert adamw([dict(param=P), dict(param=P + 64), dict(param=P)]) == -1     # the same parameter twice
    assert adamw([]) == 0
    assert adamw([dict(n=0)], step=3) == 0


def test_wrappers_refuse_cpu_tensors_and_bad_shapes():
    import torch
    rgnn, _ = lib()
    x, w, y = torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(4, 8)
    ptr = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        rgnn.typed_linear(x, ptr, w, y)
    with pytest.raises(ValueError):
        rgnn.typed_linear_wgrad(x, y, ptr, w, None)
    with pytest.raises(ValueError):
        rgnn.fp8_quantize_rows(x)
    with pytest.raises(ValueError):
        rgnn.fp8_quantize_weights(w)
    with pytest.raises(ValueError):
        rgnn.AdamwTensors([x], [x], [x], [x])
    with pytest.raises(ValueError):
        rgnn.AdamwTensors([x], [x], [x], [])
    with pytest.raises(ValueError):
        rgnn._matrix(x.t(), "X", 4)
    with pytest.raises(ValueError):
        rgnn._matrix(x, "X", 7)
    assert rgnn._matrix(torch.zeros(9, 20)[:, 3:11], "X", 8)[1:] == (9, 20)
    assert rgnn.fp8_widths(1) == (128, 4) and rgnn.fp8_widths(513) == (640, 8)


def test_stream_of_another_device_is_refused():
    from paper_2301_06284_amd import rgnn

    class Stream:
        device_index, cuda_stream = 1, 64
    with pytest.raises(ValueError, match="stream is on device 1"):
        rgnn._stream_on(Stream(), 0)
    assert rgnn._stream_on(Stream(), 1).value == 64
    assert rgnn._stream_on(64, 0).value == 64


def test_adamw_refuses_tensors_whose_memory_has_moved(monkeypatch):
    """The addresses are kept from one step to the next: a tensor that has been given other memory
    is refused before anything is enqueued, and the list made again is taken."""
    import torch
    rgnn, _ = lib()

    class OnGpu(torch.Tensor):          # host memory that says it is on device 0: nothing is launched here
        def get_device(self):
            return 0

    class Library:
        calls = 0

        def rgnn_adamw_step(self, *args):
            Library.calls += 1
            return 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(rgnn, "_lib", Library())
    monkeypatch.setattr(rgnn, "_stream_on", lambda stream, device: None)

    def make(n, dtype=torch.float32):
        return torch.zeros(n, dtype=dtype).as_subclass(OnGpu)

    def lists(bits):
        d = dict(params=[make(600), make(0), make(7)], grads=[make(600), make(0), make(7)], copies=[make(600, torch.bfloat16), None, None])
        if bits == 32:
            return dict(d, m=[make(600), make(0), make(7)], v=[make(600), make(0), make(7)])
        return dict(d, m=[make(n, torch.int8) for n in (600, 0, 7)], v=[make(n, torch.uint8) for n in (600, 0, 7)],
                    m_scale=[make(3), make(0), make(1)], v_scale=[make(3), make(0), make(1)])

    moves = {
        "data": lambda t: setattr(t, "data", torch.zeros(t.numel(), dtype=t.dtype)),
        "set_": lambda t: t.set_(torch.zeros(t.numel() + 5, dtype=t.dtype)[5:]),
        "resize_": lambda t: t.resize_(1 << 20),
        "storage": lambda t: t.untyped_storage().resize_(0),
        "twice": lambda t: (setattr(t, "data", torch.zeros(1, dtype=t.dtype)), setattr(t, "data", torch.zeros(2, dtype=t.dtype))),
    }
    for bits in (32, 8):
        for name in lists(bits):
            for move in moves.values():
                d = lists(bits)
                kept = rgnn.AdamwTensors(**d)
                before = Library.calls
                rgnn.adamw_step(kept, 1, 1e-3)
                rgnn.adamw_step(kept, 2, 1e-3)
                assert Library.calls == before + 2
                move(d[name][0])
                with pytest.raises(ValueError, match="tensor 0.*moved"):
                    rgnn.adamw_step(kept, 3, 1e-3)
                assert Library.calls == before + 2
        d = lists(bits)
        kept = rgnn.AdamwTensors(**d)
        moves["data"](d["grads"][2])
        with pytest.raises(ValueError, match="tensor 2.*moved"):
            rgnn.adamw_step(kept, 3, 1e-3)
        rgnn.adamw_step(rgnn.AdamwTensors(**d), 3, 1e-3)
