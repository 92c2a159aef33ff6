"""The layer's entry points on a CPU with a fake runtime: what they refuse, and what they queue for calls of no or some rows."""
import ctypes

import pytest

import fake_cuda as F
from paper_2608_03676_b200 import NormParams, RouteParams, RowsParams

OK, NULL, PARAM, UNSUPPORTED, CUDA, ALIGN = 0, -1, -2, -3, -4, -5
AT = [F.DEVICE + (i << 36) for i in range(16)]        # made-up device addresses, far apart


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return F.load(str(tmp_path_factory.mktemp("fake")))


def call(so, name, params, *args):
    so.fake_reset()
    conv = [ctypes.c_void_p(a) if isinstance(a, int) and a > 1 << 30 else a for a in args]
    return getattr(so, name)(ctypes.byref(params) if params is not None else None, *conv, ctypes.c_void_p(F.CALLER))


def norm_params(**kw):
    p = NormParams(ctypes.sizeof(NormParams), 1, 8, 64, 0, 1e-6, 0, 64, 64, 64, 64, 64)
    for name, v in kw.items():
        setattr(p, name, v)
    return p


def norm(so, x=AT[1], residual=None, weight=AT[2], h=None, y=AT[3], q=None, scales=None, rstd=AT[4], **kw):
    return call(so, "taot_rms_norm", norm_params(**kw), x, residual, weight, h, y, q, scales, rstd)


def norm_grad(so, dy=AT[1], dh=None, h=AT[2], weight=AT[3], rstd=AT[4], dx=AT[5], dweight=AT[6], ws=AT[7], **kw):
    return call(so, "taot_rms_norm_backward", norm_params(**kw), dy, dh, h, weight, rstd, dx, dweight, ws)


def route(so, logits=AT[1], bias=None, mask=None, topk=AT[2], weights=AT[3], **kw):
    p = RouteParams(ctypes.sizeof(RouteParams), 0, 1, 8, 64, 4, 0, 1, 1, 1, 1, 1.0, 64, 64)
    for name, v in kw.items():
        setattr(p, name, v)
    return call(so, "taot_route", p, logits, bias, mask, topk, weights)


def route_grad(so, logits=AT[1], topk=AT[2], dweights=AT[3], dlogits=AT[4], **kw):
    p = RouteParams(ctypes.sizeof(RouteParams), 0, 1, 8, 64, 4, 0, 1, 1, 1, 1, 1.0, 64, 64)
    for name, v in kw.items():
        setattr(p, name, v)
    return call(so, "taot_route_backward", p, logits, topk, dweights, dlogits)


def rows_params(kw):
    p = RowsParams(ctypes.sizeof(RowsParams), 1, 2, 8, 4, 64, 0, 0, 64, 64, 64)
    for name in list(kw):
        if hasattr(p, name):
            setattr(p, name, kw.pop(name))
    return p


def send(so, x=AT[1], scales=None, cols=0, perm=AT[2], counts=None, rows=AT[3], row_scales=None, info=AT[5], elem=2, **kw):
    return call(so, "taot_send", rows_params(kw), ctypes.c_int32(elem), x, scales, ctypes.c_int32(cols), perm, counts, rows, row_scales, info)


def combine(so, y=AT[1], perm=AT[2], counts=None, weights=None, residual=None, out=AT[3], info=AT[5], **kw):
    return call(so, "taot_combine", rows_params(kw), y, perm, counts, weights, residual, out, info)


def combine_grad(so, dout=AT[1], y=AT[2], perm=AT[3], counts=None, weights=AT[8], dy=AT[4], dweights=AT[5], info=AT[6], **kw):
    return call(so, "taot_combine_backward", rows_params(kw), dout, y, perm, counts, weights, dy, dweights, info)


CALLS = [norm, norm_grad, route, route_grad, send, combine, combine_grad]


def only_on_the_callers_stream(so):
    return all(e.stream == F.CALLER for e in F.log(so)) and not [e for e in F.log(so) if e.kind in (F.DEVICE_ALLOC, F.STREAM_CREATE)]


@pytest.mark.parametrize("f", CALLS)
def test_a_call_queues_kernels_on_its_stream_and_reports_a_failing_launch(so, f):
    assert f(so) == OK
    n = len(F.kernels(so))
    assert 1 <= n <= 3 and only_on_the_callers_stream(so)
    for after in range(n):
        so.fake_reset()
        so.fake_fail(F.LAUNCH, after)
        real, so.fake_reset = so.fake_reset, lambda: None
        try:
            assert f(so) == CUDA
        finally:
            so.fake_reset = real
    assert f(so) == OK and len(F.kernels(so)) == n


@pytest.mark.parametrize("f", CALLS)
@pytest.mark.parametrize("wrong,want", [(dict(struct_size=8), PARAM), (dict(dtype=3), PARAM), (dict(dtype=-1), PARAM)])
def test_the_struct_is_checked(so, f, wrong, want):
    if f is send and "dtype" in wrong:
        want = OK                                    # moves bytes, whatever they are
    assert f(so, **wrong) == want
    assert want == OK or not F.log(so)


@pytest.mark.parametrize("name", ["taot_rms_norm", "taot_rms_norm_backward", "taot_route", "taot_route_backward", "taot_combine"])
def test_no_params(so, name):
    so.fake_reset()
    args = {"taot_rms_norm": 9, "taot_rms_norm_backward": 9, "taot_route": 6, "taot_route_backward": 5, "taot_combine": 8}[name]
    assert getattr(so, name)(*([None] * (args + 1))) == NULL and not F.log(so)


REFUSED = [
    # norm
    (norm, dict(x=None), NULL), (norm, dict(weight=None), NULL), (norm, dict(y=None), NULL), (norm, dict(residual=AT[5]), NULL),
    (norm, dict(q=AT[5], group=32), NULL), (norm, dict(h=AT[5]), PARAM), (norm, dict(scales=AT[5]), PARAM), (norm, dict(group=32), PARAM),
    (norm, dict(q=AT[5], scales=AT[6], group=0), PARAM), (norm, dict(q=AT[5], scales=AT[6], group=96), PARAM),
    (norm, dict(q=AT[5], scales=AT[6], group=512), PARAM), (norm, dict(eps=-1e-6), PARAM), (norm, dict(eps=float("nan")), PARAM),
    (norm, dict(eps=float("inf")), PARAM), (norm, dict(N=-1), PARAM), (norm, dict(D=0), PARAM), (norm, dict(N=1 << 31), UNSUPPORTED),
    (norm, dict(D=(1 << 20) + 1, ld_x=1 << 21, ld_y=1 << 21), UNSUPPORTED), (norm, dict(ld_x=63), PARAM), (norm, dict(ld_y=63), PARAM),
    (norm, dict(ld_x=(1 << 28) + 1), PARAM), (norm, dict(reserved=1), PARAM),
    (norm, dict(residual=AT[5], h=AT[6], ld_residual=10), PARAM), (norm, dict(residual=AT[5], h=AT[6], ld_h=10), PARAM),
    (norm, dict(q=AT[5], scales=AT[6], group=32, ld_q=10), PARAM),
    (norm, dict(x=AT[1] + 1), ALIGN), (norm, dict(weight=AT[2] + 1), ALIGN), (norm, dict(y=AT[3] + 1), ALIGN), (norm, dict(rstd=AT[4] + 2), ALIGN),
    (norm, dict(q=AT[5], scales=AT[6] + 1, group=32), ALIGN),
    (norm, dict(y=AT[1] + 2), PARAM), (norm, dict(y=AT[1], ld_y=128), PARAM), (norm, dict(y=AT[2]), PARAM), (norm, dict(rstd=AT[1]), PARAM),
    (norm, dict(residual=AT[5], h=AT[3]), PARAM), (norm, dict(residual=AT[5], h=AT[5], ld_h=72), PARAM), (norm, dict(residual=AT[5], h=AT[6], y=AT[5]), PARAM),
    (norm, dict(q=AT[1], scales=AT[6], group=32), PARAM), (norm, dict(q=AT[3], scales=AT[6], group=32), PARAM),
    # its gradient
    (norm_grad, dict(dy=None), NULL), (norm_grad, dict(h=None), NULL), (norm_grad, dict(weight=None), NULL), (norm_grad, dict(rstd=None), NULL),
    (norm_grad, dict(dx=None), NULL), (norm_grad, dict(ws=None), NULL), (norm_grad, dict(ld_x=5), PARAM), (norm_grad, dict(ld_y=5), PARAM),
    (norm_grad, dict(ld_h=5), PARAM), (norm_grad, dict(dh=AT[9], ld_residual=5), PARAM), (norm_grad, dict(ws=AT[7] + 8), ALIGN),
    (norm_grad, dict(dweight=AT[6] + 2), ALIGN), (norm_grad, dict(dx=AT[5] + 1), ALIGN), (norm_grad, dict(dx=AT[2]), PARAM),
    (norm_grad, dict(dx=AT[1] + 2), PARAM), (norm_grad, dict(dx=AT[1], ld_x=72), PARAM), (norm_grad, dict(dweight=AT[5]), PARAM),
    (norm_grad, dict(ws=AT[6]), PARAM), (norm_grad, dict(ws=AT[1]), PARAM), (norm_grad, dict(dweight=AT[4]), PARAM),
    # router
    (route, dict(logits=None), NULL), (route, dict(topk=None), NULL), (route, dict(L=-1), PARAM), (route, dict(T=-1), PARAM), (route, dict(E=0), PARAM),
    (route, dict(k=0), PARAM), (route, dict(k=65, E=64), UNSUPPORTED), (route, dict(k=33, E=32), PARAM), (route, dict(E=1025, ld_logits=2000), UNSUPPORTED),
    (route, dict(L=1 << 16, T=1 << 16), UNSUPPORTED), (route, dict(L=1 << 62, T=4), UNSUPPORTED), (route, dict(score=2), PARAM), (route, dict(score=-1), PARAM),
    (route, dict(renormalise=2), PARAM), (route, dict(scale=float("nan")), PARAM), (route, dict(scale=float("inf")), PARAM), (route, dict(groups=0), PARAM),
    (route, dict(groups=3), PARAM), (route, dict(groups=128), PARAM), (route, dict(groups=128, E=1024, ld_logits=1024), UNSUPPORTED),
    (route, dict(groups=8, groups_kept=0), PARAM), (route, dict(groups=8, groups_kept=9), PARAM), (route, dict(groups=32, groups_kept=1), PARAM),
    (route, dict(groups=8, groups_kept=4, group_top=0), PARAM), (route, dict(group_top=3), PARAM), (route, dict(ld_logits=63), PARAM),
    (route, dict(logits=AT[1] + 2), ALIGN), (route, dict(topk=AT[2] + 2), ALIGN), (route, dict(weights=AT[3] + 1), ALIGN), (route, dict(bias=AT[5] + 2), ALIGN),
    (route, dict(topk=AT[1]), PARAM), (route, dict(weights=AT[1]), PARAM), (route, dict(weights=AT[2]), PARAM), (route, dict(bias=AT[3]), PARAM),
    (route, dict(mask=AT[2]), PARAM),
    # its gradient
    (route_grad, dict(logits=None), NULL), (route_grad, dict(topk=None), NULL), (route_grad, dict(dweights=None), NULL), (route_grad, dict(dlogits=None), NULL),
    (route_grad, dict(ld_dlogits=63), PARAM), (route_grad, dict(k=65), UNSUPPORTED), (route_grad, dict(dlogits=AT[1]), PARAM), (route_grad, dict(dlogits=AT[2]), PARAM),
    (route_grad, dict(dlogits=AT[3]), PARAM), (route_grad, dict(dlogits=AT[4] + 2), ALIGN),
    # rows
    (send, dict(x=None), NULL), (send, dict(perm=None), NULL), (send, dict(rows=None), NULL), (send, dict(scales=AT[6], cols=2), NULL),
    (send, dict(row_scales=AT[6], cols=2), NULL), (send, dict(C=4), NULL), (send, dict(elem=3), PARAM), (send, dict(elem=8), PARAM), (send, dict(elem=0), PARAM),
    (send, dict(scales=AT[6], row_scales=AT[7], cols=0), PARAM), (send, dict(B=-1), PARAM), (send, dict(n=-1), PARAM), (send, dict(k=-1), PARAM),
    (send, dict(D=0), PARAM), (send, dict(C=-1), PARAM), (send, dict(k=65), UNSUPPORTED), (send, dict(C=4097), UNSUPPORTED), (send, dict(n=1 << 28), UNSUPPORTED),
    (send, dict(B=1 << 40), UNSUPPORTED), (send, dict(D=(1 << 20) + 1, ld_rows=1 << 21, ld_tokens=1 << 21), UNSUPPORTED), (send, dict(ld_rows=63), PARAM),
    (send, dict(ld_tokens=63), PARAM), (send, dict(reserved=1), PARAM), (send, dict(x=AT[1] + 1), ALIGN), (send, dict(rows=AT[3] + 1), ALIGN),
    (send, dict(perm=AT[2] + 1), ALIGN), (send, dict(info=AT[5] + 1), ALIGN), (send, dict(rows=AT[1]), PARAM), (send, dict(info=AT[2]), PARAM),
    (combine, dict(y=None), NULL), (combine, dict(perm=None), NULL), (combine, dict(out=None), NULL), (combine, dict(C=2), NULL),
    (combine, dict(residual=AT[6], ld_residual=63), PARAM), (combine, dict(out=AT[1]), PARAM), (combine, dict(residual=AT[3], ld_residual=72), PARAM),
    (combine, dict(weights=AT[6] + 2), ALIGN), (combine, dict(out=AT[3] + 1), ALIGN), (combine, dict(weights=AT[3]), PARAM), (combine, dict(info=AT[3]), PARAM),
    (combine_grad, dict(dout=None), NULL), (combine_grad, dict(y=None), NULL), (combine_grad, dict(dy=None, dweights=None), NULL), (combine_grad, dict(dy=AT[1]), PARAM),
    (combine_grad, dict(dy=AT[2] + 2), PARAM), (combine_grad, dict(dweights=AT[8]), PARAM), (combine_grad, dict(dweights=AT[5] + 2), ALIGN),
    (combine_grad, dict(dweights=AT[4]), PARAM),
    # columns of one wider array that meet
    (combine_grad, dict(dy=AT[2] + 126, ld_rows=128), PARAM), (combine_grad, dict(dy=AT[2] + 130, ld_rows=128), PARAM),
    (combine_grad, dict(y=AT[2] + 130, dy=AT[2], ld_rows=128), PARAM), (norm, dict(y=AT[1] + 126, ld_x=200, ld_y=200), PARAM),
    (norm, dict(y=AT[1] + 128, ld_x=200, ld_y=204), PARAM), (route_grad, dict(dlogits=AT[1] + 252, ld_logits=128, ld_dlogits=128), PARAM),
]


@pytest.mark.parametrize("f,args,want", REFUSED, ids=lambda v: getattr(v, "__name__", str(v)[:40]))
def test_refusals_queue_nothing(so, f, args, want):
    assert f(so, **args) == want
    assert not F.log(so)


TAKEN = [(combine_grad, dict(dy=AT[2] + 128, ld_rows=128)), (combine_grad, dict(y=AT[2] + 128, dy=AT[2], ld_rows=128)),
         (norm, dict(y=AT[1] + 128, ld_x=200, ld_y=200)), (norm, dict(x=AT[1] + 400 * 3 + 128, y=AT[1], ld_x=200, ld_y=200)),
         (route_grad, dict(dlogits=AT[1] + 256, ld_logits=128, ld_dlogits=128)),
         (norm, dict(residual=AT[5], h=AT[5])), (norm, dict(residual=AT[5], h=AT[1])), (norm, dict(y=AT[1])), (norm, dict(rstd=None)),
         (norm, dict(y=None, q=AT[5], scales=AT[6], group=256)), (norm, dict(dtype=0)), (norm, dict(dtype=2)), (norm_grad, dict(dx=AT[1])),
         (norm_grad, dict(dh=AT[9], dx=AT[9])), (norm_grad, dict(dweight=None, ws=None)), (route, dict(weights=None)), (route, dict(bias=AT[5], mask=AT[6])),
         (route, dict(k=64)), (route, dict(E=1024, ld_logits=1024, k=64)), (route, dict(groups=64, groups_kept=4)), (route_grad, dict(k=64, E=8)),
         (send, dict(C=4, counts=AT[6])), (send, dict(info=None)), (send, dict(elem=1, scales=AT[6], row_scales=AT[7], cols=9)), (send, dict(elem=4)),
         (combine, dict(residual=AT[3])), (combine, dict(weights=AT[6], C=2, counts=AT[7])), (combine, dict(info=None, dtype=0)),
         (combine_grad, dict(dy=None)), (combine_grad, dict(y=None, dweights=None)), (combine_grad, dict(dy=AT[2])), (combine_grad, dict(weights=None))]


@pytest.mark.parametrize("f,args", TAKEN, ids=lambda v: getattr(v, "__name__", str(v)[:40]))
def test_what_the_documentation_allows_is_taken(so, f, args):
    assert f(so, **args) == OK
    assert F.kernels(so) and only_on_the_callers_stream(so)


def test_calls_of_no_rows_launch_nothing(so):
    for f, args in [(norm, dict(N=0)), (norm, dict(N=0, x=None, y=None)), (route, dict(L=0)), (route, dict(T=0, logits=None)), (route_grad, dict(T=0)),
                    (send, dict(B=0)), (send, dict(n=0)), (send, dict(k=0)), (combine, dict(n=0)), (combine, dict(B=0)), (combine_grad, dict(k=0)),
                    (norm_grad, dict(N=0, dweight=None))]:
        assert f(so, **args) == OK and not F.log(so), (f, args)
    assert norm_grad(so, N=0) == OK and [e.kind for e in F.log(so)] == [F.SET] and only_on_the_callers_stream(so)
    assert combine(so, k=0, y=None, perm=None) == OK and F.kernels(so)           # the residual, or zero


def test_the_workspace_is_asked_for(so):
    n = ctypes.c_size_t()
    assert so.taot_rms_norm_backward_workspace(ctypes.byref(norm_params()), ctypes.byref(n)) == OK and n.value > 0
    assert so.taot_rms_norm_backward_workspace(ctypes.byref(norm_params(D=0)), ctypes.byref(n)) == PARAM
    assert so.taot_rms_norm_backward_workspace(ctypes.byref(norm_params()), None) == NULL
    assert so.taot_rms_norm_backward_workspace(None, ctypes.byref(n)) == NULL


def test_a_call_makes_its_tensors_device_current_and_takes_that_devices_stream(monkeypatch):
    import torch
    from paper_2608_03676_b200 import layer
    current, log = [0], []

    class Device:
        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    def entry(params, *args):
        log.append((current[0], args))
        return 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(layer, "_stream_of", lambda index: 1000 + index)
    monkeypatch.setitem(layer._functions, "taot_route", entry)
    for index in (0, 1, 0):
        layer._call(torch.device("cuda", index), "taot_route", RouteParams(), 7)
    assert log == [(0, (7, 1000)), (1, (7, 1001)), (0, (7, 1000))] and current == [0]
    monkeypatch.setitem(layer._functions, "taot_route", lambda *a: PARAM)
    with pytest.raises(layer.TaotError, match="out of range"):
        layer._call(torch.device("cuda", 1), "taot_route", RouteParams(), 7)
    assert current == [0]


def test_which_strides_are_rows():
    import torch
    from paper_2608_03676_b200 import layer
    cpu = torch.device("cpu")
    rows = lambda t: layer._rows(t, "t", t.shape, t.dtype, cpu)
    x = torch.zeros((2, 3, 4, 10))
    assert rows(x) == 10 and rows(x[..., 2:7]) == 10 and rows(x[:, :, ::2, :5]) == 20 and rows(x[1:, 2:, 3:, 1:4]) == 3
    assert rows(x[0, 0, :, :1]) == 10 and rows(x[0, 0, 0, 3:5]) == 2 and rows(torch.zeros((0, 5))) == 5 and rows(torch.zeros((4, 1)).expand(4, 1)) == 1
    for bad in (x.transpose(2, 3), x[..., ::2], x[:, :2], x[:, :, :3], torch.zeros((1, 6)).expand(4, 6), torch.zeros(6).as_strided((3, 4), (1, 1)),
                x.transpose(0, 1)):
        with pytest.raises(layer.TaotError):
            rows(bad)
    with pytest.raises(layer.TaotError, match="expected a tensor"):
        layer._rows(x, "t", (2, 3, 4, 9), x.dtype, cpu)
    with pytest.raises(layer.TaotError, match="expected a tensor"):
        layer._rows(x, "t", x.shape, torch.bfloat16, cpu)
    with pytest.raises(layer.TaotError):
        layer._dense(x[..., :5], "t", (2, 3, 4, 5), x.dtype, cpu)
    layer._dense(None, "t", (1,), x.dtype, cpu)
