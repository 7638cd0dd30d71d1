"""Host side of the matrix operators: what needs no GPU."""
import copy
import io
import pickle

import pytest
import torch

import paper_2005_10761_b200 as rt


class Recorder:
    """Stands in for the library: keeps the arguments of every call."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


def context(device=-1):
    """A context without a device: tensors of the CPU count as its own."""
    ctx = rt.MatrixContext.__new__(rt.MatrixContext)
    ctx._lib, ctx._h, ctx.device, ctx._stream = Recorder(), None, device, lambda: 0
    return ctx


def addresses(ctx, coded, x, y):
    """What code_weights, coded_product and coded_gradients pass for the codes, their row strides and the scales."""
    ctx._lib.calls.clear()
    ctx.code_weights(torch.zeros(coded.n_out, coded.n_in), coded)
    ctx.coded_product(x, coded, y)
    ctx.coded_gradients(y, x, coded, torch.zeros_like(x), torch.zeros(coded.n_out, coded.n_in))
    (_, a), (_, b), (_, c) = ctx._lib.calls
    return a[6:11], b[4:7], c[6:9]


def expected(coded):
    c, t, s = coded.codes, coded.codes_t, coded.scales
    return ((c.data_ptr(), c.stride(0), t.data_ptr(), t.stride(0), s.data_ptr()), (c.data_ptr(), c.stride(0), s.data_ptr()),
            (t.data_ptr(), t.stride(0), s.data_ptr()))


def test_calls_use_the_tensors_that_coded_weights_hold():
    ctx, x, y = context(), torch.zeros(3, 30), torch.zeros(3, 40)
    coded = rt.CodedWeights(40, 30, device="cpu")
    assert addresses(ctx, coded, x, y) == expected(coded)
    coded.codes = torch.zeros((40, 256), dtype=torch.int8)                  # as received from elsewhere
    coded.scales, coded.codes_t = torch.zeros(40), torch.zeros((30, 48), dtype=torch.int8)
    assert addresses(ctx, coded, x, y) == expected(coded)
    other = copy.deepcopy(coded)
    assert other.codes.data_ptr() != coded.codes.data_ptr()
    assert addresses(ctx, other, x, y) == expected(other)
    again = pickle.loads(pickle.dumps(coded))
    assert addresses(ctx, again, x, y) == expected(again)
    buffer = io.BytesIO()
    torch.save(coded, buffer)
    buffer.seek(0)
    loaded = torch.load(buffer, weights_only=False)
    assert addresses(ctx, loaded, x, y) == expected(loaded)


def test_coded_weights_that_do_not_fit_are_refused():
    ctx, x, y = context(), torch.zeros(3, 30), torch.zeros(3, 40)
    for name, bad in (("codes", torch.zeros((39, 128), dtype=torch.int8)), ("codes", torch.zeros((40, 16), dtype=torch.int8)),
                      ("codes", torch.zeros((128, 40), dtype=torch.int8).t()), ("codes", torch.zeros(40 * 128, dtype=torch.int8)),
                      ("codes", torch.zeros((40, 128), dtype=torch.float32)), ("codes_t", torch.zeros((30, 16), dtype=torch.int8)),
                      ("codes_t", torch.zeros((29, 128), dtype=torch.int8)), ("scales", torch.zeros(39)), ("scales", torch.zeros(80)[::2]),
                      ("scales", torch.zeros(40, dtype=torch.float64))):
        coded = rt.CodedWeights(40, 30, device="cpu")
        with pytest.raises((ValueError, TypeError)):
            setattr(coded, name, bad)
            addresses(ctx, coded, x, y)
    coded = rt.CodedWeights(40, 30, device="cpu")
    with pytest.raises(AttributeError):
        coded.n_out = 41


def test_tensors_of_another_device_are_refused_before_the_library_sees_them():
    """A context of device 0 and tensors of the CPU: their addresses mean nothing there."""
    ctx, f = context(device=0), torch.zeros
    coded = rt.CodedWeights(40, 30, device="cpu")
    for call in (lambda: ctx.orthogonalize(f(4, 5), f(4, 5)), lambda: ctx.orthogonal_update(f(4, 5), f(4, 5), f(4, 5), 0.1, 0.9),
                 lambda: ctx.code_weights(f(40, 30), coded), lambda: ctx.coded_product(f(3, 30), coded, f(3, 40)),
                 lambda: ctx.coded_gradients(f(3, 40), f(3, 30), coded, f(3, 30), f(40, 30))):
        with pytest.raises(ValueError):
            call()
    assert not ctx._lib.calls


def test_codes_of_another_device_are_refused(monkeypatch):
    ctx, f = context(device=0), torch.zeros
    for name in ("codes", "codes_t", "scales"):
        coded = rt.CodedWeights(40, 30, device="cpu")
        away = getattr(coded, name)
        monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1 if t is away else 0)
        calls = [lambda: ctx.code_weights(f(40, 30), coded)]
        if name != "codes":
            calls.append(lambda: ctx.coded_gradients(f(3, 40), None, coded, f(3, 30)))
        if name != "codes_t":
            calls.append(lambda: ctx.coded_product(f(3, 30), coded, f(3, 40)))
        for call in calls:
            with pytest.raises(ValueError):
                call()
    assert not ctx._lib.calls


def test_gradients_without_x_name_what_is_missing():
    ctx, coded = context(), rt.CodedWeights(40, 30, device="cpu")
    with pytest.raises(ValueError, match="x"):
        ctx.coded_gradients(torch.zeros(3, 40), None, coded, dw=torch.zeros(40, 30))
    assert not ctx._lib.calls


def test_scratch_sizes_are_sizes_or_refusals():
    """Either at least the bytes of X in its three forms, or UNSUPPORTED; never a wrapped number."""
    import itertools
    for batch, m, n in itertools.product((1, 3, 65535), (1, 1000, 1 << 20, 1 << 30), (1, 1500, 1 << 24, 1 << 30)):
        try:
            assert rt.orthogonalize_scratch(batch, m, n) >= 8 * batch * m * n
        except rt.RTopKError as e:
            assert e.status == 4 and batch * m * n >= 1 << 50, (batch, m, n)
    with pytest.raises(rt.RTopKError):
        rt.orthogonalize_scratch(1, 1 << 30, 1 << 30)
    for tokens, n_out, n_in in itertools.product((0, 1, 1 << 30), (1, 1 << 30), (1, 1 << 30)):
        assert rt.coded_scratch(tokens, n_out, n_in) >= tokens * (n_in + n_out) + (n_in + n_out) * max(tokens, 128)
