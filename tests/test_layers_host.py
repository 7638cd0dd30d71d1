"""Host side of a worker's layers: what needs no GPU."""
import copy
import ctypes
import os
import pickle

import pytest
import torch

import paper_2005_10761_b200 as rt
from test_matrix_host import context


def test_micro_layout_and_scratch_sizes():
    for rows, cols, ld, scales in ((1, 1, 16, 1024), (128, 256, 128, 1024), (129, 257, 144, 4096), (10000, 1500, 752, 79 * 6 * 1024)):
        assert rt.micro_layout(rows, cols) == (ld, scales)
    for bad in ((0, 1), (1, 0), (1 << 31, 1)):
        with pytest.raises(rt.RTopKError):
            rt.micro_layout(*bad)
    for tokens in (0, 1, 1 << 20):
        for n_out, n_in in ((1, 1), (10000, 1500), (1 << 20, 1 << 20)):
            assert rt.micro_scratch(tokens, n_out, n_in) >= tokens * (n_in + n_out) // 2 + (n_in + n_out) * max(tokens, 32) // 2
    assert rt.layer_norm_scratch(1 << 30, 1 << 30) >= 8 << 30
    for call in (lambda: rt.layer_norm_scratch(-1, 5), lambda: rt.layer_norm_scratch(5, 0), lambda: rt.micro_scratch(-1, 1, 1)):
        with pytest.raises(rt.RTopKError):
            call()


def test_dense_reads_the_documented_layout():
    m = rt.MicroWeights(130, 300, transposed=False, tile=1, device="cpu")
    m.codes[129, 299 // 2] = 0x7 << 4 | 0x1              # the last two codes of the last row: 0.5, then 6
    m.codes[5, 0] = 0xD                                  # -3
    m.scales[(1 * 4 + 2) * 512 + 1 * 16 + 0 * 4 + 1] = 127 + 3      # row 129, block 9
    m.scales[5 * 16] = 0                                 # 2^-127
    m.scales[7 * 16] = 255
    want = torch.zeros(130, 300)
    want[129, 298], want[129, 299], want[5, 0] = 4.0, 48.0, -3 * 2.0 ** -127
    want[7, :32] = float("nan")
    assert torch.equal(m.dense().nan_to_num(-1.0), want.nan_to_num(-1.0))


def test_calls_use_the_tensors_that_micro_weights_hold():
    ctx, x, y = context(), torch.zeros(3, 30), torch.zeros(3, 40)
    m = rt.MicroWeights(40, 30, device="cpu")
    for q in (m, copy.deepcopy(m), pickle.loads(pickle.dumps(m))):
        q.codes, q.scales = torch.zeros((40, 64), dtype=torch.uint8), torch.zeros(1024, dtype=torch.uint8)
        ctx._lib.calls.clear()
        ctx.micro_weights(torch.zeros(40, 30), q)
        ctx.micro_product(x, q, y)
        ctx.micro_gradients(y, x, q, torch.zeros_like(x), torch.zeros(40, 30))
        (_, a), (_, b), (_, c) = ctx._lib.calls
        forward, backward = (q.codes.data_ptr(), 64, q.scales.data_ptr()), (q.codes_t.data_ptr(), q.codes_t.stride(0), q.scales_t.data_ptr())
        assert a[7:13] == forward + backward and b[4:7] == forward and c[6:9] == backward


def test_micro_weights_that_do_not_fit_are_refused():
    u8 = dict(dtype=torch.uint8)
    for name, bad in (("codes", torch.zeros((39, 16), **u8)), ("codes", torch.zeros((40, 8), **u8)), ("codes", torch.zeros((16, 40), **u8).t()),
                      ("codes", torch.zeros((40, 16), dtype=torch.int8)), ("codes_t", torch.zeros((30, 16), **u8)), ("scales", torch.zeros(1023, **u8)),
                      ("scales", torch.zeros(2048, **u8)[::2]), ("scales_t", torch.zeros((1, 1024), **u8)), ("scales", torch.zeros(1024))):
        m = rt.MicroWeights(40, 33, device="cpu")
        with pytest.raises((ValueError, TypeError)):
            setattr(m, name, bad)
    for args in (dict(tile=16), dict(tile=1)):
        with pytest.raises(ValueError):
            rt.MicroWeights(40, 33, device="cpu", **args)
    ctx, m = context(), rt.MicroWeights(40, 33, device="cpu")
    m.scales_t = None
    with pytest.raises(ValueError):
        ctx.micro_weights(torch.zeros(40, 33), m)
    assert not ctx._lib.calls


def test_tensors_of_another_device_are_refused_before_the_library_sees_them():
    ctx, f = context(device=0), torch.zeros
    m = rt.MicroWeights(40, 30, device="cpu")
    for call in (lambda: ctx.micro_weights(f(40, 30), m), lambda: ctx.micro_product(f(3, 30), m, f(3, 40)), lambda: ctx.micro_gradients(f(3, 40), f(3, 30), m, f(3, 30), f(40, 30)),
                 lambda: ctx.dropout(f(3, 30), f(3, 30), rt.Mask(0.5, 1)), lambda: ctx.layer_norm(f(3, 30), None, None, f(3, 30)),
                 lambda: ctx.layer_norm_gradients(f(3, 30), f(3, 30), f(3), f(3), None, f(3, 30))):
        with pytest.raises(ValueError):
            call()
    assert not ctx._lib.calls


def test_a_mask_reaches_the_library_as_it_is_when_the_call_is_made():
    seen = []

    class Library:
        def rtopk_dropout(self, *args):
            s = args[6]._obj
            seen.append((s.p, s.seed, s.step_ptr, s.step, s.worker, s.site))
            return 0
    ctx, x = context(), torch.zeros(3, 30)
    ctx._lib = Library()
    mask = rt.Mask(0.25, (1 << 64) - 1, 7, worker=3, site=2)
    ctx.dropout(x, x, mask)
    mask.step = 8
    ctx.dropout(x, x, mask)
    word = torch.zeros(1, dtype=torch.int32)
    mask.step = word
    ctx.dropout(x, x, mask)
    for copied in (copy.deepcopy(mask), pickle.loads(pickle.dumps(mask))):
        seen_before = len(seen)
        ctx.dropout(x, x, copied)
        assert seen.pop(seen_before)[2] == copied.step.data_ptr() != word.data_ptr()
    assert seen == [(0.25, (1 << 64) - 1, None, 7, 3, 2), (0.25, (1 << 64) - 1, None, 8, 3, 2), (0.25, (1 << 64) - 1, word.data_ptr(), 0, 3, 2)]
    assert ctypes.sizeof(mask._struct) == 40


def test_the_tests_philox_against_its_published_answers():
    """The form that the GPU tests' masks are made with."""
    path = os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_known_answers.txt")
    lines = [line.split()[1:] for line in open(path) if line.startswith("kat")]
    assert len(lines) == 2
    for n in ([int(w, 16) for w in words] for words in lines):
        c, key, want = n[:4], n[4:6], n[6:]
        for i in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            k0, k1 = (key[0] + i * 0x9E3779B9) % 2 ** 32, (key[1] + i * 0xBB67AE85) % 2 ** 32
            c = [(b >> 32) ^ c[1] ^ k0, b % 2 ** 32, (a >> 32) ^ c[3] ^ k1, a % 2 ** 32]
        assert c == want
