"""Rotary positions, page plans and rows held in 4 bits without a GPU: frequencies, sizes, and what is refused before anything could
be launched.  (The addresses below are never read.)"""
import ctypes
import math

import numpy as np
import pytest
import torch

import _cache4 as plain
from paper_2606_10944_b200 import binding

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
A = 1 << 20                                     # a 256-byte aligned address
FREQ = (ctypes.c_double * 128)(*[1.0] * 128)


def _lib():
    return binding.load_library()


def test_frequencies():
    for rotary in (2, 64, 128, 256):
        rope = binding.Rope(rotary, base=500000.0)
        assert np.allclose(rope.inv_freq, plain.frequencies(rotary, 500000.0), rtol=1e-14) and rope.scale == 1.0
    f = plain.frequencies(128)
    assert np.allclose(binding.Rope(128, scaling="linear", factor=4).inv_freq, f / 4, rtol=1e-14)
    # base: the fastest pair stays, the slowest is divided by the factor
    g = np.array(binding.Rope(128, scaling="base", factor=8).inv_freq)
    assert g[0] == 1.0 and g[-1] == pytest.approx(f[-1] / 8, rel=1e-12) and (np.diff(g / f) < 0).all()
    ramp = binding.Rope(128, scaling="ramp", factor=16, original=4096)
    g = np.array(ramp.inv_freq) / f
    turns = 4096 * f / (2 * math.pi)
    assert ramp.scale == pytest.approx(0.1 * math.log(16) + 1, rel=1e-15)
    assert np.allclose(g[turns > 33.5], 1, rtol=1e-14) and np.allclose(g[turns < 0.85], 1 / 16, rtol=1e-12) and (np.diff(g) <= 1e-14).all()
    smooth = np.array(binding.Rope(128, scaling="smooth", factor=8, original=8192, low=1, high=4).inv_freq) / f
    turns = 8192 * f / (2 * math.pi)
    share = np.clip((turns - 1) / 3, 0, 1)
    assert np.allclose(smooth, share + (1 - share) / 8, rtol=1e-12)


@pytest.mark.parametrize("args", [(1, 10000.0, 0, 1.0, 0, 0, 0), (0, 10000.0, 0, 1.0, 0, 0, 0), (258, 10000.0, 0, 1.0, 0, 0, 0), (64, 1.0, 0, 1.0, 0, 0, 0),
                                  (64, math.nan, 0, 1.0, 0, 0, 0), (64, 10000.0, 5, 1.0, 0, 0, 0), (64, 10000.0, -1, 1.0, 0, 0, 0),
                                  (64, 10000.0, 1, 0.5, 0, 0, 0), (64, 10000.0, 1, math.inf, 0, 0, 0), (2, 10000.0, 2, 2.0, 0, 0, 0),
                                  (64, 10000.0, 3, 2.0, 0, 1, 32), (64, 10000.0, 3, 2.0, 4096, 0, 32), (64, 10000.0, 4, 2.0, 4096, 4, 1),
                                  (64, 10000.0, 4, 2.0, 4096, 1, math.inf)])
def test_frequencies_refused(args):
    s = ctypes.c_double()
    assert _lib().elm_rope_frequencies(*args, FREQ, ctypes.byref(s)) == SHAPE
    assert _lib().elm_rope_frequencies(*args[:6], args[6], None, ctypes.byref(s)) == NULL


def _rope_params(**kw):
    p = binding.RopeParams(2, 3, 5, 128, 1, 128, 0, 0, 1.0, ctypes.cast(FREQ, ctypes.POINTER(ctypes.c_double)))
    for k, v in kw.items():
        if k.endswith("stride"):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), SHAPE), (dict(heads=0), SHAPE), (dict(n_tokens=0), SHAPE), (dict(d=3), SHAPE), (dict(d=258), SHAPE), (dict(d=0), SHAPE),
    (dict(rotary_dim=130), SHAPE), (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=63), SHAPE), (dict(layout=2), SHAPE), (dict(dtype=2), DTYPE),
    (dict(dtype=7), DTYPE), (dict(scale=math.inf), SHAPE), (dict(scale=math.nan), SHAPE), (dict(out_stride=(0, 128, 384)), SHAPE),
    (dict(out_stride=(1, 0, 128)), SHAPE), (dict(out_stride=(1, 128, 0)), SHAPE), (dict(batch=1 << 20, n_tokens=1 << 12), SHAPE),
    (dict(heads=70000), SHAPE)])
def test_rope_refused(kw, code):
    assert _lib().elm_rope(A, A, 0, ctypes.byref(_rope_params(**kw)), 2 * A, None) == code


def test_rope_refused_pointers():
    p = _rope_params()
    r = ctypes.byref(p)
    assert _lib().elm_rope(None, A, 0, r, A, None) == NULL and _lib().elm_rope(A, A, 0, r, None, None) == NULL
    assert _lib().elm_rope(A, A, 0, None, A, None) == NULL
    assert _lib().elm_rope(A + 1, A, 0, r, A, None) == ALIGN and _lib().elm_rope(A, A + 2, 0, r, A, None) == ALIGN
    assert _lib().elm_rope(A, A, 0, ctypes.byref(_rope_params(x_stride=(1920, 640, 128), out_stride=(1920, 128, 384))), A, None) == SHAPE      # in place, other strides
    bad = (ctypes.c_double * 64)(*[1.0] * 63 + [math.nan])
    assert _lib().elm_rope(A, A, 0, ctypes.byref(_rope_params(inv_freq=ctypes.cast(bad, ctypes.POINTER(ctypes.c_double)))), A, None) == SHAPE
    p = _rope_params()
    p.inv_freq = ctypes.POINTER(ctypes.c_double)()
    assert _lib().elm_rope(A, A, 0, ctypes.byref(p), A, None) == NULL


PAGES = dict(batch=4, max_pages=8, page_rows=16, max_tokens=10, n_free=5)


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=65537), dict(max_pages=0), dict(page_rows=8), dict(page_rows=24), dict(page_rows=2048),
                                dict(max_tokens=-1), dict(n_free=-1), dict(max_pages=1 << 28)])
def test_plan_refused(kw):
    p = binding.PageParams(**{**PAGES, **kw})
    assert _lib().elm_page_plan(A, A, A, A, A, ctypes.byref(p), A, A, A, A, A, A, None) == SHAPE
    assert _lib().elm_page_release(A, A, A, A, A, ctypes.byref(p), None) == SHAPE


def test_plan_refused_pointers():
    p = ctypes.byref(binding.PageParams(**PAGES))
    for i in range(12):
        if i == 5:
            continue
        args = [A] * 5 + [p] + [A] * 6
        args[i] = None
        assert _lib().elm_page_plan(*args, None) == NULL, i
        args[i] = A + 2
        assert _lib().elm_page_plan(*args, None) == ALIGN, i
    for i in range(5):
        args = [A] * 5
        args[i] = None
        assert _lib().elm_page_release(*args, p, None) == NULL
        args[i] = A + 1
        assert _lib().elm_page_release(*args, p, None) == ALIGN


def test_row_bytes():
    assert binding.cache4_row_bytes(64) == plain.row_bytes(64) and binding.cache4_row_bytes(128) == plain.row_bytes(128)
    with pytest.raises(binding.ElmError):
        binding.cache4_row_bytes(96)


def _append(**kw):
    p = binding.AppendParams(3, 4, 2, 128, 1, 16, 8, 128, 0, 1.0, ctypes.cast(FREQ, ctypes.POINTER(ctypes.c_double)))
    for k, v in kw.items():
        if k.endswith("stride"):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(n_tokens=0), SHAPE), (dict(q_heads=-1), SHAPE), (dict(kv_heads=0), SHAPE), (dict(d=96), SHAPE), (dict(dtype=2), DTYPE),
    (dict(page_rows=15), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 28), SHAPE), (dict(n_pages=1 << 26, kv_heads=8), SHAPE),
    (dict(rotary_dim=130), SHAPE), (dict(rotary_dim=3), SHAPE), (dict(rotary_dim=-2), SHAPE), (dict(layout=9), SHAPE), (dict(scale=math.nan), SHAPE),
    (dict(q_out_stride=(0, 128)), SHAPE), (dict(q_out_stride=(512, 0)), SHAPE)])
def test_append_refused(kw, code):
    assert _lib().elm_cache4_append(A, A, A, A, A, ctypes.byref(_append(**kw)), 2 * A, A, None) == code


def test_append_refused_pointers():
    p = ctypes.byref(_append())
    for i in (0, 1, 2, 3, 4, 6, 7):
        args = [A, A, A, A, A, p, A, A]
        args[i] = None
        assert _lib().elm_cache4_append(*args, None) == NULL, i
        args[i] = A + (8 if i == 7 else 1)
        assert _lib().elm_cache4_append(*args, None) == ALIGN, i
    assert _lib().elm_cache4_append(A, A, A, A, A, ctypes.byref(_append(q_stride=(768, 128))), A, A, None) == SHAPE      # in place, other strides


def _cache(**kw):
    base = dict(batch=2, q_heads=4, kv_heads=2, d=128, dtype=1, page_rows=16, n_pages=10, max_pages=5, n_kv=0, n_q=1, n_tokens=0, causal=1)
    strides = {k: kw.pop(k) for k in list(kw) if k.endswith("stride")}
    p = binding.Cache4Params(**{**base, **kw})
    for k, v in strides.items():
        getattr(p, k)[:] = v
    return p


BAD = [(dict(batch=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(d=32), SHAPE), (dict(dtype=2), DTYPE), (dict(page_rows=17), SHAPE), (dict(n_pages=0), SHAPE),
       (dict(max_pages=0), SHAPE), (dict(n_kv=-1), SHAPE)]


@pytest.mark.parametrize("kw,code", BAD + [(dict(n_kv=0), SHAPE)])
def test_read_refused(kw, code):
    assert _lib().elm_cache4_read(A, A, None, None, ctypes.byref(_cache(**{"n_kv": 7, **kw})), A, A, None) == code


def test_read_refused_pointers():
    p = ctypes.byref(_cache(n_kv=7))
    for i in (0, 1, 5, 6):
        args = [A, A, A, A, p, A, A]
        args[i] = None
        assert _lib().elm_cache4_read(*args, None) == NULL
    for i in (0, 1, 2, 3, 5, 6):
        args = [A, A, A, A, p, A, A]
        args[i] = A + 1
        assert _lib().elm_cache4_read(*args, None) == ALIGN


@pytest.mark.parametrize("kw,code", BAD + [
    (dict(q_heads=3), SHAPE), (dict(q_heads=0), SHAPE), (dict(batch=1025), SHAPE), (dict(n_q=0), SHAPE), (dict(n_tokens=-1), SHAPE),
    (dict(batch=1000, q_heads=128), SHAPE), (dict(max_pages=1 << 27), SHAPE), (dict(n_q=1 << 30), SHAPE)])
def test_attend_refused(kw, code):
    p = _cache(**kw)
    b = ctypes.c_size_t(0)
    assert _lib().elm_cache4_attend_workspace_bytes(ctypes.byref(p), 0, ctypes.byref(b)) == code
    assert _lib().elm_cache4_attend(A, A, A, A, None, None, None, ctypes.byref(p), A, A, 1 << 40, None) == code
    s = ctypes.c_int32()
    assert _lib().elm_cache4_attend_status(A, ctypes.byref(p), 0, ctypes.byref(s), None) == code


def test_attend_refused_forms_and_pointers():
    lib, p = _lib(), _cache()
    r = ctypes.byref(p)
    big = 1 << 40
    assert lib.elm_cache4_attend(A, A, A, None, None, None, None, r, A, A, big, None) == NULL           # neither form
    q = _cache(n_kv=9)
    s = ctypes.byref(q)
    assert lib.elm_cache4_attend(A, A, A, A, None, A, A, s, A, A, big, None) == SHAPE                   # both
    assert lib.elm_cache4_attend(A, A, A, None, A, A, A, s, A, A, big, None) == SHAPE                   # a list with cu
    assert lib.elm_cache4_attend(A, A, A, None, None, A, None, s, A, A, big, None) == NULL
    assert lib.elm_cache4_attend(A, A, A, None, None, A, A, r, A, A, big, None) == SHAPE                # a list of 0 entries
    for i in (0, 1, 2, 8, 9):
        args = [A, A, A, A, None, None, None, r, A, A, big, None]
        args[i] = None
        assert lib.elm_cache4_attend(*args) == NULL
        args[i] = A + (128 if i == 9 else 2)
        assert lib.elm_cache4_attend(*args) == ALIGN
    args = [A, A, A, A + 1, None, None, None, r, A, A, big, None]
    assert lib.elm_cache4_attend(*args) == ALIGN
    need = binding.cache4_attend_workspace_bytes(p, False)
    assert lib.elm_cache4_attend(A, A, A, A, None, None, None, r, A, A, need - 1, None) == WORKSPACE
    for st in ((0, 128, 128), (512, 0, 512), (512, 128, 0)):
        z = _cache(n_q=2, o_stride=st)
        assert lib.elm_cache4_attend(A, A, A, A, None, None, None, ctypes.byref(z), A, A, big, None) == SHAPE


def test_binding_refuses():
    x = torch.zeros(1, 2, 3, 64)
    rope = binding.Rope(64)
    with pytest.raises(binding.ElmError):
        binding.rope(x, 0, rope)                                # not on a GPU
    with pytest.raises(binding.ElmError):
        binding.Rope(64, layout="thirds")
    with pytest.raises(binding.ElmError):
        binding.Rope(64, scaling="cubic")
    with pytest.raises(binding.ElmError):
        binding.Rope(63)
    pool = torch.zeros(2, 1, 16, 80, dtype=torch.uint8)
    for call in (lambda: binding.cache4_append(pool, x[0], x[0], torch.zeros(2, dtype=torch.int32)),
                 lambda: binding.cache4_read(pool, torch.zeros(1, 1, dtype=torch.int32), 3),
                 lambda: binding.cache4_attend(x, pool, torch.zeros(1, 1, dtype=torch.int32), length=torch.zeros(1, dtype=torch.int32)),
                 lambda: binding.page_plan(*[torch.zeros(1, dtype=torch.int32)] * 5, 16, 1)):
        with pytest.raises(binding.ElmError):
            call()
    # what the wrappers look at themselves (CPU tensors serve)
    with pytest.raises(binding.ElmError):
        binding._rows(torch.zeros(2, 3, 8, 4).transpose(2, 3), 4, "X")
    with pytest.raises(binding.ElmError):
        binding._rows(torch.zeros(0, 3, 8, 4), 4, "X")
    with pytest.raises(binding.ElmError):
        binding._int32(torch.zeros(3, dtype=torch.int64), "idx")
    with pytest.raises(binding.ElmError):
        binding._pool_d(torch.zeros(2, 1, 16, 96, dtype=torch.uint8))
    one, st = binding._rows(torch.zeros(64).expand(2, 3, 4, 64), 4, "X")
    assert one.is_contiguous() and st == (768, 256, 64, 1)


def test_plain_statement_of_rows():
    """The test statement itself: what it stores is the nearest number it can hold, by trying all of them."""
    r = np.random.default_rng(0)
    x = r.standard_normal((50, 64)) * np.exp(2 * r.standard_normal((50, 1)))
    code, byte = plain.quantise(x)
    back = plain.value(code, byte)
    s = plain.scale_value(byte)
    every = np.concatenate([plain.LEVELS, -plain.LEVELS])
    for i in range(50):
        for j in range(64):
            assert abs(back[i, j] - x[i, j]) == np.abs(every * s[i, j // 16] - x[i, j]).min()
    a = np.abs(x).reshape(50, 4, 16).max(-1)
    values = plain.scale_value(np.arange(0xf8))
    assert np.allclose(np.abs(s - a / 6), np.abs(values[:, None, None] - a / 6).min(0), rtol=1e-6)
    assert plain.nearest_scale(np.array([0.0, 1e9, 61440.0])).tolist() == [0, 0xe2, 0xe2] and plain.scale_value(0xe2) == 10240


def test_list_workspace_is_bounded():
    """The copy that the tensor-core form makes of a list takes 552 bytes an entry (d = 128) or 296: up to 8 GiB; longer lists take
    the other form, whose workspace does not grow with them."""
    most = 8 << 30
    for d in (128, 64):
        copied = []
        for batch, n_kv in [(1, 1024), (8, 16384), (64, 1 << 20), (64, 1 << 22), (1, 1 << 26), (64, 1 << 25)]:
            p = _cache(batch=batch, q_heads=8, kv_heads=8, d=d, n_kv=n_kv, n_q=8192, max_pages=1 << 20)
            need = binding.cache4_attend_workspace_bytes(p, True)
            assert need <= most, (d, batch, n_kv, need)
            p.dtype = 0                                       # (fp32 queries: always the other form)
            copied.append(need != binding.cache4_attend_workspace_bytes(p, True))
        assert copied == [True, True, False, False, False, False]


def test_status_is_asked_on_the_workspaces_device(monkeypatch):
    """cache4_attend_status runs on the device that its workspace is on and on that device's stream, whatever the current device is
    (a library that notes what it is given stands in for two GPUs)."""
    seen, entered = [], []

    class Lib:
        def elm_cache4_attend_status(self, workspace, params, with_list, out, stream):
            seen.append((workspace, with_list, stream, list(entered)))
            out._obj.value = 7
            return 0

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *_):
            entered.pop()

    class Workspace:
        def get_device(self):
            return 1

        def data_ptr(self):
            return 4096

    monkeypatch.setattr(binding, "load_library", Lib)
    monkeypatch.setattr(binding, "_stream_of", lambda device: 1000 + device)
    monkeypatch.setattr(binding, "_stream", lambda: 1000)
    monkeypatch.setattr(torch.cuda, "device", Device)
    assert binding.cache4_attend_status(Workspace(), _cache(n_kv=5), True) == 7
    assert seen == [(4096, 1, 1001, [1])]
    with pytest.raises(binding.ElmError):
        monkeypatch.undo()
        binding.cache4_attend_status(torch.zeros(16, dtype=torch.uint8), _cache(n_kv=5), True)      # not on a GPU
