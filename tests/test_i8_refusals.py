"""Arguments that the 8-bit row calls refuse, before they touch a device (CPU only)."""
import ctypes as C

import numpy as np
import pytest
import torch

BADARG, SHAPE = -1, -3


@pytest.fixture(scope="module")
def L():
    import os
    from paper_2102_08481_amd import LIB_PATH, build, lib
    if not os.path.exists(LIB_PATH):
        build.build()
    return lib()


A = 4096   # an address that is never read: every call here is refused, or has no rows


def test_pitch_is_whole_lines(L):
    for k, pitch in ((1, 128), (127, 128), (128, 128), (129, 256), (12544, 12544), (65536, 65536)):
        assert L.thia_i8_pitch(k) == pitch
    for k in (0, -1, 65537, 2 ** 31 - 1, -2 ** 31):
        assert L.thia_i8_pitch(k) == 0


QUANTIZE = dict(x=A, ldx=8, precision=1, rows=2, k=8, codes=A, scales=A, stream=None)
NORM = dict(x=A, ldx=8, r=A, ldr=8, gain=A, eps=1e-6, precision=1, rows=2, k=8, sum=A, ldsum=8, codes=A, scales=A, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), BADARG), (dict(codes=None), BADARG), (dict(scales=None), BADARG), (dict(rows=-1), BADARG), (dict(k=0), BADARG),
    (dict(k=-5), BADARG), (dict(ldx=7), BADARG), (dict(ldx=-8), BADARG), (dict(precision=2), BADARG), (dict(precision=-1), BADARG), (dict(x=A + 1), BADARG),
    (dict(x=A + 2, precision=0), BADARG), (dict(codes=A + 8), BADARG), (dict(scales=A + 2), BADARG), (dict(k=65537, ldx=65537), SHAPE)])
def test_quantize_refuses(L, change, code):
    assert L.thia_quantize_rows(*{**QUANTIZE, **change}.values()) == code
    assert len(L.thia_i8_last_error()) > 5


@pytest.mark.parametrize("change,code", [
    (dict(x=None), BADARG), (dict(gain=None), BADARG), (dict(codes=None), BADARG), (dict(scales=None), BADARG), (dict(rows=-1), BADARG), (dict(k=0), BADARG),
    (dict(eps=0.0), BADARG), (dict(eps=-1.0), BADARG), (dict(eps=float("nan")), BADARG), (dict(eps=float("inf")), BADARG), (dict(r=None), BADARG),
    (dict(ldx=7), BADARG), (dict(ldr=7), BADARG), (dict(ldsum=7), BADARG), (dict(ldsum=9), BADARG), (dict(sum=A + 64, r=A + 64, ldr=9), BADARG), (dict(r=A + 1), BADARG), (dict(sum=A + 1), BADARG), (dict(gain=A + 2), BADARG),
    (dict(precision=2), BADARG), (dict(k=65537, ldx=65537, ldr=65537, ldsum=65537), SHAPE)])
def test_norm_refuses(L, change, code):
    assert L.thia_rms_norm_i8(*{**NORM, **change}.values()) == code
    assert len(L.thia_i8_last_error()) > 5


def test_no_rows_is_nothing(L):
    assert L.thia_quantize_rows(None, 8, 1, 0, 8, None, None, None) == 0
    assert L.thia_rms_norm_i8(None, 8, None, 8, None, 1e-6, 0, 0, 8, None, 8, None, None, None) == 0


def test_layers_refuse(L):
    h = C.c_void_p(1)
    w, s = np.ones((4, 8), np.float32), np.ones(4, np.float32)
    for n, k, code in ((0, 8, BADARG), (4, 0, BADARG), (-1, 8, BADARG), (4, 65537, SHAPE), (2 ** 20 + 1, 8, SHAPE)):
        h.value = 1
        assert L.thia_linear_i8_load(w.ctypes.data, None, n, k, C.byref(h)) == code and h.value is None
        h.value = 1
        assert L.thia_linear_i8_load_codes(w.ctypes.data, s.ctypes.data, None, n, k, C.byref(h)) == code and h.value is None
    assert L.thia_linear_i8_load(None, None, 4, 8, C.byref(h)) == BADARG
    assert L.thia_linear_i8_load(w.ctypes.data, None, 4, 8, None) == BADARG
    assert L.thia_linear_i8_load_codes(w.ctypes.data, None, None, 4, 8, C.byref(h)) == BADARG
    assert L.thia_linear_i8_run(None, A, A, 1, None, 0, 0, 1, A, 8, None) == BADARG
    n, k = C.c_int(), C.c_int()
    assert L.thia_linear_i8_shape(None, C.byref(n), C.byref(k)) == BADARG
    L.thia_linear_i8_free(None)


def test_messages_belong_to_their_thread(L):
    import threading
    assert L.thia_quantize_rows(None, 8, 1, 1, 8, None, None, None) == BADARG
    mine, seen = L.thia_i8_last_error(), []
    t = threading.Thread(target=lambda: seen.append((L.thia_i8_last_error(), L.thia_quantize_rows(A, 7, 1, 1, 8, A, A, None))))
    t.start()
    t.join()
    assert seen == [(b"", BADARG)] and L.thia_i8_last_error() == mine


def test_binding_refuses_what_is_not_on_the_gpu():
    import paper_2102_08481_amd as thia
    x = torch.zeros(2, 8)
    for call in (lambda: thia.thia_quantize_rows(x), lambda: thia.thia_quantize_rows(x.numpy()), lambda: thia.thia_rms_norm_i8(x, torch.ones(8)),
                 lambda: thia.thia_linear_i8_load(torch.zeros(8)), lambda: thia.thia_linear_i8_load(torch.zeros(4, 8), torch.zeros(5)),
                 lambda: thia.thia_linear_i8_load_codes(torch.zeros(4, 8), torch.zeros(4))):
        with pytest.raises(ValueError):
            call()
