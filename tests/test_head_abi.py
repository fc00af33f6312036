"""C ABI of the head's training operators (include/reno_head.h): the binding
lists the header's functions and structures, and every argument error is
returned before anything touches a device.  CPU only."""
import ctypes
import os
import re

import pytest

import paper_2503_12382_amd as reno

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "reno_head.h")

pytestmark = pytest.mark.skipif(not os.path.exists(reno.LIB_PATH),
                                reason="libreno.so not built (run __graft_entry__.build())")


def source():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_header_and_binding_agree():
    decl = set(re.findall(r"\b(reno_[a-z_0-9]+)\s*\(", source()))
    assert decl == set(reno._HEAD_SIGS)
    L = ctypes.CDLL(reno.LIB_PATH)
    assert all(hasattr(L, name) for name in decl)
    assert not decl & set(reno._SIGS)


@pytest.mark.parametrize("name,cls", [("reno_head", reno.reno_head), ("reno_head_data", reno.reno_head_data)])
def test_struct_layouts_agree(name, cls):
    body = re.search(r"typedef struct \{([^{}]*)\}\s*" + name + r"\s*;", source()).group(1)
    assert [m.group(1) for m in re.finditer(r"(\w+)\s*;", body)] == [f[0] for f in cls._fields_]


def test_constants_agree():
    text = source()
    assert f"RENO_HEAD_MAX_CHANNELS {reno.RENO_HEAD_MAX_CHANNELS}" in text
    assert "RENO_HEAD_MAX_SYMBOLS (1 << 20)" in text and reno.RENO_HEAD_MAX_SYMBOLS == 1 << 20
    assert f"RENO_HEAD_MAX_TOP {reno.RENO_HEAD_MAX_TOP}" in text


GOOD = dict(rows=100, channels=32, symbols=256, type=reno.RENO_T_FP32, h_stride=32, w_stride=256)
BAD = [dict(rows=-1), dict(rows=1 << 31), dict(channels=0), dict(channels=16385), dict(symbols=0),
       dict(symbols=(1 << 20) + 1), dict(type=3), dict(type=-1), dict(h_stride=31), dict(w_stride=255),
       dict(h_stride=1 << 31), dict(w_stride=1 << 31)]


def head(**kw):
    return reno.reno_head(**{**GOOD, **kw})


def workspace(**kw):
    n = ctypes.c_int64(-1)
    L = reno.lib()
    assert L.reno_head_workspace(ctypes.byref(head(**kw)), 1, 1, ctypes.byref(n)) == reno.RENO_OK
    return n.value


def test_workspace_sizes():
    L = reno.lib()
    n = ctypes.c_int64(-1)
    for bad in BAD:
        assert L.reno_head_workspace(ctypes.byref(head(**bad)), 1, 1, ctypes.byref(n)) == reno.RENO_E_INVALID, bad
        assert L.reno_last_error(None)
    p = head()
    for k in (0, -1, 129):
        assert L.reno_head_workspace(ctypes.byref(p), k, 0, ctypes.byref(n)) == reno.RENO_E_INVALID
    assert L.reno_head_workspace(None, 1, 0, ctypes.byref(n)) == reno.RENO_E_INVALID
    assert L.reno_head_workspace(ctypes.byref(p), 1, 0, None) == reno.RENO_E_INVALID
    assert L.reno_head_workspace(ctypes.byref(p), 1, 0, ctypes.byref(n)) == reno.RENO_OK
    assert 0 < n.value < workspace()
    # the logits are not kept: scratch stops growing with the rows' logits
    big = dict(channels=64, symbols=1 << 20, h_stride=64, w_stride=1 << 20, type=reno.RENO_T_BF16)
    assert workspace(rows=1 << 20, **big) < 8 << 30
    for rows in (0, 1, (1 << 31) - 1):
        assert workspace(rows=rows) > 0


def test_code_length_rejects_bad_arguments():
    L = reno.lib()
    p, ws = ctypes.c_void_p(256), 1 << 40            # never dereferenced: every case fails its checks first
    good = dict(h=256, w=256, b=256, row_weight=256, bits=256, lse=256, dh=256, dw=256, db=256)

    def call(d=good, symbol=p, work=p, nbytes=ws, **kw):
        return L.reno_head_code_length(ctypes.byref(head(**kw)), ctypes.byref(reno.reno_head_data(**d)), symbol, work,
                                       nbytes, None)
    for bad in BAD:
        assert call(**bad) == reno.RENO_E_INVALID, bad
    for name in ("h", "w", "bits"):
        assert call({**good, name: None}) == reno.RENO_E_INVALID, name
    for name in good:
        assert call({**good, name: 258}) == reno.RENO_E_INVALID, name
        if name in ("h", "w", "b", "dh", "dw", "db"):
            assert call({**good, name: 257}, type=reno.RENO_T_BF16) == reno.RENO_E_INVALID, name
    assert call(symbol=None) == reno.RENO_E_INVALID
    assert call(symbol=ctypes.c_void_p(257)) == reno.RENO_E_INVALID
    assert call(work=None) == reno.RENO_E_INVALID
    assert call(work=ctypes.c_void_p(128)) == reno.RENO_E_INVALID
    assert call(nbytes=workspace() - 1) == reno.RENO_E_INVALID
    assert call(nbytes=-1) == reno.RENO_E_INVALID
    assert L.reno_head_code_length(None, ctypes.byref(reno.reno_head_data(**good)), p, p, ws, None) == reno.RENO_E_INVALID
    assert L.reno_head_code_length(ctypes.byref(head()), None, p, p, ws, None) == reno.RENO_E_INVALID


def test_distill_rejects_bad_arguments():
    L = reno.lib()
    p, ws = ctypes.c_void_p(256), 1 << 40
    d = reno.reno_head_data(h=256, w=256, bits=256)

    def call(index=p, logit=p, k=4, T=1.0, work=p, nbytes=ws):
        return L.reno_head_distill(ctypes.byref(head()), ctypes.byref(d), index, logit, k, T, work, nbytes, None)
    for kw in (dict(k=0), dict(k=129), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")),
               dict(T=1e-45), dict(T=1e39), dict(index=None), dict(logit=None), dict(work=None), dict(nbytes=0),
               dict(logit=ctypes.c_void_p(258))):
        assert call(**kw) == reno.RENO_E_INVALID, kw
        assert L.reno_last_error(None)


@pytest.mark.parametrize("T", [4e-39, 1e-39, 3e38])
def test_distill_rejects_temperatures_whose_scale_is_not_a_normal_float(T):
    """log2(e) / T multiplies the logits: at 4e-39 it is 3.6e38, past the largest float, though 1 / T is not."""
    p, d = ctypes.c_void_p(256), reno.reno_head_data(h=256, w=256, bits=256)
    assert reno.lib().reno_head_distill(ctypes.byref(head()), ctypes.byref(d), p, p, 4, T, p, 1 << 40,
                                        None) == reno.RENO_E_INVALID


def test_top_logits_rejects_bad_arguments():
    L = reno.lib()
    p = ctypes.c_void_p(256)

    def call(z=p, type=0, rows=4, symbols=10, stride=10, k=3, index=p, value=p, lse=p):
        return L.reno_top_logits(z, type, rows, symbols, stride, k, index, value, lse, None)
    for kw in (dict(z=None), dict(type=3), dict(rows=-1), dict(rows=1 << 31), dict(symbols=0),
               dict(symbols=(1 << 20) + 1, stride=1 << 21), dict(stride=9), dict(stride=1 << 31), dict(k=0), dict(k=129),
               dict(index=None), dict(value=None), dict(z=ctypes.c_void_p(258)), dict(lse=ctypes.c_void_p(257))):
        assert call(**kw) == reno.RENO_E_INVALID, kw
    assert call(rows=0, z=None, index=None, value=None) == reno.RENO_OK


def test_features_rejects_a_null_context():
    assert reno.lib().reno_features(None, 5, None) == reno.RENO_E_INVALID
