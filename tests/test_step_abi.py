"""C ABI of the step after a gradient (include/reno_step.h) and of symbols drawn from logits (include/reno_head.h):
the binding lists the headers' functions and structures, and every argument error is returned before anything touches a
device.  CPU only."""
import ctypes
import os
import re

import pytest

import paper_2503_12382_amd as reno

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include")

pytestmark = pytest.mark.skipif(not os.path.exists(reno.LIB_PATH),
                                reason="libreno.so not built (run __graft_entry__.build())")
INVALID = reno.RENO_E_INVALID


def source(name):
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(INCLUDE, name)).read(), flags=re.S)


def test_header_and_binding_agree():
    text = source("reno_step.h")
    decl = set(re.findall(r"\b(reno_[a-z_0-9]+)\s*\(", text))
    assert decl == set(reno._STEP_SIGS)
    L = ctypes.CDLL(reno.LIB_PATH)
    assert all(hasattr(L, name) for name in decl)
    assert not decl & (set(reno._SIGS) | set(reno._HEAD_SIGS))
    assert "RENO_STEP_MAX_TENSORS (1 << 20)" in text and reno.RENO_STEP_MAX_TENSORS == 1 << 20


@pytest.mark.parametrize("header,name,cls", [
    ("reno_step.h", "reno_gradient", reno.reno_gradient), ("reno_step.h", "reno_parameter", reno.reno_parameter),
    ("reno_step.h", "reno_adamw", reno.reno_adamw), ("reno_head.h", "reno_sample", reno.reno_sample)])
def test_struct_layouts_agree(header, name, cls):
    body = re.search(r"typedef struct \{([^{}]*)\}\s*" + name + r"\s*;", source(header)).group(1)
    fields = [x for m in re.finditer(r"([^;]*);", body) for x in re.findall(r"(\w+)\s*(?:,|$)", m.group(1).strip())]
    assert fields == [f[0] for f in cls._fields_]


P = 4096   # a pointer that is never dereferenced: every case fails its checks first


def grads(*entries):
    return (reno.reno_gradient * max(len(entries), 1))(*[reno.reno_gradient(**{**dict(n=4, type=0, grad=P, out=8 * P), **e})
                                                         for e in entries])


def test_grad_norm_rejects_bad_arguments():
    L = reno.lib()
    n = ctypes.c_int64(-1)

    def call(*entries, count=None, lst=True, scale=1.0, norm=P, ws=P, size=1 << 40):
        a = grads(*entries)
        return L.reno_grad_norm(ctypes.addressof(a) if lst else None, len(entries) if count is None else count, scale,
                                norm, ws, size, None)
    for bad in (dict(n=-1), dict(n=1 << 40), dict(type=3), dict(type=-1), dict(grad=None), dict(grad=P + 2),
                dict(grad=P + 1, type=1)):
        assert call({}, bad) == INVALID, bad
        a = grads({}, bad)
        assert L.reno_grad_workspace(ctypes.addressof(a), 2, ctypes.byref(n)) == INVALID, bad
        assert L.reno_last_error(None)
    for kw in (dict(count=-1), dict(count=(1 << 20) + 1), dict(lst=False), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(norm=None), dict(norm=P + 2), dict(ws=None),
               dict(ws=P + 8), dict(size=7)):
        assert call({}, **kw) == INVALID, kw
    a = grads({}, dict(n=0, grad=None), dict(n=100000))
    assert L.reno_grad_workspace(ctypes.addressof(a), 3, ctypes.byref(n)) == reno.RENO_OK and n.value >= 16
    assert L.reno_grad_workspace(None, 0, ctypes.byref(n)) == reno.RENO_OK and n.value >= 0
    assert L.reno_grad_workspace(ctypes.addressof(a), 3, None) == INVALID


def test_grad_norm_rejects_what_overlaps():
    """What the call writes, the norm and the workspace, lies in nothing that it reads or writes besides."""
    L = reno.lib()
    n = ctypes.c_int64()
    a = grads(dict(n=1000), dict(n=1 << 24, grad=1 << 30, type=1))
    assert L.reno_grad_workspace(ctypes.addressof(a), 2, ctypes.byref(n)) == reno.RENO_OK and n.value > 16

    def call(norm, ws):
        return L.reno_grad_norm(ctypes.addressof(a), 2, 1.0, norm, ws, n.value, None)
    end = (1 << 30) + (1 << 25)
    for norm, ws in ((P, 1 << 20), (P + 3996, 1 << 20), (end - 4, 1 << 20),                   # the norm in a gradient
                     (1 << 28, P), (1 << 28, P + 3840), (1 << 28, (1 << 30) + 4096), (1 << 28, end - 256),
                     (1 << 28, (1 << 30) - 256),                                              # the workspace
                     (1 << 20, 1 << 20), ((1 << 20) + n.value - 4, 1 << 20)):                 # one in the other
        assert call(norm, ws) == INVALID, (norm, ws)
        assert b"overlaps" in L.reno_last_error(None)


def test_grad_clip_rejects_bad_arguments():
    L = reno.lib()

    def call(*entries, norm=P * 32, scale=1.0, most=1.0):
        a = grads(*entries)
        return L.reno_grad_clip(ctypes.addressof(a), len(entries), norm, scale, most, None)
    for bad in (dict(n=-1), dict(type=3), dict(grad=None), dict(out=None), dict(out=8 * P + 2), dict(grad=P + 2)):
        assert call(bad) == INVALID, bad
    for kw in (dict(norm=None), dict(norm=P + 2), dict(scale=0.0), dict(most=0.0), dict(most=float("nan"))):
        assert call({}, **kw) == INVALID, kw
    # outputs over other operands: another output, another gradient, its own shifted, the norm
    for pair in ((dict(), dict(grad=2 * P)), (dict(), dict(grad=8 * P, out=9 * P)), (dict(out=P + 8),),
                 (dict(out=32 * P),), (dict(out=P), dict(grad=P + 8, out=9 * P))):
        assert call(*pair) == INVALID, pair


GOOD = dict(n=4, type=0, grad_type=0, param=P, grad=2 * P, master=None, exp_avg=3 * P, exp_avg_sq=4 * P)
HOW = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, scale=1.0, max_norm=1.0, norm=32 * P, steps=33 * P)


def test_adamw_rejects_bad_arguments():
    L = reno.lib()

    def call(*entries, count=None, **how):
        a = (reno.reno_parameter * len(entries))(*[reno.reno_parameter(**{**GOOD, **e}) for e in entries])
        h = reno.reno_adamw(**{**HOW, **how})
        return L.reno_adamw_step(ctypes.addressof(a), len(entries) if count is None else count, ctypes.byref(h), None)
    bf = dict(type=1, grad_type=1)
    for bad in (dict(n=-1), dict(n=1 << 40), dict(type=3), dict(grad_type=1), dict(type=1, grad_type=2), dict(master=5 * P),
                dict(param=None), dict(grad=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(param=P + 2),
                dict(exp_avg=3 * P + 2), dict(**bf, grad=2 * P + 1), dict(**bf, master=5 * P + 2),
                dict(grad=P), dict(exp_avg=4 * P + 8), dict(**bf, master=P + 4), dict(exp_avg=33 * P + 4),
                dict(param=32 * P)):
        assert call(bad) == INVALID, bad
    assert call({}, {}) == INVALID                      # the same weights twice
    nan, inf = float("nan"), float("inf")
    for how in (dict(lr=-1.0), dict(lr=nan), dict(lr=1e39), dict(weight_decay=-1.0), dict(weight_decay=inf), dict(beta1=1.0),
                dict(beta1=-0.1), dict(beta2=nan), dict(beta2=0.99999999999), dict(eps=0.0), dict(eps=1e-50), dict(eps=nan),
                dict(scale=0.0), dict(scale=inf), dict(max_norm=0.0), dict(max_norm=nan), dict(steps=None),
                dict(steps=P * 33 + 2), dict(norm=P * 32 + 1), dict(lr_factor=P * 40 + 2)):
        assert call({}, **how) == INVALID, how
    for count in (-1, (1 << 20) + 1):
        assert call({}, count=count) == INVALID
    assert L.reno_adamw_step(None, 1, ctypes.byref(reno.reno_adamw(**HOW)), None) == INVALID
    a = (reno.reno_parameter * 1)(reno.reno_parameter(**GOOD))
    assert L.reno_adamw_step(ctypes.addressof(a), 1, None, None) == INVALID


def test_sample_rejects_bad_arguments():
    L = reno.lib()
    good = dict(rows=4, symbols=100000, type=0, row_stride=100000, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0)

    def call(z=P, u=P, symbol=P, bits=P, **kw):
        return L.reno_sample_symbols(ctypes.byref(reno.reno_sample(**{**good, **kw})), z, u, symbol, bits, None)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(symbols=0), dict(symbols=(1 << 20) + 1, row_stride=1 << 21),
               dict(type=3), dict(row_stride=99999), dict(row_stride=1 << 31), dict(temperature=-1.0), dict(temperature=nan),
               dict(temperature=inf), dict(temperature=2.0 ** -127), dict(temperature=2.0 ** 127), dict(top_p=-0.1),
               dict(top_p=1.1), dict(top_p=nan), dict(min_p=-0.1), dict(min_p=1.1), dict(min_p=nan), dict(top_k=-1),
               dict(allowed=P, allowed_stride=99999), dict(allowed=P, allowed_stride=-1), dict(allowed=P, allowed_stride=1 << 31)):
        assert call(**kw) == INVALID, kw
        assert L.reno_last_error(None)
    for kw in (dict(z=None), dict(u=None), dict(symbol=None), dict(bits=None), dict(z=P + 2), dict(u=P + 1),
               dict(symbol=P + 2), dict(bits=P + 2), dict(temperature_rows=P + 2), dict(top_k_rows=P + 1),
               dict(top_p_rows=P + 2), dict(min_p_rows=P + 3)):
        assert call(**kw) == INVALID, kw
    assert call(rows=0, z=None, u=None, symbol=None, bits=None) == reno.RENO_OK
    assert L.reno_sample_symbols(None, P, P, P, P, None) == INVALID
