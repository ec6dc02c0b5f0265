"""Bounded views of the prefix on the CPU: refusals of the C ABI and of the binding,
the host code under sanitizers, and the oracle against brute force."""

import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import oracle
import paper_2609_19868_amd as Z
from paper_2609_19868_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_19868_amd", "csrc")


def _hipcc():
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    return None


def test_host_code_under_sanitizers(tmp_path):
    hipcc = _hipcc()
    if hipcc is None:
        pytest.skip("hipcc is not available")
    exe = str(tmp_path / "view_harness")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           *(os.path.join(CSRC, f) for f in ("api.hip", "api_view.hip", "mdm_plan.hip")),
           "-x", "hip", os.path.join(ROOT, "tests", "host", "view_harness.cpp"), "-o", exe]
    b = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert b.returncode == 0, b.stdout[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout[-5000:]
    assert "Sanitizer" not in r.stdout and " 0 failures" in r.stdout, r.stdout[-3000:]


# ------------------------------------------------------------------ refusals

INV, UNS, WS = _lib.ERR_INVALID_ARGUMENT, _lib.ERR_UNSUPPORTED, _lib.ERR_WORKSPACE_TOO_SMALL
P = ctypes.c_void_p(4096)


def _desc(**kw):
    base = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, prefix_len=3000, kv_capacity=3008, n_slots=1,
                slot_len=1, softmax_scale=0.088, pass_=0, cross_slot=0, dtype=1, prefix_splits=0)
    base.update(kw)
    return _lib.SlotAttnDesc(**base)


def _window(desc, win, ptrs=None, ws=P, ws_bytes=1 << 40):
    a = [P, P, P, P, P, None, None, P, None]
    for i, v in (ptrs or {}).items():
        a[i] = v
    w = None if win is None else ctypes.byref(_lib.AttnWindow(*win))
    return _lib.lib().zarya_slot_attn_window(ctypes.byref(desc) if desc else None, w, *a, ws, ws_bytes, None)


def _q4(desc, win, ptrs=None, ws=P, ws_bytes=1 << 40):
    a = [P, P, P, P, P, P, P, None, None, P, None]
    for i, v in (ptrs or {}).items():
        a[i] = v
    w = None if win is None else ctypes.byref(_lib.AttnWindow(*win))
    return _lib.lib().zarya_slot_attn_q4(ctypes.byref(desc) if desc else None, w, *a, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), INV), (dict(n_q_heads=3), INV), (dict(kv_capacity=50), INV), (dict(softmax_scale=0.0), INV),
    (dict(pass_=2), INV), (dict(cross_slot=5), INV), (dict(dtype=7), INV), (dict(prefix_splits=65), INV),
    (dict(head_dim=96), UNS), (dict(batch=1 << 20, n_q_heads=64, n_kv_heads=64), UNS),
    (dict(batch=1, n_q_heads=1, n_kv_heads=1, prefix_len=2**31 - 1, kv_capacity=2**31 - 1), UNS),
])
def test_attention_rejects_bad_descriptors(bad, code):
    n = ctypes.c_size_t(0)
    for call, size in ((_window, _lib.lib().zarya_slot_attn_window_workspace_size),
                       (_q4, _lib.lib().zarya_slot_attn_q4_workspace_size)):
        d = _desc(**bad)
        assert call(d, (5, 0)) == code
        assert len(_lib.lib().zarya_last_error()) > 0
        assert size(ctypes.byref(d), ctypes.byref(_lib.AttnWindow(5, 0)), ctypes.byref(n)) == code


def test_attention_rejects_bad_windows():
    for win in ((-1, 0), (5, -1), (-2**31, 0)):
        assert _window(_desc(), win) == INV and _q4(_desc(), win) == INV
    assert _window(_desc(), (0, 0)) == INV and _window(_desc(), None) == INV  # a window is what the call is for
    n = ctypes.c_size_t(0)
    L, d = _lib.lib(), ctypes.byref(_desc())
    assert L.zarya_slot_attn_window_workspace_size(d, None, ctypes.byref(n)) == INV
    assert L.zarya_slot_attn_q4_workspace_size(d, None, ctypes.byref(n)) == _lib.OK and n.value > 0
    assert L.zarya_slot_attn_q4_workspace_size(d, None, None) == INV
    assert L.zarya_slot_attn_q4_workspace_size(None, None, ctypes.byref(n)) == INV


def test_attention_rejects_missing_misaligned_and_short_buffers():
    odd = ctypes.c_void_p(4096 + 8)
    for i in (0, 1, 2, 3, 4, 7):
        assert _window(_desc(), (5, 0), {i: None}) == INV
        assert _window(_desc(), (5, 0), {i: odd}) == INV
    for i in (0, 1, 2, 3, 4, 5, 6, 9):
        assert _q4(_desc(), None, {i: None}) == INV
        if i not in (2, 4):
            assert _q4(_desc(), None, {i: odd}) == INV
    for i in (2, 4):  # a row of scales is D/32 bytes
        for D, by in ((128, 1), (128, 2), (64, 1)):
            assert _q4(_desc(head_dim=D), None, {i: ctypes.c_void_p(4096 + by)}) == INV
    need = _lib.slot_attn_q4_workspace_size(_desc())
    assert need > 0
    assert _q4(_desc(), None, ws_bytes=need - 1) == WS
    assert _q4(_desc(), None, ws=None, ws_bytes=need) == INV
    assert _q4(_desc(), None, ws=odd, ws_bytes=need) == INV
    d = _desc(prefix_len=20000, kv_capacity=20000)
    need = _lib.slot_attn_window_workspace_size(d, _lib.AttnWindow(9000, 4))
    assert need > 0 and _window(d, (9000, 4), ws_bytes=need - 1) == WS
    # a short window needs no splits, and none of the workspace that the prefix would
    assert _lib.slot_attn_window_workspace_size(d, _lib.AttnWindow(10, 4)) == 0


@pytest.mark.parametrize("shape", [
    dict(batch=1, n_q_heads=4, n_kv_heads=1, n_slots=2, slot_len=16, head_dim=64, cross_slot=0),
    dict(batch=1, n_q_heads=20, n_kv_heads=4, n_slots=2, slot_len=8, head_dim=128, cross_slot=1),
])
def test_workspace_of_the_longest_prefix_serves_all(shape):
    """At every length: where two numbers of splits cost the same to a nanosecond, a
    longer prefix must not fall back to the smaller one."""
    sizes = [_lib.slot_attn_q4_workspace_size(_desc(prefix_len=n, kv_capacity=20000, **shape)) for n in range(0, 20000)]
    assert sizes[-1] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), INV), (dict(n_kv_heads=0), INV), (dict(n_rows=-1), INV), (dict(kv_capacity=-1, n_rows=0), INV),
    (dict(dtype=5), INV), (dict(n_rows=4097), INV), (dict(head_dim=80), UNS),
    (dict(batch=4096, n_kv_heads=64, kv_capacity=1 << 14), UNS), (dict(batch=1 << 20, n_kv_heads=1 << 20), UNS),
])
def test_quantize_rejects_bad_descriptors(bad, code):
    base = dict(batch=2, n_kv_heads=8, head_dim=128, kv_capacity=4096, n_rows=100, dtype=1)
    base.update(bad)
    d = _lib.KvQ4Desc(**base)
    L = _lib.lib()
    assert L.zarya_kv_quantize(ctypes.byref(d), P, P, None, None, P, P, P, P, None) == code
    assert L.zarya_kv_dequantize(ctypes.byref(d), P, P, P, P, None, P, P, None) == code
    assert len(L.zarya_last_error()) > 0


def test_quantize_and_append_require_every_tensor():
    L, odd = _lib.lib(), ctypes.c_void_p(4096 + 4)
    d = _lib.KvQ4Desc(batch=2, n_kv_heads=8, head_dim=128, kv_capacity=4096, n_rows=100, dtype=1)
    for i in range(6):
        for value in (None, odd):
            a = [P] * 6
            a[i] = value
            want = INV if value is None or i in (0, 1, 2, 4) else None  # scales are written by the byte
            if want is None:
                continue
            assert L.zarya_kv_quantize(ctypes.byref(d), a[0], a[1], None, None, *a[2:], None) == want
            assert L.zarya_kv_dequantize(ctypes.byref(d), *a[2:], None, a[0], a[1], None) == want
    assert L.zarya_kv_quantize(None, P, P, None, None, P, P, P, P, None) == INV
    d = _lib.KvAppendDesc(batch=2, n_kv_heads=8, head_dim=128, kv_capacity=4096, n_slots=8, slot_len=8, dtype=1)
    for i in range(9):
        a = [P] * 9
        a[i] = None
        assert L.zarya_kv_append_q4(ctypes.byref(d), *a, None) == INV
    for bad, code in ((dict(n_slots=1025, slot_len=1), UNS), (dict(batch=65536), INV), (dict(head_dim=32), UNS)):
        base = dict(batch=2, n_kv_heads=8, head_dim=128, kv_capacity=4096, n_slots=8, slot_len=8, dtype=1)
        base.update(bad)
        d = _lib.KvAppendDesc(**base)
        assert L.zarya_kv_append_q4(ctypes.byref(d), *[P] * 9, None) == code


def test_binding_refusals():
    q = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    cache = Z.q4_cache(1, 2, 8, 64, "cpu")
    assert [tuple(t.shape) for t in cache] == [(1, 2, 8, 32), (1, 2, 8, 2), (1, 2, 8, 32), (1, 2, 8, 2)]
    for call in (lambda: Z.slot_attn_q4(q, cache, q, q, 1, 1), lambda: Z.kv_quantize(q, q, cache),
                 lambda: Z.kv_dequantize(cache), lambda: Z.slot_attn(q, q, q, q, q, 1, 1, window=3),
                 lambda: Z.kv_append_q4(cache, torch.zeros(1, dtype=torch.int32), q, q,
                                        torch.zeros(1, 1, 1, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32))):
        with pytest.raises(ValueError, match="cuda"):
            call()
    with pytest.raises(ValueError, match="sinks need a window"):
        Z._window(None, 4)
    with pytest.raises(ValueError, match="32 bits"):
        Z._window(2**32 + 5, 0)
    with pytest.raises(ValueError, match="32 bits"):
        Z._window(5, 2**31)
    assert Z._window(None, 0) is None and (Z._window(7, 2).window, Z._window(7, 2).sinks) == (7, 2)


# ------------------------------------------------------------- the oracle's pins


def test_oracle_window_against_loops():
    """Visibility decided key by key from the places, and the whole prefix without a window."""
    rng = np.random.default_rng(0)
    for _ in range(200):
        P_, S, L = int(rng.integers(0, 12)), int(rng.integers(1, 4)), int(rng.integers(1, 5))
        pass_, cross = int(rng.integers(0, 2)), int(rng.integers(0, 2))
        w, sinks = int(rng.integers(1, 20)), int(rng.integers(0, 15))
        got = oracle.window_visibility(P_, S, L, pass_, cross, None, w, sinks)
        base = oracle.visibility(P_, S, L, pass_, cross)
        assert np.array_equal(oracle.window_visibility(P_, S, L, pass_, cross, None, None, 0), base)
        for t in range(S * L):
            assert got[t, P_ + t]  # no token loses itself
            for j in range(P_ + S * L):
                assert got[t, j] == (base[t, j] and (j < sinks or P_ + t - j < w))


def test_oracle_attention_is_slot_attention_without_a_window():
    rng = np.random.default_rng(1)
    q, kc, vc = (rng.standard_normal(s) for s in ((2, 4, 6, 8), (2, 2, 9, 8), (2, 2, 9, 8)))
    ks, vs = (rng.standard_normal((2, 2, 6, 8)) for _ in range(2))
    for pass_ in (0, 1):
        O, L, A = oracle.view_attention(q, kc, vc, ks, vs, [9, 4], 2, 3, 0.3, pass_)
        O2, L2 = oracle.slot_attention(q, kc, vc, ks, vs, [9, 4], 2, 3, 0.3, pass_)
        assert np.allclose(O, O2, atol=1e-12) and np.allclose(L, L2, atol=1e-12) and np.all(A >= np.abs(O) - 1e-12)


def test_oracle_quantizer_by_search():
    """For every block the scale is the smallest that holds it, and every code the nearest
    by a scalar search; a block's relative error stays within half a step of its largest."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((40, 32)) * np.exp(4 * rng.standard_normal((40, 1)))
    x[0, :] = 7.0 * 2.0 ** 3
    x[1, :] = np.nextafter(7.0, 0) * 2.0 ** 3
    codes, scales = oracle.q4_quantize(x)
    back = oracle.q4_dequantize(codes, scales)
    assert scales[0, 0] == 127 + 4 and scales[1, 0] == 127 + 3
    for i in range(40):
        unit = 2.0 ** (int(scales[i, 0]) - 127)
        top = np.abs(x[i]).max()
        assert top / unit < 7 and top / (unit / 2) >= 7
        for j in range(32):
            best = min(abs(abs(x[i, j]) / unit - m) for m in oracle.view.Q4_MAGNITUDES)
            assert math.isclose(abs(back[i, j] - x[i, j]) / unit, best, rel_tol=1e-9, abs_tol=1e-12)
    assert np.abs(back - x).max(1).max() <= 1.0 * 2.0 ** (scales.max() - 127.0)
    # every code, and what has no value
    c = np.arange(16, dtype=np.uint8)
    codes = (np.resize(c, 32)[0::2] | (np.resize(c, 32)[1::2] << 4))[None]
    v = oracle.q4_dequantize(codes, np.array([[128]], np.uint8))[0]
    assert v[:8].tolist() == [0, 1, 2, 3, 4, 6, 8, 12] and v[9:16].tolist() == [-1, -2, -3, -4, -6, -8, -12]
    assert np.isnan(oracle.q4_dequantize(codes, np.array([[255]], np.uint8))).all()
    x[5, 3], x[6, 0] = np.nan, np.inf
    assert oracle.q4_quantize(x)[1][[5, 6], 0].tolist() == [255, 255]
