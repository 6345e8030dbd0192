"""The transformer operators' kernels on the host SIMT stand-in, every buffer fenced at its last byte
(EMU_GUARD=start fences the first), against the float64 oracle: odd sizes, strided rows, lengths, windows,
sinks, empty rows, cells that must stay as they were."""
import ctypes
import os
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "emu"))

import operator_cases as C  # noqa: E402
import run_emu  # noqa: E402
from oracle import operators as O  # noqa: E402
from paper_2601_09921_amd import pwdec  # noqa: E402
from test_emu_host import emu  # noqa: E402,F401

CODE = {"fp32": pwdec.DTYPE_F32, "bf16": pwdec.DTYPE_BF16}


def buf(lib, a, dtype):
    return run_emu.Buf(lib, C.to_bf16_bits(a) if dtype == "bf16" else np.ascontiguousarray(a, np.float32))


def back(b, dtype):
    return C.from_bf16_bits(b.get()) if dtype == "bf16" else b.get()


def pad_rows(a, pad, fill=np.nan):
    """Rows of a wider buffer that ends with the last row's last element."""
    w = np.full((a.shape[0], a.shape[1] + pad), fill, a.dtype)
    w[:, :a.shape[1]] = a
    return w.reshape(-1)[:w.size - pad] if a.size else w.reshape(-1)


@pytest.mark.parametrize("dtype,out,act,pad", [("bf16", "bf16", "relu", 0), ("bf16", "fp32", "gelu", 3), ("fp32", "fp32", "silu", 0),
                                               ("bf16", "bf16", "none", 8), ("fp32", "bf16", "gelu_tanh", 1)])
@pytest.mark.parametrize("m,n,k", C.LINEAR_SHAPES)
def test_linear(emu, m, n, k, dtype, out, act, pad):  # noqa: F811
    c = C.linear_inputs(m, n, k, dtype, out, pad != 8, pad != 1, m + n + k)
    x, w = buf(emu, pad_rows(c["x"], pad), dtype), buf(emu, pad_rows(c["w"], pad), dtype)
    b = buf(emu, c["bias"], "fp32") if c["bias"] is not None else None
    r = buf(emu, c["residual"], out) if c["residual"] is not None else None
    y = buf(emu, pad_rows(np.full((m, n), 7.0, np.float32), pad, 7.0), out)
    a = pwdec.LinearArgs(m, n, k, x.ptr, k + pad, w.ptr, k + pad, b and b.ptr, r and r.ptr, n, y.ptr, n + pad,
                         CODE[dtype], CODE[out], pwdec.ACTIVATIONS[act])
    need = emu.pwd_linear_workspace(ctypes.byref(a))
    ws = run_emu.Buf(emu, np.full(max(need, 1), 0xff, np.uint8))
    a.d_workspace, a.workspace_bytes = ws.ptr, need
    assert emu.pwd_linear(ctypes.byref(a), None) == 0, emu.decoder_last_error()
    assert emu.emu_errors() == 0
    got = np.full(m * (n + pad), 7.0, np.float32)
    flat = back(y, out)
    got[:flat.size] = flat
    got = got.reshape(m, n + pad)
    assert (got[:, n:] == 7.0).all()
    ref, mag = O.linear(c["x"], c["w"], c["bias"], act, c["residual"])
    C.check(got[:, :n], ref, C.linear_bound(ref, mag, k, act, out, c["residual"]), "linear")
    for q in (x, w, b, r, y, ws):
        if q is not None:
            q.free()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("t,hq,hk,dh,pairs,layout,shared", C.ROPE_SHAPES)
def test_rope(emu, t, hq, hk, dh, pairs, layout, shared, norm, dtype):  # noqa: F811
    rng = np.random.default_rng(dh + t)
    qkv = C.values(rng, (t, hq + hk + 1, dh), dtype)
    pos = rng.integers(-5, 1 << 20, (t, max(len(pairs), 1))).astype(np.int32)
    gains = [(1 + 0.2 * rng.standard_normal(dh)).astype(np.float32) for _ in range(2)]
    src, pb = buf(emu, qkv, dtype), run_emu.Buf(emu, pos)
    gb = [buf(emu, g, "fp32") for g in gains]
    ko = buf(emu, np.zeros((t, hk, dh), np.float32), dtype)
    es = 2 if dtype == "bf16" else 4
    a = pwdec.RopeArgs(t, hq, hk, dh, CODE[dtype])
    row = (hq + hk + 1) * dh
    # queries in place inside the packed buffer, keys into one of their own
    a.d_q, a.q_token_stride, a.q_head_stride = src.ptr, row, dh
    a.d_q_out, a.q_out_token_stride, a.q_out_head_stride = src.ptr, row, dh
    a.d_k, a.k_token_stride, a.k_head_stride = src.ptr + hq * dh * es, row, dh
    a.d_k_out, a.k_out_token_stride, a.k_out_head_stride = ko.ptr, hk * dh, dh
    a.d_positions, a.axes, a.pairs = (pb.ptr if pairs else None), len(pairs), (ctypes.c_int32 * 3)(*pairs)
    a.layout, a.frequencies, a.inverse, a.theta = pwdec.ROPE_LAYOUTS[layout], int(shared), int(not norm and hk == 2), 500.0
    if norm:
        rc = emu.pwd_qk_norm_rope(ctypes.byref(a), gb[0].ptr, None, 1e-5, None)
    else:
        rc = emu.pwd_rope(ctypes.byref(a), None)
    assert rc == 0 and emu.emu_errors() == 0, emu.decoder_last_error()
    got = back(src, dtype)
    assert np.array_equal(got[:, hq:], qkv[:, hq:])
    for x, y, gain in ((qkv[:, :hq], got[:, :hq], gains[0]), (qkv[:, hq:hq + hk], back(ko, dtype), np.ones(dh))):
        z = O.rms_norm(x, gain, 1e-5) if norm else x
        ref = O.rope(z, pos, pairs, 500.0, layout, shared, bool(a.inverse))
        C.check(y, ref, C.rope_bound(ref, z, dtype, pairs, layout, gain if norm else None, dh), "rope")
    for q in (src, pb, ko, *gb):
        q.free()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("b,sq,sk,hq,hk,dh,window,sinks,ql,kl", C.ATTENTION_SHAPES)
def test_attention(emu, b, sq, sk, hq, hk, dh, window, sinks, ql, kl, dtype):  # noqa: F811
    rng = np.random.default_rng(sq + sk + dh)
    q = C.values(rng, (b, sq, hq, dh), dtype)
    k, v = C.values(rng, (b, sk, hk, dh), dtype), C.values(rng, (b, sk, hk, dh), dtype)
    hold_k, hold_v = k.copy(), v.copy()
    for s in range(b):   # what lies past a sequence's keys must not matter
        if kl is not None:
            hold_k[s, kl[s]:], hold_v[s, kl[s]:] = np.nan, np.inf
        seen = C.seen_keys(sq if ql is None else ql[s], sk if kl is None else kl[s], sk, window, sinks)
        hold_k[s, ~seen], hold_v[s, ~seen] = np.inf, np.nan   # nor keys that no query sees
    bufs = [buf(emu, t, dtype) for t in (q, hold_k, hold_v, np.full(q.shape, 7.0, np.float32))]
    lens = [run_emu.Buf(emu, np.array(n, np.int32)) if n is not None else None for n in (ql, kl)]
    a = pwdec.AttentionArgs(b, sq, sk, hq, hk, dh, CODE[dtype])
    for name, t, h, n in (("q", bufs[0], hq, sq), ("k", bufs[1], hk, sk), ("v", bufs[2], hk, sk), ("out", bufs[3], hq, sq)):
        setattr(a, f"d_{name}", t.ptr)
        setattr(a, f"{name}_stride", (ctypes.c_int64 * 3)(n * h * dh, h * dh, dh))
    a.d_q_lengths, a.d_k_lengths = (t.ptr if t else None for t in lens)
    a.window_left, a.window_right, a.sinks, a.scale = *window, sinks, dh ** -0.5
    need = emu.pwd_attention_workspace(ctypes.byref(a))
    ws = run_emu.Buf(emu, np.full(max(need, 1), 0xff, np.uint8))
    a.d_workspace, a.workspace_bytes = ws.ptr, need
    assert emu.pwd_attention(ctypes.byref(a), None) == 0, emu.decoder_last_error()
    assert emu.emu_errors() == 0
    ref, mag, top = O.attention(q, k, v, *window, sinks, None, ql, kl)
    got = back(bufs[3], dtype)
    untouched = np.isnan(ref)
    assert (got[untouched] == 7.0).all()
    bound = C.attention_bound(ref, mag, top, dtype, dh, sk)
    C.check(np.where(untouched, 0, got), np.where(untouched, 0, ref), np.where(untouched, 0, bound), "attention")
    for t in (*bufs, ws, *lens):
        if t is not None:
            t.free()
