"""Rotary networks decoded by the library's sources on the host SIMT stand-in, against the oracle; the
oracle itself against the plain decoder's where the options change nothing; and what their
configuration refuses."""
import ctypes
import os
import sys

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "emu"))

import rotary_cases as R  # noqa: E402
import run_emu  # noqa: E402
from oracle import decoder as O  # noqa: E402
from oracle import rotary as OR  # noqa: E402
from paper_2601_09921_amd import pwdec, synth  # noqa: E402
from test_emu_host import BF16_ATOL, emu  # noqa: E402,F401


def test_oracle_without_options_is_the_decoder():
    c = R.CASES[-1]
    wl = R.wl(5, 7, 3, 32, 2, 4, R.F32)
    w = synth.make_weights(wl, seed=1)
    meas, types = synth.make_windows(wl, seed=2)
    rot = dict(pairs=(0, 0), theta=100.0, qk_norm=False, norm_eps=0.0, window=-1, sinks=0)
    a, _ = OR.forward_windows(meas, types, w, 5, 4, rot)
    b, _ = O.forward_windows(meas, types, w, 5, 4)
    assert np.abs(a - b).max() < 1e-12 and c.window == -1


def test_rotation_is_relative():
    """Scores depend on row and column differences only: a shift of every cell leaves attention as it is."""
    rng = np.random.default_rng(0)
    lw = {k: rng.standard_normal((16, 16)) for k in ("Wq", "Wk", "Wv", "Wo")}
    lw.update({k: rng.standard_normal(16) for k in ("bq", "bk", "bv", "bo")})
    rot = dict(pairs=(2, 2), theta=50.0, qk_norm=False, norm_eps=0.0, window=-1, sinks=0)
    X, cells = rng.standard_normal((2, 5, 16)), [(0, 1), (1, 0), (1, 1), (2, 3), (3, 2)]
    a = OR.attention(X, lw, 2, cells, rot)
    assert np.abs(a - OR.attention(X, lw, 2, [(r + 7, c + 3) for r, c in cells], rot)).max() < 1e-12
    assert np.abs(a - OR.attention(X, lw, 2, [(2 * r, c) for r, c in cells], rot)).max() > 1e-3


def create(lib, c, blob, n):
    wl = c.wl
    g = pwdec.geometry(wl.d, wl.W, n)
    m = pwdec.dims(wl.D, wl.L, wl.H, wl.mlp_ratio, wl.dtype, int(wl.grid), int(wl.resnet))
    h, buf, r = ctypes.c_void_p(), ctypes.create_string_buffer(blob, len(blob)), c.options()
    return lib.decoder_create_rotary(ctypes.byref(g), ctypes.byref(m), ctypes.byref(r), buf, len(blob), ctypes.byref(h)), h


def blob_of(c, w):
    wl = c.wl
    return pwdec.make_blob(wl.d, wl.W, wl.D, wl.L, wl.H, wl.F, wl.dtype, w, int(wl.grid), c.options())


@pytest.mark.parametrize("c", R.SMALL, ids=[c.name for c in R.SMALL])
@pytest.mark.parametrize("call", ["decode_windows", "decode_windows_recurrent", "decode_windows_noalloc"])
def test_decode(emu, c, call):  # noqa: F811
    wl = c.wl
    w = c.weights(3)
    meas, types = synth.make_windows(wl, seed=4, realistic_boundaries=False)
    rc, h = create(emu, c, blob_of(c, w), wl.B)
    assert rc == 0, emu.decoder_last_error()
    rec = call == "decode_windows_recurrent"
    k = wl.d if rec else 1
    bufs = [run_emu.Buf(emu, a) for a in (synth.pack_bits(meas).view(np.uint32), types.astype(np.uint8),
                                          np.full(wl.B * k, np.nan, np.float32), np.full(wl.B * k, 7, np.uint8))]
    vp = ctypes.c_void_p
    assert getattr(emu, call)(h, vp(bufs[0].ptr), vp(bufs[1].ptr), wl.B, vp(bufs[2].ptr), vp(bufs[3].ptr), None) == 0
    assert emu.decoder_sync_status(h, None) == 0 and emu.emu_errors() == 0
    ref, _ = OR.forward_windows(meas, types, w, wl.d, wl.H, c.oracle(), wl.grid, rec)
    got = bufs[2].get().reshape(ref.shape)
    tol = BF16_ATOL if wl.dtype == R.BF16 else 1e-4 * np.abs(ref) + 1e-5
    assert (np.abs(got - ref) <= tol).all(), (got, ref)
    assert np.array_equal(bufs[3].get().reshape(ref.shape), (got > 0).astype(np.uint8))
    emu.decoder_destroy(h)
    for b in bufs:
        b.free()


def validate(d=5, W=10, B=4, D=192, L=2, H=8, r=5, dt=1, ts=0, emb=0, dil=(0, 0, 0), **rot):
    lib = pwdec.load_library()
    g, m = pwdec.geometry(d, W, B), pwdec.dims(D, L, H, r, dt, ts, emb, dil)
    return lib.decoder_validate_rotary(ctypes.byref(g), ctypes.byref(m), ctypes.byref(pwdec.rotary_dims(**rot)))


@pytest.mark.parametrize("kw", [dict(), dict(pairs=(6, 6)), dict(pairs=(0, 12)), dict(D=1024, H=4), dict(D=16, H=1), dict(dt=0, D=80, H=20),
                                dict(d=63, W=63, D=64), dict(d=45, W=90, ts=1), dict(window=0), dict(window=5, sinks=900), dict(emb=1, qk_norm=True)])
def test_supported(kw):
    assert validate(**kw) == pwdec.PWD_OK


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=2), -2), (dict(dt=3), -2), (dict(D=200), -2), (dict(D=1040, H=5), -2), (dict(D=0, H=1), -2), (dict(D=96, H=8, dt=1, r=3), -2),
    (dict(H=16), -2), (dict(D=512, H=1), -2), (dict(ts=1, dil=(1, 2, 4)), -2), (dict(d=4), -2), (dict(W=40), -2), (dict(H=0), -2),
    (dict(pairs=(7, 6)), -1), (dict(pairs=(-1, 2)), -1), (dict(theta=0.0), -1), (dict(theta=float("nan")), -1), (dict(norm_eps=-1.0), -1),
    (dict(window=-2), -1), (dict(window=3, sinks=-1), -1), (dict(B=1 << 24), -2)])
def test_refused(kw, rc):
    assert validate(**kw) == rc
    assert pwdec.load_library().decoder_last_error()


def test_blob_checks():
    """The gains are counted, the header's rotary words and the size are checked before any device use."""
    lib, c = pwdec.load_library(), R.SMALL[0]
    wl, w = c.wl, c.weights(1)
    blob = blob_of(c, w)
    g, m = pwdec.geometry(wl.d, wl.W, 2), pwdec.dims(wl.D, wl.L, wl.H, wl.mlp_ratio, wl.dtype)
    n = lib.decoder_rotary_blob_floats(ctypes.byref(g), ctypes.byref(m), ctypes.byref(c.options()))
    assert len(blob) == 64 + 4 * n and n == lib.decoder_blob_floats(ctypes.byref(g), ctypes.byref(m)) + wl.L * 2 * wl.D // wl.H
    for bad in (blob[:-4], blob[:56] + b"\1\0\0\0" + blob[60:], blob[:60] + b"\0\0\0\0" + blob[64:]):
        rc, h = create(lib, c, bad, 2)
        assert rc == pwdec.PWD_EBLOB and not h.value
    assert lib.decoder_create_rotary(ctypes.byref(g), ctypes.byref(m), None, blob, len(blob), None) == pwdec.PWD_EINVAL
    assert lib.decoder_validate_rotary(ctypes.byref(g), ctypes.byref(m), None) == pwdec.PWD_EINVAL
    assert lib.decoder_rotary_blob_floats(None, None, None) == 0
