"""Rotary networks on the GPU against the oracle: every entry point of the handle, batches of other sizes,
captured graphs, and the operators called one after another from outside with the same result."""
import numpy as np
import pytest

import rotary_cases as R
from gpu_helpers import say, to_device
from oracle import decoder as O
from oracle import rotary as OR
from paper_2601_09921_amd import pwdec, synth
from test_emu_host import BF16_ATOL

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    before = torch.get_default_dtype()   # other modules may have left theirs
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def run(dec, fn, meas, types, k=1):
    m, t = to_device(meas, types)
    n = types.shape[0]
    logits = torch.full((n * k,), float("nan"), device="cuda")
    bits = torch.full((n * k,), 7, dtype=torch.uint8, device="cuda")
    getattr(dec, fn)(m, t, logits, bits)
    assert dec.sync_status() == pwdec.PWD_OK
    return logits.cpu().numpy().reshape((n, k) if k > 1 else (n,)), bits.cpu().numpy()


@pytest.mark.parametrize("c", R.CASES, ids=[c.name for c in R.CASES])
def test_decode(c):
    say(f"rotary {c.name}")
    wl, w = c.wl, c.weights(3)
    meas, types = synth.make_windows(wl, seed=4, realistic_boundaries=False)
    dec = pwdec.Decoder.from_workload(wl, w, rotary=c.options())
    ref, _ = OR.forward_windows(meas, types, w, wl.d, wl.H, c.oracle(), wl.grid, True)
    tol = BF16_ATOL if wl.dtype == R.BF16 else 1e-4 * np.abs(ref) + 1e-5
    got, bits = run(dec, "decode_recurrent", meas, types, wl.d)
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()
    assert np.array_equal(bits, (got.reshape(-1) > 0).astype(np.uint8))
    last, _ = run(dec, "decode", meas, types)
    assert np.array_equal(last, got[:, -1])
    # a window's result does not depend on its batch
    for n in (1, max(1, wl.B // 3)):
        part, _ = run(dec, "decode", meas[:n], types[:n])
        assert np.array_equal(part, last[:n])
    fixed, _ = run(dec, "decode_noalloc", meas, types)
    assert np.array_equal(fixed, last)
    dec.close()


def test_plain_options_agree_with_the_fused_kernels():
    """Without rotation, norm and window the network is the plain one: both decoders within the bf16 bound of
    each other's oracle, on the same weights."""
    wl = synth.WORKLOADS["d7"]
    w = synth.make_weights(wl, seed=5)
    meas, types = synth.make_windows(wl, B=40, seed=6)
    a, b = pwdec.Decoder.from_workload(wl, w, 40), pwdec.Decoder.from_workload(wl, w, 40, rotary=pwdec.rotary_dims())
    x, y = run(a, "decode", meas, types)[0], run(b, "decode", meas, types)[0]
    ref, _ = O.forward_windows(meas, types, w, wl.d, wl.H)
    assert np.abs(x - ref).max() <= BF16_ATOL and np.abs(y - ref).max() <= BF16_ATOL
    a.close(), b.close()


def test_stream_types_and_limits():
    c = R.CASES[5]
    wl, w = c.wl, c.weights(7)
    dec = pwdec.Decoder.from_workload(wl, w, 12, rotary=c.options())
    rng = np.random.default_rng(1)
    rounds = np.cumsum(rng.random((60, wl.N)) < 0.05, 0).astype(np.uint8) & 1
    bit, prob = torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
    logits = torch.zeros(9, device="cuda")
    dec.decode_stream(torch.from_numpy(synth.pack_bits(rounds).view(np.int32)).cuda(), bit, prob, logits)
    assert dec.sync_status() == pwdec.PWD_OK
    meas, types = O.split_stream(rounds, wl.d, wl.W)
    ref, _ = OR.forward_windows(meas, types, w, wl.d, wl.H, c.oracle())
    assert np.abs(logits.cpu().numpy() - ref).max() <= BF16_ATOL
    assert int(bit) == int(O.combine_bits((logits.cpu().numpy() > 0).astype(np.uint8)))
    types[2] = 5   # an invalid window: NaN, reported once, the others as before
    m, t = to_device(meas, types)
    out, bits = torch.zeros(9, device="cuda"), torch.zeros(9, dtype=torch.uint8, device="cuda")
    dec.decode(m, t, out, bits)
    assert dec.sync_status() == pwdec.PWD_EDEVICE and dec.sync_status() == pwdec.PWD_OK
    keep = np.arange(9) != 2
    assert np.isnan(out.cpu().numpy()[2]) and np.array_equal(out.cpu().numpy()[keep], logits.cpu().numpy()[keep])
    with pytest.raises(pwdec.PwdError):
        dec.schedule(pwdec.SCHEDULE_RESIDENT)
    dec.schedule(pwdec.SCHEDULE_LAYERS)
    dec.profile(True)
    types[2] = 1
    dec.decode(*to_device(meas, types), out, bits)
    assert set(dec.profile_read()) == {"embed_qkv", "post_qkv", "attention", "out_proj", "post", "readout"}
    dec.close()


def test_graph_replays():
    c = R.CASES[6]
    wl, w = c.wl, c.weights(8)
    meas, types = synth.make_windows(wl, seed=9)
    dec = pwdec.Decoder.from_workload(wl, w, rotary=c.options())
    want, _ = run(dec, "decode", meas, types)
    m, t = to_device(meas, types)
    logits, bits = torch.zeros(wl.B, device="cuda"), torch.zeros(wl.B, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dec.decode(m, t, logits, bits)
    for _ in range(3):
        logits.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(logits.cpu().numpy(), want)
        assert np.array_equal(run(dec, "decode", meas, types)[0], want)
    dec.close()
