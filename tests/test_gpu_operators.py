"""The transformer operators on the GPU, through the binding, against the float64 oracle: the sizes of
the CPU runs and larger ones that reach every kernel, strided operands, in-place calls, streams,
captured graphs, refusals, and a run of them together as a layer uses them."""
import numpy as np
import pytest

import operator_cases as C
from gpu_helpers import say
from oracle import operators as O
from paper_2601_09921_amd import pwdec

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    before = torch.get_default_dtype()   # other modules may have left theirs
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(before)


def dev(a, dtype=None):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.to(DT[dtype]) if dtype else t


def host(t):
    return t.double().cpu().numpy()


def strided(a, dtype, pad):
    """The same values as columns of a wider buffer, NaN around them."""
    t = torch.full((a.shape[0], a.shape[1] + pad), float("nan"), dtype=DT[dtype], device="cuda")
    t[:, :a.shape[1]] = dev(a, dtype)
    return t[:, :a.shape[1]]


BIG = [(300, 200, 1000), (1, 1000, 4096), (48, 512, 2050), (129, 1024, 4096), (513, 257, 130), (1500, 2048, 192), (4100, 1031, 65),
       (2560, 2560, 128), (4096, 4100, 70)]


@pytest.mark.parametrize("dtype,out,act,pad", [("bf16", "bf16", "relu", 0), ("bf16", "fp32", "gelu", 3), ("fp32", "fp32", "silu", 0),
                                               ("bf16", "bf16", "none", 8), ("fp32", "bf16", "gelu_tanh", 1)])
@pytest.mark.parametrize("m,n,k", C.LINEAR_SHAPES + BIG)
def test_linear(m, n, k, dtype, out, act, pad):
    say(f"linear {m} {n} {k} {dtype} {out} {act} {pad}")
    c = C.linear_inputs(m, n, k, dtype, out, pad != 8, pad != 1, m + n + k)
    x, w = strided(c["x"], dtype, pad), strided(c["w"], dtype, pad)
    whole = torch.full((m, n + pad), 7.0, dtype=DT[out], device="cuda")
    pwdec.linear(x, w, whole[:, :n], bias=dev(c["bias"]), activation=act,
                 residual=dev(c["residual"], out) if c["residual"] is not None else None)
    got = host(whole)
    assert (got[:, n:] == 7.0).all()
    ref, mag = O.linear(c["x"], c["w"], c["bias"], act, c["residual"])
    C.check(got[:, :n], ref, C.linear_bound(ref, mag, k, act, out, c["residual"]), "linear")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("t,hq,hk,dh,pairs,layout,shared", C.ROPE_SHAPES + [(3000, 8, 8, 32, (8, 8), "half", False),
                                                                             (999, 7, 1, 48, (7, 8, 9), "half", True)])
def test_rope(t, hq, hk, dh, pairs, layout, shared, norm, dtype):
    say(f"rope {t} {hq} {hk} {dh} {pairs} {layout} {norm} {dtype}")
    rng = np.random.default_rng(dh + t)
    qkv = C.values(rng, (t, hq + hk + 1, dh), dtype)
    pos = rng.integers(-(1 << 30), 1 << 30, (t, len(pairs))).astype(np.int32)
    gain = (1 + 0.2 * rng.standard_normal(dh)).astype(np.float32)
    buf = dev(qkv, dtype)
    q, k = buf[:, :hq], buf[:, hq:hq + hk] if hk else None
    k_out = torch.empty(t, hk, dh, dtype=DT[dtype], device="cuda") if hk else None
    p, kw = dev(pos) if pairs else None, dict(pairs=pairs, theta=500.0, layout=layout, frequencies="shared" if shared else "axis")
    inverse = not norm and hk == 2
    if norm:
        pwdec.qk_norm_rope(q, k, dev(gain), None, p, eps=1e-5, k_out=k_out, **kw)
    else:
        pwdec.rope(q, k, p, inverse=inverse, k_out=k_out, **kw)
    got = host(buf)
    assert np.array_equal(got[:, hq:], qkv[:, hq:])
    for x, y, g in ((qkv[:, :hq], got[:, :hq], gain), (qkv[:, hq:hq + hk], host(k_out) if hk else None, np.ones(dh))):
        if y is None:
            continue
        z = O.rms_norm(x, g, 1e-5) if norm else x
        ref = O.rope(z, pos, pairs, 500.0, layout, shared, inverse)
        C.check(y, ref, C.rope_bound(ref, z, dtype, pairs, layout, g if norm else None, dh), "rope")


def test_rope_inverse_undoes_the_rotation():
    """Rotated and rotated back, fp32: each way is within the bound of its own."""
    rng = np.random.default_rng(5)
    x = C.values(rng, (50, 3, 64), "fp32")
    pos = rng.integers(0, 1 << 20, (50, 3)).astype(np.int32)
    q = dev(x)
    pwdec.rope(q, None, dev(pos), (10, 11, 11))
    assert np.abs(host(q) - x).max() > 0.5
    pwdec.rope(q, None, dev(pos), (10, 11, 11), inverse=True)
    C.check(host(q), x.astype(np.float64), 4 * C.rope_bound(x.astype(np.float64), x, "fp32", (10, 11, 11), "half"))


def test_rope_of_keys_alone():
    """Keys without queries, one axis given as [tokens], against the same call with both."""
    rng = np.random.default_rng(6)
    x, pos = C.values(rng, (9, 2, 32), "bf16"), dev(rng.integers(0, 99, 9).astype(np.int32))
    a, b, c = dev(x, "bf16"), dev(x, "bf16"), torch.empty(9, 2, 32, dtype=torch.bfloat16, device="cuda")
    pwdec.rope(a, b, pos, (16,))
    pwdec.rope(None, c.copy_(dev(x, "bf16")), pos[:, None], (16,))
    assert torch.equal(a, b) and torch.equal(a, c)
    g = torch.ones(32, device="cuda")
    pwdec.qk_norm_rope(None, c.copy_(dev(x, "bf16")), None, g, pos, (16,))
    pwdec.qk_norm_rope(a.copy_(dev(x, "bf16")), None, None, None, pos, (16,))
    assert torch.equal(a, c)


def test_offsets_past_32_bits():
    """Rows, tokens and sequences more than 2^31 elements into their buffers."""
    rng = np.random.default_rng(8)
    big = torch.empty((1 << 31) + (1 << 22), dtype=torch.bfloat16, device="cuda")   # 4 GB, each row at a stride
    ld = 1 << 21
    for m in (40, 1025):   # the kernel for few rows, and the tiles
        x = big.as_strided((m, 64), (ld if m > 64 else (1 << 31) // 39, 1))
        a, w = C.values(rng, (m, 64), "bf16"), C.values(rng, (30, 64), "bf16")
        x.copy_(dev(a, "bf16"))
        y = torch.empty(m, 30, device="cuda")
        pwdec.linear(x, dev(w, "bf16"), y)
        ref, mag = O.linear(a, w)
        C.check(host(y), ref, C.linear_bound(ref, mag, 64, "none", "fp32", None))
        out = big.as_strided((m, 64), (ld if m > 64 else (1 << 31) // 39, 1))
        pwdec.linear(dev(a, "bf16"), dev(np.eye(64, dtype=np.float32), "bf16"), out)
        assert torch.equal(out, dev(a, "bf16"))
    t = C.values(rng, (3, 2, 32), "bf16")
    q = big.as_strided((3, 2, 32), (1 << 30, 32, 1))
    q.copy_(dev(t, "bf16"))
    pos = np.array([[3], [5], [1 << 20]], np.int32)
    pwdec.rope(q, None, dev(pos), (16,))
    ref = O.rope(t, pos, (16,))
    C.check(host(q), ref, C.rope_bound(ref, t, "bf16", (16,), "half"))
    kv, qq = C.values(rng, (3, 100, 1, 32), "bf16"), C.values(rng, (3, 1, 1, 32), "bf16")
    cache = big.as_strided((3, 100, 1, 32), (1 << 30, 4096, 32, 1))
    cache.copy_(dev(kv, "bf16"))
    out = torch.empty(3, 1, 1, 32, dtype=torch.bfloat16, device="cuda")
    pwdec.attention(dev(qq, "bf16"), cache, cache, out)
    ref, mag, top = O.attention(qq, kv, kv)
    C.check(host(out), ref, C.attention_bound(ref, mag, top, "bf16", 32, 100))
    keys = big.as_strided((1, 300, 1, 32), (0, (1 << 31) // 299 // 8 * 8, 32, 1))   # one sequence, far apart tokens
    kv = C.values(rng, (1, 300, 1, 32), "bf16")
    keys.copy_(dev(kv, "bf16"))
    pwdec.attention(dev(qq[:1], "bf16"), keys, keys, out[:1])
    ref, mag, top = O.attention(qq[:1], kv, kv)
    C.check(host(out[:1]), ref, C.attention_bound(ref, mag, top, "bf16", 32, 300))


def test_workspaces_and_streams_that_are_given():
    """A workspace of the caller's gives the same result; one too small, of another type, or a call whose tensors
    do not fit is refused before anything runs."""
    q, c = torch.randn(1, 1, 4, 64, device="cuda"), torch.randn(1, 4000, 2, 64, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    need = pwdec.attention_workspace(q, c, c, a)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    pwdec.attention(q, c, c, a)
    pwdec.attention(q, c, c, b, workspace=ws)
    assert need > 0 and torch.equal(a, b)
    x, w = torch.randn(100, 4096, device="cuda"), torch.randn(300, 4096, device="cuda")
    y, z = torch.empty(100, 300, device="cuda"), torch.empty(100, 300, device="cuda")
    need = pwdec.linear_workspace(x, w, y)
    pwdec.linear(x, w, y)
    pwdec.linear(x, w, z, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert need > 0 and torch.equal(y, z)
    with pytest.raises(ValueError):
        pwdec.linear(x, w, y, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        pwdec.attention(q, c, c, b, workspace=torch.empty(1 << 20, device="cuda"))
    with pytest.raises(pwdec.PwdError):
        pwdec.linear(x, w, x[:, :300])
    with pytest.raises(pwdec.PwdError):
        pwdec.attention(q, c, c, a, scale=0.0)


ATT_BIG = [(2, 200, 200, 4, 2, 128, (-1, 0), 0, (200, 150), (200, 150)), (1, 1, 3000, 8, 1, 128, (-1, 0), 0, None, (2900,)),
           (1, 2, 2500, 4, 4, 64, (600, 0), 4, None, None), (3, 130, 130, 2, 2, 32, (-1, -1), 0, None, None),
           (1, 40, 600, 16, 2, 96, (-1, 0), 0, None, None), (2, 33, 700, 2, 1, 256, (100, 3), 5, (33, 0), (650, 700)),
           (1, 300, 300, 2, 1, 64, (17, 9), 33, None, None)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("b,sq,sk,hq,hk,dh,window,sinks,ql,kl", C.ATTENTION_SHAPES + ATT_BIG)
def test_attention(b, sq, sk, hq, hk, dh, window, sinks, ql, kl, dtype):
    say(f"attention {b} {sq} {sk} {hq} {hk} {dh} {window} {sinks} {ql} {kl} {dtype}")
    rng = np.random.default_rng(sq + sk + dh)
    q = C.values(rng, (b, sq, hq, dh), dtype)
    k, v = C.values(rng, (b, sk, hk, dh), dtype), C.values(rng, (b, sk, hk, dh), dtype)
    cache = torch.full((b, sk + 1, 2, hk, dh), float("nan"), dtype=DT[dtype], device="cuda")
    cache[:, :sk, 0], cache[:, :sk, 1] = dev(k, dtype), dev(v, dtype)
    for s in range(b):   # what lies past a sequence's keys must not matter
        if kl is not None:
            cache[s, kl[s]:, 0], cache[s, kl[s]:, 1] = float("nan"), float("inf")
        seen = C.seen_keys(sq if ql is None else ql[s], sk if kl is None else kl[s], sk, window, sinks)
        hidden = torch.from_numpy(~seen).cuda()
        cache[s, :sk, 0][hidden], cache[s, :sk, 1][hidden] = float("inf"), float("nan")   # nor keys that no query sees
    out = torch.full((b, sq, hq, dh), 7.0, dtype=DT[dtype], device="cuda")
    lens = [dev(np.array(n, np.int32)) if n is not None else None for n in (ql, kl)]
    pwdec.attention(dev(q, dtype), cache[:, :sk, 0], cache[:, :sk, 1], out, window=window, sinks=sinks, q_lengths=lens[0],
                    k_lengths=lens[1])
    got = host(out)
    ref, mag, top = O.attention(q, k, v, *window, sinks, None, ql, kl)
    untouched = np.isnan(ref)
    assert (got[untouched] == 7.0).all()
    bound = C.attention_bound(ref, mag, top, dtype, dh, sk)
    C.check(np.where(untouched, 0, got), np.where(untouched, 0, ref), np.where(untouched, 0, bound), "attention")


def test_attention_large_scores():
    """Scores of hundreds, growing along the keys so that the running maximum moves in every tile, against
    the oracle; and one query whose scores all stay far below the others'."""
    rng = np.random.default_rng(9)
    q, k, v = (C.values(rng, (1, 40, 1, 64), "fp32") for _ in range(3))
    k = k * np.linspace(0.1, 12, 40, dtype=np.float32)[None, :, None, None]
    k = np.concatenate([k, k[:, ::-1] * 4], 1)
    v = np.concatenate([v, -v], 1)
    q[:, 3] *= 1e-3
    q[:, 5] *= 20
    out = torch.empty(1, 40, 1, 64, device="cuda")
    pwdec.attention(dev(q), dev(k), dev(v), out)
    ref, mag, top = O.attention(q, k, v)
    C.check(host(out), ref, C.attention_bound(ref, mag, top, "fp32", 64, 80))


def test_activations_at_the_ends():
    """Infinite, huge, tiny and NaN arguments: as the formulas give them."""
    v = np.array([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 3.0, -3.0, 30.0, -30.0, 1e4, -1e4, 1e20, -1e20], np.float32)
    for act in pwdec.ACTIVATIONS:
        y = torch.empty(len(v), 1, device="cuda")
        pwdec.linear(dev(v[:, None]), torch.ones(1, 1, device="cuda"), y, activation=act)
        ref = O.activate(v.astype(np.float64), act)
        assert (np.abs(host(y)[:, 0] - ref) <= 2.0 ** -20 * np.abs(v) + 1e-38).all(), (act, host(y)[:, 0], ref)
        nan = torch.full((1, 1), float("nan"), device="cuda")
        pwdec.linear(nan, torch.ones(1, 1, device="cuda"), y[:1], activation=act)
        assert torch.isnan(y[0, 0])


def layer(x, w, pos, heads, out, tmp, stream=None):
    """One pre-projected attention block, as a layer runs the operators: the q/k/v projection, the norm
    and rotation of q and k in place, attention, the output projection added to the stream, and a
    feed-forward product."""
    n, d = x.shape
    qkv = tmp["qkv"]
    pwdec.linear(x, w["qkv"], qkv, bias=w["b"], stream=stream)
    q, k, v = (qkv[:, i * d:(i + 1) * d].unflatten(1, (heads, d // heads)) for i in range(3))
    p = d // heads // 2 // 2
    pwdec.qk_norm_rope(q, k, w["g"], w["g"], pos, (p, p), stream=stream)
    pwdec.attention(q[None], k[None], v[None], tmp["a"].unflatten(1, (heads, d // heads))[None], window=(50, -1), sinks=1, stream=stream)
    out.copy_(x)
    pwdec.linear(tmp["a"], w["o"], out, residual=out, stream=stream)
    pwdec.linear(out, w["f"], tmp["f"], activation="gelu", stream=stream)
    return out, tmp["f"]


def layer_inputs(n, d, heads, seed):
    rng = np.random.default_rng(seed)
    x = C.values(rng, (n, d), "bf16")
    w = {"qkv": C.values(rng, (3 * d, d), "bf16", d ** -0.5), "b": rng.standard_normal(3 * d).astype(np.float32) * 0.1,
         "g": np.ones(d // heads, np.float32) * 1.5, "o": C.values(rng, (d, d), "bf16", d ** -0.5),
         "f": C.values(rng, (2 * d, d), "bf16", d ** -0.5)}
    pos = np.stack([np.arange(n) // 12, np.arange(n) % 12], 1).astype(np.int32)
    wd = {k: dev(v, None if k in ("b", "g") else "bf16") for k, v in w.items()}
    tmp = {"qkv": torch.empty(n, 3 * d, dtype=torch.bfloat16, device="cuda"), "a": torch.empty(n, d, dtype=torch.bfloat16, device="cuda"),
           "f": torch.empty(n, 2 * d, dtype=torch.bfloat16, device="cuda")}
    return x, w, pos, wd, tmp


def test_a_layer_of_operators():
    """The operators one after another against the oracle chained the same way, rounded to bf16 where they
    store bf16. What differs are single roundings that fall the other way (2^-8 of a value), which the
    following steps average: 2^-5 of the largest value of each output covers them many times over and
    no misplaced head, position or key (which moves values by their own size)."""
    n, d, heads = 144, 192, 8
    x, w, pos, wd, tmp = layer_inputs(n, d, heads, 3)
    out, f = layer(dev(x, "bf16"), wd, dev(pos), heads, torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), tmp)
    r = lambda a: C.from_bf16_bits(C.to_bf16_bits(a)).astype(np.float64)
    qkv = r(O.linear(x, w["qkv"], w["b"])[0]).reshape(n, 3, heads, d // heads)
    q, k = (r(O.rope(O.rms_norm(qkv[:, i], w["g"]), pos, (6, 6))) for i in (0, 1))
    a = r(O.attention(q[None], k[None], qkv[None, :, 2], left=50, sinks=1)[0][0].reshape(n, d))
    y = r(O.linear(a, w["o"], residual=x)[0])
    z = O.linear(y, w["f"], act="gelu")[0]
    for got, ref in ((out, y), (f, z)):
        assert np.abs(host(got) - ref).max() <= 2.0 ** -5 * np.abs(ref).max()


def test_streams_and_graphs():
    """The same layer on another stream, and captured into two graphs that are replayed in turn, with eager
    work between the replays: every result equals the eager one bit for bit."""
    n, d, heads = 144, 192, 8
    x, _, pos, wd, tmp = layer_inputs(n, d, heads, 4)
    xs, ps, out = dev(x, "bf16"), dev(pos), torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    ref = [t.clone() for t in layer(xs, wd, ps, heads, out, tmp)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = layer(xs, wd, ps, heads, torch.empty_like(out), {k: torch.empty_like(v) for k, v in tmp.items()}, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    # a call that splits its keys (it has a workspace) beside the layer
    q, c = torch.randn(1, 1, 8, 64, device="cuda"), torch.randn(1, 3000, 2, 2, 64, device="cuda")
    kv = [c[:, :, 0], c[:, :, 1]]
    step = torch.empty_like(q)
    pwdec.attention(q, *kv, step)
    want = step.clone()
    assert pwdec.attention_workspace(q, *kv, step) > 0
    graphs = []
    for _ in range(2):
        g, o = torch.cuda.CUDAGraph(), torch.empty_like(out)
        t = {k: torch.empty_like(v) for k, v in tmp.items()}
        s = torch.empty_like(q)
        with torch.cuda.graph(g):
            res = layer(xs, wd, ps, heads, o, t)
            pwdec.attention(q, *kv, s)
        graphs.append((g, res, s))
    for _ in range(3):
        for g, res, s in graphs:
            for r in (*res, s):
                r.zero_()
            g.replay()
            pwdec.attention(q, *kv, step)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(ref, res))
            assert torch.equal(s, want) and torch.equal(step, want)


def test_repeated_calls_agree():
    """No result depends on the order in which workgroups end: bit equality over repeated calls of the
    kernels that join partial sums."""
    rng = np.random.default_rng(11)
    q, c = dev(C.values(rng, (2, 1, 8, 128), "bf16"), "bf16"), dev(C.values(rng, (2, 5000, 2, 2, 128), "bf16"), "bf16")
    x, w = dev(C.values(rng, (100, 4096), "bf16"), "bf16"), dev(C.values(rng, (200, 4096), "bf16"), "bf16")
    outs = []
    for _ in range(4):
        o, y = torch.empty_like(q), torch.empty(100, 200, device="cuda")
        pwdec.attention(q, c[:, :, 0], c[:, :, 1], o)
        pwdec.linear(x, w, y)
        outs.append((o, y))
    assert all(torch.equal(a[0], outs[0][0]) and torch.equal(a[1], outs[0][1]) for a in outs)


def test_empty_calls():
    """Sizes of zero: nothing is launched, an empty sum is the activated bias and the residual."""
    e = lambda *s: torch.empty(*s, device="cuda")
    pwdec.linear(e(0, 5), e(4, 5), e(0, 4))
    pwdec.linear(e(3, 5), e(0, 5), e(3, 0))
    y, b = e(3, 4), torch.tensor([1.0, -2.0, 0.5, 0.0], device="cuda")
    pwdec.linear(e(3, 0), e(4, 0), y, bias=b, activation="relu", residual=torch.ones(3, 4, device="cuda"))
    assert torch.equal(y, (b.clamp(min=0) + 1).expand(3, 4))
    pwdec.rope(e(0, 2, 8), None, torch.empty(0, 1, dtype=torch.int32, device="cuda"), (4,))
    pwdec.attention(e(0, 3, 2, 8), e(0, 3, 2, 8), e(0, 3, 2, 8), e(0, 3, 2, 8))
    o = torch.full((2, 3, 2, 8), 7.0, device="cuda")
    pwdec.attention(torch.ones(2, 3, 2, 8, device="cuda"), e(2, 0, 1, 8), e(2, 0, 1, 8), o)
    assert not o.any()
