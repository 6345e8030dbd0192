"""Cases that the transformer operators' speed is measured on.

A case is one call of an operator as a program that runs a transformer over syndromes, or another
network's layer, makes it:
  linear        y = act(x w^T + b) + r over row-major rows (weights [out][in]);
  rope          the position rotation of queries and keys over one to three axes (the rounds, rows and
                columns of a syndrome array; time, height and width of a clip; a text's one axis);
  qk_norm_rope  RMS norm of every head of the queries and keys, then that rotation, in one pass;
  attention     softmax(q k^T scale) v over sequences of their own lengths, with a sliding window of
                keys and the first few keys (sinks) in sight, key heads shared by query heads.
The sizes are the decoder's own (d_model 256 over the distance-25 windows), the calls of a few tokens
where latency counts, and generic transformer layers up to a teraflop. `draw` spreads over the same
ranges. Queries, keys and values are columns of a packed q/k/v buffer, as a projection writes them, or
of a key/value cache.

Inputs are synthetic: activations N(0, 1), matrices N(0, 1/fan_in), positions of real layouts.
"""
import math

import torch

own = False

FLOPS_MAX = 1.2e12   # of the largest listed product
BYTES_MAX = 1.8e9    # of the largest listed pass over memory
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _linear(name, m, n, k, dtype="bf16", out="", act="none", bias=True, residual=False, pad=0):
    c = {"op": "linear", "m": m, "n": n, "k": k, "dtype": dtype, "out": out or dtype, "act": act, "bias": bias,
         "residual": residual, "pad": pad}
    return {"name": name, **c} if name else c


def _rope(name, t, hq, hk, dh, pairs, layout="half", freq="axis", pos="grid", side=26, dtype="bf16", norm=False,
          inverse=False):
    c = {"op": "qk_norm_rope" if norm else "rope", "t": t, "hq": hq, "hk": hk, "dh": dh,
         "pairs": ",".join(map(str, pairs)), "layout": layout, "freq": freq, "pos": pos, "side": side, "dtype": dtype,
         "inverse": inverse}
    return {"name": name, **c} if name else c


def _attn(name, b, sq, sk, hq, hk, dh, left=-1, right=-1, sinks=0, lens="full", dtype="bf16"):
    c = {"op": "attention", "b": b, "sq": sq, "sk": sk, "hq": hq, "hk": hk, "dh": dh, "left": left, "right": right,
         "sinks": sinks, "lens": lens, "dtype": dtype}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token through a small square projection: the latency of a call
        _linear("linear_token", 1, 256, 256),
        # sixteen sequences a step, with the residual stream in fp32
        _linear("linear_serve_16", 16, 4096, 4096, out="fp32", residual=True),
        # a ragged batch and an odd layer: nothing is a multiple of a tile
        _linear("linear_ragged", 1999, 1003, 515, act="gelu", residual=True, pad=3),
        # fp32 throughout, a mid-sized layer with its residual
        _linear("linear_fp32", 4096, 2048, 1024, dtype="fp32", act="gelu_tanh", residual=True),
        # a large layer: the matrix rate
        _linear("linear_large", 16384, 8192, 4096, act="silu"),
        # rotation of three axes over a clip (frames of 32 x 32 patches), every head of a layer
        _rope("rope_clip", 65536, 16, 16, 128, (16, 24, 24), pos="clip", side=32),
        # fp32 rotation of a syndrome history's rows and columns, adjacent pairs, undone
        _rope("rope_grid_fp32", 20000, 8, 8, 32, (8, 8), layout="adjacent", dtype="fp32", inverse=True),
        # one new token a sequence, 8 sequences deep in their texts: the latency of a call
        _rope("qk_step", 8, 32, 8, 128, (64,), pos="far", norm=True),
        # queries and keys of 512 windows of distance 25, rotated by row and column
        _rope("qk_d25", 319488, 8, 8, 32, (8, 8), norm=True),
        # one new token a sequence against caches of up to 32768 keys: the cache's bytes
        _attn("attn_step", 8, 1, 32768, 32, 8, 128, right=0, lens="ragged"),
        # two prompts of 8192 tokens through a layer with a window of 1024 keys and 4 sinks
        _attn("attn_prompt", 2, 8192, 8192, 32, 8, 128, left=1023, right=0, sinks=4),
        # every token of 256 windows of distance 25 against every other
        _attn("attn_d25", 256, 624, 624, 8, 8, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the listed ranges: sizes spread over their logarithm, round and odd."""
    while True:
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        op = rng.choice(["linear", "linear", "rope", "attention"])
        if op == "linear":
            m, n, k = _log(rng, 1, 100000), _log(rng, 8, 8192), _log(rng, 8, 8192)
            if rng.random() < 0.6:   # layers' sizes are mostly multiples of a power of two
                n, k = max(16, n // 64 * 64), max(16, k // 64 * 64)
            c = _linear("", m, n, k, dtype, rng.choice([dtype, "fp32"]), rng.choice(ACTS), rng.random() < 0.7,
                        rng.random() < 0.5, rng.choice([0, 0, 8, 5]))
        elif op == "attention":
            hk, dh = rng.choice([1, 2, 4, 8]), rng.choice([16, 24, 32, 64, 64, 80, 96, 128, 128, 256])
            sk = _log(rng, 1, 32768)
            sq = rng.choice([sk, sk, 1, min(sk, rng.randint(1, 64))])
            right = rng.choice([-1, 0, 0, 0])
            left = rng.choice([-1, -1, _log(rng, 1, 4096)])
            c = _attn("", _log(rng, 1, 256), sq, sk, hk * rng.choice([1, 2, 4, 8]), hk, dh, left, right,
                      rng.choice([0, 1, 4, 17]) if left >= 0 else 0, rng.choice(["full", "ragged"]), dtype)
            if _pair_bound(c) > 2.5e10 / dh:
                continue
        else:
            axes = rng.choice([1, 2, 3])
            dh = rng.choice([16, 24, 32, 48, 64, 80, 96, 128, 160, 256, 34])
            each = dh // 2 // axes
            if rng.random() < 0.3 and each > 1:   # part of the head keeps its values
                each = rng.randint(1, each)
            hk = rng.choice([1, 2, 4, 8, 16])
            c = _rope("", _log(rng, 1, 200000), hk * rng.choice([1, 1, 2, 4]), hk, dh, (each,) * axes,
                      rng.choice(["half", "adjacent"]), rng.choice(["axis", "shared"]),
                      {1: rng.choice(["text", "far"]), 2: "grid", 3: "clip"}[axes], rng.randint(4, 40), dtype,
                      norm=rng.random() < 0.6)
            if c["op"] == "rope":
                c["inverse"] = rng.random() < 0.3
        w = work(c)
        if w["flops"] <= FLOPS_MAX * (1 if dtype == "bf16" else 0.1) and w["bytes"] <= BYTES_MAX:
            return c


def work(c):
    s = SIZE[c["dtype"]]
    if c["op"] == "linear":
        m, n, k, so = c["m"], c["n"], c["k"], SIZE[c["out"]]
        return {"bytes": (m * k + n * k) * s + 4 * n * c["bias"] + m * n * so * (2 if c["residual"] else 1),
                "flops": 2 * m * n * k}
    if c["op"] == "attention":
        klen = _lengths(c)
        qo = 2 * sum(_queries(c, n) for n in klen) * c["hq"] * c["dh"]
        seen = [_visible(c, n) for n in klen]
        return {"bytes": (qo + 2 * sum(kept for kept, _ in seen) * c["hk"] * c["dh"]) * s + 4 * c["b"],
                "flops": 4 * sum(p for _, p in seen) * c["hq"] * c["dh"]}
    pairs = _pairs(c)
    values = c["t"] * (c["hq"] + c["hk"]) * c["dh"]
    rotated = c["t"] * (c["hq"] + c["hk"]) * sum(pairs)
    norm = c["op"] == "qk_norm_rope"
    return {"bytes": 2 * values * s + 4 * c["t"] * len(pairs) + (8 * c["dh"] if norm else 0),
            "flops": 6 * rotated + (4 * values if norm else 0)}


def _pair_bound(c):
    return c["b"] * c["sq"] * c["sk"] * c["hq"]


def _lengths(c):
    """Keys of each sequence: all, or spread over the upper seven eighths of the room (one is empty
    where there are many)."""
    if c["lens"] == "full":
        return [c["sk"]] * c["b"]
    n = [max(1, c["sk"] - i * 7919 % (1 + 7 * c["sk"] // 8)) for i in range(c["b"])]
    if c["b"] > 4:
        n[3] = 0
    return n


def _queries(c, n):
    """Queries of a sequence of n keys: in a padded batch of prompts as many as keys, else all."""
    return n if c["sq"] == c["sk"] else c["sq"]


def _visible(c, n):
    """(keys that any query of a sequence of n keys sees, pairs of query and key that see each other);
    the sequence's queries are its last positions."""
    pairs, last_lo, last_hi, sink, nq = 0, None, 0, 0, _queries(c, n)
    for i in range(nq) if c["left"] >= 0 or c["right"] >= 0 else ():
        p = n - nq + i
        hi = min(n, p + c["right"] + 1) if c["right"] >= 0 else n
        lo = max(0, p - c["left"]) if c["left"] >= 0 else 0
        if hi <= 0:
            continue
        s = min(c["sinks"], lo, hi)
        pairs += max(0, hi - lo) + s
        sink = max(sink, s)
        last_lo = lo if last_lo is None else min(last_lo, lo)
        last_hi = max(last_hi, hi)
    if c["left"] < 0 and c["right"] < 0:
        return (n if nq else 0), n * nq
    if last_lo is None:
        return 0, 0
    return max(0, last_hi - last_lo) + min(sink, last_lo), pairs


def _pairs(c):
    return tuple(int(p) for p in c["pairs"].split(","))


def _positions(c, axes, g):
    """int32 [t][axes]: the cells of a side x side array again and again (grid), those cells in frame
    after frame (clip), 0 1 2 ... (text), or anywhere up to a million (far)."""
    i = torch.arange(c["t"], device="cuda")
    s = c["side"]
    if c["pos"] == "grid":
        p = [i // s % s, i % s]
    elif c["pos"] == "clip":
        p = [i // (s * s), i // s % s, i % s]
    elif c["pos"] == "text":
        p = [i]
    else:
        p = [torch.randint(0, 1 << 20, (c["t"],), device="cuda", generator=g)]
    return torch.stack(p[:axes], 1).to(torch.int32).contiguous()


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    dt = DT[c["dtype"]]
    st = {"case": c}
    if c["op"] == "linear":
        m, n, k, pad = c["m"], c["n"], c["k"], c["pad"]
        st["x"] = rnd(m, k + pad).to(dt)[:, :k]   # pad: the rows of a wider buffer
        st["w"] = (rnd(n, k) / math.sqrt(k)).to(dt)
        st["bias"] = rnd(n) * 0.1 if c["bias"] else None
        st["residual"] = rnd(m, n).to(DT[c["out"]]) if c["residual"] else None
        if own:
            st["y"] = torch.empty(m, n, dtype=DT[c["out"]], device="cuda")
        return st
    if c["op"] == "attention":
        b, sq, sk, hq, hk, dh = c["b"], c["sq"], c["sk"], c["hq"], c["hk"], c["dh"]
        if sq == sk:   # self attention: the columns of one projection
            qkv = rnd(b, sq, (hq + 2 * hk) * dh).to(dt)
            q, kv = qkv[..., :hq * dh], qkv[..., hq * dh:]
        else:          # new tokens against a cache
            q, kv = rnd(b, sq, hq * dh).to(dt), rnd(b, sk, 2 * hk * dh).to(dt)
        st["q"] = q.unflatten(2, (hq, dh))
        st["k"] = kv[..., :hk * dh].unflatten(2, (hk, dh))
        st["v"] = kv[..., hk * dh:].unflatten(2, (hk, dh))
        st["len"] = None
        if c["lens"] != "full":
            st["len"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
        if own:   # rows of padding are left as they are: zeros
            st["out"] = torch.zeros(b, sq, hq, dh, dtype=dt, device="cuda")
        return st
    t, hq, hk, dh = c["t"], c["hq"], c["hk"], c["dh"]
    qkv = rnd(t, (hq + 2 * hk) * dh).to(dt)
    st["q"] = qkv[:, :hq * dh].unflatten(1, (hq, dh))
    st["k"] = qkv[:, hq * dh:(hq + hk) * dh].unflatten(1, (hk, dh))
    st["pos"] = _positions(c, len(_pairs(c)), g)
    if c["op"] == "qk_norm_rope":
        st["gq"], st["gk"] = 1 + 0.1 * rnd(dh), 1 + 0.1 * rnd(dh)
    if own:
        st["q_out"] = torch.empty(t, hq, dh, dtype=dt, device="cuda")
        st["k_out"] = torch.empty(t, hk, dh, dtype=dt, device="cuda")
    return st


THETA, EPS = 10000.0, 1e-6


def run(st):
    c = st["case"]
    if own:
        return _run_own(c, st)
    if c["op"] == "linear":
        y = st["x"].float() @ st["w"].float().t()
        if st["bias"] is not None:
            y = y + st["bias"]
        y = _act(y, c["act"])
        if st["residual"] is not None:
            y = y + st["residual"].float()
        return y.to(DT[c["out"]])
    if c["op"] == "attention":
        return _attention(c, st)
    cos, sin = _tables(c, st["pos"])
    out = []
    for x, gain in ((st["q"], st.get("gq")), (st["k"], st.get("gk"))):
        y = x.float()
        if gain is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain
        out.append(_rotate(y, cos, sin, c["layout"]).to(x.dtype))
    return out


def _run_own(c, st):
    from paper_2601_09921_amd import pwdec
    if c["op"] == "linear":
        pwdec.linear(st["x"], st["w"], st["y"], bias=st["bias"], activation=c["act"], residual=st["residual"])
        return st["y"]
    if c["op"] == "attention":
        pwdec.attention(st["q"], st["k"], st["v"], st["out"], window=(c["left"], c["right"]), sinks=c["sinks"],
                        k_lengths=st["len"], q_lengths=st["len"] if c["sq"] == c["sk"] else None)
        return st["out"]
    kw = dict(pairs=_pairs(c), theta=THETA, layout=c["layout"], frequencies=c["freq"], q_out=st["q_out"],
              k_out=st["k_out"])
    if c["op"] == "rope":
        pwdec.rope(st["q"], st["k"], st["pos"], inverse=c["inverse"], **kw)
    else:
        pwdec.qk_norm_rope(st["q"], st["k"], st["gq"], st["gk"], st["pos"], eps=EPS, **kw)
    return [st["q_out"], st["k_out"]]


def _mask(c, n):
    """[sq][sk] for a sequence of n keys: does query i see key j? Queries past the sequence see none."""
    j = torch.arange(c["sk"], device="cuda")[None]
    i = torch.arange(c["sq"], device="cuda")[:, None]
    nq = _queries(c, n)
    p = n - nq + i
    see = (j < n) & (i < nq)
    if c["right"] >= 0:
        see = see & (j <= p + c["right"])
    if c["left"] >= 0:
        see = see & ((j >= p - c["left"]) | (j < c["sinks"]))
    return see


def _attention(c, st):
    """A block of the sequences and one key head at a time; hidden scores are minus infinity, and a
    query that sees nothing gives zeros."""
    b, sq, hq, hk, dh = c["b"], c["sq"], c["hq"], c["hk"], c["dh"]
    g, out = hq // hk, torch.zeros(b, sq, hq, dh, device="cuda")
    room = max(1, (1 << 28) // max(1, g * sq * c["sk"]))
    masked = st["len"] is not None or c["left"] >= 0 or c["right"] >= 0
    for i in range(0, b, room):
        e = min(b, i + room)
        if masked:
            n = st["len"][i:e, None, None].long() if st["len"] is not None else c["sk"]
            see = _mask(c, n).expand(e - i, sq, c["sk"])[:, None]
        for h in range(hk):
            q = st["q"][i:e, :, h * g:(h + 1) * g].float().transpose(1, 2).contiguous()
            k = st["k"][i:e, :, h].float().transpose(1, 2).contiguous()[:, None]
            v = st["v"][i:e, :, h].float().contiguous()[:, None]
            s = torch.matmul(q, k) * dh ** -0.5
            if masked:
                s = torch.where(see, s, float("-inf"))
            p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
            total = p.sum(-1, keepdim=True)
            y = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
            out[i:e, :, h * g:(h + 1) * g] = y.transpose(1, 2)
    return out.to(st["q"].dtype)


def _act(y, act):
    if act == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == "silu":
        return y / (1 + torch.exp(-y))
    return y


def _tables(c, pos):
    """cos and sin [t][pairs] of the rotation, from angles in 64 bits (a position of a million turns
    its first pair 160,000 times: 32 bits leave that angle two digits)."""
    pairs = _pairs(c)
    total, cols, start = sum(pairs), [], 0
    for a, n in enumerate(pairs):
        j = torch.arange(n, device=pos.device, dtype=torch.float64)
        power = j / n if c["freq"] == "axis" else (j + start) / total
        cols.append(pos[:, a:a + 1].double() * THETA ** -power)
        start += n
    ang = torch.cat(cols, 1)
    if c["inverse"]:
        ang = -ang
    return ang.cos().float(), ang.sin().float()


def _rotate(y, cos, sin, layout):
    n = cos.shape[1]
    cos, sin = cos[:, None], sin[:, None]
    y = y.clone()
    if layout == "half":
        u, v = y[..., :n].clone(), y[..., n:2 * n].clone()
        y[..., :n], y[..., n:2 * n] = u * cos - v * sin, u * sin + v * cos
    else:
        u, v = y[..., 0:2 * n:2].clone(), y[..., 1:2 * n:2].clone()
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = u * cos - v * sin, u * sin + v * cos
    return y


def exact(c, seed):
    """The definition in float64: for the product, rows in blocks; for the rotation, complex numbers
    u + iv times e^(i angle) with the pairs gathered by index."""
    st = prepare(c, seed)
    if c["op"] == "linear":
        w = st["w"].double().t().contiguous()
        y = torch.empty(c["m"], c["n"], dtype=torch.float64, device="cuda")
        for i in range(0, c["m"], 1 << 15):
            z = st["x"][i:i + (1 << 15)].double() @ w
            if c["bias"]:
                z += st["bias"].double()
            if c["act"] == "relu":
                z = z.clamp(min=0)
            elif c["act"] == "gelu":
                z = z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
            elif c["act"] == "gelu_tanh":
                z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * z * (1 + 0.044715 * z.square()))
            elif c["act"] == "silu":
                z = z * torch.sigmoid(z)
            if c["residual"]:
                z += st["residual"][i:i + (1 << 15)].double()
            y[i:i + (1 << 15)] = z
        return y
    if c["op"] == "attention":
        return _attention_exact(c, st)
    pairs = _pairs(c)
    total, dh = sum(pairs), c["dh"]
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    within = [j for n in pairs for j in range(n)]
    freq = [THETA ** (-within[j] / pairs[axis[j]] if c["freq"] == "axis" else -j / total) for j in range(total)]
    ang = st["pos"].double()[:, axis] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    turn = torch.exp(1j * (-ang if c["inverse"] else ang))[:, None]
    first = torch.arange(total, device="cuda") * (1 if c["layout"] == "half" else 2)
    second = first + (total if c["layout"] == "half" else 1)
    out = []
    for x, gain in ((st["q"], st.get("gq")), (st["k"], st.get("gk"))):
        y = x.double()
        if gain is not None:
            y = gain.double() * y / torch.sqrt(y.square().sum(-1, keepdim=True) / dh + EPS)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y = y.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def _attention_exact(c, st):
    """Sequence by sequence and head by head in float64, a block of queries at a time against the
    keys that the sequence has."""
    if _pair_bound(c) * c["dh"] > 1.5e12 or c["b"] * c["hq"] > 5000:
        return None
    out = torch.zeros(c["b"], c["sq"], c["hq"], c["dh"], dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        j, nq = torch.arange(n, device="cuda"), _queries(c, n)
        for h in range(c["hq"]):
            kv = h // (c["hq"] // c["hk"])
            k, v = st["k"][i, :n, kv].double().t().contiguous(), st["v"][i, :n, kv].double().contiguous()
            for a in range(0, nq, 8192):
                q = st["q"][i, a:min(a + 8192, nq), h].double()
                p = torch.arange(a, a + q.shape[0], device="cuda") + (n - nq)
                hidden = torch.zeros(q.shape[0], n, dtype=torch.bool, device="cuda")
                if c["right"] >= 0:
                    hidden |= j[None] > (p + c["right"])[:, None]
                if c["left"] >= 0:
                    hidden |= (j[None] < (p - c["left"])[:, None]) & (j >= c["sinks"])[None]
                s = (q @ k / math.sqrt(c["dh"])).masked_fill(hidden, -math.inf)
                w = torch.softmax(s, -1).masked_fill(hidden, 0.0)
                out[i, a:a + q.shape[0], h] = torch.nan_to_num(w) @ v
    return out
