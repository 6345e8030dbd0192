"""Host-only checks of the transformer operators: what the C ABI refuses and with which status, before
any device is touched, what the binding refuses before the library is called, workspace sizes, and
that the staged product's kernels are among those whose waits test_wait_counts.py checks."""
import ctypes
import math

import pytest

import test_wait_counts as W
from paper_2601_09921_amd import pwdec

BAD, NO = pwdec.PWD_EINVAL, pwdec.PWD_EUNSUPPORTED
PTR, OUT = 0x10000, 0x400000   # never read: every call below is refused


@pytest.fixture(scope="module")
def lib():
    return pwdec.load_library()


def linear_args(**kw):
    a = pwdec.LinearArgs(100, 64, 32, PTR, 32, PTR, 32, PTR, OUT, 64, OUT, 64, 1, 1, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,rc", [
    (dict(m=-1), BAD), (dict(n=-1), BAD), (dict(k=-1), BAD), (dict(m=1 << 31), NO), (dict(k=(1 << 31) - 511), NO),
    (dict(dtype=2), NO), (dict(dtype=-1), NO), (dict(out_dtype=2), NO), (dict(activation=5), NO), (dict(activation=-1), NO),
    (dict(d_x=None), BAD), (dict(d_w=None), BAD), (dict(d_y=None), BAD), (dict(ld_x=31), BAD), (dict(ld_w=31), BAD),
    (dict(ld_y=63), BAD), (dict(ld_residual=63), BAD), (dict(d_x=PTR + 1), BAD), (dict(d_bias=PTR + 2), BAD),
    (dict(d_y=OUT + 1), BAD), (dict(dtype=0, d_w=PTR + 2), BAD), (dict(ld_residual=70), BAD),
    # over an input: the same place, the end of x, the bias, a residual that is not y itself
    (dict(d_y=PTR), BAD), (dict(d_y=PTR + 100 * 64 - 2), BAD), (dict(d_bias=OUT + 12), BAD), (dict(d_residual=OUT + 2), BAD),
    (dict(d_x=OUT + 200, ld_x=32), BAD), (dict(d_y=PTR, ld_y=500), BAD),
    (dict(m=(1 << 31) - 512, n=(1 << 31) - 512, ld_y=1 << 31), NO),
])
def test_linear_refuses(lib, kw, rc):
    assert lib.pwd_linear(ctypes.byref(linear_args(**kw)), None) == rc
    assert lib.decoder_last_error().startswith(b"linear")


def test_linear_nothing_to_do(lib):
    assert lib.pwd_linear(None, None) == BAD and lib.pwd_linear_workspace(None) == 0
    for kw in (dict(m=0), dict(n=0)):
        assert lib.pwd_linear(ctypes.byref(linear_args(d_x=None, d_w=None, d_y=None, d_bias=None, d_residual=None, **kw)), None) == 0


def rope_args(**kw):
    a = pwdec.RopeArgs(10, 4, 2, 32, 1)
    for name, heads in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2)):
        setattr(a, f"d_{name}", PTR + 0x1000 * ("out" in name))
        setattr(a, f"{name}_token_stride", 32 * heads)
        setattr(a, f"{name}_head_stride", 32)
    a.d_positions, a.axes, a.pairs, a.theta = PTR, 2, (ctypes.c_int32 * 3)(8, 8, 0), 1e4
    for k, v in kw.items():
        setattr(a, k, (ctypes.c_int32 * 3)(*v) if k == "pairs" else v)
    return a


@pytest.mark.parametrize("kw,rc", [
    (dict(tokens=-1), BAD), (dict(q_heads=-1), BAD), (dict(dtype=2), NO), (dict(head_dim=0), NO), (dict(head_dim=33), NO),
    (dict(head_dim=258), NO), (dict(q_heads=65536), NO), (dict(axes=4), NO), (dict(axes=-1), NO), (dict(layout=2), NO),
    (dict(frequencies=2), NO), (dict(theta=0.0), BAD), (dict(theta=math.inf), BAD), (dict(theta=math.nan), BAD),
    (dict(pairs=(8, 9, 0)), BAD), (dict(pairs=(8, -1, 0)), BAD), (dict(axes=1), BAD), (dict(pairs=(1 << 30, 1 << 30, 0)), BAD),
    (dict(d_q=None), BAD), (dict(d_k_out=None), BAD), (dict(d_positions=None), BAD), (dict(d_positions=PTR + 2), BAD),
    (dict(d_q=PTR + 1), BAD), (dict(q_head_stride=31), BAD), (dict(q_token_stride=127), BAD), (dict(k_out_token_stride=0), BAD),
    (dict(d_q_out=PTR, q_out_token_stride=200), BAD), (dict(tokens=(1 << 31) + 1), NO),
])
def test_rope_refuses(lib, kw, rc):
    assert lib.pwd_rope(ctypes.byref(rope_args(**kw)), None) == rc
    assert lib.pwd_qk_norm_rope(ctypes.byref(rope_args(**kw)), PTR, PTR, 1e-6, None) == rc
    assert lib.decoder_last_error()


def test_qk_norm_refuses(lib):
    call = lambda a, gq=PTR, eps=1e-6: lib.pwd_qk_norm_rope(ctypes.byref(a), gq, PTR, eps, None)
    assert call(rope_args(), eps=-1.0) == BAD and call(rope_args(), eps=math.nan) == BAD
    assert call(rope_args(), gq=PTR + 2) == BAD
    assert call(rope_args(inverse=1)) == NO
    assert lib.pwd_rope(None, None) == BAD and lib.pwd_qk_norm_rope(None, None, None, 0.0, None) == BAD
    assert lib.pwd_rope(ctypes.byref(rope_args(tokens=0, d_q=None, d_positions=None)), None) == 0
    assert lib.pwd_rope(ctypes.byref(rope_args(q_heads=0, k_heads=0, d_q=None)), None) == 0


def attention_args(**kw):
    a = pwdec.AttentionArgs(2, 10, 20, 4, 2, 32, 1)
    for name, n, h in (("q", 10, 4), ("k", 20, 2), ("v", 20, 2), ("out", 10, 4)):
        setattr(a, f"d_{name}", OUT if name == "out" else PTR)
        setattr(a, f"{name}_stride", (ctypes.c_int64 * 3)(n * h * 32, h * 32, 32))
    a.window_left = a.window_right = -1
    a.scale = 0.2
    for k, v in kw.items():
        setattr(a, k, (ctypes.c_int64 * 3)(*v) if k.endswith("stride") else v)
    return a


@pytest.mark.parametrize("kw,rc", [
    (dict(batch=-1), BAD), (dict(q_len=-1), BAD), (dict(k_len=-1), BAD), (dict(sinks=-1), BAD), (dict(dtype=2), NO),
    (dict(head_dim=0), NO), (dict(head_dim=12), NO), (dict(head_dim=264), NO), (dict(dtype=0, head_dim=6), NO),
    (dict(q_heads=3), BAD), (dict(k_heads=0), BAD), (dict(k_len=(1 << 30) + 1), NO), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=1e-21), BAD), (dict(scale=1e21), BAD),
    (dict(scale=math.inf), BAD), (dict(scale=math.nan), BAD), (dict(d_q=None), BAD), (dict(d_v=None), BAD), (dict(d_out=None), BAD),
    (dict(d_k=PTR + 1), BAD), (dict(d_q_lengths=PTR + 2), BAD), (dict(out_stride=(1280, 128, 31)), BAD),
    (dict(k_stride=(1280, -64, 32)), BAD), (dict(d_out=PTR), BAD), (dict(v_stride=(1 << 40, (1 << 24) + 1, 32)), NO), (dict(batch=1 << 30, q_len=1 << 20), NO),
])
def test_attention_refuses(lib, kw, rc):
    assert lib.pwd_attention(ctypes.byref(attention_args(**kw)), None) == rc
    assert lib.decoder_last_error().startswith(b"attention")


def test_attention_workspace(lib):
    """One new token against many keys is split over workgroups and needs a workspace; one that is missing,
    too small or misaligned is refused; short calls need none."""
    a = attention_args(q_len=1, k_len=20000)
    need = lib.pwd_attention_workspace(ctypes.byref(a))
    assert need > 0 and need % (2 * 4 * (32 + 2) * 4) == 0
    for ptr, size in ((None, need), (PTR, need - 1), (PTR + 4, need)):
        a.d_workspace, a.workspace_bytes = ptr, size
        assert lib.pwd_attention(ctypes.byref(a), None) == BAD
    assert lib.pwd_attention_workspace(ctypes.byref(attention_args())) == 0
    assert lib.pwd_attention_workspace(ctypes.byref(attention_args(k_heads=0))) == 0
    assert lib.pwd_attention_workspace(None) == 0 and lib.pwd_attention(None, None) == BAD
    for kw in (dict(batch=0), dict(q_len=0), dict(q_heads=0, k_heads=0)):
        assert lib.pwd_attention(ctypes.byref(attention_args(d_q=None, d_out=None, **kw)), None) == 0


class Fake:
    """Stands in for a torch tensor in the binding's checks."""

    def __init__(self, *shape, dtype="bfloat16", cuda=True, index=0, strides=None, ptr=PTR):
        self.shape, self.dtype, self.is_cuda, self.ptr = tuple(shape), f"torch.{dtype}", cuda, ptr
        self.device = type("Dev", (), {"index": index})()
        packed = [1]
        for n in reversed(shape[1:]):
            packed.append(packed[-1] * n)
        self.strides = strides or tuple(reversed(packed))

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def get_device(self):
        return self.device.index

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return 4 if "32" in self.dtype else 2

    def data_ptr(self):
        return self.ptr

    def is_contiguous(self):
        return True


def at(i):
    return dict(ptr=PTR + (i << 20))


def test_binding_refuses():
    """Shapes, types, devices and strides that the kernels would read past raise ValueError."""
    x, w, y = Fake(5, 8, **at(0)), Fake(3, 8, **at(1)), Fake(5, 3, **at(2))
    lin = [((Fake(5, 8, cuda=False), w, y), {}), ((x, Fake(3, 9), y), {}), ((x, w, Fake(5, 4)), {}), ((x, w, Fake(3, 5)), {}),
           ((x, Fake(3, 8, dtype="float32"), y), {}), ((Fake(5, 8, dtype="float16"), w, y), {}), ((x, Fake(3, 8, index=1), y), {}),
           ((Fake(5, 8, strides=(1, 5)), w, y), {}), ((x, w, y), dict(bias=Fake(3))), ((x, w, y), dict(bias=Fake(4, dtype="float32"))),
           ((x, w, y), dict(residual=Fake(5, 3, dtype="float32"))), ((x, w, y), dict(activation="tanh")), ((x, None, y), {}),
           ((Fake(5, 8, 1), w, y), {})]
    for args, kw in lin:
        with pytest.raises(ValueError):
            pwdec.linear(*args, **kw)
    q, k, p = Fake(4, 2, 16, **at(0)), Fake(4, 1, 16, **at(1)), Fake(4, 2, dtype="int32", **at(2))
    for args, kw in [((None, None, p, (4, 4)), {}), ((q, Fake(5, 1, 16), p, (4, 4)), {}), ((q, Fake(4, 1, 8), p, (4, 4)), {}),
                     ((q, k, p, (4, 4, 0)), {}), ((q, k, None, (4, 4)), {}), ((q, k, Fake(4, 2, dtype="int64"), (4, 4)), {}),
                     ((q, k, p, ()), {}), ((q, k, p, (4, 4)), dict(layout="split")), ((q, k, p, (4, 4)), dict(frequencies="all")),
                     ((q, None, p, (4, 4)), dict(k_out=k)), ((q, k, p, (4, 4)), dict(q_out=Fake(4, 2, 8))),
                     ((Fake(4, 2, 16, index=1), k, p, (4, 4)), {}), ((q, k, Fake(3, 2, dtype="int32"), (4, 4)), {}),
                     ((q, k, p, (1, 1, 1, 1)), {})]:
        with pytest.raises(ValueError):
            pwdec.rope(*args, **kw)
    with pytest.raises(ValueError):
        pwdec.qk_norm_rope(q, k, Fake(16), None, p, (4, 4))
    q, k, v, o = Fake(2, 3, 4, 16, **at(0)), Fake(2, 5, 2, 16, **at(1)), Fake(2, 5, 2, 16, **at(2)), Fake(2, 3, 4, 16, **at(3))
    for args, kw in [((q, Fake(1, 5, 2, 16), v, o), {}), ((q, k, Fake(2, 6, 2, 16), o), {}), ((q, k, v, Fake(2, 3, 4, 8)), {}),
                     ((q, k, v, o), dict(k_lengths=Fake(2, dtype="int64"))), ((q, k, v, o), dict(q_lengths=Fake(3, dtype="int32"))),
                     ((q, k, v, Fake(2, 3, 4, 16, dtype="float32")), {}), ((q, Fake(2, 5, 2, 16, strides=(160, 32, 1, 2)), v, o), {})]:
        with pytest.raises(ValueError):
            pwdec.attention(*args, **kw)


def test_staged_products_are_inspected():
    """Every tile kernel that stages by direct loads is among the kernels whose waits are checked."""
    objs = [obj for src, obj in W.OBJECTS if src == "linear.hip"]
    direct = [n for o in objs for n, insts in W.kernels(o).items() if any(W.DMA.match(mn) for _, mn, _, _ in insts)]
    assert len([n for n in direct if "linear_tile_kernel" in n]) >= 5
