"""Rotary networks that the CPU (host stand-in) and GPU tests decode."""
import dataclasses

import numpy as np

from paper_2601_09921_amd import pwdec, synth

F32, BF16 = synth.DTYPE_F32, synth.DTYPE_BF16


@dataclasses.dataclass(frozen=True)
class Case:
    name: str
    wl: synth.Workload
    pairs: tuple = (0, 0)
    qk_norm: bool = False
    window: int = -1
    sinks: int = 0

    def options(self):
        return pwdec.rotary_dims(self.pairs, 100.0, self.qk_norm, 1e-5, self.window, self.sinks)

    def oracle(self):
        return dict(pairs=self.pairs, theta=100.0, qk_norm=self.qk_norm, norm_eps=float(np.float32(1e-5)), window=self.window,
                    sinks=self.sinks)

    def weights(self, seed):
        w = synth.make_weights(self.wl, seed=seed)
        rng = np.random.default_rng(seed)
        dh = self.wl.D // self.wl.H
        for lw in w["layers"]:
            if self.qk_norm:   # gains above one: scores as peaked as without the norm
                lw["gq"], lw["gk"] = (np.float32(1.5 + 0.1 * rng.standard_normal(dh)).astype(np.float64) for _ in range(2))
        return w


def wl(d, W, B, D, L, H, dtype, mlp=4, **kw):
    return synth.Workload(f"r{d}", d, W, B, 0.05, 0.0, D, L, H, mlp, dtype, **kw)


SMALL = [
    Case("norm_f32", wl(3, 5, 3, 48, 2, 4, F32), (3, 3), True),
    Case("plain_f32", wl(3, 4, 2, 16, 1, 1, F32, grid=True)),
    Case("window_f32", wl(3, 4, 2, 32, 1, 2, F32, mlp=5, resnet=True), (4, 2), False, 2, 1),
    Case("paper_width", wl(3, 3, 2, 192, 1, 8, BF16, mlp=5), (6, 6), True),
]
CASES = SMALL + [
    Case("d5_192", wl(5, 10, 20, 192, 3, 8, BF16, mlp=5, grid=True, resnet=True), (6, 6), True),
    Case("d7_128", wl(7, 14, 33, 128, 3, 8, BF16), (4, 4)),
    Case("d7_320", wl(7, 9, 5, 320, 2, 5, BF16), (16, 16), True, 10, 4),
    Case("d9_f32", wl(9, 12, 7, 80, 2, 4, F32), (5, 5), True, 20, 2),
    Case("d11_sinusoid", wl(11, 13, 6, 256, 2, 8, BF16)),
]
