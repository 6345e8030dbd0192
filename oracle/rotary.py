"""CPU float64 oracle of rotary networks: oracle/decoder.py's network with the attention options of
decoder_create_rotary. TEST INFRASTRUCTURE ONLY.

Per layer Q and K heads take an RMS norm (optional) and turn by the token's row and column on the
(d+1) x (d+1) lattice; a token sees the tokens within a window of it in row-major order and the first
few. With a rotation the embedding has no sinusoidal encoding.
"""
from __future__ import annotations

import numpy as np

from oracle import decoder as O
from oracle import operators as P


def attention(X, lw, H, cells, rot):
    B, N, D = X.shape
    dh = D // H
    heads = [(X @ lw[w] + lw[b]).reshape(B * N, H, dh) for w, b in (("Wq", "bq"), ("Wk", "bk"), ("Wv", "bv"))]
    if rot["qk_norm"]:
        heads[0], heads[1] = (P.rms_norm(h, lw[g], rot["norm_eps"]) for h, g in ((heads[0], "gq"), (heads[1], "gk")))
    pos = np.tile(np.array(cells), (B, 1))
    q, k = (P.rope(h, pos, rot["pairs"], rot["theta"]).reshape(B, N, H, dh).transpose(0, 2, 1, 3) for h in heads[:2])
    v = heads[2].reshape(B, N, H, dh).transpose(0, 2, 1, 3)
    s = q @ k.transpose(0, 1, 3, 2) / np.sqrt(dh)
    if rot["window"] >= 0:
        see = np.stack([P.visible(i, N, N, rot["window"], rot["window"], rot["sinks"]) for i in range(N)])
        s = np.where(see, s, -np.inf)
    return (O.softmax(s) @ v).transpose(0, 2, 1, 3).reshape(B, N, D) @ lw["Wo"] + lw["bo"]


def forward_windows(meas, types, w, d, H, rot, grid=False, recurrent=False):
    """Logits and bits [B], or [B][d] of the recurrent branch (O.forward_windows_recurrent)."""
    meas = np.asarray(meas, dtype=np.uint8)
    B, Wr, D = meas.shape[0], meas.shape[1] - 1, w["w_e"].shape[0]
    cells = O.token_cells(d, grid)
    ev = O.detection_events(meas, types, d)
    pe = O.positional_encoding((d + 1) ** 2, D)[[r * (d + 1) + c for r, c in cells]]
    if sum(rot["pairs"]) > 0:
        pe = np.zeros_like(pe)
    state, logits = np.zeros((B, len(cells), D)), []
    for n in range(1, Wr + 1):
        X = w["kappa"] * (O.embed_round(ev[:, n - 1], w, d, grid, pe) + state)
        for lw in w["layers"]:
            X = O.layer_norm(X + attention(X, lw, H, cells, rot), lw["g1"], lw["be1"], w["eps"])
            X = O.layer_norm(X + O.feed_forward(X, lw), lw["g2"], lw["be2"], w["eps"])
        state = X
        if n == Wr or (recurrent and n > Wr - d):
            logits.append(O.readout(state, types, w, d, grid))
    logits = np.stack(logits, 1) if recurrent else logits[0]
    return logits, (logits > 0).astype(np.uint8)
