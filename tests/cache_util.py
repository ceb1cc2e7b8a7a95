"""Plain form of the paged 4-bit cache for its tests: the format in fp32 arithmetic, operation by operation, and attention in 64 bits."""
from __future__ import annotations

import numpy as np
import torch

from parity_util import Guarded

GROUP = 64
LIMIT = np.float32(61440.0)


def rotate(x, cos, sin, positions, dtype):
    """x [B, T, H, D], positions [B, T]: adjacent channels turned, every operation rounded to dtype."""
    x = x.astype(dtype)
    c = cos[positions].astype(dtype)[:, :, None, :]
    s = sin[positions].astype(dtype)[:, :, None, :]
    out = np.empty_like(x)
    a, b = x[..., 0::2], x[..., 1::2]
    out[..., 0::2] = a * c - b * s
    out[..., 1::2] = a * s + b * c
    return out


def hold(x):
    """fp32 rows [..., D] -> codes uint8 [..., D], minimum and step fp16 [..., G], values fp32 [..., D]."""
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        g = np.clip(x.astype(np.float32), -LIMIT, LIMIT).reshape(*x.shape[:-1], -1, GROUP)
        low, high = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
        step = ((high - low) * np.float32(1.0 / 15.0)).astype(np.float16)
        low = low.astype(np.float16)
        wide = step.astype(np.float32)
        inverse = np.where(wide > 0, np.float32(1.0) / wide, np.float32(0.0)).astype(np.float32)
        code = np.clip(np.rint((g - low.astype(np.float32)) * inverse), 0, 15)
        code = np.where(np.isnan(code), 0, code).astype(np.float32)
        values = low.astype(np.float32) + wide * code
    return code.astype(np.uint8).reshape(x.shape), low[..., 0], step[..., 0], values.reshape(x.shape)


class Pool:
    """A guarded pool of pages, handed out in a shuffled order, and the table."""

    def __init__(self, B, kv_heads, D, page, capacity, device="cuda", seed=0, spare=2):
        rng = np.random.default_rng(seed)
        self.B, self.H, self.D, self.page = B, kv_heads, D, page
        self.width = max(1, -(-capacity // page))
        self.count = B * self.width + spare
        self.page_bytes = kv_heads * page * (D + D // GROUP * 8)
        self.guard = Guarded((self.count, self.page_bytes), torch.uint8, device)
        # whatever the memory holds before must not matter: fp16 NaN in every parameter
        self.guard.t.fill_(0xFF)
        order = rng.permutation(self.count)[: B * self.width].reshape(B, self.width).astype(np.int32)
        self.order = order
        self.table = torch.from_numpy(order).to(device)

    def split(self):
        """Copies of (K codes, V codes, K parameters, V parameters): [page, head, token, D/2] bytes and [.., G, 2] fp16."""
        p, d = self.page, self.D
        unit = self.guard.t.cpu().numpy().reshape(self.count, self.H, -1)
        a, b = p * d // 2, p * d // GROUP * 4
        cuts = [0, a, 2 * a, 2 * a + b, 2 * a + 2 * b]
        k, v, kp, vp = (np.ascontiguousarray(unit[:, :, i:j]) for i, j in zip(cuts, cuts[1:]))
        par = lambda x: x.view(np.float16).reshape(self.count, self.H, p, d // GROUP, 2)  # noqa: E731
        return k.reshape(self.count, self.H, p, d // 2), v.reshape(self.count, self.H, p, d // 2), par(kp), par(vp)

    def fill(self, k, v, first=0):
        """Writes rows k, v (fp32 [B, T, H, D], T tokens from `first`) in the format, on the host."""
        p, d = self.page, self.D
        unit = self.guard.t.cpu().numpy().reshape(self.count, self.H, -1)
        a, b = p * d // 2, d // GROUP * 4
        for w, x in enumerate((k, v)):
            code, low, step, _ = hold(x)
            packed = code[..., 0::2] | (code[..., 1::2] << 4)
            par = np.stack((low, step), -1)
            for s in range(self.B):
                t = np.arange(first, first + x.shape[1])
                pages, slots = self.order[s, t // p], t % p
                for h in range(self.H):
                    codes = unit[:, h, w * a:(w + 1) * a].reshape(self.count, p, d // 2)
                    codes[pages, slots] = packed[s, :, h]
                    unit[:, h, w * a:(w + 1) * a] = codes.reshape(self.count, -1)
                    lo = 2 * a + w * p * b
                    pars = unit[:, h, lo:lo + p * b].reshape(self.count, p, b)
                    pars[pages, slots] = np.ascontiguousarray(par[s, :, h]).view(np.uint8).reshape(x.shape[1], b)
                    unit[:, h, lo:lo + p * b] = pars.reshape(self.count, -1)
        self.guard.t.copy_(torch.from_numpy(unit.reshape(self.count, -1)))

    def values(self, b, n):
        """What the first n tokens of stream b stand for, float64 [H, n, D] twice."""
        k, v, kp, vp = self.split()
        out = []
        for codes, par in ((k, kp), (v, vp)):
            pages = self.order[b, : -(-n // self.page)]
            c = np.empty((len(pages), self.H, self.page, self.D))
            c[..., 0::2] = codes[pages] & 15
            c[..., 1::2] = codes[pages] >> 4
            pr = par[pages].astype(np.float64)
            c = c.reshape(*c.shape[:-1], -1, GROUP)
            with np.errstate(invalid="ignore"):
                x = pr[..., 0:1] + pr[..., 1:2] * c
            out.append(x.reshape(len(pages), self.H, self.page, self.D).transpose(1, 0, 2, 3).reshape(self.H, -1, self.D)[:, :n])
        return out


def attend64(q, pool, lengths, q_start, causal, scale=None, cos=None, sin=None):
    """q [B, T, H, D] -> output float64, and per element how far a result may be off: see `tolerance`."""
    B, T, H, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    rep = H // pool.H
    out, weight_v, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, T, H, 1))
    for b in range(B):
        n = int(lengths[b])
        if n <= 0:
            continue
        keys, values = pool.values(b, n)
        pos = (n - T if q_start is None else int(q_start[b])) + np.arange(T)
        x = q[b].astype(np.float64)
        if cos is not None:
            x = rotate(x[None], cos, sin, np.clip(pos, 0, len(cos) - 1)[None], np.float64)[0]
        for h in range(H):
            with np.errstate(invalid="ignore"):
                s = x[:, h] @ keys[h // rep].T * scale
            if causal:
                s = np.where(np.arange(n)[None, :] <= pos[:, None], s, -np.inf)
            m = s.max(-1, keepdims=True)
            with np.errstate(invalid="ignore"):
                e = np.where(s == -np.inf, 0.0, np.exp(s - np.where(np.isinf(m) & (m < 0), 0.0, m)))
            total = e.sum(-1, keepdims=True)
            p = e / np.where(total == 0, 1.0, total)
            v = values[h // rep]
            # a value that a row does not see does not reach it, not even as 0 * NaN
            out[b, :, h] = sum_seen(p, v)
            weight_v[b, :, h] = sum_seen(p, np.abs(v))
            reach[b, :, h, 0] = (np.abs(x[:, h]) @ np.nan_to_num(np.abs(keys[h // rep])).T).max(-1) * scale
    return out, weight_v, reach


def sum_seen(p, v):
    bad = ~np.isfinite(v).all(-1)
    if not bad.any():
        return p @ v
    out = p[:, ~bad] @ v[~bad]
    for j in np.flatnonzero(bad):
        seen = p[:, j] != 0
        with np.errstate(invalid="ignore"):
            out[seen] = out[seen] + p[seen, j][:, None] * v[j]
    return out


def tolerance(ref, weight_v, reach, dtype, keys):
    """How far each element may be off.

    A score's error is at most eps times sum_c |q_c k_c| scale ("reach"); softmax weights are then off by twice that, relatively,
    and the output by as much of sum_j p_j |v_j|.  bf16 I/O: q and k in fp16, 2^-12 each; p and v in fp16, 2^-12 each, a few fp32
    roundings; the result in bf16, 2^-9 (taken twice).  fp32 I/O: operands of 22 bits, sums of up to `keys` fp32 terms.
    """
    if dtype == "bf16":
        eps, rest, last = 2.0 ** -11, 2.0 ** -10, 2.0 ** -8
    else:
        eps, rest, last = 2.0 ** -19, 2.0 ** -18 + keys * 2.0 ** -24, 2.0 ** -22
    return last * np.abs(ref) + (2 * eps * reach + rest) * weight_v + 1e-30
