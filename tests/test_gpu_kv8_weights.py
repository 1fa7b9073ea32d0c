"""Attention over the paged 8-bit cache where small weights make the result: a key that takes nearly all of the softmax
but has no value, in front of many keys that share what is left.

Tolerance, per element: the bf16 output is off by at most half a step, 2^-8 |ref|; a weight is rounded to fp16, 2^-11 of
itself or, where fp16 has no more normal numbers, 2^-25 next to a largest weight of 2^9 or more (both taken with the
value's page scale s): with p the softmax weights, 2^-34 max(p s) sum |code|; scores as in test_gpu_kv8."""
import numpy as np
import pytest
import torch

from oracle import kv8 as ok
from test_gpu_kv8 import DEV, Case, attend

pytestmark = pytest.mark.gpu

ONE = {"e4m3": 0x38, "int8": 64}          # a code in the middle of the format: 1 or 64


def sink_case(B, n, fmt, hkv, pt, seed):
    """Key 0: a large score and no value.  The others: score 0, values of one sign in equal and random parts."""
    c = Case([n] * B, pt, fmt, hkv, 128, seed=seed, scale_exp=(-6, -6))
    for w in (0, 1):
        codes = c.pool.codes[w]
        codes[:] = 0 if w == 0 else ONE[fmt]
        if w == 1:
            codes[..., 64:] = c.rng.integers(1, ONE[fmt] + 1, codes[..., 64:].shape)
        for p in c.pages:
            codes[0, p[0], :, 0] = ONE[fmt] if w == 0 else 0
        c.t[w].view(torch.uint8).copy_(torch.from_numpy(codes))
    return c


def exact(c, q, kn, vn, i, rows):
    """The oracle's rows with their tolerance."""
    R, H, d = q.shape[1:]
    out, tol = np.zeros((len(rows), H, d)), np.zeros((len(rows), H, d))
    for h in range(c.hkv):
        k, v = (c.pool.read(w, 0, h, c.pages[i], c.lens[i]) for w in (0, 1))
        s = np.repeat([float(c.pool.scales[1][0, p, h]) for p in c.pages[i]], c.pt)[:c.lens[i]]
        new = [x[i, :, h].double().numpy() for x in (kn, vn)]
        # a new row's scale puts its largest element where a page's largest code is
        top = np.abs(new[1]).max(1)
        s_new = np.where(top > 0, 2.0 ** np.floor(np.log2(np.where(top > 0, top, 1.0))), 2.0 ** -64) * 2.0 ** (-8 if c.fmt == "e4m3" else -6)
        for j in range(h * (H // c.hkv), (h + 1) * (H // c.hkv)):
            for z, x in enumerate(rows):
                ks, vs = np.concatenate([k, new[0][:x + 1]]), np.concatenate([v, new[1][:x + 1]])
                sc = np.concatenate([s, s_new[:x + 1]])
                qq = q[i, x, j].double().numpy()
                t = ks @ qq / np.sqrt(d)
                p = np.exp(t - t.max())
                p /= p.sum()
                out[z, j] = p @ vs
                absx = (np.abs(ks) @ np.abs(qq)).max() / np.sqrt(d)
                tol[z, j] = (2.0 ** -8 * np.abs(out[z, j]) + (2.0 ** -10 + 2.0 ** -18 * absx) * (p @ np.abs(vs))
                             + 2.0 ** -34 * (p * sc).max() * (np.abs(vs) / sc[:, None]).sum(0))
    return out, tol


@pytest.mark.parametrize("score", [12.0, 16.0, 17.5, 19.0])
@pytest.mark.parametrize("B,R,H,hkv,n,fmt", [(1, 1, 5, 1, 8193, "e4m3"), (64, 1, 5, 1, 8193, "int8"), (16, 1, 8, 8, 8193, "e4m3"),
                                             (1, 24, 1, 1, 8193, "int8"), (1, 60, 5, 1, 8193, "e4m3"), (40, 60, 5, 1, 8193, "int8"),
                                             (1, 1, 8, 1, 131001, "int8"), (2, 300, 1, 1, 8193, "e4m3")])
def test_many_small_weights_next_to_a_key_without_value(B, R, H, hkv, n, fmt, score):
    if fmt == "int8":
        unit = 64 * 2.0 ** -6
    else:
        unit = 2.0 ** -6
    c = sink_case(B, n, fmt, hkv, 64, seed=R + B)
    q = torch.full((B, R, H, 128), score / (128 * unit / np.sqrt(128)), dtype=torch.bfloat16)
    kn = torch.zeros(B, R, hkv, 128, dtype=torch.bfloat16)
    vn = c.bf16(B, R, hkv, 128).abs() * 2.0 ** -6
    got = attend(c, 0, q.to(DEV), kn.to(DEV), vn.to(DEV), n).double().cpu().numpy()
    rows = sorted({0, R // 2, R - 1})
    for i in sorted({0, B // 2, B - 1}):
        want, tol = exact(c, q, kn, vn, i, rows)
        err = np.abs(got[i][rows] - want)
        assert np.all(err <= tol), (i, float((err / np.maximum(np.abs(want), 1e-30)).max()), float(np.abs(want).max()))
