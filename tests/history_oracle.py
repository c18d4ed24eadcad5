"""The operators of include/rec_history.h in 64 bits on the CPU, from their definitions, and how far
a kernel's outputs may be from them.  Shares no code with the library."""
import numpy as np
import torch

EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] +
                [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])      # the last code is NaN


def quantise(x, fmt):
    """x float64 [n, 32] -> (codes uint8 [n, 32], scale bytes [n]): the nearest value, ties to the even code."""
    table, top, over, cap = (E2M1, 2, 1.75, 125) if fmt == "mx4" else (E4M3, 8, 1.8125, 119)
    codes, scales = np.zeros(x.shape, np.uint8), np.zeros(len(x), np.uint8)
    for i, row in enumerate(x):
        amax = np.abs(row).max()
        if not np.isfinite(row).all():
            scales[i] = 255
            continue
        e = -110
        if amax > 0:
            m, e = np.frexp(amax)
            e = min(max(e - 1 - top + (2 * m > over), -110), cap)
        scales[i] = e + 127
        u = np.abs(row) * 2.0 ** -e
        for j in range(32):
            d = np.abs(table - u[j])
            best = np.flatnonzero(d == d.min())
            c = best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]
            codes[i, j] = c | ((0x80 if fmt == "mx8" else 8) if np.signbit(row[j]) else 0)
    return codes, scales


def values(codes, fmt):
    if fmt == "mx4":
        return np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    return np.where(codes & 128, -1.0, 1.0) * E4M3[codes & 127]


def scale_values(bytes_):
    return np.where(bytes_ == 255, np.nan, 2.0 ** (bytes_.astype(np.float64) - 127))


def row_of(pages, fmt, d, page_tokens, slot, head):
    """K and V of one slot and head from the pages' bytes (uint8 numpy [pages, heads, groups, bytes])."""
    page, at = divmod(int(slot), page_tokens)
    g, t = pages[page, head, at // 16], at % 16
    per = d // 2 if fmt == "mx4" else d
    k, v = g[:16 * per].reshape(16, per)[t], g[16 * per:32 * per].reshape(d // 2, 16, -1)[:, t]
    ks = g[32 * per:32 * per + d // 2].reshape(16, d // 32)[t]
    vs = g[32 * per + d // 2:].reshape(d // 32, 16)[:, t]
    if fmt == "mx4":
        k = np.stack((k & 15, k >> 4), 1).reshape(-1)
        v = np.stack((v[:, 0] & 15, v[:, 0] >> 4), 1)
    vc = np.zeros(d, np.uint8)
    for i in range(d // 32):
        vc[32 * i:32 * i + 16], vc[32 * i + 16:32 * i + 32] = v[16 * i:16 * i + 16, 0], v[16 * i:16 * i + 16, 1]
    return (values(k, fmt) * np.repeat(scale_values(ks), 32), values(vc, fmt) * np.repeat(scale_values(vs), 32))


def sees(p, j, window, sinks):
    return 0 <= j <= p and (window == 0 or p - j < window or j < sinks)


def attend_rows(q, k, v, positions, scale, window, sinks, dtype, hidden=()):
    """q [M, D], k and v [L, D] float64, positions [M] -> (outputs [M, D], how far off each may be [M, D]).
    `hidden`: keys that nobody sees.

    Errors counted, relative to A = sum_j w_j |v_j|: the output's rounding (of itself), the weights' rounding to
    the type that they are multiplied in, scores summed in fp32 (each of the D + 8 steps half an fp32 step of the sum of
    magnitudes), q held to 2^-16 of its largest element, exponentials to 2^-20; an error of a score counts twice,
    in the weight and in their sum."""
    out, off = np.zeros_like(q), np.zeros_like(q)
    u = EPS[dtype]
    for m, p in enumerate(positions):
        js = [j for j in range(min(p, len(k) - 1) + 1) if sees(p, j, window, sinks) and j not in hidden]
        if not js:
            continue
        with np.errstate(all="ignore"):
            x = k[js] @ q[m] * scale
            w = np.exp(x - x.max())
            w /= w.sum()
            out[m] = w @ v[js]
            score = abs(scale) * ((np.abs(k[js]) @ np.abs(q[m])).max() * (len(q[m]) + 8) * 2.0 ** -24
                             + 2.0 ** -16 * np.abs(q[m]).max() * np.abs(k[js]).sum(1).max())
            off[m] = u * np.abs(out[m]) + (u + 2 * score + 2.0 ** -20) * (w @ np.abs(v[js])) + 2.0 ** -25
    return out, off


def assert_close(got, want, off, what=""):
    """got: tensor; equal where the oracle is not finite, else within `off`."""
    got = got.double().cpu().numpy().reshape(want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, "NaN", np.argwhere(np.isnan(got) != np.isnan(want))[:5])
    fine = np.isfinite(want)
    bad = np.abs(got[fine] - want[fine]) > off[fine]
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got[fine] - want[fine]) / off[fine])))
