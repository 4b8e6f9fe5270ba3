"""The paged 4-bit cache from its definition: quantisation in fp32 with numpy, attention in 64 bits with its error bound."""
import numpy as np
import torch

TINY = np.float32(2.0 ** -100)


def floor_bf16(x):
    """Largest bf16 not above x, elementwise (fp32)."""
    x = np.asarray(x, np.float32)
    bits = x.view(np.uint32)
    cut = bits & np.uint32(0xffff0000)
    down = np.where((x < 0) & (cut != bits), cut + np.uint32(0x10000), cut)
    return down.astype(np.uint32).view(np.float32)


def quantise(x):
    """fp32 [..., dh] -> (codes, zero, scale, the fp32 values they stand for)."""
    with np.errstate(all="ignore"):
        x = np.asarray(x, np.float32)
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        zero = floor_bf16(lo)
        scale = -floor_bf16(-((hi - zero) / np.float32(15)))
        bad = ~(np.isfinite(x).all(-1, keepdims=True) & np.isfinite(scale))
        flat = (scale < TINY) | bad
        code = np.where(flat, 0, np.clip(np.rint((x - zero) / np.where(flat, np.float32(1), scale)), 0, 15))
        scale = np.where(bad, np.float32("nan"), np.where(flat, np.float32(0), scale)).astype(np.float32)
        zero = np.where(bad, np.float32("nan"), zero).astype(np.float32)
        return code.astype(np.float32), zero, scale, zero + scale * code.astype(np.float32)


def rotate(x, table, pos):
    """fp32 [n, heads, dh] turned by rows `pos` of table [*, dh/2, 2]; every product rounded."""
    x = np.asarray(x, np.float32)
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    c, s = table[pos][:, None, :, 0], table[pos][:, None, :, 1]
    return np.concatenate([a * c - b * s, b * c + a * s], -1).astype(np.float32)


def attention(q, K, V, scale, sees):
    """64 bits: q [n, hq, dh]; K, V = (code, zero, scale, value) of slots [s, hk, ...]; sees [n, s] -> out and a bound on the kernels'
    error before the output is rounded, as a function of whether a weight is one fp16 number (else two).

    What the kernels round: a score's sums (fp32, at most 2^-20 of the sum of the absolute values of its terms), q where it is
    fp32 (22 bits, inside the same), 2^x (2^-21), a weight times the scale of V to fp16 (2^-12 relative; 2^-34 of the largest scale
    absolute, where fp16 runs out of exponent) and the sums of the output (2^-20 of the absolute terms)."""
    n, hq, dh = q.shape
    hk = K[0].shape[1]
    G = hq // hk
    out = np.zeros((n, hq, dh))
    one, two = np.zeros((n, hq, dh)), np.zeros((n, hq, dh))
    for h in range(hq):
        k, v = K[3][:, h // G].astype(np.float64), V[3][:, h // G].astype(np.float64)
        kz, ks = np.abs(K[1][:, h // G]), K[2][:, h // G]
        vz, vs, vc = V[1][:, h // G].astype(np.float64), V[2][:, h // G].astype(np.float64), V[0][:, h // G].astype(np.float64)
        s = scale * (q[:, h].astype(np.float64) @ k.T)
        terms = scale * np.abs(q[:, h]).sum(-1, keepdims=True) * (15.0 * ks + kz).astype(np.float64).T          # [n, s]
        s = np.where(sees, s, -np.inf)
        top = s.max(-1, keepdims=True, initial=-np.inf)
        some = np.isfinite(top)
        p = np.where(sees, np.exp(s - np.where(some, top, 0.0)), 0.0)
        p = p / np.where(some, p.sum(-1, keepdims=True), 1.0)
        out[:, h] = p @ np.where(sees.any(0)[:, None], v, 0.0)
        seen = sees.any(0)[:, None]
        spread = p @ np.where(seen, vs * np.abs(vc - 8), 0.0)
        size = p @ np.where(seen, np.abs(vz) + 15 * vs, 0.0)
        off = 2.0 ** -20 * (1 + np.where(sees, terms, 0.0).max(-1, keepdims=True, initial=0.0)) * 2 * size
        under = len(k) * 2.0 ** -31 * np.where(seen, vs, 0.0).max(initial=0.0)
        one[:, h] = off + 2.0 ** -12 * spread + under
        two[:, h] = off + 2.0 ** -22 * spread + under * 2.0 ** -9
    return out, one, two


def check(got, out, one, two, dtype, what):
    half = torch.finfo(dtype).eps / 2
    bound = (two if dtype == torch.float32 else one) * (1 + half) + half * np.abs(out) + 1e-30
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25
    err = np.abs(got.double().cpu().numpy() - out)
    assert np.isfinite(err).all(), f"{what}: not finite at {np.argwhere(~np.isfinite(err))[:4].tolist()}"
    worst = float((err / bound).max(initial=0.0))
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound at {np.unravel_index(np.argmax(err / bound), err.shape)}, error {err.max():.3g}"
    return worst


def tree_masks(n, rng):
    """Ancestor sets of a random tree of n nodes: bool [n, n] and the two 64-bit words a row."""
    sees = np.zeros((n, n), bool)
    for u in range(n):
        if u:
            sees[u] = sees[rng.integers(max(0, u - 9), u)]
        sees[u, u] = True
    words = np.zeros((n, 128), bool)
    words[:, :n] = sees
    return sees, np.packbits(words, axis=1, bitorder="little").view(np.uint64).view(np.int64)
