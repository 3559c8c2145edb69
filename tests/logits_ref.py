"""Token log-probabilities, entropies, their gradients and the clipped policy loss in plain numpy (64 bits), and the
error bounds of the fp32 kernels, for their tests."""
import numpy as np

E24 = 2.0 ** -24                                       # half a step of fp32
HALF_STEP = {"f32": E24, "bf16": 2.0 ** -8}


def softmax_parts(x, T):
    """y = x/T - max, p, ln sum e^y and the entropy of rows x [R, V]."""
    y = np.asarray(x, np.float64) / T
    y = y - y.max(1, keepdims=True)
    e = np.exp(y)
    s = e.sum(1, keepdims=True)
    p = e / s
    lp = y - np.log(s)
    return y, p, lp, np.log(s)[:, 0], -(np.where(p > 0, p * np.where(p > 0, lp, 0), 0)).sum(1)


def logprobs(x, tok, T):
    """logp, entropy, norm; rows without a token are zeros."""
    x = np.asarray(x, np.float64)
    _, _, lp, ls, H = softmax_parts(x, T)
    ok = (tok >= 0) & (tok < x.shape[1])
    at = np.where(ok, tok, 0)
    logp = lp[np.arange(len(tok)), at]
    return np.where(ok, logp, 0), np.where(ok, H, 0), np.where(ok[:, None], np.stack((x.max(1), ls), 1), 0)


def gradient(x, tok, T, g, h):
    """d(sum g logp + h H)/dx, and the scale of the terms that each value is a sum of."""
    _, p, lp, _, H = softmax_parts(x, T)
    ok = (tok >= 0) & (tok < x.shape[1])
    g, h = np.where(ok, g, 0), np.where(ok, h, 0)
    lp0 = np.where(p > 0, lp, 0)
    d = -g[:, None] * p - h[:, None] * p * (lp0 + H[:, None])
    scale = p * (np.abs(g) + np.abs(h) * H)[:, None] + np.abs(h)[:, None] * p * np.abs(lp0)
    r = np.arange(len(tok))[ok]
    d[r, tok[ok]] += g[ok]
    scale[r, tok[ok]] += np.abs(g[ok])
    return d / T, scale / T


def policy(x, tok, T, old, adv, w, ref=None, beh=None, clip_low=0.2, clip_high=0.2, kl=0.0, ent=0.0, is_low=0.5, is_high=2.0):
    """stats, logp, entropy, and the gradients g, h by the rows' ln p and H."""
    logp, H, _ = logprobs(np.where(np.isfinite(x).any(1, keepdims=True), x, 0), tok, T)
    with np.errstate(invalid="ignore", over="ignore"):
        on = (w != 0) & (tok >= 0) & (tok < x.shape[1])
        keep = on.copy()
        if beh is not None:
            f = np.exp(np.asarray(old, np.float64) - beh)
            keep &= (f >= is_low) & (f <= is_high)
        z = lambda v: np.where(keep, v, 0.0).astype(np.float64)  # noqa: E731
        logp, H, w_, A = z(logp), z(H), z(w), z(adv)
        r = np.exp(logp - z(old))
        free, cut = r * A, np.clip(r, 1 - clip_low, 1 + clip_high) * A
        clipped = cut < free
        d = z(ref) - logp if ref is not None else np.zeros_like(logp)
        k = np.expm1(d) - d if ref is not None else d
        pg = -np.minimum(free, cut)
        g = w_ * (np.where(clipped, 0, -free) + (kl * -np.expm1(d) if ref is not None else 0))
        h = -ent * w_
        stats = np.array([(w_ * (pg + kl * k - ent * H)).sum(), (w_ * pg).sum(), (w_ * k).sum(), (w_ * H).sum(), (w_ * clipped).sum(),
                          np.where(on & ~keep, w, 0).sum()])
    return stats, logp, H, g, h


def sum_error(V, y_max):
    """Relative error of the sums over a row: each term's exponent is off by two roundings relative to it (|y| log2 e of
    them at most) and one of the factor log2(e)/T, its power by two steps; a thread adds at most V/64 terms one after
    another, moves its sums a few times and joins 6 + 16 more."""
    return E24 * (3 * 1.45 * y_max + 4 + V / 64 + 8 + 22)
