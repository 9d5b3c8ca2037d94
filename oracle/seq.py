"""fp64 forms of the operators around the attention and the scan (test infrastructure; numpy only).

Beside each result stands a bound on what fp32 arithmetic may differ from it (``*_bound``), from the
operations' roundings: u = 2^-24 is half a step of fp32, the hardware's exp2, reciprocal, root and
reciprocal root are within a step (2 u)."""
import numpy as np

U = 2.0 ** -24


def half_step(x, dtype):
    """The largest error of rounding x to dtype ("f32", "bf16")."""
    return np.abs(x) * (2.0 ** -8 if dtype == "bf16" else U)


# ---- norm ------------------------------------------------------------------------------------

def norm_adds(D, vec):
    """Additions on the way of one value into the sum of squares: those of a lane, then 10 over lanes and waves."""
    pieces = -(-D // vec)
    per = -(-pieces // 64) if pieces <= 256 else -(-pieces // 256) if pieces <= 1024 else -(-pieces // 1024)
    return per * vec + 10


def rms_norm(x, weight, residual=None, eps=1e-6, adds=42):
    """(y, s, rstd, relative bound on y): s one rounding; the sum's additions (halved by the root); rsq; two
    products."""
    s = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt((s * s).mean(-1) + eps)
    return s * rstd[..., None] * weight, s, rstd, (adds / 2 + 8) * U


def rms_norm_bwd(dy, s, weight, rstd, dsum=None, adds=42):
    """(dx, dweight, bound on dx, bound on dweight)."""
    n = s * rstd[..., None]
    dn = dy * weight
    along = (dn * n).mean(-1, keepdims=True)
    dx = (dn - n * along) * rstd[..., None]
    bound = rstd[..., None] * (4 * U * np.abs(dn) + np.abs(n) * (adds + 4) * U * np.abs(dn * n).mean(-1, keepdims=True)
                               + 4 * U * np.abs(n * along))
    if dsum is not None:
        dx = dx + dsum
        bound = bound + U * np.abs(dx)
    rows = dy.reshape(-1, dy.shape[-1]).shape[0]
    dw = (dy * n).reshape(-1, dy.shape[-1])
    return dx, dw.sum(0), bound + U * np.abs(dx), (rows + 30) * U * np.abs(dw).sum(0)


def e4m3(v):
    """v (|v| <= 448 up to rounding) rounded to e4m3, ties to even."""
    a = np.maximum(np.abs(v), 2.0 ** -6)
    step = np.exp2(np.floor(np.log2(a)) - 3)
    return np.rint(v / step) * step


def quantize(y, group):
    """(q, scales) of y [rows, D]: a scale for each `group` channels (0: each row)."""
    rows, D = y.shape
    group = group or max(D, 1)
    cuts = range(0, D, group)
    top = np.stack([np.abs(y[:, j:j + group]).max(1) for j in cuts], 1)
    scales = np.where(top > 0, np.maximum(top / 448.0, 2.0 ** -126), 1.0)
    q = np.concatenate([e4m3(y[:, j:j + group] / scales[:, k:k + 1]) for k, j in enumerate(cuts)], 1)
    return q, scales


# ---- rotary ----------------------------------------------------------------------------------

def rotary(x, freqs, positions, interleaved=False, mscale=1.0, inverse=False):
    """(y, bound): x [B, L, heads, d], positions [B, L] or [B, L, 2].  cos and sin are off by the rounding of
    half a turn (2 pi 2^-26) and their own (2 u each, mscale u); then two products and a sum."""
    half = len(freqs)
    pos = positions.astype(np.float64)
    if pos.ndim == 3:
        pos = np.concatenate([np.repeat(pos[..., :1], half // 2, -1), np.repeat(pos[..., 1:], half // 2, -1)], -1)
        ang = pos * freqs
    else:
        ang = pos[..., None] * freqs
    c, s = (f(ang)[:, :, None] * mscale for f in (np.cos, np.sin))
    if inverse:
        s = -s
    ia, ib = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., ia], x[..., ib]
    y, bound = x.copy(), np.zeros_like(x)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    bound[..., ia] = bound[..., ib] = (np.abs(a) + np.abs(b)) * abs(mscale) * (2 * np.pi * 2.0 ** -26 + 8 * U)
    # fp64 angles: position times frequency over 2 pi is off by a few 2^-53 turns of its size
    far = np.abs(ang).max(-1)[..., None, None] * 2.0 ** -50
    return y, bound + (np.abs(x).max(-1, keepdims=True) * 2 * abs(mscale)) * far * (bound > 0)


# ---- gated linear recurrence -----------------------------------------------------------------

def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def _gates(x, r, i, lam, c):
    rate = c * np.logaddexp(0.0, lam)
    gr, gi = _sigmoid(r), _sigmoid(i)
    z = rate * gr
    a = np.exp(-z)
    m2 = -np.expm1(-2 * z)
    return gr, gi, z, a, m2, np.sqrt(m2) * gi * x


def gated_scan(x, r, i, lam, h0=None, lengths=None, c=8.0):
    """(h, h_last, bound on h, bound on h_last); rows past a sequence's end are 0.

    Per step: z is off by 8 u z (rate, sigmoid, product), a by that and exp2's 2 u, u by 20 u (m^2 from the
    series or 1 - a^2 >= 0.22, its root, the gate, three products); twice that for the states' joining
    over runs and chunks.  A run is reduced from zero and the state that enters it added afterwards, so
    roundings are relative to the parts and not to their sum: they are counted against `mag`, the same
    recurrence over absolute values, which is at least every such part."""
    B, L, D = x.shape
    h = np.zeros((B, D)) if h0 is None else h0.copy()
    e, mag = np.zeros((B, D)), np.abs(h)
    out, bound = np.zeros_like(x), np.zeros_like(x)
    _, _, z, a, _, u = _gates(x, r, i, lam, c)
    lens = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    for t in range(L):
        live = (t < lens)[:, None]
        with np.errstate(invalid="ignore"):
            nh = a[:, t] * h + u[:, t]
            ne = a[:, t] * e + 2 * U * ((22 + 8 * z[:, t]) * a[:, t] * mag + 20 * np.abs(u[:, t]))
            nm = a[:, t] * mag + np.abs(u[:, t])
        h, e, mag = np.where(live, nh, h), np.where(live, ne, e), np.where(live, nm, mag)
        out[:, t], bound[:, t] = np.where(live, h, 0), np.where(live, e, 0)
    return out, h, bound, e + U * np.abs(h)


def gated_scan_bwd(x, r, i, lam, h0, lengths, dh, d_last, c=8.0):
    """(dx, dr, di, dlam, dh0) and a bound on each (g's roundings counted as h's are, against the recurrence over
    absolute values)."""
    B, L, D = x.shape
    gr, gi, z, a, m2, u = _gates(x, r, i, lam, c)
    h, _, eh, _ = gated_scan(x, r, i, lam, h0, lengths, c)
    h0 = np.zeros((B, D)) if h0 is None else h0
    prev = np.concatenate([h0[:, None], h[:, :-1]], 1)
    eprev = np.concatenate([np.zeros((B, 1, D)), eh[:, :-1]], 1)
    lens = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    p = np.zeros((B, D)) if d_last is None else d_last.copy()
    e, mag = np.zeros((B, D)), np.abs(p)
    dx, dr, di = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    bx, br, bi = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    share, bshare, ashare = np.zeros(D), np.zeros(D), np.zeros(D)
    for t in range(L - 1, -1, -1):
        live = (t < lens)[:, None]
        zt, at, mt, ut = z[:, t], a[:, t], m2[:, t], u[:, t]
        with np.errstate(invalid="ignore", divide="ignore"):
            g = p + (0 if dh is None else dh[:, t])
            mag_g = mag + (0 if dh is None else np.abs(dh[:, t]))
            eg = e + 2 * U * mag_g
            over = np.where(zt > 0, zt / mt, 0.5)
            t1, t2 = over * at * at * ut, zt * at * prev[:, t]
            el = g * (t1 - t2)
            bl = eg * (np.abs(t1) + np.abs(t2)) + np.abs(g) * (zt * at * eprev[:, t]
                                                               + 60 * U * (1 + zt) * (np.abs(t1) + np.abs(t2)))
            m = np.sqrt(mt)
            vals = (g * m * gi[:, t], el * (1 - gr[:, t]), g * ut * (1 - gi[:, t]), el)
            bounds = (eg * m * gi[:, t] + 24 * U * np.abs(g * m * gi[:, t]),
                      bl * (1 - gr[:, t]) + 12 * U * np.abs(el), eg * np.abs(ut) + 40 * U * np.abs(g * ut), bl)
            np_, ne = at * g, at * eg + 2 * U * (22 + 8 * zt) * at * mag_g
            nm = at * mag_g
        for dst, v in zip((dx, dr, di, bx, br, bi), (*vals[:3], *bounds)):
            dst[:, t] = np.where(live, v, 0)
        share += np.where(live, vals[3], 0).sum(0)
        ashare += np.where(live, np.abs(vals[3]), 0).sum(0)
        bshare += np.where(live, bounds[3], 0).sum(0)
        p, e, mag = np.where(live, np_, p), np.where(live, ne, e), np.where(live, nm, mag)
    f = _sigmoid(lam) / np.logaddexp(0.0, lam)
    dlam = share * f
    # shares are added over runs, chunks and sequences: a few hundred additions at most
    return (dx, dr, di, dlam, p), (bx, br, bi, f * (bshare + 300 * U * ashare) + 8 * U * np.abs(dlam),
                                   e + U * np.abs(p))
