"""GPU parity of the norm, the rotary positions and the gated linear recurrence against the fp64 forms of
oracle/seq.py, at the sizes and masks where they can go wrong.  Tolerances are the bounds derived there, plus
half a step of the output's type."""
import numpy as np
import pytest
import torch

from oracle import seq as O
from paper_2407_02109_amd import seq as S

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    S.load_seq_library()


def _say(*a):
    print("[case]", *a, flush=True)


def _f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def _close(name, got, want, bound):
    got = _f64(got)
    ok = (np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want))
    if not ok.all():
        at = tuple(np.argwhere(~ok)[0])
        raise AssertionError("%s: %d of %d off, first at %s: %r, expected %r +- %.3g" % (
            name, (~ok).sum(), ok.size, at, got[at], want[at], np.broadcast_to(bound, ok.shape)[at]))


def _out(ref, bound, dt):
    """The bound with the output's rounding; and values below the least normal fp32 (2^-126 = 1.2e-38) may vanish on
    the way, of which a sum over fewer than 10^4 tokens makes less than 2e-34."""
    return bound + O.half_step(ref, dt) + O.half_step(bound, dt) + 2e-34


def _randn(shape, dt, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(TYPES[dt]).cuda()


# ---- norm ------------------------------------------------------------------------------------

# rows, D: one token; every number of waves per row and pieces per lane; widths that no piece divides; rows
# that are read again
NORM_SHAPES = [(1, 1), (3, 7), (1, 768), (5, 512), (7, 513), (9, 1000), (1030, 130), (4, 2049), (3, 4100), (2, 8192),
               (2, 8193), (3, 16384), (2, 16385), (1, 32769), (5000, 96), (2, 40001)]


@pytest.mark.parametrize("wdt", ["same", "f32"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "%dx%d" % s)
def test_norm(shape, dt, wdt):
    _say("norm", shape, dt, wdt)
    rows, D = shape
    wdt = dt if wdt == "same" else wdt
    adds = O.norm_adds(D, 8 if dt == "bf16" else 4)
    x, r = _randn(shape, dt, 1, 3.0), _randn(shape, dt, 2)
    w = (1 + 0.2 * _randn((D,), "f32", 3)).to(TYPES[wdt])
    for res in (None, r):
        y, s, rstd = S.add_rms_norm_fwd_train(x, w, res)
        ry, rs, rr, rel = O.rms_norm(_f64(x), _f64(w), None if res is None else _f64(res), 1e-6, adds)
        _close("sum", s, rs, O.half_step(rs, dt) + 2 * O.U * np.abs(rs))
        _close("rstd", rstd, rr, rel * rr)
        _close("y", y, ry, _out(ry, rel * np.abs(ry), dt))
        y2, s2 = S.add_rms_norm(x, w, res)
        assert torch.equal(y, y2) and torch.equal(s, s2)
        dy, ds = _randn(shape, dt, 4), (None if res is None else _randn(shape, dt, 5))
        dx, dw = S.add_rms_norm_bwd(dy, s, w, rstd, ds)
        rdx, rdw, bdx, bdw = O.rms_norm_bwd(_f64(dy), _f64(s), _f64(w), _f64(rstd), None if ds is None else _f64(ds), adds)
        _close("dx", dx, rdx, _out(rdx, bdx, dt))
        _close("dw", dw, rdw, bdw)


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "%dx%d" % s)
def test_norm_q8(shape, dt, group):
    _say("q8", shape, dt, group)
    rows, D = shape
    x, r = _randn(shape, dt, 1, 3.0), _randn(shape, dt, 2)
    x[0, : D // 2] = 0
    r[0, : D // 2] = 0          # groups of zeros
    w = (1 + 0.2 * _randn((D,), "f32", 3)).to(TYPES[dt])
    q, sc, s = S.add_rms_norm_q8(x, w, r, group=group)
    ry, rs, _, rel = O.rms_norm(_f64(x), _f64(w), _f64(r), 1e-6, O.norm_adds(D, 8 if dt == "bf16" else 4))
    _, rsc = O.quantize(ry, group)
    assert q.dtype == torch.float8_e4m3fn and tuple(sc.shape) == rsc.shape
    _close("scales", sc, rsc, (rel + 4 * O.U) * rsc)
    wide = lambda t: np.repeat(t, group or D, 1)[:, :D]
    step = np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * wide(rsc))   # half a step of e4m3
    got = _f64(q) * wide(_f64(sc))
    assert (np.abs(got - ry) <= step * (1 + 1e-5) + rel * np.abs(ry)).all()
    assert torch.equal(s, S.add_rms_norm(x, w, r)[1])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_rows_of_views_and_in_place(dt):
    _say("norm views", dt)
    wide = _randn((4, 50, 300), dt, 1)
    x, r = wide[..., 3:133], wide[..., 140:270]
    w = _randn((130,), dt, 2)
    y, s = S.add_rms_norm(x, w, r)
    yc, sc = S.add_rms_norm(x.contiguous(), w, r.contiguous())
    assert torch.equal(y, yc) and torch.equal(s, sc) and y.shape == x.shape
    # the residual stream and the input overwritten
    xi, ri = x.contiguous(), r.contiguous()
    yo, so = S.add_rms_norm(xi, w, ri, out=xi, sum_out=ri)
    assert yo is xi and so is ri and torch.equal(yo, y) and torch.equal(so, s)
    xw, rw = _randn((2, 40001), dt, 3), _randn((2, 40001), dt, 4)   # rows that are read again
    ww = _randn((40001,), dt, 5)
    y, s = S.add_rms_norm(xw, ww, rw)
    S.add_rms_norm(xw, ww, rw, out=rw, sum_out=xw)
    assert torch.equal(rw, y) and torch.equal(xw, s)
    rows = S.add_rms_norm(x[:, :1].expand(4, 50, 130)[0], w)[0]     # one row many times
    assert torch.equal(rows, rows[:1].expand_as(rows))


def test_norm_carries_nan_and_infinity():
    _say("norm nan")
    x = _randn((4, 256), "bf16", 1)
    x[0, 5], x[1, 200] = float("nan"), float("inf")
    w = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    y, _ = S.add_rms_norm(x, w)
    assert torch.isnan(y[0]).all() and torch.isnan(y[1, 200]) and (y[1, :200] == 0).all()
    assert torch.isfinite(y[2:].float()).all()
    q, sc, _ = S.add_rms_norm_q8(x, w, group=128)
    assert torch.isnan(sc[0]).all() and torch.isnan(q[0].float()).all()
    assert sc[1, 0] == 1 and torch.isnan(sc[1, 1]) and torch.isfinite(sc[2:]).all()
    assert torch.isfinite(q[2:].float()).all()


def test_norm_backward_is_the_forwards_difference():
    """fp32, against central differences of the fp32 forward summed in fp64: its rounding (2^-24 of |y| over
    2 d = 0.02, over 40 channels) and the third derivative's d^2 stay below 5e-4 of the gradient's largest value."""
    _say("norm differences")
    x, w, dy = _randn((2, 40), "f32", 1), _randn((40,), "f32", 2), _randn((2, 40), "f32", 3)
    _, s, rstd = S.add_rms_norm_fwd_train(x, w)
    dx, dw = S.add_rms_norm_bwd(dy, s, w, rstd)
    f = lambda a, b: (S.add_rms_norm(a, b)[0].double() * dy.double()).sum()
    for t, g, at in ((x, dx, (1, 7)), (x, dx, (0, 0)), (w, dw, (11,))):
        d = torch.zeros_like(t)
        d[at] = 1e-2
        diff = (f(x + d, w) - f(x - d, w)) / 0.02 if t is x else (f(x, w + d) - f(x, w - d)) / 0.02
        assert abs(diff.item() - g[at].item()) <= 5e-4 * g.abs().max().item()


# ---- rotary ----------------------------------------------------------------------------------

# B, L, hq, hk, d, rot, axes
ROTARY_SHAPES = [(1, 1, 1, 0, 2, 2, 1), (32, 1, 32, 8, 128, 128, 1), (2, 37, 12, 12, 64, 64, 2), (3, 11, 4, 1, 80, 40, 1),
                 (2, 9, 3, 2, 96, 24, 2), (1, 5, 2, 2, 7, 6, 1), (2, 3, 2, 1, 512, 512, 2), (1, 2100, 1, 1, 64, 32, 1),
                 (1, 3, 2, 1, 512, 2, 1), (4, 333, 2, 0, 256, 256, 1)]


@pytest.mark.parametrize("inverse", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ROTARY_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_rotary(shape, dt, interleaved, inverse):
    _say("rotary", shape, dt, interleaved, inverse)
    B, L, hq, hk, d, rot, axes = shape
    q, k = _randn((B, L, hq, d), dt, 1), _randn((B, L, hk, d), dt, 2) if hk else None
    freqs, m = S.rotary_freqs(rot, scaling="parts" if axes == 1 else "none", factor=8.0, axes=axes)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-1000000, 1000000, (B, L) if axes == 1 else (B, L, 2), generator=g).cuda()
    fn = S.rotary_bwd if inverse else S.rotary
    got = fn(q, k, freqs, pos, interleaved, m)
    for name, y, x in (("q", got[0], q), ("k", got[1], k)):
        if x is None:
            assert y is None
            continue
        ref, bound = O.rotary(_f64(x), freqs.cpu().numpy(), pos.cpu().numpy(), interleaved, m, inverse)
        _close(name, y, ref, (bound + O.half_step(bound, dt) + O.half_step(ref, dt)) * (bound > 0))
    again = fn(q, k, freqs, pos.int(), interleaved, m)     # positions of 32 bits
    assert torch.equal(again[0], got[0]) and (k is None or torch.equal(again[1], got[1]))


def test_rotary_layouts_and_in_place():
    """Heads before tokens, q and k side by side in each token, positions shared by the batch: the same values."""
    _say("rotary layouts")
    B, L, hq, hk, d = 3, 17, 6, 2, 64
    buf = _randn((B, L, hq + hk + 1, d), "bf16", 1)
    q, k = buf[:, :, :hq], buf[:, :, hq:hq + hk]
    freqs, m = S.rotary_freqs(32, scaling="linear", factor=2.0)
    pos = torch.arange(L, device="cuda")[None].expand(B, L)
    want = S.rotary(q.contiguous(), k.contiguous(), freqs, pos.contiguous(), mscale=m)
    got = S.rotary(q, k, freqs, pos, mscale=m)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    qt, kt = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k))
    assert not qt.is_contiguous()
    got = S.rotary(qt, kt, freqs, pos, mscale=m)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    rest = buf[:, :, -1:].clone()
    S.rotary(q, k, freqs, pos, mscale=m, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(buf[:, :, -1:], rest)
    e = torch.empty(0, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert S.rotary(e, None, freqs, torch.empty(0, 5, dtype=torch.int32, device="cuda"))[0].shape == e.shape


def test_rotary_far_positions_turn_like_near_ones():
    """A frequency of one turn in 2^20 positions: the position 2^20 further is the same rotation (fp64 angles; an
    fp32 angle of 1.6 million radians would be off by 0.06)."""
    _say("rotary far")
    q = _randn((1, 4, 2, 16), "f32", 1)
    freqs = torch.full((8,), 2 * np.pi * (0.25 + 2.0 ** -20), dtype=torch.float64, device="cuda")
    near = torch.arange(4, device="cuda")[None]
    a = S.rotary(q, None, freqs, near)[0]
    b = S.rotary(q, None, freqs, near + (1 << 20))[0]
    # the fp64 product is off by 2^-53 of 1.6e6 radians; then as at the near position
    assert (a - b).abs().max().item() <= 4 * 2.0 ** -24 * q.abs().max().item() * 2


# ---- gated linear recurrence -------------------------------------------------------------------

def _scan_inputs(B, L, D, dt, seed, lam_mean=-3.0):
    x, r, i = (_randn((B, L, D), dt, seed + j) for j in range(3))
    return x, r, i, _randn((D,), "f32", seed + 3) + lam_mean, _randn((B, D), "f32", seed + 4)


# B, L, D, lengths
SCAN_SHAPES = [(1, 1, 1, None), (64, 1, 200, None), (3, 2, 9, None), (2, 16, 66, [16, 3]), (2, 17, 64, None), (1, 256, 70, None), (2, 31, 70, None), (2, 128, 64, None), (1, 129, 65, None),
               (2, 257, 130, [0, 257]), (4, 300, 66, [1, 128, 129, 300]), (1, 1000, 33, None), (2, 4100, 24, [4100, 2049]),
               (3, 640, 1001, [640, 1, 333]), (1, 9000, 8, None),
               (1, 36000, 3, None), (2, 20000, 5, [20000, 11111])]   # chains of more links than one look takes in


@pytest.mark.parametrize("h0", [True, False], ids=["h0", "zero"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SCAN_SHAPES, ids=lambda s: "x".join(map(str, s[:3])) + ("r" if s[3] else ""))
def test_scan(shape, dt, h0):
    _say("scan", shape, dt, h0)
    B, L, D, lengths = shape
    x, r, i, lam, st = _scan_inputs(B, L, D, dt, 10)
    st = st if h0 else None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    args = [_f64(t) for t in (x, r, i, lam)] + [None if st is None else _f64(st), None if lengths is None else np.array(lengths)]
    out = torch.full_like(x, 7.0)
    h, last, states = S.gated_scan_fwd_train(x, r, i, lam, st, n, out=out)
    assert h is out
    ref, rlast, bound, blast = O.gated_scan(*args)
    live = np.arange(L)[None, :, None] < (np.full(B, L) if lengths is None else args[5])[:, None, None]
    past = torch.tensor(np.broadcast_to(~live, x.shape).copy(), device="cuda")
    assert (h[past] == 7.0).all()
    _close("h", torch.where(past, 0, h), ref, _out(ref, bound, dt))
    _close("last", last, rlast, blast)
    h2, last2 = S.gated_scan(x, r, i, lam, st, n, out=torch.full_like(x, 7.0))
    assert torch.equal(h2, h) and torch.equal(last2, last)
    dh, dl = _randn((B, L, D), dt, 20), _randn((B, D), "f32", 21)
    for g, e in ((dh, dl), (None, dl), (dh, None)):
        grads = S.gated_scan_bwd(x, r, i, lam, states, g, e, n)
        refs, bounds = O.gated_scan_bwd(*args, None if g is None else _f64(g), None if e is None else _f64(e))
        for name, got, want, b in zip(("dx", "dr", "di", "dlam", "dh0"), grads, refs, bounds):
            _close(name, got, want, _out(want, b, dt if name in ("dx", "dr", "di") else "f32"))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("lam", [-30.0, -100.0, 12.0], ids=["keeps", "keeps all", "forgets"])
def test_scan_at_the_ends_of_the_gates(dt, lam):
    """Decays that round to 1 (lam = -100: softplus is 0 in fp32) and to 0, gates that are wide open and shut."""
    _say("scan gates", dt, lam)
    B, L, D = 2, 200, 72
    x, r, i, _, h0 = _scan_inputs(B, L, D, dt, 30)
    r, i = r * 30, i * 30
    r[0, 3], i[0, 5], r[1, 7], i[1, 9] = float("-inf"), float("-inf"), float("inf"), float("inf")
    lam = torch.full((D,), lam, device="cuda")
    h, last, states = S.gated_scan_fwd_train(x, r, i, lam, h0)
    args = [_f64(t) for t in (x, r, i, lam, h0)] + [None]
    with np.errstate(all="ignore"):
        ref, rlast, bound, blast = O.gated_scan(*args)
        dh = _randn((B, L, D), dt, 31)
        refs, bounds = O.gated_scan_bwd(*args, _f64(dh), None)
    # a gate's exponential passes fp32's range at 2^128, so sigmoid(r) below 2^-128 vanishes, z below rate 2^-126 with
    # it and m below sqrt(2 rate 2^-126) <= 1.5e-18 (rate <= 96); h and g are sums of at most 200 values of N(0, 1)
    # (|sum| < 400), so what m multiplies is off by less than 6e-16
    tiny = 1e-15
    _close("h", h, ref, _out(ref, bound + tiny, dt))
    _close("last", last, rlast, blast + tiny)
    for name, got, want, b in zip(("dx", "dr", "di", "dlam", "dh0"), S.gated_scan_bwd(x, r, i, lam, states, dh), refs, bounds):
        _close(name, got, want, _out(want, b + tiny, dt if name in ("dx", "dr", "di") else "f32"))


def test_scan_looks_at_no_token_past_the_end():
    _say("scan padding")
    B, L, D = 3, 300, 70
    x, r, i, lam, h0 = _scan_inputs(B, L, D, "bf16", 40)
    n = torch.tensor([129, 0, -3], dtype=torch.int32, device="cuda")
    h, last, states = S.gated_scan_fwd_train(x, r, i, lam, h0, n, out=torch.zeros_like(x))
    dh = _randn((B, L, D), "bf16", 41)
    grads = S.gated_scan_bwd(x, r, i, lam, states, dh, None, n)
    for t in (x, r, i, dh):
        t[0, 129:], t[1:] = float("nan"), float("inf")
    h2, last2, states2 = S.gated_scan_fwd_train(x, r, i, lam, h0, n, out=torch.zeros_like(x))
    assert torch.equal(h, h2) and torch.equal(last, last2) and torch.equal(last[1:], h0[1:])
    for a, b in zip(grads, S.gated_scan_bwd(x, r, i, lam, states2, dh, None, n)):
        assert torch.equal(a, b)
    assert all((g[0, 129:] == 0).all() and (g[1:] == 0).all() for g in grads[:3])


def test_scan_in_parts_and_in_steps():
    """A sequence cut into parts, each from the state that the one before left, and its last tokens one by one:
    fp32, each state within the bound of the whole."""
    _say("scan parts")
    B, L, D = 2, 421, 40
    x, r, i, lam, h0 = _scan_inputs(B, L, D, "f32", 50)
    ref, rlast, bound, blast = O.gated_scan(*(_f64(t) for t in (x, r, i, lam, h0)), None)
    state, t = h0, 0
    parts = []
    for end in (1, 130, 415):
        h, state = S.gated_scan(x[:, t:end], r[:, t:end], i[:, t:end], lam, state)
        parts.append(h)
        t = end
    state = state.clone()
    for t in range(415, L):
        h, new = S.gated_scan_step(x[:, t], r[:, t], i[:, t], lam, state, new_state=state)
        assert new is state and torch.equal(h, state)
        parts.append(h[:, None])
    _close("h", torch.cat(parts, 1), ref, 2 * bound + O.half_step(ref, "f32"))
    _close("last", state, rlast, 2 * blast)


def test_scan_strides():
    """Gates side by side in one projection, tokens before the batch, one token shared by all: the same values."""
    _say("scan strides")
    B, L, D = 2, 150, 70
    both = _randn((B, L, 3 * D + 1), "bf16", 60)
    x, r, i = both[..., :D], both[..., D:2 * D], both[..., 2 * D + 1:]
    lam = _randn((D,), "f32", 61) - 3
    want = S.gated_scan(x.contiguous(), r.contiguous(), i.contiguous(), lam)
    got = S.gated_scan(x, r, i, lam)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    xt = x.transpose(0, 1).contiguous().transpose(0, 1)
    got = S.gated_scan(xt, r, i, lam)
    assert torch.equal(got[0], want[0])
    one = r[:1, :1].expand(B, L, D)
    assert torch.equal(S.gated_scan(x, one, i, lam)[0], S.gated_scan(x, one.contiguous(), i, lam)[0])


def test_empty_problems():
    _say("empty")
    e = torch.empty(0, 5, 8, device="cuda")
    lam = torch.zeros(8, device="cuda")
    h, last = S.gated_scan(e, e, e, lam)
    assert h.shape == e.shape and last.shape == (0, 8)
    z = torch.empty(2, 0, 8, device="cuda")
    h0 = _randn((2, 8), "f32", 1)
    assert torch.equal(S.gated_scan(z, z, z, lam, h0)[1], h0)
    h, last, states = S.gated_scan_fwd_train(z, z, z, lam, h0)
    dl = _randn((2, 8), "f32", 2)
    _, _, _, dlam, dh0 = S.gated_scan_bwd(z, z, z, lam, states, z, dl)
    assert (dlam == 0).all() and torch.equal(dh0, dl)
    assert (S.gated_scan_bwd(e, e, e, lam, torch.empty(0, device="cuda"), e)[3] == 0).all()
    w = torch.ones(8, device="cuda")
    y, s = S.add_rms_norm(torch.empty(0, 8, device="cuda"), w)
    assert y.shape == (0, 8)
    x = torch.empty(0, 8, device="cuda")
    dx, dw = S.add_rms_norm_bwd(x, x, w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 8) and (dw == 0).all()


# ---- beyond 2^31 elements ------------------------------------------------------------------------

def _big(*shape):
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def test_norm_beyond_2_31_elements():
    _say("big norm")
    rows, D = 2900000, 768
    assert rows * D > 2 ** 31
    x, w = _big(rows, D), torch.ones(D, dtype=torch.bfloat16, device="cuda")
    y, s, rstd = S.add_rms_norm_fwd_train(x, w)
    for sl in (slice(0, 50), slice(rows - 50, rows)):
        ys, _, rs = S.add_rms_norm_fwd_train(x[sl], w)
        assert torch.equal(y[sl], ys) and torch.equal(rstd[sl], rs)
    q, sc, _ = S.add_rms_norm_q8(x, w, group=64)
    qs, scs, _ = S.add_rms_norm_q8(x[-50:], w, group=64)
    assert torch.equal(q[-50:].view(torch.uint8), qs.view(torch.uint8)) and torch.equal(sc[-50:], scs)
    del q, sc
    dx, _ = S.add_rms_norm_bwd(y, x, w, rstd)
    assert torch.equal(dx[-50:], S.add_rms_norm_bwd(y[-50:], x[-50:], w, rstd[-50:])[0])
    del x, y, dx
    torch.cuda.empty_cache()


def test_rotary_beyond_2_31_elements():
    _say("big rotary")
    L, hq, hk, d = 300000, 56, 4, 128
    qk = _big(1, L, hq + hk, d)
    assert qk.numel() > 2 ** 31
    freqs, m = S.rotary_freqs(64)
    pos = torch.arange(L, device="cuda")[None]
    q, k = S.rotary(qk[:, :, :hq], qk[:, :, hq:], freqs, pos)
    for sl in (slice(0, 33), slice(L - 33, L)):
        qs, ks = S.rotary(qk[:, sl, :hq], qk[:, sl, hq:], freqs, pos[:, sl])
        assert torch.equal(q[:, sl], qs) and torch.equal(k[:, sl], ks)
    del qk, q, k
    torch.cuda.empty_cache()


def test_scan_beyond_2_31_elements():
    """Gates that forget to below 2^-126 within a few hundred tokens, so that the last whole tiles alone give the same
    bits as in the whole sequence (tiles of the backward and forward both begin at multiples of 256)."""
    _say("big scan")
    L, D = 2900224, 768
    assert L * D > 2 ** 31 and L % 256 == 0
    x, r, i = (_big(1, L, D) for _ in range(3))
    r.abs_()                                     # a < exp(-8 softplus(1) / 2) < 0.006
    lam = torch.ones(D, device="cuda")
    h, last, states = S.gated_scan_fwd_train(x, r, i, lam)
    t = slice(L - 2048, L)
    hs, lasts, _ = S.gated_scan_fwd_train(x[:, t], r[:, t], i[:, t], lam)
    assert torch.equal(h[:, L - 1024:], hs[:, 1024:]) and torch.equal(last, lasts)
    grads = S.gated_scan_bwd(x, r, i, lam, states, x)
    t = slice(0, 2048)
    _, _, st = S.gated_scan_fwd_train(x[:, t], r[:, t], i[:, t], lam)
    gs = S.gated_scan_bwd(x[:, t], r[:, t], i[:, t], lam, st, x[:, t])
    for a, b in zip(grads[:3], gs[:3]):
        assert torch.equal(a[:, :1024], b[:, :1024])
    t = slice(L - 2048, L)
    _, _, st = S.gated_scan_fwd_train(x[:, t], r[:, t], i[:, t], lam)
    gs = S.gated_scan_bwd(x[:, t], r[:, t], i[:, t], lam, st, x[:, t])
    for a, b in zip(grads[:3], gs[:3]):
        assert torch.equal(a[:, L - 1024:], b[:, 1024:])
    del x, r, i, h, grads
    torch.cuda.empty_cache()
