"""Runs the host build of the kernels and the C ABI of fla_seq.h on buffers of exactly their size, under the
sanitizers, against the fp64 forms.  Usage: drive.py LIBRARY GROUP (see GROUPS)."""
import ctypes
import os
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__)))))
sys.path.insert(0, ROOT)
from oracle import seq as O  # noqa: E402
from paper_2407_02109_amd import seq as S  # noqa: E402

libc = ctypes.CDLL(None)
libc.malloc.restype, libc.malloc.argtypes = ctypes.c_void_p, [ctypes.c_size_t]
libc.free.argtypes = [ctypes.c_void_p]


class Buf:
    """A tensor on memory of exactly its size (an allocation of its own, so that the sanitizer sees its ends), as
    the kernel's type; `view`: elements of a larger row layout, strides in elements."""

    def __init__(self, shape, kind, values=None, strides=None):
        self.shape, self.kind = tuple(shape), kind
        self.np = {"f32": np.float32, "bf16": np.uint16, "i32": np.int32, "i64": np.int64, "f64": np.float64,
                   "u8": np.uint8}[kind]
        n = int(np.prod(self.shape))
        if strides is None:
            strides, step = [], 1
            for s in reversed(self.shape):
                strides.insert(0, step)
                step *= s
        self.strides = tuple(strides)
        span = 1 + sum((s - 1) * t for s, t in zip(self.shape, self.strides)) if n else 0
        size = np.dtype(self.np).itemsize
        self.ptr = libc.malloc(max(span * size, 1))
        raw = (ctypes.c_char * (span * size)).from_address(self.ptr)
        flat = np.frombuffer(raw, dtype=self.np) if n else np.zeros(0, self.np)
        # what lies between the elements is NaN
        if span:
            flat[:] = {"f32": np.float32(np.nan), "bf16": 0x7fc0, "f64": np.nan}.get(kind, 0)
        self.a = np.lib.stride_tricks.as_strided(flat, self.shape, [t * size for t in self.strides], writeable=True)
        if values is not None:
            self.a[...] = to_bits(values) if kind == "bf16" else values

    def get(self):
        return from_bits(self.a).astype(np.float64) if self.kind == "bf16" else np.array(self.a, dtype=np.float64)


def to_bits(x):
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def from_bits(u):
    return (np.ascontiguousarray(u).astype(np.uint32) << 16).view(np.float32)


def rounded(x, kind):
    return from_bits(to_bits(x)).astype(np.float64) if kind == "bf16" else x.astype(np.float32).astype(np.float64)


def close(name, got, want, bound):
    # values below the least normal fp32 (1.2e-38) may vanish on the way, of which a sum over fewer than 10^4 tokens makes
    # less than 2e-34
    bound = bound + 2e-34
    bad = ~(np.abs(got - want) <= bound) & ~(np.isnan(got) & np.isnan(want))
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError("%s: %d of %d off, first at %s: %r, expected %r +- %.3g" % (
            name, bad.sum(), bad.size, at, got[at], want[at], np.broadcast_to(bound, bad.shape)[at]))


def kinds(which):
    ctypes.c_int.in_dll(S._lib, "emu_kernel_args").value = which


CODE = {"f32": 0, "bf16": 1}


def norm(kind, rows, D, residual, wkind, pad, rng):
    kinds(0)
    vec = 8 if kind == "bf16" else 4
    x, r = (rounded(rng.standard_normal((rows, D)) * 3, kind) for _ in range(2))
    w = rounded(1 + 0.2 * rng.standard_normal(D), wkind)
    stride = D + pad
    bx, br = Buf((rows, D), kind, x, (stride, 1)), Buf((rows, D), kind, r, (stride, 1))
    bw, y, s, rstd = Buf((D,), wkind, w), Buf((rows, D), kind), Buf((rows, D), kind), Buf((rows,), "f32")
    res, rp = (r, br.ptr) if residual else (None, None)
    S.fla_add_rms_norm_fwd(bx.ptr, stride, rp, stride, bw.ptr, y.ptr, s.ptr, rstd.ptr, rows, D, 1e-6, CODE[kind],
                           CODE[wkind], 0)
    adds = O.norm_adds(D, vec)
    ry, rs, rr, rel = O.rms_norm(x, w, res, 1e-6, adds)
    close("sum", s.get(), rs, O.half_step(rs, kind) + 2 * O.U * np.abs(rs))
    close("rstd", rstd.get(), rr, rel * rr)
    close("y", y.get(), ry, rel * np.abs(ry) + O.half_step(ry, kind) * (1 + rel))
    for group in (0, 32, 64, 128):
        n = -(-D // group) if group else 1
        q, sc, s2 = Buf((rows, D), "u8"), Buf((rows, n), "f32"), Buf((rows, D), kind)
        S.fla_add_rms_norm_q8(bx.ptr, stride, rp, stride, bw.ptr, q.ptr, sc.ptr, s2.ptr, rows, D, group, 1e-6,
                              CODE[kind], CODE[wkind], 0)
        _, rsc = O.quantize(ry, group)
        close("scales", sc.get(), rsc, (rel + 4 * O.U) * rsc)
        assert (s2.a == s.a).all()
        got = E4M3[q.a] * np.repeat(sc.get(), group or D, 1)[:, :D]
        # half a step of e4m3 (2^-4 of the value, 2^-10 of the scale at least)
        close("q", got, ry, np.maximum(2.0 ** -4 * np.abs(ry), 2.0 ** -10 * np.repeat(rsc, group or D, 1)[:, :D])
              * (1 + 1e-5) + rel * np.abs(ry))
    # backward at the kept sum
    kinds(1)
    sv, dy, ds = s.get(), *(rounded(rng.standard_normal((rows, D)), kind) for _ in range(2))
    bdy, bds = Buf((rows, D), kind, dy, (stride, 1)), Buf((rows, D), kind, ds, (stride, 1))
    dx, dw = Buf((rows, D), kind), Buf((D,), "f32")
    nws = S.fla_add_rms_norm_bwd_workspace(rows, D)
    ws = Buf((nws // 4,), "f32")
    S.fla_add_rms_norm_bwd(bdy.ptr, stride, s.ptr, D, bw.ptr, rstd.ptr, bds.ptr if residual else None, stride, dx.ptr,
                           dw.ptr, ws.ptr, nws, rows, D, CODE[kind], CODE[wkind], 0)
    rdx, rdw, bdx, bdw = O.rms_norm_bwd(dy, sv, w, rstd.get(), ds if residual else None, adds)
    close("dx", dx.get(), rdx, bdx + O.half_step(rdx, kind) + O.half_step(bdx, kind))
    close("dw", dw.get(), rdw, bdw)


E4M3 = np.array([(-1 if c & 128 else 1) * (np.nan if (c & 127) == 127 else (c & 7) * 2.0 ** -9 if not c & 120 else
                 (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7)) for c in range(256)])


def norms(rng):
    for case in [("bf16", 5, 65, True, "bf16", 0), ("f32", 9, 1, True, "f32", 3), ("bf16", 11, 1000, True, "f32", 7),
                 ("f32", 3, 1001, True, "f32", 5), ("bf16", 2, 4099, False, "bf16", 0), ("f32", 1, 4096, False, "f32", 1),
                 ("bf16", 17, 130, False, "bf16", 1)]:
        print("norm", case, flush=True)
        norm(*case, rng)


def wide_norms(rng):
    for case in [("bf16", 2, 8200, True, "bf16", 0), ("f32", 3, 4101, True, "f32", 1), ("f32", 5, 16400, True, "f32", 0),
                 ("bf16", 2, 33001, True, "f32", 3)]:
        print("norm", case, flush=True)
        norm(*case, rng)


def rotaries(rng):
    kinds(2)
    # kind, B, L, hq, hk, d, rot, axes, interleaved, pos64, inverse, layout
    for case in [("bf16", 2, 3, 2, 1, 64, 64, 1, 0, 0, 0, "fused"), ("f32", 1, 5, 3, 0, 32, 8, 2, 1, 1, 0, "whole"),
                 ("bf16", 2, 2, 1, 2, 40, 20, 2, 0, 0, 1, "heads"), ("f32", 3, 1, 2, 2, 7, 6, 1, 0, 1, 1, "place"),
                 ("bf16", 1, 4, 2, 2, 80, 40, 1, 1, 0, 0, "fusedplace"), ("bf16", 1, 70, 1, 1, 8, 2, 1, 0, 0, 0, "whole"),
                 ("f32", 1, 2, 1, 1, 512, 512, 1, 1, 0, 0, "whole"), ("f32", 1, 1, 3, 1, 512, 2, 1, 1, 0, 1, "whole")]:
        print("rotary", case, flush=True)
        kind, B, L, hq, hk, d, rot, axes, inter, p64, inv, layout = case
        H = hq + hk
        vals = rounded(rng.standard_normal((B, L, H, d)), kind)
        q, k = vals[:, :, :hq], vals[:, :, hq:]
        freqs = 10000.0 ** (-2 * np.arange(rot // 2) / rot)
        pos = rng.integers(-1000000, 1000000, (B, L) if axes == 1 else (B, L, 2))
        bp, bf = Buf(pos.shape, "i64" if p64 else "i32", pos), Buf(freqs.shape, "f64", freqs)
        size = 2 if kind == "bf16" else 4
        fresh = lambda h: Buf((B, L, h, d), kind)
        if layout.startswith("fused"):   # q and k side by side in each token
            buf = Buf((B, L, H, d), kind, vals, (L * (H * d + 5), H * d + 5, d, 1))
            pq, pk, sq = buf.ptr, buf.ptr + hq * d * size, buf.strides[:3]
            sk = sq
        elif layout == "heads":          # [B, heads, L, d]
            bq, bk = (Buf(t.shape, kind, t, (t.shape[2] * L * d, d, L * d, 1)) for t in (q, k))
            pq, pk, sq, sk = bq.ptr, bk.ptr, bq.strides[:3], bk.strides[:3]
        else:
            bq, bk = Buf(q.shape, kind, q), Buf(k.shape, kind, k)
            pq, pk, sq, sk = bq.ptr, bk.ptr, bq.strides[:3], bk.strides[:3]
        if layout.endswith("place"):
            oq, ok, soq, sok = pq, pk, sq, sk
        else:
            rq, rk = fresh(hq), fresh(hk)
            oq, ok, soq, sok = rq.ptr, rk.ptr, rq.strides[:3], rk.strides[:3]
        S.fla_rotary(pq, sq, pk, sk, oq, soq, ok, sok, bp.ptr, p64, bp.strides[0], bp.strides[1], axes, bf.ptr, B, L, hq,
                     hk, d, rot, inter, 1.25, inv, CODE[kind], 0)
        if layout == "fusedplace":
            got = buf.get()
            gq, gk = got[:, :, :hq], got[:, :, hq:]
        elif layout == "place":
            gq, gk = bq.get(), bk.get()
        else:
            gq, gk = rq.get(), rk.get()
        for name, got, x in (("q", gq, q), ("k", gk, k)):
            want, bound = O.rotary(x, freqs, pos, inter, 1.25, inv) if x.size else (x, x)
            close(name, got, want, bound + O.half_step(want, kind) * (bound > 0) + O.half_step(bound, kind))


def scan(kind, B, L, D, with_h0, lengths, pad, with_dh, rng, lam_shift=0.0):
    x, r, i = (rounded(rng.standard_normal((B, L, D)), kind) for _ in range(3))
    lam = (rng.standard_normal(D) - 3 + lam_shift).astype(np.float32).astype(np.float64)
    tok = D + pad
    st = (L * tok + pad, tok)
    bx, br, bi = (Buf((B, L, D), kind, t, (*st, 1)) for t in (x, r, i))
    blam = Buf((D,), "f32", lam)
    h0 = rng.standard_normal((B, D)).astype(np.float32).astype(np.float64) if with_h0 else None
    bh0 = Buf((B, D), "f32", h0) if with_h0 else None
    bl = Buf((B,), "i32", lengths) if lengths is not None else None
    ptr = lambda b: b.ptr if b is not None else None
    h, last = Buf((B, L, D), kind, np.full((B, L, D), 7.0)), Buf((B, D), "f32")
    states = Buf((S.fla_gated_scan_states(B, L, D) // 4,), "f32")
    nws = S.fla_gated_scan_workspace(B, L, D)
    ws = Buf((nws,), "u8", rng.integers(0, 256, nws))
    kinds(3)
    S.fla_gated_scan_fwd(bx.ptr, st, br.ptr, st, bi.ptr, st, blam.ptr, ptr(bh0), ptr(bl), h.ptr, last.ptr, states.ptr,
                         ws.ptr, nws, B, L, D, 8.0, CODE[kind], 0)
    ref, rlast, bound, blast = O.gated_scan(x, r, i, lam, h0, lengths)
    live = np.arange(L)[None, :, None] < (np.full(B, L) if lengths is None else np.clip(lengths, 0, L))[:, None, None]
    got = h.get()
    assert (got[np.broadcast_to(~live, got.shape)] == 7.0).all()
    close("h", np.where(live, got, 0), ref, bound + O.half_step(ref, kind) + O.half_step(bound, kind))
    close("last", last.get(), rlast, blast)
    # again without the kept states, in place of h0
    h2 = Buf((B, L, D), kind, np.full((B, L, D), 7.0))
    inplace = Buf((B, D), "f32", h0) if with_h0 else Buf((B, D), "f32")
    S.fla_gated_scan_fwd(bx.ptr, st, br.ptr, st, bi.ptr, st, blam.ptr, inplace.ptr if with_h0 else None, ptr(bl), h2.ptr,
                         inplace.ptr, None, ws.ptr, nws, B, L, D, 8.0, CODE[kind], 0)
    assert (h2.a == h.a).all() and (inplace.a == last.a).all()
    dh = rounded(rng.standard_normal((B, L, D)), kind) if with_dh else None
    dl = rng.standard_normal((B, D)).astype(np.float32).astype(np.float64)
    bdh, bdl = Buf((B, L, D), kind, dh, (*st, 1)) if with_dh else None, Buf((B, D), "f32", dl)
    dx, dr, di = (Buf((B, L, D), kind) for _ in range(3))
    dlam, dh0 = Buf((D,), "f32"), Buf((B, D), "f32")
    nws = S.fla_gated_scan_bwd_workspace(B, L, D)
    ws = Buf((nws,), "u8", rng.integers(0, 256, nws))
    kinds(4)
    S.fla_gated_scan_bwd(bx.ptr, st, br.ptr, st, bi.ptr, st, blam.ptr, states.ptr, ptr(bl), ptr(bdh), st, bdl.ptr,
                         dx.ptr, dr.ptr, di.ptr, dlam.ptr, dh0.ptr, ws.ptr, nws, B, L, D, 8.0, CODE[kind], 0)
    grads, bounds = O.gated_scan_bwd(x, r, i, lam, h0, lengths, dh, dl)
    for name, b, g, e in zip(("dx", "dr", "di", "dlam", "dh0"), (dx, dr, di, dlam, dh0), grads, bounds):
        k = kind if name in ("dx", "dr", "di") else "f32"
        close(name, b.get(), g, e + O.half_step(g, k) + O.half_step(e, k))


def scans(rng):
    # kind, B, L, D, h0, lengths, pad, dh
    for case in [("bf16", 2, 1, 64, True, None, 0, True), ("f32", 1, 130, 70, False, None, 3, True),
                 ("bf16", 2, 300, 65, True, [137, 300], 1, True), ("f32", 3, 140, 5, True, [0, 1, 140], 0, False),
                 ("bf16", 1, 517, 9, False, None, 0, True), ("f32", 2, 257, 66, True, [-5, 900], 1, True),
                 ("f32", 2, 0, 66, True, None, 0, False)]:
        print("scan", case, flush=True)
        kind, B, L, D, with_h0, lengths, pad, with_dh = case
        scan(kind, B, L, D, with_h0, None if lengths is None else np.array(lengths), pad, with_dh, rng)
    print("scan with gates that hardly forget, and that forget all", flush=True)
    scan("f32", 1, 150, 8, True, None, 0, True, rng, -14.0)
    scan("f32", 1, 150, 8, True, None, 0, True, rng, 8.0)


GROUPS = {"norm": norms, "norm_wide": wide_norms, "rotary": rotaries, "scan": scans}

if __name__ == "__main__":
    S._lib = ctypes.CDLL(sys.argv[1])
    S._declare(S._lib)
    GROUPS[sys.argv[2]](np.random.default_rng(7))
    print("ok", flush=True)
