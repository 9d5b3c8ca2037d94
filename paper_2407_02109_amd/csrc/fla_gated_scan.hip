// Gated linear recurrence over the tokens, forward and backward, gfx950.
//
// Per channel: z_t = c softplus(lam) sigmoid(r_t), a_t = exp(-z_t), u_t = sqrt(1 - a_t^2) sigmoid(i_t) x_t,
// h_t = a_t h_{t-1} + u_t.  Backward, with p_t = a_t g_t what token t hands to the one before it:
//   g_t = dh_t + p_{t+1},   v_t = g_t u_t,
//   dx_t = g_t m_t sigmoid(i_t),  di_t = v_t (1 - sigmoid(i_t)),  m_t = sqrt(1 - a_t^2),
//   e_t = z_t dL/dz_t = (z_t / m_t^2) a_t^2 v_t - z_t a_t h_{t-1} g_t,
//   dr_t = e_t (1 - sigmoid(r_t)),   dlam = sigmoid(lam) / softplus(lam) sum_t e_t.
// Bound by memory: x, both gates (backward: and dh) read once, h (dx, dr, di) written once.
//
// A workgroup takes a chunk of 128 tokens of a column of 64 channels; a thread S consecutive tokens of N
// channels (16 bytes of each row).  Each thread reduces its tokens to their decay and their state from
// zero, one wave carries a state over those in token order, and each thread runs over its tokens again
// from the state that enters them.  Tokens past a sequence's end keep the state: a = 1, u = 0.
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

namespace fla {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T>
struct Tile {
    static constexpr int N = kVec<T>;                // channels of a thread
    static constexpr int X = kScanChannels / N;      // threads across the column
    static constexpr int SEG = 256 / X;              // runs of tokens
    static constexpr int S = kScanChunk / SEG;       // tokens of a run
};

__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e));
}
// c softplus(lam), in units of log2
__device__ __forceinline__ float decay_rate(float lam, float c) {
    return c * kLog2e * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam))));
}
// 1 - a^2 for a = 2^-z2: near a = 1 from the series of 1 - exp(-w), w = 2 z2 ln 2, whose first dropped term is
// w^6 / 5040 (5e-8 at w = 1/4); there 1 - a^2 in fp32 would lose what a's rounding takes
__device__ __forceinline__ float one_minus_square(float a, float z2) {
    const float w = z2 * (2.f * kLn2);
    float p = __builtin_fmaf(w, -1.f / 6.f, 1.f);
    p = __builtin_fmaf(w * p, -1.f / 5.f, 1.f);
    p = __builtin_fmaf(w * p, -1.f / 4.f, 1.f);
    p = __builtin_fmaf(w * p, -1.f / 3.f, 1.f);
    p = __builtin_fmaf(w * p, -1.f / 2.f, 1.f);
    return w < 0.25f ? w * p : __builtin_fmaf(-a, a, 1.f);
}

// tokens of sequence b
__device__ __forceinline__ int length_of(const int* lengths, int b, int L) {
    if (!lengths) return L;
    const int n = lengths[b];
    return n < 0 ? 0 : n < L ? n : L;
}

template <typename T>
__device__ __forceinline__ const T* row_of(const ScanInput& m, int b, int64_t t) {
    return static_cast<const T*>(m.p) + (b * m.batch + t * m.token);
}

// One thread for each piece of channels of a sequence, token by token.
template <typename T>
__global__ __launch_bounds__(256) void scan_serial(ScanArgs a) {
    constexpr int N = kVec<T>, X = Tile<T>::X;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per_b = a.columns * X;
    if (id >= (int64_t)a.B * per_b) return;
    const int b = (int)(id / per_b), piece = (int)(id - (int64_t)b * per_b);
    const int ch = piece * N, n = a.D - ch;
    if (n <= 0) return;
    float s2[N], h[N];
    load_piece(a.lam + ch, n, s2);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        s2[j] = decay_rate(s2[j], a.c);
        h[j] = 0.f;
    }
    if (a.h0) load_piece(a.h0 + (int64_t)b * a.D + ch, n, h);
    const int len = length_of(a.lengths, b, a.L);
    for (int t = 0; t < a.L; ++t) {
        if (a.states && t % kScanChunk == 0) {
            float* st = a.states + (((int64_t)b * a.columns + piece / X) * a.chunks + t / kScanChunk) * kScanChannels +
                        ch % kScanChannels;
#pragma unroll
            for (int j = 0; j < N; ++j) st[j] = h[j];
        }
        if (t >= len) continue;
        float x[N], r[N], i[N];
        load_piece(row_of<T>(a.x, b, t) + ch, n, x);
        load_piece(row_of<T>(a.r, b, t) + ch, n, r);
        load_piece(row_of<T>(a.i, b, t) + ch, n, i);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float z2 = s2[j] * sigmoid(r[j]);
            const float d = __builtin_amdgcn_exp2f(-z2);
            const float u = __builtin_amdgcn_sqrtf(one_minus_square(d, z2)) * sigmoid(i[j]) * x[j];
            h[j] = __builtin_fmaf(d, h[j], u);
        }
        store_piece(static_cast<T*>(a.h) + ((int64_t)b * a.L + t) * a.D + ch, n, h);
    }
    if (a.h_last) {
        float* last = a.h_last + (int64_t)b * a.D + ch;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) last[j] = h[j];
    }
}

// Backward: a workgroup takes a column of a sequence and goes over its chunks from the last.
template <typename T>
__global__ __launch_bounds__(256) void scan_bwd(ScanBwdArgs a) {
    constexpr int N = Tile<T>::N, X = Tile<T>::X, SEG = Tile<T>::SEG, S = Tile<T>::S;
    // of each run: its decay, its state from zero and what it hands on from zero; then the state that
    // enters it and what it is handed
    __shared__ float run_a[SEG][kScanChannels], run_h[SEG][kScanChannels], run_p[SEG][kScanChannels];
    __shared__ float rate[kScanChannels];
    const int tid = (int)threadIdx.x, seg = tid / X, lc = tid % X * N;
    const int g = (int)(blockIdx.x % (unsigned)a.columns), b = (int)(blockIdx.x / (unsigned)a.columns);
    const int ch = g * kScanChannels + lc, n = a.D - ch;
    const int c1 = g * kScanChannels + (tid & 63);   // the carrying waves' channel
    const int len = length_of(a.lengths, b, a.L);
    if (tid < 64) rate[tid] = c1 < a.D ? decay_rate(a.lam[c1], a.c) : 0.f;
    __syncthreads();
    float s2[N], esum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        s2[j] = rate[lc + j];
        esum[j] = 0.f;
    }
    float handed = a.d_last && c1 < a.D ? a.d_last[(int64_t)b * a.D + c1] : 0.f;   // (wave 1's)
    for (int k = a.chunks - 1; k >= 0; --k) {
        const int t0 = k * kScanChunk + seg * S;
        float d[S][N], u[S][N], gi[S][N], gr[S][N], gg[S][N];
        float zs[N], h[N], p[N];
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const bool live = t0 + t < len;
            const int m = live ? n : 0;
            load_piece(row_of<T>(a.r, b, t0 + t) + ch, m, gr[t]);
            load_piece(row_of<T>(a.i, b, t0 + t) + ch, m, gi[t]);
            load_piece(row_of<T>(a.x, b, t0 + t) + ch, m, u[t]);
            load_piece(row_of<T>(a.dh.p ? a.dh : a.x, b, t0 + t) + ch, a.dh.p ? m : 0, gg[t]);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                gr[t][j] = live ? sigmoid(gr[t][j]) : 0.f;
                gi[t][j] = sigmoid(gi[t][j]);
                const float z2 = s2[j] * gr[t][j];
                d[t][j] = __builtin_amdgcn_exp2f(-z2);
                u[t][j] *= __builtin_amdgcn_sqrtf(one_minus_square(d[t][j], z2)) * gi[t][j];
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            zs[j] = h[j] = p[j] = 0.f;
#pragma unroll
            for (int t = 0; t < S; ++t) {
                zs[j] = __builtin_fmaf(s2[j], gr[t][j], zs[j]);
                h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
                p[j] = d[S - 1 - t][j] * (gg[S - 1 - t][j] + p[j]);
            }
            run_a[seg][lc + j] = __builtin_amdgcn_exp2f(-zs[j]);
            run_h[seg][lc + j] = h[j];
            run_p[seg][lc + j] = p[j];
        }
        __syncthreads();
        if (tid < 64) {
            float st = a.states[(((int64_t)b * a.columns + g) * a.chunks + k) * kScanChannels + tid];
            for (int s = 0; s < SEG; ++s) {
                const float next = __builtin_fmaf(run_a[s][tid], st, run_h[s][tid]);
                run_h[s][tid] = st;
                st = next;
            }
        } else if (tid < 128) {
            const int l = tid - 64;
            for (int s = SEG - 1; s >= 0; --s) {
                const float next = __builtin_fmaf(run_a[s][l], handed, run_p[s][l]);
                run_p[s][l] = handed;
                handed = next;
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            h[j] = run_h[seg][lc + j];
            p[j] = run_p[seg][lc + j];
#pragma unroll
            for (int t = S - 1; t >= 0; --t) {
                gg[t][j] += p[j];
                p[j] = d[t][j] * gg[t][j];
            }
        }
#pragma unroll
        for (int t = 0; t < S; ++t) {
            float dx[N], dr[N], di[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float z2 = s2[j] * gr[t][j], z = z2 * kLn2, m2 = one_minus_square(d[t][j], z2);
                const float v = gg[t][j] * u[t][j];
                // z / m^2 -> 1/2 as z -> 0, where u is 0 too
                const float over = z > 1e-30f ? z * __builtin_amdgcn_rcpf(m2) : 0.5f;
                const float e = over * d[t][j] * d[t][j] * v - z * d[t][j] * h[j] * gg[t][j];
                h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
                dx[j] = gg[t][j] * __builtin_amdgcn_sqrtf(m2) * gi[t][j];
                di[j] = v * (1.f - gi[t][j]);
                dr[j] = e * (1.f - gr[t][j]);
                esum[j] += e;
            }
            if (t0 + t < a.L) {
                if (t0 + t >= len) {
#pragma unroll
                    for (int j = 0; j < N; ++j) dx[j] = dr[j] = di[j] = 0.f;
                }
                const int64_t at = ((int64_t)b * a.L + t0 + t) * a.D + ch;
                store_piece(static_cast<T*>(a.dx) + at, n, dx);
                store_piece(static_cast<T*>(a.dr) + at, n, dr);
                store_piece(static_cast<T*>(a.di) + at, n, di);
            }
        }
        __syncthreads();   // the runs' values are taken
    }
    if (tid >= 64 && tid < 128 && a.dh0 && c1 < a.D) a.dh0[(int64_t)b * a.D + c1] = handed;
#pragma unroll
    for (int j = 0; j < N; ++j) run_a[seg][lc + j] = esum[j];
    __syncthreads();
    if (tid < 64) {
        float s = run_a[0][tid];
        for (int q = 1; q < SEG; ++q) s += run_a[q][tid];
        a.shares[((int64_t)b * a.columns + g) * kScanChannels + tid] = s;
    }
}

// dlam: one thread for each channel, the sequences' shares in order
__global__ __launch_bounds__(256) void scan_dlam(ScanBwdArgs a) {
    const int c = (int)(blockIdx.x * 256 + threadIdx.x);
    if (c >= a.D) return;
    float s = 0.f;
    for (int b = 0; b < a.B; ++b) s += a.shares[(int64_t)b * a.columns * kScanChannels + c];
    // d softplus / softplus; both are exp(lam) far below 0
    const float lam = a.lam[c];
    const float f = lam < -20.f ? 1.f : 1.f / ((1.f + expf(-lam)) * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam)))));
    a.dlam[c] = s * f;
}

template <typename T>
hipError_t fwd(const ScanArgs& a, hipStream_t stream) {
    const int64_t pieces = (int64_t)a.B * a.columns * Tile<T>::X;
    return launch<ScanArgs>(&scan_serial<T>, (pieces + 255) / 256, 256, a, stream);
}
template <typename T>
hipError_t bwd(const ScanBwdArgs& a, hipStream_t stream) {
    if (a.B > 0) {
        const hipError_t e = launch<ScanBwdArgs>(&scan_bwd<T>, (int64_t)a.B * a.columns, 256, a, stream);
        if (e != hipSuccess) return e;
    }
    return launch<ScanBwdArgs>(&scan_dlam, ((int64_t)a.D + 255) / 256, 256, a, stream);
}

}  // namespace

hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream);
}
hipError_t launch_scan_bwd(const ScanBwdArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream);
}

}  // namespace fla
