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
//
// The state that enters a chunk comes from the chunk before it, in one pass over the data: as soon as a
// workgroup has its chunk's decay A and state from zero H, it publishes both, then looks back over the
// chunks before it for the nearest one whose outgoing state is known, runs A and H of those between
// over it, and publishes its own outgoing state.  The values are their own flags: a word is all ones
// until it is published, and no value has that pattern.  The states meet in chunk order whatever is found
// first, so the result does not depend on timing.  Workgroups draw the chunks of a column in order, so
// a workgroup waits only for ones that have begun, and the first of a column waits for none: every
// wait ends.
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

namespace fla {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T, int THREADS>
struct Tile {
    static constexpr int N = kVec<T>;                // channels of a thread
    static constexpr int X = kScanChannels / N;      // threads across the column
    static constexpr int SEG = THREADS / X;          // runs of tokens
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
    constexpr int N = kVec<T>, X = kScanChannels / N;
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

// ---- the chain over the chunks of a column.  Words of the workspace, all ones until published:
//      for each (column, chunk, channel) A and H in one 64-bit word, and the outgoing state.
struct Chain {
    unsigned long long* part;   // [chunks][64] of this column, in the order in which the chain runs
    unsigned* out;
};
__device__ __forceinline__ Chain chain_of(void* ws, int64_t columns, int chunks, int64_t column) {
    const int64_t all = columns * chunks * kScanChannels, mine = column * chunks * kScanChannels;
    Chain c;
    c.part = static_cast<unsigned long long*>(ws) + mine;
    c.out = reinterpret_cast<unsigned*>(static_cast<unsigned long long*>(ws) + all) + mine;
    return c;
}
// the next chunk of the column, in order (one draw a workgroup)
__device__ __forceinline__ unsigned draw(void* ws, int64_t columns, int chunks, int64_t column) {
    unsigned* tickets = reinterpret_cast<unsigned*>(static_cast<unsigned char*>(ws) +
                                                    columns * chunks * kScanChannels * 12);
    return __scoped_atomic_fetch_add(tickets + column * kScanTicketWords, 1u, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
constexpr unsigned kUnset = 0xffffffffu;
__device__ __forceinline__ unsigned word_of(float v) {
    const unsigned u = f32_bits(v);
    return u == kUnset ? 0x7fc00000u : u;   // (that NaN becomes another)
}
__device__ __forceinline__ void publish(const Chain& c, int k, int lane, float v) {
    __scoped_atomic_store_n(c.out + k * kScanChannels + lane, word_of(v), __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
__device__ __forceinline__ void publish(const Chain& c, int k, int lane, float A, float H) {
    __scoped_atomic_store_n(c.part + k * kScanChannels + lane,
                            (unsigned long long)word_of(A) << 32 | word_of(H), __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
// The outgoing state of link k - 1, for one wave (a lane each channel).  A turn reads kLook links; a lane has
// its state once an outgoing state and the parts of all links behind it are there.
constexpr int kLook = 8;
constexpr int kMostTurns = 1 << 22;   // seconds: only a workspace that another call overwrites makes a wait that long
__device__ __forceinline__ float look_back(const Chain& c, int k, int lane) {
    float state = 0.f;
    bool found = false;
    for (int turn = 0; turn < kMostTurns; ++turn) {
        if (!found) {
            unsigned out[kLook];
            unsigned long long part[kLook];
#pragma unroll
            for (int i = 0; i < kLook; ++i) {
                const int at = (k - 1 - i > 0 ? k - 1 - i : 0) * kScanChannels + lane;
                out[i] = __scoped_atomic_load_n(c.out + at, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
                part[i] = __scoped_atomic_load_n(c.part + at, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
            }
            // the nearest outgoing state with every part behind it
            int near = -1;
            bool parts = true;
#pragma unroll
            for (int i = 0; i < kLook; ++i) {
                if (near < 0 && parts && i < k && out[i] != kUnset) near = i;
                parts = parts && part[i] != ~0ull;
            }
            if (near >= 0) {
                found = true;
#pragma unroll
                for (int i = kLook - 1; i >= 0; --i) {
                    if (i == near) state = bits_f32(out[i]);
                    if (i < near)
                        state = __builtin_fmaf(bits_f32((unsigned)(part[i] >> 32)), state, bits_f32((unsigned)part[i]));
                }
            }
        }
        if (__builtin_amdgcn_ballot_w64(!found) == 0) return state;
        __builtin_amdgcn_s_sleep(1);
    }
    return found ? state : __builtin_nanf("");
}

// the words of a workspace before a chain: all ones, and the tickets 0
template <typename A>
__global__ __launch_bounds__(256) void chain_clear(A a) {
    unsigned* ws = static_cast<unsigned*>(a.ws);
    const int64_t columns = (int64_t)a.B * a.columns, words = columns * a.chunks * kScanChannels * 3;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words + columns * kScanTicketWords;
         w += (int64_t)gridDim.x * 256)
        ws[w] = w < words ? kUnset : 0u;
}

template <typename T, bool CHAIN>
__global__ __launch_bounds__(256) void scan_tiles(ScanArgs a) {
    using Ti = Tile<T, 256>;
    constexpr int N = Ti::N, X = Ti::X, SEG = Ti::SEG, S = Ti::S;
    // of each run: its decay and its state from zero; then the state that enters it
    __shared__ float run_a[SEG][kScanChannels], run_h[SEG][kScanChannels];
    __shared__ float rate[kScanChannels];
    __shared__ int drawn;
    const int tid = (int)threadIdx.x, seg = tid / X, lc = tid % X * N;
    const unsigned columns = (unsigned)(a.B * a.columns), column = blockIdx.x % columns;
    const int g = (int)(column % (unsigned)a.columns), b = (int)(column / (unsigned)a.columns);
    const int ch = g * kScanChannels + lc, n = a.D - ch;
    const int c1 = g * kScanChannels + (tid & 63);   // the carrying wave's channel
    if (CHAIN && tid == 0) drawn = (int)draw(a.ws, columns, a.chunks, column);
    if (tid < 64) rate[tid] = c1 < a.D ? decay_rate(a.lam[c1], a.c) : 0.f;
    __syncthreads();
    const int k = CHAIN ? drawn : 0;
    const int len = length_of(a.lengths, b, a.L);
    const int t0 = k * kScanChunk + seg * S;
    float d[S][N], u[S][N], gi[S][N];
#pragma unroll
    for (int t = 0; t < S; ++t) {
        const int m = t0 + t < len ? n : 0;
        load_piece(row_of<T>(a.r, b, t0 + t) + ch, m, d[t]);
        load_piece(row_of<T>(a.i, b, t0 + t) + ch, m, gi[t]);
        load_piece(row_of<T>(a.x, b, t0 + t) + ch, m, u[t]);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float s2 = rate[lc + j];
        float zs = 0.f, h = 0.f;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const float z2 = t0 + t < len ? s2 * sigmoid(d[t][j]) : 0.f;
            d[t][j] = __builtin_amdgcn_exp2f(-z2);
            u[t][j] *= __builtin_amdgcn_sqrtf(one_minus_square(d[t][j], z2)) * sigmoid(gi[t][j]);
            zs += z2;
            h = __builtin_fmaf(d[t][j], h, u[t][j]);
        }
        run_a[seg][lc + j] = __builtin_amdgcn_exp2f(-zs);
        run_h[seg][lc + j] = h;
    }
    __syncthreads();
    if (tid < 64) {
        float st = 0.f;
        if (k == 0) {
            if (a.h0 && c1 < a.D) st = a.h0[(int64_t)b * a.D + c1];
            if (a.h_last && len == 0 && c1 < a.D) a.h_last[(int64_t)b * a.D + c1] = st;
        }
        if constexpr (CHAIN) {
            const Chain c = chain_of(a.ws, columns, a.chunks, column);
            float A = 1.f, H = 0.f;
#pragma unroll 8
            for (int s = 0; s < SEG; ++s) {
                H = __builtin_fmaf(run_a[s][tid], H, run_h[s][tid]);
                A *= run_a[s][tid];
            }
            if (k > 0) {
                publish(c, k, tid, A, H);
                st = look_back(c, k, tid);
            }
            publish(c, k, tid, __builtin_fmaf(A, st, H));
        }
        if (a.states) a.states[((int64_t)column * a.chunks + k) * kScanChannels + tid] = st;
#pragma unroll 8
        for (int s = 0; s < SEG; ++s) {
            const float next = __builtin_fmaf(run_a[s][tid], st, run_h[s][tid]);
            run_h[s][tid] = st;
            st = next;
        }
    }
    __syncthreads();
    float h[N];
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = run_h[seg][lc + j];
#pragma unroll
    for (int t = 0; t < S; ++t) {
        if (t0 + t >= len) break;
#pragma unroll
        for (int j = 0; j < N; ++j) h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
        store_piece(static_cast<T*>(a.h) + ((int64_t)b * a.L + t0 + t) * a.D + ch, n, h);
        if (a.h_last && t0 + t == len - 1) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) a.h_last[(int64_t)b * a.D + ch + j] = h[j];
        }
    }
}

// Backward: the chain runs from the last chunk to the first, over what a chunk hands on: q from zero, its decay
// the forward's.  The states that enter the chunks are the forward's, kept.
template <typename T>
__global__ __launch_bounds__(512) void scan_bwd(ScanBwdArgs a) {
    using Ti = Tile<T, 512>;
    constexpr int N = Ti::N, X = Ti::X, SEG = Ti::SEG, S = Ti::S;
    // of each run: its decay, its state from zero and what it hands on from zero; then the state that
    // enters it and what it is handed
    __shared__ float run_a[SEG][kScanChannels], run_h[SEG][kScanChannels], run_p[SEG][kScanChannels];
    __shared__ float rate[kScanChannels];
    __shared__ int drawn;
    const int tid = (int)threadIdx.x, seg = tid / X, lc = tid % X * N;
    const unsigned columns = (unsigned)(a.B * a.columns), column = blockIdx.x % columns;
    const int g = (int)(column % (unsigned)a.columns), b = (int)(column / (unsigned)a.columns);
    const int ch = g * kScanChannels + lc, n = a.D - ch;
    const int c1 = g * kScanChannels + (tid & 63);   // the carrying waves' channel
    if (tid == 0) drawn = a.chunks > 1 ? (int)draw(a.ws, columns, a.chunks, column) : 0;
    if (tid < 64) rate[tid] = c1 < a.D ? decay_rate(a.lam[c1], a.c) : 0.f;
    __syncthreads();
    const int link = drawn, k = a.chunks - 1 - link;
    const int len = length_of(a.lengths, b, a.L);
    const int t0 = k * kScanChunk + seg * S;
    float d[S][N], u[S][N], gi[S][N], gr[S][N], gg[S][N];
#pragma unroll
    for (int t = 0; t < S; ++t) {
        const int m = t0 + t < len ? n : 0;
        load_piece(row_of<T>(a.r, b, t0 + t) + ch, m, gr[t]);
        load_piece(row_of<T>(a.i, b, t0 + t) + ch, m, gi[t]);
        load_piece(row_of<T>(a.x, b, t0 + t) + ch, m, u[t]);
        load_piece(row_of<T>(a.dh.p ? a.dh : a.x, b, t0 + t) + ch, a.dh.p ? m : 0, gg[t]);
    }
    float s2[N], h[N], p[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float zs = 0.f;
        s2[j] = rate[lc + j];
        h[j] = p[j] = 0.f;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            gr[t][j] = t0 + t < len ? sigmoid(gr[t][j]) : 0.f;
            gi[t][j] = sigmoid(gi[t][j]);
            const float z2 = s2[j] * gr[t][j];
            d[t][j] = __builtin_amdgcn_exp2f(-z2);
            u[t][j] *= __builtin_amdgcn_sqrtf(one_minus_square(d[t][j], z2)) * gi[t][j];
            zs += z2;
            h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
        }
#pragma unroll
        for (int t = S - 1; t >= 0; --t) p[j] = d[t][j] * (gg[t][j] + p[j]);
        run_a[seg][lc + j] = __builtin_amdgcn_exp2f(-zs);
        run_h[seg][lc + j] = h[j];
        run_p[seg][lc + j] = p[j];
    }
    __syncthreads();
    if (tid < 64) {
        float handed = 0.f;
        if (link == 0) {
            if (a.d_last && c1 < a.D) handed = a.d_last[(int64_t)b * a.D + c1];
        }
        if (a.chunks > 1) {
            const Chain c = chain_of(a.ws, columns, a.chunks, column);
            float A = 1.f, Q = 0.f;
#pragma unroll 8
            for (int s = SEG - 1; s >= 0; --s) {
                Q = __builtin_fmaf(run_a[s][tid], Q, run_p[s][tid]);
                A *= run_a[s][tid];
            }
            if (link > 0) {
                publish(c, link, tid, A, Q);
                handed = look_back(c, link, tid);
            }
            publish(c, link, tid, __builtin_fmaf(A, handed, Q));
        }
#pragma unroll 8
        for (int s = SEG - 1; s >= 0; --s) {
            const float next = __builtin_fmaf(run_a[s][tid], handed, run_p[s][tid]);
            run_p[s][tid] = handed;
            handed = next;
        }
    } else if (tid < 128) {
        const int l = tid - 64;
        float st = a.states[((int64_t)column * a.chunks + k) * kScanChannels + l];
#pragma unroll 8
        for (int s = 0; s < SEG; ++s) {
            const float next = __builtin_fmaf(run_a[s][l], st, run_h[s][l]);
            run_h[s][l] = st;
            st = next;
        }
    }
    __syncthreads();
    float esum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        h[j] = run_h[seg][lc + j];
        p[j] = run_p[seg][lc + j];
        esum[j] = 0.f;
#pragma unroll
        for (int t = S - 1; t >= 0; --t) {
            gg[t][j] += p[j];
            p[j] = d[t][j] * gg[t][j];
        }
    }
    if (a.dh0 && k == 0 && seg == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) a.dh0[(int64_t)b * a.D + ch + j] = p[j];
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
    // the chunk's share of dlam, its runs added in order (run_a is taken)
#pragma unroll
    for (int j = 0; j < N; ++j) run_a[seg][lc + j] = esum[j];
    __syncthreads();
    if (tid < 64) {
        float s = run_a[0][tid];
#pragma unroll 8
        for (int q = 1; q < SEG; ++q) s += run_a[q][tid];
        a.shares[((int64_t)column * a.chunks + k) * kScanChannels + tid] = s;
    }
}

// dh0 of sequences without tokens
__global__ __launch_bounds__(256) void scan_bwd_empty(ScanBwdArgs a) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id < (int64_t)a.B * a.D) a.dh0[id] = a.d_last ? a.d_last[id] : 0.f;
}

// dlam: a workgroup takes a column, its 16 waves every 16th share each, added in wave order
__global__ __launch_bounds__(1024) void scan_dlam(ScanBwdArgs a) {
    __shared__ float part[16][kScanChannels];
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const int c = (int)blockIdx.x * kScanChannels + lane;
    const int64_t shares = (int64_t)a.B * a.chunks;
    float t[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t s = wave; s < shares; s += 64)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t q = s + 16 * v;
            if (q < shares) {
                const int64_t b = q / a.chunks, k = q - b * a.chunks;
                t[v] += a.shares[((b * a.columns + blockIdx.x) * a.chunks + k) * kScanChannels + lane];
            }
        }
    part[wave][lane] = (t[0] + t[1]) + (t[2] + t[3]);
    __syncthreads();
    if (wave == 0 && c < a.D) {
        float s = part[0][lane];
#pragma unroll
        for (int w = 1; w < 16; ++w) s += part[w][lane];
        // d softplus / softplus; both are exp(lam) far below 0
        const float lam = a.lam[c];
        const float f = lam < -20.f ? 1.f : 1.f / ((1.f + expf(-lam)) * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam)))));
        a.dlam[c] = s * f;
    }
}

template <typename A>
hipError_t clear_chain(const A& a, hipStream_t stream) {
    const int64_t groups = scan_chain_bytes((int64_t)a.B * a.columns, a.chunks) / 4096 + 1;
    return launch<A>(&chain_clear<A>, groups < 1024 ? groups : 1024, 256, a, stream);
}

template <typename T>
hipError_t fwd(const ScanArgs& a, hipStream_t stream) {
    const int64_t columns = (int64_t)a.B * a.columns;
    // a few tokens: a thread for each piece of channels, nothing to meet
    if (a.L <= 4)
        return launch<ScanArgs>(&scan_serial<T>, (columns * (kScanChannels / kVec<T>) + 255) / 256, 256, a, stream);
    if (a.chunks == 1) return launch<ScanArgs>(&scan_tiles<T, false>, columns, 256, a, stream);
    const hipError_t e = clear_chain(a, stream);
    if (e != hipSuccess) return e;
    return launch<ScanArgs>(&scan_tiles<T, true>, columns * a.chunks, 256, a, stream);
}
template <typename T>
hipError_t bwd(const ScanBwdArgs& a, hipStream_t stream) {
    const int64_t columns = (int64_t)a.B * a.columns;
    hipError_t e = hipSuccess;
    if (columns > 0 && a.chunks > 0) {
        if (a.chunks > 1) e = clear_chain(a, stream);
        if (e == hipSuccess) e = launch<ScanBwdArgs>(&scan_bwd<T>, columns * a.chunks, 512, a, stream);
    } else if (columns > 0 && a.dh0) {
        e = launch<ScanBwdArgs>(&scan_bwd_empty, ((int64_t)a.B * a.D + 255) / 256, 256, a, stream);
    }
    if (e != hipSuccess) return e;
    return launch<ScanBwdArgs>(&scan_dlam, a.columns, 1024, a, stream);
}

}  // namespace

hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream);
}
hipError_t launch_scan_bwd(const ScanBwdArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream);
}

}  // namespace fla
