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
// A workgroup takes a tile: a chunk of 256 tokens (backward 128) of a column of 64 channels; a thread S consecutive
// tokens of N channels (16 bytes of each row).  Each thread reduces its tokens (a run) to their decay and their state
// from zero, each wave its runs, one wave the waves' sums; the state that enters the chunk goes the same way back,
// and each thread runs over its tokens again.  Tokens past a sequence's end keep the state: a = 1, u = 0.
//
// The state that enters a chunk comes from the chunk before it, in one pass over the data: as soon as a workgroup has
// its chunk's decay A and state from zero H, it publishes both, then looks back over the chunks before it for the
// nearest one whose outgoing state is known, runs A and H of those between over it, and publishes its own outgoing
// state.  The states meet in chunk order whatever is found first, so the result does not depend on timing.
// Workgroups draw the chunks of a column in order, so a workgroup waits only for ones that have begun, and the first
// of a column waits for none: every wait ends.
//
// Measured (MI355X), 65536 tokens x 768 channels, bf16: forward 96 to 102 us, 3.9 to 4.2 TB/s where a copy of that size
// reaches 5.2; without waiting for the chain it took 82.  A tile's rows come after about 7 us, its state 4 us later
// (three round trips to words of another XCD, each 1 to 2 us while the memory is busy), during which nothing of it
// loads; asking for the next tile's rows before the wait (a workgroup staying for several tiles) took 48 registers
// and was slower, 143 us.  Every word read bypasses the L2s and costs as a memory access: reading 8 links on suspicion
// with the marks took 139 us instead of 107.  Backward, 2 x 16384 tokens x 1024 channels: 129 to 137 us, 3.4 to 3.6
// TB/s; 11 us of it the chain, 14 to 20 the arithmetic (76 vector operations a value, eight of them transcendental)
// that two workgroups on a compute unit do not hide, 10 the rows of 128 bytes (of 256 bytes a copy of the
// same tensors takes 88 us instead of 97).
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

#include <type_traits>

namespace fla {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A tile of CHUNK tokens in a workgroup of THREADS.
template <typename T, int CHUNK, int THREADS>
struct Tile {
    static constexpr int N = kVec<T>;                // channels of a thread
    static constexpr int X = kScanChannels / N;      // threads across the column
    static constexpr int SEG = THREADS / X;          // runs of tokens
    static constexpr int S = CHUNK / SEG;            // tokens of a run
    static constexpr int WAVES = THREADS / 64;
};
// Forward: up to kSerial tokens a thread runs over them for two channels (us a call, bf16, serial against tiles of 128:
// 64 x 16 tokens x 2048 channels 18.5, 24.3; 64 x 32 33.7, 23.1; 1 x 16 x 768 10.7, 9.4; 1 x 1 x 768 3.2, 7.8).  More
// tokens: tiles of kFwdChunk, or of half of it where that holds all of them (16 x 128 x 1024 7.6, in tiles of 256
// 11.3).  Tiles of 128 in a chain have twice the links to wait for: 1 x 65536 x 256 72.7 instead of 50.1,
// 1 x 30450 x 768 70.6 instead of 61.0, 8 x 1024 x 2048 37.5 and 39.0.
constexpr int kFwdChunk = 256;
constexpr int kSerial = 16;
constexpr int kBwdThreads = 512;

__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e));
}
// c softplus(lam), in units of log2
__device__ __forceinline__ float decay_rate(float lam, float c) {
    return c * kLog2e * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam))));
}
// 1 - a^2 for a = 2^-z2: near a = 1 from the series of 1 - exp(-w), w = 2 z2 ln 2, in powers of z2; its first dropped
// term is w^6 / 5040 of the value (5e-8 at w = 1/4).  There 1 - a^2 in fp32 would lose what a's rounding takes.
__device__ __forceinline__ float one_minus_square(float a, float z2) {
    constexpr float w = 2.f * kLn2;
    float p = __builtin_fmaf(z2, -w * w * w * w * w * w / 720.f, w * w * w * w * w / 120.f);
    p = __builtin_fmaf(z2, p, -w * w * w * w / 24.f);
    p = __builtin_fmaf(z2, p, w * w * w / 6.f);
    p = __builtin_fmaf(z2, p, -w * w / 2.f);
    p = __builtin_fmaf(z2, p, w) * z2;
    const float q = __builtin_fmaf(-a, a, 1.f);
    return z2 < 0.25f / w ? p : q;
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

// A thread for two channels of a sequence, token by token.
template <typename T>
__global__ __launch_bounds__(256) void scan_serial(ScanArgs a) {
    constexpr int N = 2, X = kScanChannels / N;
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

// ---- the chain over the chunks of a column, in the order in which it runs ("links").  Words of the workspace, all
//      ones until published: for each (column, link, channel) A and H in one 64-bit word, and the outgoing
//      state.  And a mark for each link: 1 with A and H, 2 with the outgoing state, so that one load of 64 marks
//      shows how far back to go; the words tell for themselves whether they are there.
struct Chain {
    unsigned long long* part;   // [links][64] of this column
    unsigned* out;              // [links][64]
    unsigned* mark;             // [links]
    unsigned* ticket;
};
__device__ __forceinline__ Chain chain_of(void* ws, int64_t columns, int links, int64_t column) {
    const int64_t all = columns * links, mine = column * links;
    Chain c;
    c.part = static_cast<unsigned long long*>(ws) + mine * kScanChannels;
    unsigned* w = reinterpret_cast<unsigned*>(static_cast<unsigned long long*>(ws) + all * kScanChannels);
    c.out = w + mine * kScanChannels;
    w += all * kScanChannels;
    c.mark = w + mine;
    c.ticket = w + all + column * kScanTicketWords;
    return c;
}
template <typename W>
__device__ __forceinline__ W seen(const W* p) {
    return __scoped_atomic_load_n(p, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
template <typename W>
__device__ __forceinline__ void put(W* p, W v) {
    __scoped_atomic_store_n(p, v, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
// the next link of the column, in order (one draw a workgroup)
__device__ __forceinline__ int draw(const Chain& c) {
    return (int)__scoped_atomic_fetch_add(c.ticket, 1u, __ATOMIC_RELAXED, __MEMORY_SCOPE_DEVICE);
}
constexpr unsigned kUnset = 0xffffffffu;
__device__ __forceinline__ unsigned word_of(float v) {
    const unsigned u = f32_bits(v);
    return u == kUnset ? 0x7fc00000u : u;   // (that NaN becomes another)
}
__device__ __forceinline__ void publish(const Chain& c, int link, int lane, float v) {
    put(c.out + (int64_t)link * kScanChannels + lane, word_of(v));
    if (lane == 0) put(c.mark + link, 2u);
}
__device__ __forceinline__ void publish(const Chain& c, int link, int lane, float A, float H) {
    put(c.part + (int64_t)link * kScanChannels + lane, (unsigned long long)word_of(A) << 32 | word_of(H));
    if (lane == 0) put(c.mark + link, 1u);
}
// The outgoing state of link - 1, for one wave (a lane each channel): the nearest outgoing state, and A and H of the
// links behind it over it, in order.
constexpr int kMostTurns = 1 << 22;   // seconds: only a workspace that another call overwrites makes a wait that long
__device__ __forceinline__ float look_back(const Chain& c, int link, int lane) {
    constexpr int kBatch = 4;
    for (int turn = 0; turn < kMostTurns; ++turn) {
        const unsigned m = lane < link ? seen(c.mark + (link - 1 - lane)) : 0u;
        const unsigned long long outs = __builtin_amdgcn_ballot_w64(m == 2u), parts = __builtin_amdgcn_ballot_w64(m != 0u);
        if (outs != 0) {
            const int near = __builtin_ctzll(outs);   // links behind the nearest outgoing state
            const unsigned long long behind = (1ull << near) - 1;
            if ((parts & behind) == behind) {
                const int first = link - 1 - near;
                const unsigned w = seen(c.out + (int64_t)first * kScanChannels + lane);
                bool there = true;
                float state = bits_f32(w);
                for (int at = first + 1; at < link; at += kBatch) {
                    // (a batch is asked for at once, without a condition, past the last link that one again)
                    unsigned long long p[kBatch];
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
                        p[i] = seen(c.part + (int64_t)(at + i < link ? at + i : link - 1) * kScanChannels + lane);
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
                        if (at + i < link) {
                            there = there && p[i] != ~0ull;
                            state = __builtin_fmaf(bits_f32((unsigned)(p[i] >> 32)), state, bits_f32((unsigned)p[i]));
                        }
                }
                there = there && w != kUnset;
                if (__builtin_amdgcn_ballot_w64(!there) == 0) return state;
            }
        }
        __builtin_amdgcn_s_sleep(1);
    }
    return __builtin_nanf("");
}

// The column of a workgroup.  Ids go to the 8 XCDs in turn: in long chains groups of 8 take a column each, so that the
// tiles of one chunk mostly meet in one XCD's L2 -- where the columns' rows are not whole cache lines and share some,
// or HBM pages.  us a call, each id the next column / groups of 8: 1 x 20000 x 1001 bf16 79.5, 65.7; 4 x 5001 x 1001
// 74.8, 64.2; 1 x 65536 x 768 102, 99.  Of few links the start of the chain counts: 4 x 2048 x 512 15.0, 15.9; and a
// last group that is not full draws for nothing: 8 x 1024 x 2048 38.4, 44.3.
__host__ __device__ constexpr int column_shift(int links, int lines) { return links >= (lines ? 32 : 16) ? 3 : 0; }
__device__ __forceinline__ unsigned column_of(unsigned id, unsigned columns, int links, int lines) {
    return (id >> column_shift(links, lines)) % columns;
}

// the words of a workspace before a chain: all ones; the marks and tickets 0
template <typename A>
__global__ __launch_bounds__(256) void chain_clear(A a) {
    unsigned* ws = static_cast<unsigned*>(a.ws);
    const int64_t columns = (int64_t)a.B * a.columns, words = columns * a.links * kScanChannels * 3;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words + columns * (a.links + kScanTicketWords);
         w += (int64_t)gridDim.x * 256)
        ws[w] = w < words ? kUnset : 0u;
}

// Runs of one column and their joining.  The runs of a wave are neighbours, and a lane takes a channel of
// them: it reduces the wave's runs to one, and once the state that enters the wave is known, runs over
// them again.  Only the waves' sums cross the workgroup.
template <int SEG, int WAVES>
struct Runs {
    static constexpr int PER = SEG / WAVES;   // runs of a wave
    float a[SEG][kScanChannels];              // decay of each run
    float h[SEG][kScanChannels];              // its state from zero; then the state that enters it
    float wave_a[WAVES][kScanChannels], wave_h[WAVES][kScanChannels];   // the same of a wave's runs
};
// the order of LDS accesses within a wave is theirs in the program
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// runs [s0, s0 + PER) in order (BACK: from the last) to one, in (A, H)
template <int PER, bool BACK>
__device__ __forceinline__ void join(const float (*ra)[kScanChannels], const float (*rh)[kScanChannels], int s0, int lane,
                                     float& A, float& H) {
    A = 1.f;
    H = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = s0 + (BACK ? PER - 1 - i : i);
        H = __builtin_fmaf(ra[s][lane], H, rh[s][lane]);
        A *= ra[s][lane];
    }
}
// the states that enter the runs, from the one that enters the first, in place of rh
template <int PER, bool BACK>
__device__ __forceinline__ float enter(const float (*ra)[kScanChannels], float (*rh)[kScanChannels], int s0, int lane,
                                       float st) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int s = s0 + (BACK ? PER - 1 - i : i);
        const float next = __builtin_fmaf(ra[s][lane], st, rh[s][lane]);
        rh[s][lane] = st;
        st = next;
    }
    return st;
}

// (32 values a thread; four waves on a SIMD)
template <typename T, int CHUNK, bool CHAIN>
__global__ __launch_bounds__(2 * CHUNK, 4) void scan_tiles(ScanArgs a) {
    using Ti = Tile<T, CHUNK, 2 * CHUNK>;
    constexpr int N = Ti::N, X = Ti::X, SEG = Ti::SEG, S = Ti::S, WAVES = Ti::WAVES;
    using R = Runs<SEG, WAVES>;
    __shared__ R runs;
    __shared__ float rate[kScanChannels];
    __shared__ int drawn;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, seg = tid / X, lc = tid % X * N;
    const unsigned columns = (unsigned)(a.B * a.columns), column = CHAIN ? column_of(blockIdx.x, columns, a.links, a.lines) : blockIdx.x;
    const int g = (int)(column % (unsigned)a.columns), b = (int)(column / (unsigned)a.columns);
    const int ch = g * kScanChannels + lc, n = a.D - ch;
    const int c1 = g * kScanChannels + lane;   // the channel of a joining lane
    if (CHAIN && tid == 0) drawn = draw(chain_of(a.ws, columns, a.links, column));
    if (tid < 64) rate[tid] = c1 < a.D ? decay_rate(a.lam[c1], a.c) : 0.f;
    __syncthreads();
    const int k = CHAIN ? drawn : 0;
    if (k >= a.links) return;
    const int len = length_of(a.lengths, b, a.L);
    const int t0 = k * CHUNK + seg * S;
    float d[S][N], u[S][N];
    // WHOLE: every token and channel of the tile is there
    auto load = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        float gi[S][N];
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const int m = WHOLE ? N : t0 + t < len ? n : 0;
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
                const float z2 = WHOLE || t0 + t < len ? s2 * sigmoid(d[t][j]) : 0.f;
                d[t][j] = __builtin_amdgcn_exp2f(-z2);
                u[t][j] *= __builtin_amdgcn_sqrtf(one_minus_square(d[t][j], z2)) * sigmoid(gi[t][j]);
                zs += z2;
                h = __builtin_fmaf(d[t][j], h, u[t][j]);
            }
            runs.a[seg][lc + j] = __builtin_amdgcn_exp2f(-zs);
            runs.h[seg][lc + j] = h;
        }
    };
    const bool whole = (int64_t)(k + 1) * CHUNK <= len && (g + 1) * kScanChannels <= a.D;
    if (whole)
        load(std::true_type{});
    else
        load(std::false_type{});
    wave_order();
    float A, H;
    join<R::PER, false>(runs.a, runs.h, wave * R::PER, lane, A, H);
    runs.wave_a[wave][lane] = A;
    runs.wave_h[wave][lane] = H;
    __syncthreads();
    if (wave == 0) {
        float st = 0.f;
        if (k == 0) {
            if (a.h0 && c1 < a.D) st = a.h0[(int64_t)b * a.D + c1];
            if (a.h_last && len == 0 && c1 < a.D) a.h_last[(int64_t)b * a.D + c1] = st;
        }
        if constexpr (CHAIN) {
            const Chain c = chain_of(a.ws, columns, a.links, column);
            join<WAVES, false>(runs.wave_a, runs.wave_h, 0, lane, A, H);
            if (k > 0) {
                publish(c, k, lane, A, H);
                st = look_back(c, k, lane);
            }
            publish(c, k, lane, __builtin_fmaf(A, st, H));
        }
        enter<WAVES, false>(runs.wave_a, runs.wave_h, 0, lane, st);
        if (a.states)
#pragma unroll
            for (int q = 0; q < CHUNK / kScanChunk; ++q)
                if (k * (CHUNK / kScanChunk) + q < a.chunks)
                    a.states[((int64_t)column * a.chunks + k * (CHUNK / kScanChunk) + q) * kScanChannels + lane] =
                        runs.wave_h[q * WAVES / (CHUNK / kScanChunk)][lane];
    }
    __syncthreads();
    enter<R::PER, false>(runs.a, runs.h, wave * R::PER, lane, runs.wave_h[wave][lane]);
    wave_order();
    float h[N];
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = runs.h[seg][lc + j];
#pragma unroll
    for (int t = 0; t < S; ++t) {
        if (!whole && t0 + t >= len) break;
#pragma unroll
        for (int j = 0; j < N; ++j) h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
        T* row = static_cast<T*>(a.h) + ((int64_t)b * a.L + t0 + t) * a.D + ch;
        if (whole && a.lines)
            store_piece<true>(row, N, h);
        else
            store_piece(row, n, h);
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
__global__ __launch_bounds__(kBwdThreads, 4) void scan_bwd(ScanBwdArgs a) {
    using Ti = Tile<T, kScanChunk, kBwdThreads>;
    constexpr int N = Ti::N, X = Ti::X, SEG = Ti::SEG, S = Ti::S, WAVES = Ti::WAVES;
    using R = Runs<SEG, WAVES>;
    __shared__ R runs;
    __shared__ float run_p[SEG][kScanChannels];   // what a run hands on from zero; then what it is handed
    __shared__ float wave_p[WAVES][kScanChannels], wave_b[WAVES][kScanChannels];
    __shared__ float rate[kScanChannels];
    __shared__ int drawn;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, seg = tid / X, lc = tid % X * N;
    const unsigned columns = (unsigned)(a.B * a.columns), column = column_of(blockIdx.x, columns, a.links, a.lines);
    const int g = (int)(column % (unsigned)a.columns), b = (int)(column / (unsigned)a.columns);
    const int ch = g * kScanChannels + lc, n = a.D - ch;
    const int c1 = g * kScanChannels + lane;   // the channel of a joining lane
    if (tid == 0) drawn = a.chunks > 1 ? draw(chain_of(a.ws, columns, a.links, column)) : 0;
    if (tid < 64) rate[tid] = c1 < a.D ? decay_rate(a.lam[c1], a.c) : 0.f;
    __syncthreads();
    const int link = drawn, k = a.chunks - 1 - link;
    if (link >= a.links) return;
    const int len = length_of(a.lengths, b, a.L);
    const int t0 = k * kScanChunk + seg * S;
    float d[S][N], u[S][N], gi[S][N], gr[S][N], gg[S][N];
    const bool whole = (int64_t)(k + 1) * kScanChunk <= len && (g + 1) * kScanChannels <= a.D;
    auto load = [&](auto is_whole) {
        constexpr bool WHOLE = decltype(is_whole)::value;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const int m = WHOLE ? N : t0 + t < len ? n : 0;
            load_piece(row_of<T>(a.r, b, t0 + t) + ch, m, gr[t]);
            load_piece(row_of<T>(a.i, b, t0 + t) + ch, m, gi[t]);
            load_piece(row_of<T>(a.x, b, t0 + t) + ch, m, u[t]);
            load_piece(row_of<T>(a.dh.p ? a.dh : a.x, b, t0 + t) + ch, a.dh.p ? m : 0, gg[t]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float s2 = rate[lc + j];
            float zs = 0.f, h = 0.f, p = 0.f;
#pragma unroll
            for (int t = 0; t < S; ++t) {
                gr[t][j] = WHOLE || t0 + t < len ? sigmoid(gr[t][j]) : 0.f;
                gi[t][j] = sigmoid(gi[t][j]);
                const float z2 = s2 * gr[t][j];
                d[t][j] = __builtin_amdgcn_exp2f(-z2);
                u[t][j] *= __builtin_amdgcn_sqrtf(one_minus_square(d[t][j], z2)) * gi[t][j];
                zs += z2;
                h = __builtin_fmaf(d[t][j], h, u[t][j]);
            }
#pragma unroll
            for (int t = S - 1; t >= 0; --t) p = d[t][j] * (gg[t][j] + p);
            runs.a[seg][lc + j] = __builtin_amdgcn_exp2f(-zs);
            runs.h[seg][lc + j] = h;
            run_p[seg][lc + j] = p;
        }
    };
    if (whole)
        load(std::true_type{});
    else
        load(std::false_type{});
    wave_order();
    float A, H, Q;
    join<R::PER, false>(runs.a, runs.h, wave * R::PER, lane, A, H);
    runs.wave_a[wave][lane] = A;
    runs.wave_h[wave][lane] = H;
    join<R::PER, true>(runs.a, run_p, wave * R::PER, lane, A, Q);
    wave_b[wave][lane] = A;
    wave_p[wave][lane] = Q;
    __syncthreads();
    if (wave == 0) {
        float handed = 0.f;
        if (link == 0 && a.d_last && c1 < a.D) handed = a.d_last[(int64_t)b * a.D + c1];
        if (a.chunks > 1) {
            const Chain c = chain_of(a.ws, columns, a.links, column);
            join<WAVES, true>(wave_b, wave_p, 0, lane, A, Q);
            if (link > 0) {
                publish(c, link, lane, A, Q);
                handed = look_back(c, link, lane);
            }
            publish(c, link, lane, __builtin_fmaf(A, handed, Q));
        }
        enter<WAVES, true>(wave_b, wave_p, 0, lane, handed);
    } else if (wave == 1) {
        enter<WAVES, false>(runs.wave_a, runs.wave_h, 0, lane, a.states[((int64_t)column * a.chunks + k) * kScanChannels + lane]);
    }
    __syncthreads();
    enter<R::PER, false>(runs.a, runs.h, wave * R::PER, lane, runs.wave_h[wave][lane]);
    enter<R::PER, true>(runs.a, run_p, wave * R::PER, lane, wave_p[wave][lane]);
    wave_order();
    float h[N], esum[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        h[j] = runs.h[seg][lc + j];
        float p = run_p[seg][lc + j];
        esum[j] = 0.f;
#pragma unroll
        for (int t = S - 1; t >= 0; --t) {
            gg[t][j] += p;
            p = d[t][j] * gg[t][j];
        }
        if (a.dh0 && k == 0 && seg == 0 && j < n) a.dh0[(int64_t)b * a.D + ch + j] = p;
    }
#pragma unroll
    for (int t = 0; t < S; ++t) {
        float dx[N], dr[N], di[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float z2 = rate[lc + j] * gr[t][j], z = z2 * kLn2, m2 = one_minus_square(d[t][j], z2);
            const float v = gg[t][j] * u[t][j];
            // z / m^2, which is about 1/2 as both vanish; u vanishes there too, so what keeps 0 / 0 away does not count
            const float over = z * __builtin_amdgcn_rcpf(m2 + 1e-36f);
            const float e = gg[t][j] * d[t][j] * __builtin_fmaf(-z, h[j], over * d[t][j] * u[t][j]);
            h[j] = __builtin_fmaf(d[t][j], h[j], u[t][j]);
            dx[j] = gg[t][j] * __builtin_amdgcn_sqrtf(m2) * gi[t][j];
            di[j] = v * (1.f - gi[t][j]);
            dr[j] = e * (1.f - gr[t][j]);
            esum[j] += e;
        }
        const int64_t at = ((int64_t)b * a.L + t0 + t) * a.D + ch;
        if (whole && a.lines) {
            store_piece<true>(static_cast<T*>(a.dx) + at, N, dx);
            store_piece<true>(static_cast<T*>(a.dr) + at, N, dr);
            store_piece<true>(static_cast<T*>(a.di) + at, N, di);
        } else if (t0 + t < a.L) {
            if (t0 + t >= len) {
#pragma unroll
                for (int j = 0; j < N; ++j) dx[j] = dr[j] = di[j] = 0.f;
            }
            store_piece(static_cast<T*>(a.dx) + at, n, dx);
            store_piece(static_cast<T*>(a.dr) + at, n, dr);
            store_piece(static_cast<T*>(a.di) + at, n, di);
        }
    }
    // the chunk's share of dlam, its runs added in order (the wave's runs.a are taken)
#pragma unroll
    for (int j = 0; j < N; ++j) runs.a[seg][lc + j] = esum[j];
    wave_order();
    float s = runs.a[wave * R::PER][lane];
#pragma unroll
    for (int q = 1; q < R::PER; ++q) s += runs.a[wave * R::PER + q][lane];
    runs.wave_a[wave][lane] = s;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += runs.wave_a[w][lane];
        a.shares[(((int64_t)b * a.chunks + k) * a.columns + g) * kScanChannels + lane] = s;
    }
}

// dh0 of sequences without tokens
__global__ __launch_bounds__(256) void scan_bwd_empty(ScanBwdArgs a) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id < (int64_t)a.B * a.D) a.dh0[id] = a.d_last ? a.d_last[id] : 0.f;
}

__global__ __launch_bounds__(1024) void scan_dlam(ScanBwdArgs a) {
    const int64_t c0 = (int64_t)blockIdx.x * kSumColumns, c = c0 + threadIdx.x;
    const float s = column_sum(a.shares, (int64_t)a.B * a.chunks, (int64_t)a.columns * kScanChannels, c0, a.D);
    if (threadIdx.x < kSumColumns && c < a.D) {
        // d softplus / softplus; both are exp(lam) far below 0
        const float lam = a.lam[c];
        const float f = lam < -20.f ? 1.f : 1.f / ((1.f + expf(-lam)) * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam)))));
        a.dlam[c] = s * f;
    }
}

template <typename A>
hipError_t clear_chain(const A& a, hipStream_t stream) {
    const int64_t groups = scan_chain_bytes((int64_t)a.B * a.columns, a.links) / 4096 + 1;
    return launch<A>(&chain_clear<A>, groups < 1024 ? groups : 1024, 256, a, stream);
}

// one workgroup for each tile, whole groups for each column (a workgroup that draws past the last link ends)
template <typename A>
int64_t chain_groups(const A& a) {
    const int group = 1 << column_shift(a.links, a.lines);
    return (int64_t)a.B * a.columns * ((a.links + group - 1) / group * group);
}

template <typename T>
hipError_t fwd(const ScanArgs& args, hipStream_t stream) {
    ScanArgs a = args;
    const int64_t columns = (int64_t)a.B * a.columns;
    if (a.L <= kSerial) return launch<ScanArgs>(&scan_serial<T>, (columns * (kScanChannels / 2) + 255) / 256, 256, a, stream);
    a.links = (int)(((int64_t)a.L + kFwdChunk - 1) / kFwdChunk);
    if (a.L <= kFwdChunk / 2)
        return launch<ScanArgs>(&scan_tiles<T, kFwdChunk / 2, false>, columns, kFwdChunk, a, stream);
    if (a.links == 1) return launch<ScanArgs>(&scan_tiles<T, kFwdChunk, false>, columns, 2 * kFwdChunk, a, stream);
    const hipError_t e = clear_chain(a, stream);
    if (e != hipSuccess) return e;
    return launch<ScanArgs>(&scan_tiles<T, kFwdChunk, true>, chain_groups(a), 2 * kFwdChunk, a, stream);
}
template <typename T>
hipError_t bwd(const ScanBwdArgs& a, hipStream_t stream) {
    const int64_t columns = (int64_t)a.B * a.columns;
    hipError_t e = hipSuccess;
    if (columns > 0 && a.chunks > 0) {
        if (a.chunks > 1) e = clear_chain(a, stream);
        if (e == hipSuccess) e = launch<ScanBwdArgs>(&scan_bwd<T>, chain_groups(a), kBwdThreads, a, stream);
    } else if (columns > 0 && a.dh0) {
        e = launch<ScanBwdArgs>(&scan_bwd_empty, ((int64_t)a.B * a.D + 255) / 256, 256, a, stream);
    }
    if (e != hipSuccess) return e;
    return launch<ScanBwdArgs>(&scan_dlam, ((int64_t)a.D + kSumColumns - 1) / kSumColumns, 1024, a, stream);
}

}  // namespace

hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream);
}
hipError_t launch_scan_bwd(const ScanBwdArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream);
}

}  // namespace fla
