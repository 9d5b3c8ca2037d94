// Residual addition and root-mean-square norm, forward (in the input's type or in 8 bits with scales)
// and backward, gfx950.
//
// Bound by memory: every value is read once and written once, a handful of operations each.  W waves
// share a row; a lane holds K pieces of 16 bytes of it (pieces of consecutive lanes are consecutive), so
// a row is read once and its values stay in registers between the sum of squares and the output.  Rows of
// more than 16 waves hold are read again instead (the *_wide kernels).
//
// Measured (MI355X; a copy reaches 5.2 TB/s): forward with residual, sum and 1 / rms, 65536 rows of 768 bf16 77 us, 5.2
// TB/s; 8-bit output with a scale for 128 channels, 121800 rows of 1024 140 us, 6.2 TB/s; backward with dsum, 65536 rows
// of 768 bf16 74 us, 5.4 TB/s, 16384 of 4096 100 us, 5.4 TB/s, 4099 of 1001 fp32 16.5 us (12.4 and the sum of the
// shares of dweight, 4.0).  Eight rows of 768: 3.6 us.
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

#include <type_traits>

namespace fla {
namespace {

// Where a lane stands in its row, and the sums over the row's waves.
template <int W>
struct Row {
    static constexpr int kThreads = W == 1 ? 256 : 64 * W;   // one wave per row: four rows per workgroup
    static constexpr int kRows = W == 1 ? 4 : 1;
    int lane, wave, first;
    __device__ __forceinline__ Row() {
        lane = (int)threadIdx.x & 63;
        wave = (int)threadIdx.x >> 6;
        first = W == 1 ? lane : (int)threadIdx.x;
    }
    __device__ __forceinline__ int64_t row0() const { return (int64_t)blockIdx.x * kRows + (W == 1 ? wave : 0); }
};

// OP over all waves of a row; `red` alternates between two buffers, so one barrier per call is enough
template <int W, typename OP>
__device__ __forceinline__ unsigned over_row(unsigned x, unsigned (*red)[16], int& buf, int wave) {
    x = over_lanes<OP>(x, 64);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) red[buf][wave] = x;
        __syncthreads();
        x = red[buf][0];
#pragma unroll
        for (int w = 1; w < W; ++w) x = OP::of(x, red[buf][w]);
        buf ^= 1;
    }
    return x;
}
template <int W>
__device__ __forceinline__ float row_sum(float x, unsigned (*red)[16], int& buf, int wave) {
    return bits_f32(over_row<W, SumOp>(f32_bits(x), red, buf, wave));
}

template <typename T, int N>
__device__ __forceinline__ void load_weight(const void* w, int f32, int col, int n, float (&v)[N]) {
    if (f32)
        load_piece(static_cast<const float*>(w) + col, n, v);
    else
        load_piece(static_cast<const T*>(w) + col, n, v);
}

// ---- 8-bit output: a scale for max|y| of a group of channels (or of the row), and the values over it
__device__ __forceinline__ float scale_of(unsigned top_bits) {
    const float top = bits_f32(top_bits);
    if (top == 0.f) return 1.f;
    const float s = top / 448.f;
    return s < 0x1p-126f ? 0x1p-126f : s;   // (a NaN stays)
}
// N values times 1 / scale as e4m3 bytes.  |y| / scale is at most 448 (1 + 2^-22), which rounds to 448.
template <int N>
__device__ __forceinline__ void store_q(bool nt, unsigned char* p, int n, const float (&y)[N], float inv) {
    unsigned w[N / 4];
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j] * inv, y[4 * j + 1] * inv, 0, false);
        u = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j + 2] * inv, y[4 * j + 3] * inv, u, true);
        w[j] = (unsigned)u;
    }
    if (n >= N) {
        if constexpr (N == 8) {
            const u32x2_any v = {w[0], w[1]};
            if (nt)
                store8<true>(p, v);
            else
                store8<false>(p, v);
        } else {
            __builtin_memcpy(p, w, N);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) p[j] = (unsigned char)(w[j / 4] >> (8 * (j % 4)));
    }
}

template <typename T, int W, int K, bool Q8>
__global__ __launch_bounds__(Row<W>::kThreads) void norm_fwd(NormArgs a) {
    constexpr int N = kVec<T>;
    __shared__ unsigned red[2][16];
    int buf = 0;
    const Row<W> rw;
    float w[K][N];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * 64 * W + rw.first) * N;
        load_weight<T>(a.weight, a.weight_f32, col, a.D - col, w[k]);
    }
    for (int64_t row = rw.row0(); row < a.rows; row += (int64_t)gridDim.x * Row<W>::kRows) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.residual_stride : nullptr;
        float s[K][N];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (k * 64 * W + rw.first) * N;
            load_piece<true>(x + col, a.D - col, s[k]);
        }
        if (res) {
            float t[K][N];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (k * 64 * W + rw.first) * N;
                load_piece<true>(res + col, a.D - col, t[k]);
            }
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) s[k][j] += t[k][j];
        }
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) ss = __builtin_fmaf(s[k][j], s[k][j], ss);
        if (a.sum) {
            T* out = static_cast<T*>(a.sum) + row * a.D;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (k * 64 * W + rw.first) * N;
                store_piece(a.nt, out + col, a.D - col, s[k]);
            }
        }
        const float rstd = __builtin_amdgcn_rsqf(
            __builtin_fmaf(row_sum<W>(ss, red, buf, rw.wave), a.inv_D, a.eps));
        if (a.rstd && rw.first == 0) a.rstd[row] = rstd;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) s[k][j] = s[k][j] * rstd * w[k][j];
        if constexpr (!Q8) {
            T* y = static_cast<T*>(a.y) + row * a.D;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (k * 64 * W + rw.first) * N;
                store_piece(a.nt, y + col, a.D - col, s[k]);
            }
        } else {
            unsigned top[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                top[k] = 0;
#pragma unroll
                for (int j = 0; j < N; ++j) top[k] = MaxOp::of(top[k], f32_bits(s[k][j]) & 0x7fffffffu);
            }
            if (a.group == 0) {
#pragma unroll
                for (int k = 1; k < K; ++k) top[0] = MaxOp::of(top[0], top[k]);
                top[0] = over_row<W, MaxOp>(top[0], red, buf, rw.wave);
            }
            unsigned char* q = static_cast<unsigned char*>(a.y) + row * a.D;
            const int lanes = a.group / N;   // of one group
            const int groups = a.group ? (a.D + a.group - 1) / a.group : 1;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int piece = k * 64 * W + rw.first, col = piece * N;
                if (a.group) top[k] = over_lanes<MaxOp>(top[k], lanes);
                const float scale = scale_of(a.group ? top[k] : top[0]);
                if (col < a.D && (a.group ? (piece & (lanes - 1)) == 0 : piece == 0))
                    a.scales[row * groups + (a.group ? col / a.group : 0)] = scale;
                store_q(a.nt, q + col, a.D - col, s[k], 1.f / scale);
            }
        }
    }
}

// Rows of any width: the row is read again for each of its uses (from the caches).  In place is fine:
// a thread reads its pieces before it writes them, and reads none that another writes.
template <typename T, bool Q8>
__global__ __launch_bounds__(1024) void norm_fwd_wide(NormArgs a) {
    constexpr int N = kVec<T>, W = 16;
    __shared__ unsigned red[2][16];
    int buf = 0;
    const Row<W> rw;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.residual_stride : nullptr;
        auto load = [&](int col, float (&s)[N]) {
            load_piece(x + col, a.D - col, s);
            if (res) {
                float t[N];
                load_piece(res + col, a.D - col, t);
#pragma unroll
                for (int j = 0; j < N; ++j) s[j] += t[j];
            }
        };
        float ss = 0.f;
        for (int64_t c = rw.first * N; c < a.D; c += 1024 * N) {
            float s[N];
            load((int)c, s);
#pragma unroll
            for (int j = 0; j < N; ++j) ss = __builtin_fmaf(s[j], s[j], ss);
        }
        const float rstd = __builtin_amdgcn_rsqf(
            __builtin_fmaf(row_sum<W>(ss, red, buf, rw.wave), a.inv_D, a.eps));
        if (a.rstd && rw.first == 0) a.rstd[row] = rstd;
        auto norm = [&](int col, float (&s)[N], float (&y)[N]) {
            float w[N];
            load(col, s);
            load_weight<T>(a.weight, a.weight_f32, col, a.D - col, w);
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = s[j] * rstd * w[j];
        };
        auto top_of = [&](const float (&y)[N]) {
            unsigned t = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) t = MaxOp::of(t, f32_bits(y[j]) & 0x7fffffffu);
            return t;
        };
        unsigned row_top = 0;
        if (Q8 && a.group == 0) {
            for (int64_t c = rw.first * N; c < a.D; c += 1024 * N) {
                float s[N], y[N];
                norm((int)c, s, y);
                row_top = MaxOp::of(row_top, top_of(y));
            }
            row_top = over_row<W, MaxOp>(row_top, red, buf, rw.wave);
            if (rw.first == 0) a.scales[row] = scale_of(row_top);
        }
        const int lanes = a.group / N;
        const int groups = a.group ? (a.D + a.group - 1) / a.group : 1;
        // whole workgroups of pieces, so that a group's lanes meet in over_lanes
        for (int64_t c0 = 0; c0 < a.D; c0 += 1024 * N) {
            const int64_t c = c0 + rw.first * N;
            const int col = c < a.D ? (int)c : a.D;   // past the end: no value
            float s[N], y[N];
            norm(col, s, y);
            if (a.sum) store_piece(static_cast<T*>(a.sum) + row * a.D + col, a.D - col, s);
            if constexpr (!Q8) {
                store_piece(static_cast<T*>(a.y) + row * a.D + col, a.D - col, y);
            } else {
                const unsigned top = a.group ? over_lanes<MaxOp>(top_of(y), lanes) : row_top;
                const float scale = scale_of(top);
                if (a.group && col < a.D && (rw.first & (lanes - 1)) == 0)
                    a.scales[row * groups + col / a.group] = scale;
                store_q(false, static_cast<unsigned char*>(a.y) + row * a.D + col, a.D - col, y, 1.f / scale);
            }
        }
    }
}

// ---- backward: a workgroup takes every gridDim-th row (of W = 1: four at a time) and keeps its share of
//      dweight in registers, which goes to the workspace at the end and is summed by norm_bwd_weight.
// (NT: rows of whole cache lines, read non-temporally)
template <typename T, int W, int K, bool NT>
__global__ __launch_bounds__(Row<W>::kThreads) void norm_bwd(NormBwdArgs a) {
    constexpr int N = kVec<T>;
    __shared__ unsigned red[2][16];
    int buf = 0;
    const Row<W> rw;
    float w[K][N], dw[K][N];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * 64 * W + rw.first) * N;
        load_weight<T>(a.weight, a.weight_f32, col, a.D - col, w[k]);
#pragma unroll
        for (int j = 0; j < N; ++j) dw[k][j] = 0.f;
    }
    // A row's pieces as they lie in memory; the next row's are asked for before this one's sum is waited for, where the
    // registers hold both (65536 rows of 768 bf16 90 -> 73 us; with four pieces of fp32 a lane two waves fewer on a SIMD,
    // 4099 of 1001 18.9 -> 20.1; 16 waves of two pieces of bf16 spill).
    constexpr bool AHEAD = K <= 2 && !(W == 16 && K == 2 && sizeof(T) == 2);
    struct Raw {
        u32x4_any s[K], dy[K], ds[K];
        float rstd;
    };
    auto ask = [&](Raw& r, int64_t row) {
        const T* sp = static_cast<const T*>(a.s) + row * a.s_stride;
        const T* dyp = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const T* dsp = static_cast<const T*>(a.dsum) + (a.dsum ? row * a.dsum_stride : 0);
        r.rstd = a.rstd[row];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (k * 64 * W + rw.first) * N;
            r.s[k] = load_raw<NT>(sp + col, a.D - col);
            r.dy[k] = load_raw<NT>(dyp + col, a.D - col);
            r.ds[k] = a.dsum ? load_raw<NT>(dsp + col, a.D - col) : u32x4_any{0u, 0u, 0u, 0u};
        }
    };
    const int64_t step = (int64_t)gridDim.x * Row<W>::kRows;
    int64_t row = rw.row0();
    Raw now, next;
    if (AHEAD && row < a.rows) ask(now, row);
    for (; row < a.rows; row += step) {
        if constexpr (!AHEAD)
            ask(now, row);
        else if (row + step < a.rows)
            ask(next, row + step);
        float along = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s[N], dy[N];
            unpack(now.s[k], s);
            unpack(now.dy[k], dy);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float v = dy[j] * (s[j] * now.rstd);
                dw[k][j] += v;
                along = __builtin_fmaf(v, w[k][j], along);
            }
        }
        along = row_sum<W>(along, red, buf, rw.wave) * a.inv_D;
        T* dx = static_cast<T*>(a.dx) + row * a.D;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (k * 64 * W + rw.first) * N;
            float s[N], dy[N], t[N];
            unpack(now.s[k], s);
            unpack(now.dy[k], dy);
            unpack(now.ds[k], t);
#pragma unroll
            for (int j = 0; j < N; ++j)
                t[j] = __builtin_fmaf(__builtin_fmaf(-(s[j] * now.rstd), along, dy[j] * w[k][j]), now.rstd, t[j]);
            store_piece(dx + col, a.D - col, t);
        }
        if constexpr (AHEAD) now = next;
    }
    float* out = a.ws + (int64_t)blockIdx.x * a.D;
    if constexpr (W == 1) {
        // the four waves' shares, in wave order
        __shared__ float part[4][K * N * 64];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < N; ++j) part[rw.wave][(k * 64 + rw.lane) * N + j] = dw[k][j];
        __syncthreads();
        for (int c = (int)threadIdx.x; c < a.D; c += 256)
            out[c] = part[0][c] + part[1][c] + part[2][c] + part[3][c];
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (k * 64 * W + rw.first) * N;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (col + j < a.D) out[col + j] = dw[k][j];
        }
    }
}

// Rows of any width: read again for the output, the shares of dweight kept in the workspace.
template <typename T>
__global__ __launch_bounds__(1024) void norm_bwd_wide(NormBwdArgs a) {
    constexpr int N = kVec<T>, W = 16;
    __shared__ unsigned red[2][16];
    int buf = 0;
    const Row<W> rw;
    float* share = a.ws + (int64_t)blockIdx.x * a.D;
    bool first = true;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* sp = static_cast<const T*>(a.s) + row * a.s_stride;
        const T* dyp = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const float rstd = a.rstd[row];
        float along = 0.f;
        for (int64_t c = rw.first * N; c < a.D; c += 1024 * N) {
            const int col = (int)c, n = a.D - col;
            float s[N], dy[N], w[N];
            load_piece(sp + col, n, s);
            load_piece(dyp + col, n, dy);
            load_weight<T>(a.weight, a.weight_f32, col, n, w);
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < n) {
                    const float v = dy[j] * (s[j] * rstd);
                    share[col + j] = first ? v : share[col + j] + v;
                    along = __builtin_fmaf(v, w[j], along);
                }
        }
        first = false;
        along = row_sum<W>(along, red, buf, rw.wave) * a.inv_D;
        T* dx = static_cast<T*>(a.dx) + row * a.D;
        const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.dsum_stride : nullptr;
        for (int64_t c = rw.first * N; c < a.D; c += 1024 * N) {
            const int col = (int)c, n = a.D - col;
            float s[N], dy[N], w[N], t[N];
            load_piece(sp + col, n, s);
            load_piece(dyp + col, n, dy);
            load_weight<T>(a.weight, a.weight_f32, col, n, w);
#pragma unroll
            for (int j = 0; j < N; ++j) t[j] = 0.f;
            if (ds) load_piece(ds + col, n, t);
#pragma unroll
            for (int j = 0; j < N; ++j)
                t[j] = __builtin_fmaf(__builtin_fmaf(-(s[j] * rstd), along, dy[j] * w[j]), rstd, t[j]);
            store_piece(dx + col, n, t);
        }
    }
}

__global__ __launch_bounds__(1024) void norm_bwd_weight(NormBwdArgs a) {
    const int64_t c0 = (int64_t)blockIdx.x * kSumColumns;
    const float s = column_sum(a.ws, a.blocks, a.D, c0, a.D);
    if (threadIdx.x < kSumColumns && c0 + threadIdx.x < a.D) a.dweight[c0 + threadIdx.x] = s;
}

// Waves per row and pieces per lane by the width.
#define FLA_WIDTH(W, K) \
    if (pieces <= 64 * W * K) { f(std::integral_constant<int, W>{}, std::integral_constant<int, K>{}); return true; }
// Forward: one wave up to 4 pieces a lane, then 4, then 16.
template <typename F>
bool fwd_width(int64_t pieces, F&& f) {
    FLA_WIDTH(1, 1)
    FLA_WIDTH(1, 2)
    FLA_WIDTH(1, 4)
    FLA_WIDTH(4, 2)
    FLA_WIDTH(4, 4)
    FLA_WIDTH(16, 2)
    FLA_WIDTH(16, 4)
    return false;
}
// Backward, where a lane keeps more for each channel: as few pieces of bf16 as the waves allow (with 4 in a lane two
// waves fit a SIMD: 8192 rows of 2048 43 us, with one and four waves a row 35), up to 4 of fp32.
template <typename T, typename F>
bool bwd_width(int64_t pieces, F&& f) {
    FLA_WIDTH(1, 1)
    FLA_WIDTH(1, 2)
    if constexpr (sizeof(T) == 4) {
        FLA_WIDTH(1, 4)
        FLA_WIDTH(4, 2)
        FLA_WIDTH(4, 4)
        FLA_WIDTH(16, 2)
        FLA_WIDTH(16, 4)
    } else {
        FLA_WIDTH(4, 1)
        FLA_WIDTH(4, 2)
        FLA_WIDTH(16, 1)
        FLA_WIDTH(16, 2)
    }
    return false;
}
#undef FLA_WIDTH

template <typename T, bool Q8>
hipError_t fwd(const NormArgs& args, int cus, hipStream_t stream) {
    NormArgs a = args;
    const int64_t per_row = (int64_t)a.D * (sizeof(T) * (1 + (a.residual != nullptr) + (a.sum != nullptr)) + (Q8 ? 1 : sizeof(T)));
    a.nt = a.rows > kLastLevelCache / per_row;
    hipError_t e = hipErrorInvalidValue;
    const bool kept = fwd_width(((int64_t)a.D + kVec<T> - 1) / kVec<T>, [&](auto w, auto k) {
        constexpr int W = decltype(w)::value, K = decltype(k)::value;
        const int64_t need = (a.rows + Row<W>::kRows - 1) / Row<W>::kRows;
        const int64_t most = (int64_t)cus * (W == 16 ? 4 : 16);
        e = launch<NormArgs>(&norm_fwd<T, W, K, Q8>, need < most ? need : most, Row<W>::kThreads, a, stream);
    });
    if (kept) return e;
    const int64_t most = (int64_t)cus * 2;
    return launch<NormArgs>(&norm_fwd_wide<T, Q8>, a.rows < most ? a.rows : most, 1024, a, stream);
}

template <typename T>
hipError_t bwd(const NormBwdArgs& a, hipStream_t stream) {
    hipError_t e = hipSuccess;
    NormBwdArgs args = a;
    args.blocks = 0;
    if (a.rows > 0) {
        const int most = norm_bwd_blocks(a.rows, a.D);
        const bool kept = bwd_width<T>(((int64_t)a.D + kVec<T> - 1) / kVec<T>, [&](auto w, auto k) {
            constexpr int W = decltype(w)::value, K = decltype(k)::value;
            const int64_t need = (a.rows + Row<W>::kRows - 1) / Row<W>::kRows;
            args.blocks = (int)(need < most ? need : most);
            e = launch<NormBwdArgs>(a.lines ? &norm_bwd<T, W, K, true> : &norm_bwd<T, W, K, false>, args.blocks,
                                    Row<W>::kThreads, args, stream);
        });
        if (!kept) {
            args.blocks = most;
            e = launch<NormBwdArgs>(&norm_bwd_wide<T>, args.blocks, 1024, args, stream);
        }
        if (e != hipSuccess) return e;
    }
    return launch<NormBwdArgs>(&norm_bwd_weight, ((int64_t)a.D + kSumColumns - 1) / kSumColumns, 1024, args, stream);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, int cus, hipStream_t stream) {
    return bf16 ? fwd<bf16_t, false>(a, cus, stream) : fwd<float, false>(a, cus, stream);
}
hipError_t launch_norm_q8(const NormArgs& a, bool bf16, int cus, hipStream_t stream) {
    return bf16 ? fwd<bf16_t, true>(a, cus, stream) : fwd<float, true>(a, cus, stream);
}
hipError_t launch_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream);
}

}  // namespace fla
