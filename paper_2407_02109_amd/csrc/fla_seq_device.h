// Device helpers shared by the kernels of fla_seq.h: 16-byte pieces of rows as fp32 values, and sums
// and maxima over the lanes of a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace fla {

typedef __bf16 bf16_t;
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
// 16, 8 and 4 bytes at any element's address (global memory takes them at any alignment)
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// 16 or 8 bytes, of values that are not used again soon (NT: the non-temporal cache policy) or as usual.  (The
// types are named here: as a template's argument they would lose their alignment.)
template <bool NT>
__device__ __forceinline__ u32x4_any load16(const void* p) {
    const u32x4_any* q = static_cast<const u32x4_any*>(p);
    if constexpr (NT)
        return __builtin_nontemporal_load(q);
    else
        return *q;
}
template <bool NT>
__device__ __forceinline__ void store16(void* p, const u32x4_any& v) {
    u32x4_any* q = static_cast<u32x4_any*>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(v, q);
    else
        *q = v;
}
template <bool NT>
__device__ __forceinline__ void store8(void* p, const u32x2_any& v) {
    u32x2_any* q = static_cast<u32x2_any*>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(v, q);
    else
        *q = v;
}

// values of a type in 16 bytes
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ float bits_f32(unsigned u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ unsigned f32_bits(float x) { return __builtin_bit_cast(unsigned, x); }

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
    const bf16x2_t p = {(bf16_t)a, (bf16_t)b};   // rounded to nearest even
    return __builtin_bit_cast(unsigned, p);
}

// the first n values of a 16-byte piece at p (the others 0); n >= kVec: the whole piece
template <bool NT = false>
__device__ __forceinline__ void load_piece(const float* p, int n, float (&v)[4]) {
    if (n >= 4) {
        const u32x4_any w = load16<NT>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = bits_f32(w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < n ? p[j] : 0.f;
    }
}
__device__ __forceinline__ void unpack_piece(const u32x4_any& w, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = bits_f32(w[j] << 16);
        v[2 * j + 1] = bits_f32(w[j] & 0xffff0000u);
    }
}
template <bool NT = false>
__device__ __forceinline__ void load_piece(const bf16_t* p, int n, float (&v)[8]) {
    if (n >= 8) {
        unpack_piece(load16<NT>(p), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? (float)p[j] : 0.f;
    }
}
// a piece as it lies in memory: its first n values, the others 0
template <bool NT = false>
__device__ __forceinline__ u32x4_any load_raw(const float* p, int n) {
    u32x4_any w = {0u, 0u, 0u, 0u};
    if (n >= 4) {
        w = load16<NT>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) w[j] = f32_bits(p[j]);
    }
    return w;
}
template <bool NT = false>
__device__ __forceinline__ u32x4_any load_raw(const bf16_t* p, int n) {
    u32x4_any w = {0u, 0u, 0u, 0u};
    if (n >= 8) {
        w = load16<NT>(p);
    } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) w[j / 2] |= (unsigned)h[j] << 16 * (j % 2);
    }
    return w;
}
__device__ __forceinline__ void unpack(const u32x4_any& w, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = bits_f32(w[j]);
}
__device__ __forceinline__ void unpack(const u32x4_any& w, float (&v)[8]) { unpack_piece(w, v); }
// eight fp32 values beside a piece of eight bf16
__device__ __forceinline__ void load_piece(const float* p, int n, float (&v)[8]) {
    float a[4], b[4];
    load_piece(p, n, a);
    load_piece(p + 4, n - 4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
    }
}
template <bool NT = false>
__device__ __forceinline__ void store_piece(float* p, int n, const float (&v)[4]) {
    if (n >= 4) {
        u32x4_any w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = f32_bits(v[j]);
        store16<NT>(p, w);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < n) p[j] = v[j];
    }
}
template <bool NT = false>
__device__ __forceinline__ void store_piece(bf16_t* p, int n, const float (&v)[8]) {
    if (n >= 8) {
        u32x4_any w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
        store16<NT>(p, w);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (bf16_t)v[j];
    }
}

// two values
template <typename T>
__device__ __forceinline__ void load_piece(const T* p, int n, float (&v)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) v[j] = j < n ? (float)p[j] : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, int n, const float (&v)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
        if (j < n) p[j] = (T)v[j];
}

// a piece, non-temporally if nt (which is the same for the whole launch)
template <typename T, int N>
__device__ __forceinline__ void store_piece(bool nt, T* p, int n, const float (&v)[N]) {
    if (nt)
        store_piece<true>(p, n, v);
    else
        store_piece<false>(p, n, v);
}
// Whether outputs are stored non-temporally: where the call's bytes pass the last-level cache, so that what it writes would
// not be found there anyway.  us a call, as usual / non-temporally: norm of 65536 rows of 768 83, 76; 8-bit norm of 121800
// of 1024 162, 148; rotary of 65536 x 24 heads x 64 83, 79; below it, rotary of 16382 x 20 x 128 (168 MB) 37.4, 39.2.
constexpr int64_t kLastLevelCache = int64_t(256) << 20;

// ---- over the lanes of a wave.  Lane permutations inside 16 lanes are operands of the vector ALU:
//      with the lane's neighbour, its pair's, its quad's and its eight's mirror image.
template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned x) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kSwapPair = 0xB1, kSwapTwo = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;

struct SumOp {
    __device__ __forceinline__ static unsigned of(unsigned a, unsigned b) { return f32_bits(bits_f32(a) + bits_f32(b)); }
};
// the larger of two bit patterns of |x|: their order is that of the values, and a NaN is above all
struct MaxOp {
    __device__ __forceinline__ static unsigned of(unsigned a, unsigned b) { return a > b ? a : b; }
};

// over groups of `lanes` neighbouring lanes (4 .. 64, a power of two): every lane gets the result
template <typename OP>
__device__ __forceinline__ unsigned over_lanes(unsigned x, int lanes) {
    x = OP::of(x, dpp<kSwapPair>(x));
    x = OP::of(x, dpp<kSwapTwo>(x));
    if (lanes >= 8) x = OP::of(x, dpp<kMirror8>(x));
    if (lanes >= 16) x = OP::of(x, dpp<kMirror16>(x));
    if (lanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = OP::of(r[0], r[1]);
    }
    if (lanes >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = OP::of(r[0], r[1]);
    }
    return x;
}
__device__ __forceinline__ float wave_sum(float x) { return bits_f32(over_lanes<SumOp>(f32_bits(x), 64)); }

// ---- sums of columns: column c of [rows, stride] over the rows, for a workgroup of 1024 and kSumColumns columns from
//      c0 on (those below `columns`); the result in the threads below kSumColumns.  Each thread adds every 64th row of
//      a column, eight loads at a time; then the 64 sums in order.  Few columns a workgroup: a few hundred rows of some
//      hundred columns are all there is, and only as many workgroups as that gives read them.
constexpr int kSumColumns = 16;
__device__ __forceinline__ float column_sum(const float* p, int64_t rows, int64_t stride, int64_t c0, int64_t columns) {
    __shared__ float part[64][kSumColumns], quarter[16][kSumColumns];
    const int col = (int)threadIdx.x % kSumColumns, slot = (int)threadIdx.x / kSumColumns;
    float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c0 + col < columns) {
        const float* q = p + c0 + col;
        int64_t r = slot;
        for (; r + 7 * 64 < rows; r += 8 * 64)
#pragma unroll
            for (int u = 0; u < 8; ++u) t[u] += q[(r + u * 64) * stride];
#pragma unroll
        for (int u = 0; u < 7; ++u)
            if (r + u * 64 < rows) t[u] += q[(r + u * 64) * stride];
    }
    part[slot][col] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    __syncthreads();
    if (slot < 16)
        quarter[slot][col] = (part[4 * slot][col] + part[4 * slot + 1][col]) + (part[4 * slot + 2][col] + part[4 * slot + 3][col]);
    __syncthreads();
    float s = 0.f;
    if (slot == 0)
#pragma unroll
        for (int w = 0; w < 16; ++w) s += quarter[w][col];
    return s;
}

// ---- host side
template <typename A>
inline hipError_t launch(void (*kernel)(A), int64_t groups, int threads, const A& args, hipStream_t stream) {
    A copy = args;
    void* params[] = {&copy};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)groups), dim3((unsigned)threads), params,
                           0, stream);
}

}  // namespace fla
