// Rotary positions of q and k, gfx950: the first `rot` channels of each head turn by the token's
// position(s), the others are copied.
//
// Bound by memory: every value is read and written once.  A workgroup takes some tokens with all their
// heads: it first puts the (cos, sin) of each token and pair into LDS, one for all heads, then turns the
// heads in pieces of 16 bytes (pairs that lie rot / 2 apart: a piece of either half).
// The angle is formed in revolutions in fp64 and reduced to half a turn before it is rounded to fp32: at
// position 10^6 an fp32 angle would be off by 0.03 radians.
//
// Measured (MI355X; a copy reaches 5.2 TB/s): 65536 tokens x 24 heads x 64, bf16, pairs side by side, two axes 79 us, 5.1
// TB/s; 16382 x 20 heads x 128, half of each turned, halves apart 37 us, 4.5 TB/s; 32 tokens x 40 heads x 128 4.1 us.
// Addresses are taken from a table of the tokens' places: computed for each piece they were 60 vector operations of
// 64-bit products (77 us where the table took 74, results over each other).  One head in flight instead of two 80 us.
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

#include <type_traits>

namespace fla {
namespace {

constexpr int kRows = 2;     // heads that a thread has in flight
constexpr int kTokens = 64;  // of one turn, at most

// WHOLE: every piece of a head is a whole one.  NT: outputs are stored non-temporally.
template <typename T, bool PAIRS, bool WHOLE, bool NT>
__global__ __launch_bounds__(256) void rotary(RotaryArgs a) {
    constexpr int N = kVec<T>;
    __shared__ float2 table[kRotaryTable + N];   // a last piece reads past its pairs, and drops that
    __shared__ T* place[2][2][kTokens];          // of each token's first head: q and k, in and out
    const int half = a.rot >> 1;
    const int slots = 256 / a.pieces;            // heads that the workgroup turns at a time
    const int slot = (int)threadIdx.x / a.pieces, piece = (int)threadIdx.x - slot * a.pieces;
    const bool turns_here = piece < a.turn_pieces;
    const int c = turns_here ? piece * N : a.rot + (piece - a.turn_pieces) * N;
    const int n = WHOLE ? N : !turns_here ? a.d - c : PAIRS ? a.rot - c : half - c;
    // channels that are copied have nothing to do in place
    const bool idle_q = !turns_here && a.q.in == a.q.out, idle_k = !turns_here && a.k.in == a.k.out;
    const int64_t turns = (a.n_tokens + a.tokens - 1) / a.tokens;
    for (int64_t g = blockIdx.x; g < turns; g += gridDim.x) {
        const unsigned tok0 = (unsigned)(g * a.tokens);
        const int nt = (int)(a.n_tokens - tok0 < a.tokens ? a.n_tokens - tok0 : a.tokens);
        for (int e = (int)threadIdx.x; e < nt * half; e += 256) {
            const int t = (int)a.div_half.div((unsigned)e), j = e - t * half;
            const unsigned b = a.div_L.div(tok0 + t), l = tok0 + t - b * (unsigned)a.L;
            const int64_t at = b * a.pos_batch + l * a.pos_token + (a.axes == 2 && 2 * j >= half ? 1 : 0);
            const double pos = a.pos64 ? (double)static_cast<const int64_t*>(a.positions)[at]
                                       : (double)static_cast<const int*>(a.positions)[at];
            double rev = pos * a.freqs[j] * 0.15915494309189533577;   // 1 / (2 pi)
            rev -= __builtin_rint(rev);
            float s, co;
            sincospif(2.f * (float)rev, &s, &co);
            table[e] = make_float2(co * a.mscale, s * a.mscale * a.sign);
        }
        if ((int)threadIdx.x < nt) {
            const unsigned b = a.div_L.div(tok0 + threadIdx.x), l = tok0 + threadIdx.x - b * (unsigned)a.L;
            auto first = [&](const void* p, int64_t batch, int64_t token) {
                return const_cast<T*>(static_cast<const T*>(p)) + (b * batch + l * token);
            };
            place[0][0][threadIdx.x] = first(a.q.in, a.q.in_batch, a.q.in_token);
            place[0][1][threadIdx.x] = first(a.q.out, a.q.out_batch, a.q.out_token);
            place[1][0][threadIdx.x] = first(a.k.in, a.k.in_batch, a.k.in_token);
            place[1][1][threadIdx.x] = first(a.k.out, a.k.out_batch, a.k.out_token);
        }
        __syncthreads();
        const int rows = slot < slots ? nt * a.heads : 0;
        // kRows heads at a time: their loads before the first store, which may be in place of them
        for (int row0 = slot; row0 < rows; row0 += kRows * slots) {
            u32x4_any v[kRows], w[kRows];
            T* out[kRows];
            int pair[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                out[u] = nullptr;
                const int row = row0 + u * slots;
                if (row >= rows) continue;
                const int t = (int)a.div_heads.div((unsigned)row);
                const int head = row - t * a.heads;
                const bool is_q = head < a.hq;
                if (is_q ? idle_q : idle_k) continue;
                const unsigned h = (unsigned)(is_q ? head : head - a.hq);
                const T* in = place[is_q ? 0 : 1][0][t] + (uint64_t)h * (is_q ? a.q.in_head : a.k.in_head) + c;
                out[u] = place[is_q ? 0 : 1][1][t] + (uint64_t)h * (is_q ? a.q.out_head : a.k.out_head) + c;
                pair[u] = t * half + (PAIRS ? c >> 1 : c);
                v[u] = load_raw<true>(in, n);
                if (!PAIRS && turns_here) w[u] = load_raw<true>(in + half, n);
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if (!out[u]) continue;
                float x[N], y[N];
                unpack(v[u], x);
                if (!turns_here) {
                    store_piece<NT>(out[u], n, x);
                } else if constexpr (PAIRS) {
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) {
                        const float2 cs = table[pair[u] + j];
                        const float a0 = x[2 * j], b0 = x[2 * j + 1];
                        x[2 * j] = a0 * cs.x - b0 * cs.y;
                        x[2 * j + 1] = b0 * cs.x + a0 * cs.y;
                    }
                    store_piece<NT>(out[u], n, x);
                } else {
                    unpack(w[u], y);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float2 cs = table[pair[u] + j];
                        const float t0 = x[j] * cs.x - y[j] * cs.y;
                        y[j] = y[j] * cs.x + x[j] * cs.y;
                        x[j] = t0;
                    }
                    store_piece<NT>(out[u], n, x);
                    store_piece<NT>(out[u] + half, n, y);
                }
            }
        }
        __syncthreads();   // the next turn writes the table
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& args, bool bf16, bool interleaved, int cus, hipStream_t stream) {
    RotaryArgs a = args;
    const int vec = bf16 ? 8 : 4, half = a.rot / 2;
    a.turn_pieces = interleaved ? (a.rot + vec - 1) / vec : (half + vec - 1) / vec;
    a.pieces = a.turn_pieces + (a.d - a.rot + vec - 1) / vec;
    // a table entry for each thread, but eight workgroups for each compute unit before several tokens in one
    const int64_t spread = (a.n_tokens + 8 * cus - 1) / (8 * cus);
    const int fit = half >= 256 ? 1 : half > 256 / kTokens ? 256 / half : kTokens;
    a.tokens = (int)(spread < fit ? spread : fit);
    a.div_L = FastDiv::make((unsigned)a.L);
    a.div_half = FastDiv::make((unsigned)half);
    a.div_heads = FastDiv::make((unsigned)a.heads);
    const int64_t turns = (a.n_tokens + a.tokens - 1) / a.tokens, most = (int64_t)cus * 64;
    const bool whole = (interleaved ? a.rot : half) % vec == 0 && (a.d - a.rot) % vec == 0;
    const bool large = 2 * a.n_tokens * a.heads * a.d * (bf16 ? 2 : 4) > kLastLevelCache;
    auto pick = [&](auto t, auto pairs) {
        using T = decltype(t);
        constexpr bool P = decltype(pairs)::value;
        return !whole ? &rotary<T, P, false, false> : large ? &rotary<T, P, true, true> : &rotary<T, P, true, false>;
    };
    auto* kernel = bf16 ? (interleaved ? pick(bf16_t{}, std::true_type{}) : pick(bf16_t{}, std::false_type{}))
                        : (interleaved ? pick(float{}, std::true_type{}) : pick(float{}, std::false_type{}));
    return launch<RotaryArgs>(kernel, turns < most ? turns : most, 256, a, stream);
}

}  // namespace fla
