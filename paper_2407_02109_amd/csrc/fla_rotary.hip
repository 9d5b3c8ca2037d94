// Rotary positions of q and k, gfx950: the first `rot` channels of each head turn by the token's
// position(s), the others are copied.
//
// Bound by memory: every value is read and written once.  A workgroup takes some tokens with all their
// heads: it first puts the (cos, sin) of each token and pair into LDS, one for all heads, then turns the
// heads in pieces of 16 bytes (pairs that lie rot / 2 apart: a piece of either half).
// The angle is formed in revolutions in fp64 and reduced to half a turn before it is rounded to fp32: at
// position 10^6 an fp32 angle would be off by 0.03 radians.
#include "fla_seq_device.h"
#include "fla_seq_internal.h"

namespace fla {
namespace {

template <typename T, bool PAIRS>
__global__ __launch_bounds__(256) void rotary(RotaryArgs a) {
    constexpr int N = kVec<T>;
    __shared__ float2 table[kRotaryTable + N];   // a last piece reads past its pairs, and drops that
    const int half = a.rot >> 1;
    const int slots = 256 / a.pieces;            // heads that the workgroup turns at a time
    const int slot = (int)threadIdx.x / a.pieces, piece = (int)threadIdx.x - slot * a.pieces;
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
            float s, c;
            sincospif(2.f * (float)rev, &s, &c);
            table[e] = make_float2(c * a.mscale, s * a.mscale * a.sign);
        }
        __syncthreads();
        if (slot < slots)
            for (int row = slot; row < nt * a.heads; row += slots) {
                const int t = (int)a.div_heads.div((unsigned)row);
                int h = row - t * a.heads;
                const unsigned b = a.div_L.div(tok0 + t), l = tok0 + t - b * (unsigned)a.L;
                const bool is_q = h < a.hq;
                if (!is_q) h -= a.hq;
                const RotaryTensor& m = is_q ? a.q : a.k;
                const T* in = static_cast<const T*>(m.in) + (b * m.in_batch + l * m.in_token + h * m.in_head);
                T* out = static_cast<T*>(m.out) + (b * m.out_batch + l * m.out_token + h * m.out_head);
                if (piece >= a.turn_pieces) {
                    const int c = a.rot + (piece - a.turn_pieces) * N;
                    float v[N];
                    if (m.in != m.out) {
                        load_piece(in + c, a.d - c, v);
                        store_piece(out + c, a.d - c, v);
                    }
                } else if constexpr (PAIRS) {
                    const int c = piece * N, n = a.rot - c;
                    const float2* cs = table + t * half + (c >> 1);
                    float v[N];
                    load_piece(in + c, n, v);
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) {
                        const float2 w = cs[j];
                        const float x = v[2 * j], y = v[2 * j + 1];
                        v[2 * j] = x * w.x - y * w.y;
                        v[2 * j + 1] = y * w.x + x * w.y;
                    }
                    store_piece(out + c, n, v);
                } else {
                    const int c = piece * N, n = half - c;
                    const float2* cs = table + t * half + c;
                    float x[N], y[N];
                    load_piece(in + c, n, x);
                    load_piece(in + half + c, n, y);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float2 w = cs[j];
                        const float u = x[j] * w.x - y[j] * w.y;
                        y[j] = y[j] * w.x + x[j] * w.y;
                        x[j] = u;
                    }
                    store_piece(out + c, n, x);
                    store_piece(out + half + c, n, y);
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
    // a table entry for each thread, but four workgroups for each compute unit before several tokens in one
    const int64_t spread = (a.n_tokens + 4 * cus - 1) / (4 * cus);
    const int fit = half < 256 ? 256 / half : 1;
    a.tokens = (int)(spread < fit ? spread : fit);
    a.div_L = FastDiv::make((unsigned)a.L);
    a.div_half = FastDiv::make((unsigned)half);
    a.div_heads = FastDiv::make((unsigned)a.heads);
    const int64_t turns = (a.n_tokens + a.tokens - 1) / a.tokens, most = (int64_t)cus * 64;
    auto* kernel = bf16 ? (interleaved ? &rotary<bf16_t, true> : &rotary<bf16_t, false>)
                        : (interleaved ? &rotary<float, true> : &rotary<float, false>);
    return launch<RotaryArgs>(kernel, turns < most ? turns : most, 256, a, stream);
}

}  // namespace fla
