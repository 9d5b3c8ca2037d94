// Arguments and launchers shared by the C ABI of fla_seq.h and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "fla_swin_internal.h"   // FastDiv

namespace fla {

// ---- residual + root-mean-square norm (fla_rms_norm.hip)
struct NormArgs {
    const void* x;
    const void* residual;    // NULL: none
    const void* weight;
    void* y;                 // T, or bytes of the 8-bit output
    void* sum;               // NULL: not kept
    float* rstd;             // NULL: not kept
    float* scales;           // 8-bit output
    int64_t x_stride, residual_stride;
    int64_t rows;
    int D;
    int group;               // channels per scale, 0: one per row
    int weight_f32;
    int nt;                  // outputs are stored non-temporally (set by the launcher)
    float eps, inv_D;
};
hipError_t launch_norm_fwd(const NormArgs& a, bool bf16, int cus, hipStream_t stream);
hipError_t launch_norm_q8(const NormArgs& a, bool bf16, int cus, hipStream_t stream);

struct NormBwdArgs {
    const void* dy;
    const void* s;
    const void* weight;
    const float* rstd;
    const void* dsum;        // NULL: none
    void* dx;
    float* dweight;
    float* ws;               // [blocks, D]: each block's share of dweight
    int64_t dy_stride, s_stride, dsum_stride;
    int64_t rows;
    int D;
    int weight_f32;
    float inv_D;
    int blocks;
    int lines;               // rows are whole cache lines
};
// Workgroups of the backward at most, each with a share of dweight in the workspace: about as many as the chip holds
// of them.  us a call, bf16, with 768 / 1024 / 2048 of them (131072 of 256: 1024 / 1536 / 2048): 65536 rows of 768 73,
// 86, 80; 16384 of 4096 100, 105, 104; 131072 of 256 59, 73, 63; of 16 waves, with 256 / 512 / 1024: 4096 of 16384 117,
// 128, 156.
inline int norm_bwd_blocks(int64_t rows, int D) {
    const int most = D <= 512 ? 1024 : D <= 4096 ? 768 : 256;
    return rows < most ? (int)rows : most;
}
hipError_t launch_norm_bwd(const NormBwdArgs& a, bool bf16, hipStream_t stream);

// ---- rotary positions (fla_rotary.hip)
struct RotaryTensor {
    const void* in;
    void* out;               // == in: in place
    int64_t in_batch, in_token, out_batch, out_token;
    unsigned in_head, out_head;
};
struct RotaryArgs {
    RotaryTensor q, k;
    const void* positions;
    const double* freqs;
    int64_t pos_batch, pos_token;
    int pos64, axes;
    int B, L, hq, heads;     // heads: of q and k
    int d, rot;
    int turn_pieces;         // 16-byte pieces (of both halves, where pairs lie apart) that turn, per head
    int pieces;              // with those that are copied
    int tokens;              // tokens of a workgroup's turn
    int64_t n_tokens;        // B * L
    float mscale, sign;      // sign: -1 turns back
    FastDiv div_L, div_half, div_heads;
};
constexpr int kRotaryTable = 512;   // (cos, sin) of one turn: tokens * rot / 2 at most
hipError_t launch_rotary(const RotaryArgs& a, bool bf16, bool interleaved, int cus, hipStream_t stream);

// ---- gated linear recurrence (fla_gated_scan.hip)
constexpr int kScanChunk = 128;     // tokens from one kept state to the next
constexpr int kScanChannels = 64;   // of a column
struct ScanInput {
    const void* p;
    int64_t batch, token;
};
struct ScanArgs {
    ScanInput x, r, i;
    const float* lam;
    const float* h0;         // NULL: 0
    const int* lengths;      // NULL: L
    void* h;
    float* h_last;           // NULL: not kept
    float* states;           // [B, columns, chunks, 64]: the state that enters each chunk (NULL: not kept)
    void* ws;                // the chain's words (several chunks)
    int B, L, D;
    int columns, chunks;
    int links;               // of the chain: tiles of a column (set by the launcher)
    int cus;
    int lines;               // the columns' rows of h are whole cache lines
    float c;
};
struct ScanBwdArgs {
    ScanInput x, r, i, dh;   // dh.p NULL: 0
    const float* lam;
    const float* states;
    const int* lengths;
    const float* d_last;     // NULL: 0
    void* dx;
    void* dr;
    void* di;
    float* dlam;
    float* dh0;              // NULL: not wanted
    void* ws;                // the chain's words (several chunks)
    float* shares;           // [B, chunks, columns, 64]: shares of dlam
    int B, L, D;
    int columns, chunks;
    int links;               // == chunks
    int lines;               // the columns' rows of dx, dr and di are whole cache lines
    float c;
};
// The chain's words: 12 bytes for each (column, chunk, channel), a mark for each (column, chunk), and a ticket for each
// column in cache lines of its own.
constexpr int kScanTicketWords = 32;
inline int64_t scan_chain_bytes(int64_t columns, int64_t chunks) {
    return chunks > 1 ? columns * (chunks * (kScanChannels * 12 + 4) + kScanTicketWords * 4) : 0;
}
hipError_t launch_scan_fwd(const ScanArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_scan_bwd(const ScanBwdArgs& a, bool bf16, hipStream_t stream);

}  // namespace fla
