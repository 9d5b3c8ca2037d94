// Host definitions of the further gfx950 builtins and HIP pieces that the kernels of fla_seq.h use, beside those
// of host_emu/amdgcn_host.h (test infrastructure; force-included into every file of the host build).
#pragma once
#include "amdgcn_host.h"
#include "hip/hip_runtime.h"

extern thread_local emu_index gridDim;

// (the host's own want aligned addresses)
#define __builtin_nontemporal_load(p) (*(p))
#define __builtin_nontemporal_store(v, p) (*(p) = (v))

inline float __builtin_amdgcn_rcpf(float x) { return 1.f / x; }
inline float __builtin_amdgcn_rsqf(float x) { return 1.f / std::sqrt(x); }
inline float __builtin_amdgcn_sqrtf(float x) { return std::sqrt(x); }
inline void __builtin_amdgcn_s_sleep(int) {}
inline void __builtin_amdgcn_wave_barrier() { emu_wave_barrier(); }
inline void __builtin_amdgcn_fence(int, const char*) {}
inline void sincospif(float x, float* s, float* c) {
    const double t = 3.14159265358979323846 * (double)x;
    *s = (float)std::sin(t);
    *c = (float)std::cos(t);
}

// the lane permutations in use: pairs, pairs of pairs, mirrors of 8 and 16 lanes
inline int __builtin_amdgcn_update_dpp(int, int x, int ctrl, int, int, bool) {
    int* s = reinterpret_cast<int*>(emu_wave_slots());
    const unsigned l = emu_lane_id();
    s[l] = x;
    emu_wave_barrier();
    switch (ctrl) {
        case 0xB1: return s[l ^ 1];
        case 0x4E: return s[l ^ 2];
        case 0x141: return s[l ^ 7];
        case 0x140: return s[l ^ 15];
    }
    std::abort();
}
// swaps the odd rows of 16 lanes of the first operand with the even rows of the second
inline emu_u32x2 __builtin_amdgcn_permlane16_swap(unsigned x, unsigned y, bool, bool) {
    unsigned* s = reinterpret_cast<unsigned*>(emu_wave_slots());
    const unsigned l = emu_lane_id();
    s[2 * l] = x;
    s[2 * l + 1] = y;
    emu_wave_barrier();
    emu_u32x2 r;
    if (l & 16) {
        r[0] = s[2 * (l - 16) + 1];
        r[1] = y;
    } else {
        r[0] = x;
        r[1] = s[2 * (l + 16)];
    }
    return r;
}

// e4m3 (OCP), round to nearest even, no infinities
inline unsigned emu_e4m3(float x) {
    if (std::isnan(x)) return 0x7f;
    const unsigned sign = std::signbit(x) ? 0x80 : 0;
    const double v = std::fabs((double)x);
    if (v >= 464) return sign | 0x7f;   // (never asked for)
    const double q = v < 0.015625 ? 0x1p-9 : std::exp2(std::floor(std::log2(v)) - 3);
    const double r = std::nearbyint(v / q) * q;
    if (r < 0.015625) return sign | (unsigned)(r * 512);
    const int e = (int)std::floor(std::log2(r));
    return sign | (unsigned)((e + 7) << 3) | (unsigned)((r / std::exp2(e) - 1) * 8);
}
inline int __builtin_amdgcn_cvt_pk_fp8_f32(float a, float b, int old, bool high) {
    const unsigned w = emu_e4m3(a) | emu_e4m3(b) << 8;
    return high ? (int)(((unsigned)old & 0xffffu) | w << 16) : (int)(((unsigned)old & 0xffff0000u) | w);
}
