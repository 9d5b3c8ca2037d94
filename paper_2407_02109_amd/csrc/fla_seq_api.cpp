// C ABI of libfla_seq.so (include/fla_seq.h): argument checks, launch geometry, frequencies.
#include "fla_seq.h"

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "fla_seq_internal.h"

namespace {

constexpr int64_t kMaxElems = int64_t(1) << 40;
constexpr int64_t kMaxGroups = (int64_t(1) << 22) - 1;   // grid.x * 1024 threads < 2^32
constexpr int64_t kMaxLen = (int64_t(1) << 31) - 1024;   // tokens of a sequence
constexpr int kMaxWidth = 1 << 24;                       // channels of a norm's row or of a scan

// Per-device probe result: 0 = not probed yet, -1 = not gfx950, > 0 = gfx950 with that many compute units.
std::atomic<int> g_cus[64];

int check_arch(int* cus) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0) {
        (void)hipGetLastError();
        return FLA_ERR_ARCH;
    }
    int st = dev < 64 ? g_cus[dev].load(std::memory_order_acquire) : 0;
    if (st == 0) {
        hipDeviceProp_t prop;
        if (hipGetDeviceProperties(&prop, dev) != hipSuccess) {
            (void)hipGetLastError();
            return FLA_ERR_ARCH;
        }
        const char* name = prop.gcnArchName;
        st = std::strncmp(name, "gfx950", 6) == 0 && (name[6] == 0 || name[6] == ':') && prop.multiProcessorCount > 0
                 ? prop.multiProcessorCount
                 : -1;
        if (dev < 64) g_cus[dev].store(st, std::memory_order_release);
    }
    if (st < 0) return FLA_ERR_ARCH;
    *cus = st;
    return FLA_OK;
}

int launched(hipError_t e) {
    if (e == hipSuccess) return FLA_OK;
    (void)hipGetLastError();
    return FLA_ERR_LAUNCH;
}

bool type_ok(int dtype) { return dtype == FLA_F32 || dtype == FLA_BF16; }
int size_of(int dtype) { return dtype == FLA_BF16 ? 2 : 4; }
bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

struct Range {
    const void* p;
    int64_t bytes;   // 0: absent
};
bool overlap(const Range& a, const Range& b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    return a0 < b0 + (uint64_t)b.bytes && b0 < a0 + (uint64_t)a.bytes;
}
// (n - 1) * stride in 64 bits, or a value past every limit
int64_t reach(int64_t n, int64_t stride) {
    if (n <= 1 || stride == 0) return 0;
    return stride >= kMaxElems || n - 1 >= kMaxElems / stride + 1 ? kMaxElems : (n - 1) * stride;
}

// A tensor of tokens: `wide` elements from the first to the last of a token.
struct Tokens {
    const void* p;
    int64_t batch, token;
    int64_t B, L, wide;
    int elem;
    int64_t elements() const {
        const int64_t b = reach(B, batch), t = reach(L, token);
        return b >= kMaxElems || t >= kMaxElems ? kMaxElems : b + t + wide;
    }
    Range range() const { return {p, elements() * elem}; }
};

// Whether two tensors share an element.  Views that lie side by side in every token of one buffer (equal
// strides) do not, although their ranges meet.
bool share(const Tokens& a, const Tokens& b) {
    if (!overlap(a.range(), b.range())) return false;
    if (a.token != b.token || a.elem != b.elem || a.token == 0) return true;
    if ((a.B > 1 && a.batch % a.token != 0) || (b.B > 1 && b.batch % b.token != 0)) return true;
    const int64_t period = a.token * a.elem;
    int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % period;
    if (d < 0) d += period;
    return d < a.wide * a.elem || d + b.wide * b.elem > period;
}

// whether rows of `stride` elements from p on begin at cache lines
bool lines(const void* p, int64_t stride, int elem) {
    return stride * elem % 128 == 0 && reinterpret_cast<uintptr_t>(p) % 128 == 0;
}

// ---- norm

int norm_checks(int64_t rows, int D, const int64_t* strides, int n_strides, float eps, int dtype, int weight_dtype) {
    if (rows < 0 || D < 0) return FLA_ERR_SHAPE;
    for (int i = 0; i < n_strides; ++i)
        if (strides[i] < 0) return FLA_ERR_SHAPE;
    if (!type_ok(dtype) || (weight_dtype != dtype && weight_dtype != FLA_F32)) return FLA_ERR_UNSUPPORTED;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return FLA_ERR_UNSUPPORTED;
    return FLA_OK;
}

bool norm_too_large(int64_t rows, int D, const int64_t* strides, int n_strides) {
    if (D > kMaxWidth || rows > kMaxElems / D) return true;
    for (int i = 0; i < n_strides; ++i)
        if (reach(rows, strides[i]) + D >= kMaxElems) return true;
    return false;
}

Range rows_range(const void* p, int64_t rows, int64_t stride, int D, int elem) {
    return {p, p ? (reach(rows, stride) + D) * elem : 0};
}

int norm_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const void* weight, void* y,
             float* scales, void* sum, float* rstd, int64_t rows, int D, int group, float eps, int dtype,
             int weight_dtype, bool q8, hipStream_t stream) {
    const int64_t strides[] = {x_stride, residual ? residual_stride : 0};
    int st = norm_checks(rows, D, strides, 2, eps, dtype, weight_dtype);
    if (st != FLA_OK) return st;
    if (q8 && group != 0 && group != 32 && group != 64 && group != 128) return FLA_ERR_UNSUPPORTED;
    if (rows == 0 || D == 0) return FLA_OK;
    if (!x || !weight || !y || (q8 && !scales)) return FLA_ERR_NULL;
    const int e = size_of(dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, size_of(weight_dtype)) ||
        !aligned(y, q8 ? 1 : e) || !aligned(sum, e) || !aligned(rstd, 4) || !aligned(scales, 4))
        return FLA_ERR_ALIGN;
    if (norm_too_large(rows, D, strides, 2)) return FLA_ERR_TOO_LARGE;
    const int64_t groups = group ? ((int64_t)D + group - 1) / group : 1;
    const Range in[] = {rows_range(x, rows, x_stride, D, e), rows_range(residual, rows, residual_stride, D, e)};
    const Range w = {weight, (int64_t)D * size_of(weight_dtype)};
    const Range out[] = {{y, rows * D * (q8 ? 1 : e)}, {sum, rows * D * e}, {rstd, rows * 4}, {scales, rows * groups * 4}};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 2; ++i) {
            const bool in_place = (o == 1 || (o == 0 && !q8)) && out[o].p == in[i].p &&
                                  (strides[i] == D || rows == 1);
            if (!in_place && overlap(out[o], in[i])) return FLA_ERR_ALIAS;
        }
        if (overlap(out[o], w)) return FLA_ERR_ALIAS;
        for (int p = 0; p < o; ++p)
            if (overlap(out[o], out[p])) return FLA_ERR_ALIAS;
    }
    int cus = 0;
    st = check_arch(&cus);
    if (st != FLA_OK) return st;
    fla::NormArgs a{};
    a.x = x;
    a.residual = residual;
    a.weight = weight;
    a.y = y;
    a.sum = sum;
    a.rstd = rstd;
    a.scales = scales;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.rows = rows;
    a.D = D;
    a.group = group;
    a.weight_f32 = weight_dtype == FLA_F32;
    a.eps = eps;
    a.inv_D = (float)(1.0 / D);
    return launched(q8 ? fla::launch_norm_q8(a, dtype == FLA_BF16, cus, stream)
                       : fla::launch_norm_fwd(a, dtype == FLA_BF16, cus, stream));
}

// ---- scan

int scan_sizes(int B, int L, int D) { return B < 0 || L < 0 || D < 0 ? FLA_ERR_SHAPE : FLA_OK; }
int64_t scan_columns(int D) { return ((int64_t)D + fla::kScanChannels - 1) / fla::kScanChannels; }
int64_t scan_chunks(int L) { return ((int64_t)L + fla::kScanChunk - 1) / fla::kScanChunk; }
bool scan_too_large(int B, int L, int D) {
    if (L > kMaxLen || D > kMaxWidth) return true;
    const int64_t columns = scan_columns(D), chunks = scan_chunks(L);
    if ((int64_t)B * columns > kMaxGroups) return true;
    return chunks > 0 && (int64_t)B * columns > kMaxGroups / chunks;
}
int64_t scan_states_bytes(int B, int L, int D) {
    return (int64_t)B * scan_columns(D) * scan_chunks(L) * fla::kScanChannels * 4;
}
int64_t scan_ws_bytes(int B, int L, int D) { return fla::scan_chain_bytes(B * scan_columns(D), scan_chunks(L)); }
// the chain's words and the chunks' shares of dlam
int64_t scan_bwd_ws_bytes(int B, int L, int D) { return scan_ws_bytes(B, L, D) + scan_states_bytes(B, L, D); }

int scan_bytes(int B, int L, int D, size_t* bytes, int64_t (*of)(int, int, int)) {
    const int st = scan_sizes(B, L, D);
    if (st != FLA_OK) return st;
    if (!bytes) return FLA_ERR_NULL;
    if (scan_too_large(B, L, D)) return FLA_ERR_TOO_LARGE;
    *bytes = (size_t)of(B, L, D);
    return FLA_OK;
}

}  // namespace

extern "C" {

int fla_add_rms_norm_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                         const void* weight, void* y, void* sum, float* rstd, int64_t rows, int D, float eps,
                         int dtype, int weight_dtype, hipStream_t stream) {
    return norm_fwd(x, x_stride, residual, residual_stride, weight, y, nullptr, sum, rstd, rows, D, 0, eps, dtype,
                    weight_dtype, false, stream);
}

int fla_add_rms_norm_q8(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                        const void* weight, void* q, float* scales, void* sum, int64_t rows, int D, int group,
                        float eps, int dtype, int weight_dtype, hipStream_t stream) {
    return norm_fwd(x, x_stride, residual, residual_stride, weight, q, scales, sum, nullptr, rows, D, group, eps, dtype,
                    weight_dtype, true, stream);
}

int fla_add_rms_norm_bwd_workspace(int64_t rows, int D, size_t* bytes) {
    if (rows < 0 || D < 0) return FLA_ERR_SHAPE;
    if (!bytes) return FLA_ERR_NULL;
    if (D > kMaxWidth) return FLA_ERR_TOO_LARGE;
    *bytes = (size_t)fla::norm_bwd_blocks(rows, D) * D * 4;
    return FLA_OK;
}

int fla_add_rms_norm_bwd(const void* dy, int64_t dy_stride, const void* s, int64_t s_stride, const void* weight,
                         const float* rstd, const void* dsum, int64_t dsum_stride, void* dx, float* dweight,
                         void* workspace, size_t workspace_bytes, int64_t rows, int D, int dtype, int weight_dtype,
                         hipStream_t stream) {
    const int64_t strides[] = {dy_stride, s_stride, dsum ? dsum_stride : 0};
    int st = norm_checks(rows, D, strides, 3, 0.f, dtype, weight_dtype);
    if (st != FLA_OK) return st;
    if (D == 0) return FLA_OK;
    if (!dweight || (rows > 0 && (!dy || !s || !weight || !rstd || !dx))) return FLA_ERR_NULL;
    const int e = size_of(dtype);
    if (!aligned(dy, e) || !aligned(s, e) || !aligned(weight, size_of(weight_dtype)) || !aligned(rstd, 4) ||
        !aligned(dsum, e) || !aligned(dx, e) || !aligned(dweight, 4) || !aligned(workspace, 4))
        return FLA_ERR_ALIGN;
    if (norm_too_large(rows, D, strides, 3)) return FLA_ERR_TOO_LARGE;
    size_t need = 0;
    (void)fla_add_rms_norm_bwd_workspace(rows, D, &need);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FLA_ERR_WORKSPACE;
    if (rows > 0) {
        const Range in[] = {rows_range(dy, rows, dy_stride, D, e), rows_range(s, rows, s_stride, D, e),
                            rows_range(dsum, rows, dsum_stride, D, e), {weight, (int64_t)D * size_of(weight_dtype)},
                            {rstd, rows * 4}};
        const Range out[] = {{dx, rows * D * e}, {dweight, (int64_t)D * 4}, {workspace, (int64_t)need}};
        for (int o = 0; o < 3; ++o) {
            for (int i = 0; i < 5; ++i) {
                const bool in_place = o == 0 && (i == 0 || i == 2) && out[o].p == in[i].p &&
                                      (strides[i] == D || rows == 1);
                if (!in_place && overlap(out[o], in[i])) return FLA_ERR_ALIAS;
            }
            for (int p = 0; p < o; ++p)
                if (overlap(out[o], out[p])) return FLA_ERR_ALIAS;
        }
    }
    int cus = 0;
    st = check_arch(&cus);
    if (st != FLA_OK) return st;
    fla::NormBwdArgs a{};
    a.dy = dy;
    a.s = s;
    a.weight = weight;
    a.rstd = rstd;
    a.dsum = dsum;
    a.dx = dx;
    a.dweight = dweight;
    a.ws = static_cast<float*>(workspace);
    a.dy_stride = dy_stride;
    a.s_stride = s_stride;
    a.dsum_stride = dsum_stride;
    a.rows = rows;
    a.D = D;
    a.weight_f32 = weight_dtype == FLA_F32;
    a.inv_D = (float)(1.0 / D);
    a.lines = lines(dy, dy_stride, e) && lines(s, s_stride, e) && (!dsum || lines(dsum, dsum_stride, e));
    return launched(fla::launch_norm_bwd(a, dtype == FLA_BF16, stream));
}

int fla_rotary_freqs(int rot, double theta, int scaling, double factor, double trained_len, double* freqs,
                     double* mscale) {
    if (rot < 2 || rot % 2 != 0 || (scaling == FLA_ROPE_BASE && rot == 2)) return FLA_ERR_HEAD_DIM;
    if (scaling < FLA_ROPE_PLAIN || scaling > FLA_ROPE_PARTS || !std::isfinite(theta) || theta <= 0 ||
        !std::isfinite(factor) || factor < 1 || !std::isfinite(trained_len) || trained_len <= 0)
        return FLA_ERR_ROPE;
    if (!freqs) return FLA_ERR_NULL;
    if (scaling == FLA_ROPE_BASE) theta *= std::pow(factor, rot / (rot - 2.0));
    for (int j = 0; j < rot / 2; ++j) {
        const double f = std::pow(theta, -2.0 * j / rot);
        double keep = scaling == FLA_ROPE_LINEAR ? 0.0 : 1.0;
        if (scaling == FLA_ROPE_PARTS) {
            const double turns = trained_len * f / 6.283185307179586477;
            keep = turns <= 1 ? 0.0 : turns >= 32 ? 1.0 : (turns - 1) / 31;
        }
        freqs[j] = f / factor * (1 - keep) + f * keep;
    }
    if (mscale) *mscale = scaling == FLA_ROPE_PARTS ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return FLA_OK;
}

int fla_rotary(const void* q, int64_t q_batch, int64_t q_token, int64_t q_head, const void* k, int64_t k_batch,
               int64_t k_token, int64_t k_head, void* q_out, int64_t qo_batch, int64_t qo_token, int64_t qo_head,
               void* k_out, int64_t ko_batch, int64_t ko_token, int64_t ko_head, const void* positions, int pos64,
               int64_t pos_batch, int64_t pos_token, int axes, const double* freqs, int B, int L, int hq, int hk, int d,
               int rot, int interleaved, double mscale, int inverse, int dtype, hipStream_t stream) {
    if (B < 0 || L < 0 || hq < 0 || hk < 0 || axes < 1 || axes > 2) return FLA_ERR_SHAPE;
    const int64_t strides[] = {q_batch,  q_token,  q_head,   k_batch,  k_token,  k_head,    qo_batch,
                               qo_token, qo_head,  ko_batch, ko_token, ko_head,  pos_batch, pos_token};
    for (int64_t s : strides)
        if (s < 0) return FLA_ERR_SHAPE;
    if (!type_ok(dtype)) return FLA_ERR_UNSUPPORTED;
    if (rot < 2 || rot % 2 != 0 || rot > d || d > 512 || (axes == 2 && rot % 4 != 0)) return FLA_ERR_HEAD_DIM;
    if (!std::isfinite(mscale)) return FLA_ERR_ROPE;
    if (B == 0 || L == 0 || (hq == 0 && hk == 0)) return FLA_OK;
    if ((hq > 0 && (!q || !q_out)) || (hk > 0 && (!k || !k_out)) || !positions || !freqs) return FLA_ERR_NULL;
    const int e = size_of(dtype);
    if ((hq > 0 && (!aligned(q, e) || !aligned(q_out, e))) || (hk > 0 && (!aligned(k, e) || !aligned(k_out, e))) ||
        !aligned(positions, pos64 ? 8 : 4) || !aligned(freqs, 8))
        return FLA_ERR_ALIGN;
    if ((int64_t)B * L > kMaxLen || (int64_t)hq + hk > 1 << 20) return FLA_ERR_TOO_LARGE;
    struct Side {
        const void* in;
        void* out;
        const int64_t* s;   // in: batch, token, head; out 6 further
        int heads;
    };
    const Side sides[] = {{q, q_out, strides, hq}, {k, k_out, strides + 3, hk}};
    Tokens in[2], out[2];
    for (int i = 0; i < 2; ++i) {
        const Side& m = sides[i];
        const int64_t wi = reach(m.heads, m.s[2]) + d, wo = reach(m.heads, m.s[8]) + d;
        in[i] = {m.heads ? m.in : nullptr, m.s[0], m.s[1], B, L, wi, e};
        out[i] = {m.heads ? m.out : nullptr, m.s[6], m.s[7], B, L, wo, e};
        if (in[i].elements() >= kMaxElems || out[i].elements() >= kMaxElems) return FLA_ERR_TOO_LARGE;
        if (m.heads > 1 && (m.s[2] > UINT32_MAX || m.s[8] > UINT32_MAX)) return FLA_ERR_TOO_LARGE;
    }
    const Range pos = {positions, (reach(B, pos_batch) + reach(L, pos_token) + axes) * (pos64 ? 8 : 4)};
    const Range table = {freqs, (int64_t)rot / 2 * 8};
    for (int i = 0; i < 2; ++i) {
        const Side& m = sides[i];
        if (!m.heads) continue;
        // the rows of an output lie apart: the strides from the smallest on step over what is below them
        struct {
            int64_t n, s;
        } dim[] = {{m.heads, m.s[8]}, {L, m.s[7]}, {B, m.s[6]}};
        for (int u = 0; u < 2; ++u)
            for (int v = 0; v < 2 - u; ++v)
                if (dim[v].s > dim[v + 1].s) {
                    const auto t = dim[v];
                    dim[v] = dim[v + 1];
                    dim[v + 1] = t;
                }
        int64_t span = d;
        for (const auto& x : dim) {
            if (x.n == 1) continue;
            if (x.s < span) return FLA_ERR_ALIAS;
            span += (x.n - 1) * x.s;
        }
        for (int j = 0; j < 2; ++j) {
            if (!sides[j].heads) continue;
            const bool in_place = i == j && m.in == m.out && (B == 1 || m.s[0] == m.s[6]) &&
                                  (L == 1 || m.s[1] == m.s[7]) && (m.heads == 1 || m.s[2] == m.s[8]);
            if (!in_place && share(out[i], in[j])) return FLA_ERR_ALIAS;
        }
        if (overlap(out[i].range(), pos) || overlap(out[i].range(), table)) return FLA_ERR_ALIAS;
    }
    if (hq > 0 && hk > 0 && share(out[0], out[1])) return FLA_ERR_ALIAS;
    int cus = 0;
    const int st = check_arch(&cus);
    if (st != FLA_OK) return st;
    fla::RotaryArgs a{};
    a.q = {q, q_out, q_batch, q_token, qo_batch, qo_token, (unsigned)q_head, (unsigned)qo_head};
    a.k = {k, k_out, k_batch, k_token, ko_batch, ko_token, (unsigned)k_head, (unsigned)ko_head};
    a.positions = positions;
    a.freqs = freqs;
    a.pos_batch = pos_batch;
    a.pos_token = pos_token;
    a.pos64 = pos64;
    a.axes = axes;
    a.B = B;
    a.L = L;
    a.hq = hq;
    a.heads = hq + hk;
    a.d = d;
    a.rot = rot;
    a.n_tokens = (int64_t)B * L;
    a.mscale = (float)mscale;
    a.sign = inverse ? -1.f : 1.f;
    return launched(fla::launch_rotary(a, dtype == FLA_BF16, interleaved != 0, cus, stream));
}

int fla_gated_scan_states(int B, int L, int D, size_t* bytes) { return scan_bytes(B, L, D, bytes, scan_states_bytes); }
int fla_gated_scan_workspace(int B, int L, int D, size_t* bytes) { return scan_bytes(B, L, D, bytes, scan_ws_bytes); }
int fla_gated_scan_bwd_workspace(int B, int L, int D, size_t* bytes) {
    return scan_bytes(B, L, D, bytes, scan_bwd_ws_bytes);
}

int fla_gated_scan_fwd(const void* x, int64_t x_batch, int64_t x_token, const void* r, int64_t r_batch,
                       int64_t r_token, const void* i, int64_t i_batch, int64_t i_token, const float* lam,
                       const float* h0, const int* lengths, void* h, float* h_last, float* states, void* workspace,
                       size_t workspace_bytes, int B, int L, int D, float c, int dtype, hipStream_t stream) {
    int st = scan_sizes(B, L, D);
    if (st != FLA_OK) return st;
    if (x_batch < 0 || x_token < 0 || r_batch < 0 || r_token < 0 || i_batch < 0 || i_token < 0) return FLA_ERR_SHAPE;
    if (!type_ok(dtype) || !(c > 0.f) || !std::isfinite(c)) return FLA_ERR_UNSUPPORTED;
    if (B == 0 || D == 0) return FLA_OK;
    if (L > 0 && (!x || !r || !i || !lam || !h)) return FLA_ERR_NULL;
    const int e = size_of(dtype);
    if (!aligned(x, e) || !aligned(r, e) || !aligned(i, e) || !aligned(h, e) || !aligned(lam, 4) || !aligned(h0, 4) ||
        !aligned(lengths, 4) || !aligned(h_last, 4) || !aligned(states, 4) || !aligned(workspace, 8))
        return FLA_ERR_ALIGN;
    if (scan_too_large(B, L, D)) return FLA_ERR_TOO_LARGE;
    const Tokens in[] = {{x, x_batch, x_token, B, L, D, e}, {r, r_batch, r_token, B, L, D, e}, {i, i_batch, i_token, B, L, D, e}};
    for (const Tokens& t : in)
        if (t.elements() >= kMaxElems) return FLA_ERR_TOO_LARGE;
    const int64_t need = scan_ws_bytes(B, L, D);
    if (need > 0 && (!workspace || workspace_bytes < (size_t)need)) return FLA_ERR_WORKSPACE;
    const int64_t state = (int64_t)B * D * 4;
    const Range ins[] = {L ? in[0].range() : Range{}, L ? in[1].range() : Range{}, L ? in[2].range() : Range{},
                         {lam, (int64_t)D * 4}, {h0, state}, {lengths, (int64_t)B * 4}};
    const Range outs[] = {{h, (int64_t)B * L * D * e}, {h_last, state}, {states, scan_states_bytes(B, L, D)}, {workspace, need}};
    for (int o = 0; o < 4; ++o) {
        for (int q = 0; q < 6; ++q)
            if (!(o == 1 && q == 4 && h_last == h0) && overlap(outs[o], ins[q])) return FLA_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (overlap(outs[o], outs[q])) return FLA_ERR_ALIAS;
    }
    if (L == 0 && !h_last) return FLA_OK;
    if (!lam) return FLA_ERR_NULL;
    int cus = 0;
    st = check_arch(&cus);
    if (st != FLA_OK) return st;
    fla::ScanArgs a{};
    a.x = {x, x_batch, x_token};
    a.r = {r, r_batch, r_token};
    a.i = {i, i_batch, i_token};
    a.lam = lam;
    a.h0 = h0;
    a.lengths = lengths;
    a.h = h;
    a.h_last = h_last;
    a.states = states;
    a.ws = workspace;
    a.B = B;
    a.L = L;
    a.D = D;
    a.columns = (int)scan_columns(D);
    a.chunks = (int)scan_chunks(L);
    a.cus = cus;
    a.lines = lines(h, D, e);
    a.c = c;
    return launched(fla::launch_scan_fwd(a, dtype == FLA_BF16, stream));
}

int fla_gated_scan_bwd(const void* x, int64_t x_batch, int64_t x_token, const void* r, int64_t r_batch,
                       int64_t r_token, const void* i, int64_t i_batch, int64_t i_token, const float* lam,
                       const float* states, const int* lengths, const void* dh, int64_t dh_batch, int64_t dh_token,
                       const float* d_last, void* dx, void* dr, void* di, float* dlam, float* dh0, void* workspace,
                       size_t workspace_bytes, int B, int L, int D, float c, int dtype, hipStream_t stream) {
    int st = scan_sizes(B, L, D);
    if (st != FLA_OK) return st;
    if (x_batch < 0 || x_token < 0 || r_batch < 0 || r_token < 0 || i_batch < 0 || i_token < 0 || dh_batch < 0 ||
        dh_token < 0)
        return FLA_ERR_SHAPE;
    if (!type_ok(dtype) || !(c > 0.f) || !std::isfinite(c)) return FLA_ERR_UNSUPPORTED;
    if (D == 0) return FLA_OK;
    if (!lam || !dlam || (B > 0 && L > 0 && (!x || !r || !i || !states || !dx || !dr || !di))) return FLA_ERR_NULL;
    const int e = size_of(dtype);
    if (!aligned(x, e) || !aligned(r, e) || !aligned(i, e) || !aligned(dh, e) || !aligned(dx, e) || !aligned(dr, e) ||
        !aligned(di, e) || !aligned(lam, 4) || !aligned(states, 4) || !aligned(lengths, 4) || !aligned(d_last, 4) ||
        !aligned(dlam, 4) || !aligned(dh0, 4) || !aligned(workspace, 8))
        return FLA_ERR_ALIGN;
    if (scan_too_large(B, L, D)) return FLA_ERR_TOO_LARGE;
    const Tokens in[] = {{x, x_batch, x_token, B, L, D, e}, {r, r_batch, r_token, B, L, D, e},
                         {i, i_batch, i_token, B, L, D, e}, {dh, dh_batch, dh_token, B, L, D, e}};
    for (const Tokens& t : in)
        if (t.elements() >= kMaxElems) return FLA_ERR_TOO_LARGE;
    const int64_t need = scan_bwd_ws_bytes(B, L, D);
    if (need > 0 && (!workspace || workspace_bytes < (size_t)need)) return FLA_ERR_WORKSPACE;
    const int64_t state = (int64_t)B * D * 4, full = (int64_t)B * L * D * e;
    const bool any = B > 0 && L > 0;
    const Range ins[] = {any ? in[0].range() : Range{}, any ? in[1].range() : Range{}, any ? in[2].range() : Range{},
                         any ? in[3].range() : Range{}, {lam, (int64_t)D * 4}, {states, scan_states_bytes(B, L, D)},
                         {lengths, (int64_t)B * 4}, {d_last, state}};
    const Range outs[] = {{dx, full}, {dr, full}, {di, full}, {dlam, (int64_t)D * 4}, {dh0, state}, {workspace, need}};
    for (int o = 0; o < 6; ++o) {
        for (const Range& q : ins)
            if (overlap(outs[o], q)) return FLA_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (overlap(outs[o], outs[q])) return FLA_ERR_ALIAS;
    }
    int cus = 0;
    st = check_arch(&cus);
    if (st != FLA_OK) return st;
    fla::ScanBwdArgs a{};
    a.x = {x, x_batch, x_token};
    a.r = {r, r_batch, r_token};
    a.i = {i, i_batch, i_token};
    a.dh = {dh, dh_batch, dh_token};
    a.lam = lam;
    a.states = states;
    a.lengths = lengths;
    a.d_last = d_last;
    a.dx = dx;
    a.dr = dr;
    a.di = di;
    a.dlam = dlam;
    a.dh0 = dh0;
    a.ws = workspace;
    a.shares = reinterpret_cast<float*>(static_cast<char*>(workspace) + scan_ws_bytes(B, L, D));
    a.B = B;
    a.L = L;
    a.D = D;
    a.columns = (int)scan_columns(D);
    a.chunks = a.links = (int)scan_chunks(L);
    a.lines = lines(dx, D, e) && lines(dr, D, e) && lines(di, D, e);
    a.c = c;
    return launched(fla::launch_scan_bwd(a, dtype == FLA_BF16, stream));
}

}  // extern "C"
