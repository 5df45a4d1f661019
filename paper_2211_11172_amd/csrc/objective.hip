// Policy objectives on the logits of any actor: log-probabilities of chosen actions with their
// gradient, the clipped policy loss with a KL term, and the pairwise preference loss of log ratios.
//
// A row of logits z is cut into segments; of each, with m = max z,
//   s = sum e^(z - m), u = sum e^(z - m) (z - m), lse = m + log s, H = log s - u / s,
// and the row's log-probability is the sum over segments of z[action] - lse.  Every objective reaches
// the logits through the row's two gradients g_logp and g_H:
//   dz_i = g_logp (1[i = action] - p_i) - g_H p_i (log p_i + H_s),  p_i = e^(z_i - m) / s.
//
// Bytes bound all of it: a row read once for the sums and its gradient written once, with some 20 instruction
// slots a column (two exponentials of four among them) of about 30 that a copy's rate leaves.
//   k_loss         clipped loss, one segment: a row stays in registers between its sums and its gradient
//   k_stats        sums of rows, or of chunks of rows where few of them would leave the machine idle
//   k_grad         gradient of rows whose sums are known: of harl_policy_logp_grad, of the preference loss
//                  (whose gradient needs all of a pair's rows first) and of few rows' clipped loss
//   k_pairs        a pair's log ratios, loss terms and row gradients
//   k_types        heads of several segments: a wave's rows in LDS through all steps
//   k_types_pairs  the preference loss of short tracks of such heads in one launch
// Sums over a row are fp32 relative to its maximum, in a fixed order; over rows and segments fp64.  The gradient is
// rounded once, to the logits' type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "internal.hpp"

namespace harl {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxGrid = 1 << 20;  // workgroups of a launch; kernels step over rows by the grid

struct Rows {
    const void *z;
    int64_t ld;
    int M, a, n_seg;
    const int32_t *act;
    const float *weight;     // rows of weight 0 count for nothing, or null
    const int32_t *seq_ptr;  // only rows of [seq_ptr[0], seq_ptr[n_seq]) count, or null
    int n_seq;
    int32_t off[HARL_SELECT_MAX_SEGMENTS + 1];
};

// A chunk of a row's sums, and the row's logit at its action.
struct Stat {
    float m, s, u, zact;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void store(float *p, float x) { *p = x; }
__device__ __forceinline__ void store(uint16_t *p, float x) {  // to nearest, ties to even; NaN stays NaN
    const uint32_t b = __float_as_uint(x);
    *p = x != x ? (uint16_t)0x7fc0u : (uint16_t)((b + 0x7fffu + ((b >> 16) & 1)) >> 16);
}

__device__ __forceinline__ int clamp_row(int r, int M) { return r < 0 ? 0 : r > M ? M : r; }

__device__ __forceinline__ bool row_counts(const Rows &q, int r) {
    if (q.seq_ptr && (r < clamp_row(q.seq_ptr[0], q.M) || r >= clamp_row(q.seq_ptr[q.n_seq], q.M))) return false;
    return !q.weight || q.weight[r] != 0.f;
}

struct LossArgs {
    const float *logp_old, *logp_ref, *adv, *weight;
    float clip_low, clip_high, w_kl, w_entropy;
    float inv_m;
};

// The ratio of two probabilities ends at e^690 (a product with any advantage but 0 is infinite in fp32 long before), so
// that an advantage of 0 gives 0 whatever the ratio is, and not 0 times infinity.
constexpr double kTopLog = 690.0;

// One row's terms of the clipped loss, weighted.
__device__ __forceinline__ void loss_row(const LossArgs &a, int64_t r, float w, double logp, double H, double (&term)[3]) {
    const double d = logp - (double)a.logp_old[r], ratio = exp(d > kTopLog ? kTopLog : d);
    const double adv = a.adv[r], lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
    const double s1 = ratio * adv, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
    double kl = 0.0;
    if (a.logp_ref) {
        const double x = (double)a.logp_ref[r] - logp;
        kl = x < INFINITY ? expm1(x) - x : x;  // x = inf (an excluded action): inf, not inf - inf
    }
    term[0] = (double)w * -(s2 < s1 ? s2 : s1);
    term[1] = (double)w * kl;
    term[2] = (double)w * H;
}

// ------------------------------------------------------------------------------------------------
// Heads of one segment.  A row is moved as 16-byte vectors behind its first aligned column; the columns
// before it and behind the last whole vector (at most 2 (16 / element - 1)) are an element a thread.
//
// The exponentials are 2^y, y = (z - m) log2 e, with s = sum 2^y and u = sum 2^y y, so that
//   log s = ln 2 log2 s,  H = ln 2 (log2 s - u / s).
// log2 e is rounded to fp32 once for all columns: 2^y is e^(z - m) to the power 1 - 1.3e-8, which moves log s
// by 1.3e-8 ln 2 u / s (6e-8 for a vocabulary's logits, the same sign in every row of a track); log_sum
// adds it back.
// ------------------------------------------------------------------------------------------------
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr double kLn2d = 0.69314718055994530942, kLog2eRest = 1.44269504088896340736 - (double)kLog2e;
constexpr float kYMin = -160.f;  // 2^y is 0 from here on; keeps 0 times y a number for excluded actions

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float exp2_hw(float y) { return __builtin_amdgcn_exp2f(y); }
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ void unpack(const uint4 &r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x);
    x[1] = __uint_as_float(r.y);
    x[2] = __uint_as_float(r.z);
    x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(const uint4 &r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, bf16x2));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ uint4 all_excluded() {
    constexpr uint32_t w = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    return make_uint4(w, w, w, w);
}

// The parts of a row: `head` columns, `full` vectors, `tail` columns.
template <typename T>
struct Parts {
    int head, full, tail;
    __device__ __forceinline__ Parts(const T *p, int a) {
        const int mis = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T)) & (kVec<T> - 1);
        head = mis ? min(kVec<T> - mis, a) : 0;
        full = (a - head) / kVec<T>;
        tail = a - head - full * kVec<T>;
    }
    // the column of thread t's single element, or -1
    __device__ __forceinline__ int edge(int t) const {
        return t < head ? t : t < head + tail ? full * kVec<T> + t : -1;
    }
};

// A row's vectors as TPR-wide slices through buffer descriptors: thread t's vector of slice j lies at byte
// 16 t of the slice, and the descriptor ends with the row (loads beyond give 0, stores go nowhere), so that
// loads and stores need neither masks nor an address of their own a vector.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t slice(const void *base, int bytes, int from) {
    char *p = static_cast<char *>(const_cast<void *>(base)) + from;
    return __builtin_amdgcn_make_buffer_rsrc(p, 0, max(bytes - from, 0), 0x00027000);
}
__device__ __forceinline__ uint4 load_vec(__amdgpu_buffer_rsrc_t b, int byte) {
    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(b, byte, 0, 0);
    return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void put_vec(__amdgpu_buffer_rsrc_t b, int byte, const uint4 &v) {
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{v.x, v.y, v.z, v.w}, b, byte, 0, 0);
}

// Running sums of one lane, wave or workgroup relative to its own largest value.
struct Sums {
    float m, s, u;
};

__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }

// FINE: u is not the entropy's sum but sum 2^y (d log2 e - y), d = z - m: what the products y = d log2 e were
// rounded by and log2 e misses.  The difference of two log-probabilities summed over a track's rows needs it: bf16
// logits are few values, whose roundings do not cancel (1e-8 a row).  log s is then ln s + ln 2 u / s.
__device__ __forceinline__ float missed(float d, float y) { return fmaf(d, (float)kLog2eRest, fmaf(d, kLog2e, -y)); }

// Moves the sums to a larger maximum (its shift ms = shift_of(m_new)).
template <bool FINE = false>
__device__ __forceinline__ void rescale(Sums &q, float m_new, float ms) {
    if (FINE) {
        const float d = fmaxf(q.m - ms, -1e4f), y = d * kLog2e, f = q.m == -INFINITY ? 0.f : exp2_hw(y);
        q.u = f * fmaf(q.s, missed(d, y), q.u);
        q.s *= f;
        if (q.m != q.m || m_new != m_new) q.s = __builtin_nanf("");
    } else {
        const float d = (q.m - ms) * kLog2e, f = exp2_hw(d);
        q.u = f * (q.u + q.s * fmaxf(d, -1e4f));
        q.s *= f;
    }
    q.m = m_new;
}

// Adds NV vectors or single values to a lane's sums, with one change of the maximum.
template <bool FINE, int NV, int N>
__device__ __forceinline__ void add_values(Sums &q, const float (&x)[NV][N]) {
    float gm = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) gm = max_nan(gm, x[j][i]);
    const float m = max_nan(q.m, gm), ms = shift_of(m);
    rescale<FINE>(q, m, ms);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (FINE) {
                const float d = fmaxf(x[j][i] - ms, kYMin), y = d * kLog2e, e = exp2_hw(y);
                q.s += e;
                q.u = fmaf(e, missed(d, y), q.u);
            } else {
                const float y = fmaxf((x[j][i] - ms) * kLog2e, kYMin), e = exp2_hw(y);
                q.s += e;
                q.u = fmaf(e, y, q.u);
            }
        }
}
template <bool FINE, int N, int NV>
__device__ __forceinline__ void add_vectors(Sums &q, const uint4 *raw) {
    float x[NV][N];
#pragma unroll
    for (int j = 0; j < NV; ++j) unpack(raw[j], x[j]);
    add_values<FINE, NV, N>(q, x);
}

// Reductions over the first W lanes of a wave (W a power of two up to 64); the result in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float x, float old) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <int W, typename Op>
__device__ __forceinline__ float lanes_reduce(float x, float none, Op op) {
    if constexpr (W > 1) x = op(x, dpp<0x111, 0xf>(x, none));   // row_shr:1
    if constexpr (W > 2) x = op(x, dpp<0x112, 0xf>(x, none));   // row_shr:2
    if constexpr (W > 4) x = op(x, dpp<0x114, 0xf>(x, none));   // row_shr:4
    if constexpr (W > 8) x = op(x, dpp<0x118, 0xf>(x, none));   // row_shr:8
    if constexpr (W > 16) x = op(x, dpp<0x142, 0xa>(x, none));  // row_bcast:15 into rows 1 and 3
    if constexpr (W > 32) x = op(x, dpp<0x143, 0xc>(x, none));  // row_bcast:31 into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), W - 1));
}
template <int W, bool FINE = false>
__device__ __forceinline__ Sums lanes_join(Sums q) {
    const float m = lanes_reduce<W>(q.m, -INFINITY, [](float a, float b) { return max_nan(a, b); });
    rescale<FINE>(q, m, shift_of(m));
    const auto add = [](float a, float b) { return a + b; };
    return Sums{m, lanes_reduce<W>(q.s, 0.f, add), lanes_reduce<W>(q.u, 0.f, add)};
}

// Sum of 64 bits over a wave, in lane order by pairs; the result in every lane.
__device__ __forceinline__ double wave_sum(double x) {
    const auto move = [](double v, auto f) {
        return __hiloint2double(__float_as_int(f(__int_as_float(__double2hiint(v)))), __float_as_int(f(__int_as_float(__double2loint(v)))));
    };
    x += move(x, [](float v) { return dpp<0x111, 0xf>(v, 0.f); });
    x += move(x, [](float v) { return dpp<0x112, 0xf>(v, 0.f); });
    x += move(x, [](float v) { return dpp<0x114, 0xf>(v, 0.f); });
    x += move(x, [](float v) { return dpp<0x118, 0xf>(v, 0.f); });
    x += move(x, [](float v) { return dpp<0x142, 0xa>(v, 0.f); });
    x += move(x, [](float v) { return dpp<0x143, 0xc>(v, 0.f); });
    return move(x, [](float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63)); });
}

// The sums of a row from those of its TPR threads, in every thread.  `red` has 2 halves of TPR / 64
// entries, used in turn, so that one barrier a row is enough.
template <int TPR, bool FINE = false>
__device__ __forceinline__ Sums row_join(Sums q, Sums (*red)[16], int &half) {
    q = lanes_join<64, FINE>(q);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        if (threadIdx.x % 64 == 0) red[half][threadIdx.x / 64] = q;
        __syncthreads();
        q = lanes_join<W, FINE>(red[half][threadIdx.x % W]);
        half ^= 1;
    }
    // NaN or +inf among the values: everything that follows is NaN
    if (!(q.m < INFINITY)) q.s = q.u = __builtin_nanf("");
    return q;
}

__device__ __forceinline__ double log_sum(const Sums &q) {
    return log((double)q.s) + kLog2eRest * kLn2d * kLn2d * (double)q.u / (double)q.s;
}
__device__ __forceinline__ double log_prob(const Sums &q, float zact) {
    return q.s == 0.f ? 0.0 : ((double)zact - (double)q.m) - log_sum(q);
}
__device__ __forceinline__ double entropy_of(const Sums &q) {
    return q.s == 0.f ? 0.0 : log_sum(q) - kLn2d * (double)q.u / (double)q.s;
}

// The same in fp32, for what is rounded to fp32 next.  The hardware's log2 s is good to a step of its own size
// (1.9e-6 for a vocabulary); s 2^-(that) - 1 is what it misses.
struct LogSum {
    float l2s, ls, mean_y, inv_s;
};
__device__ __forceinline__ LogSum log_sum_f32(const Sums &q) {
    const float l2s = __builtin_amdgcn_logf(q.s), inv_s = 1.f / q.s, mean_y = q.u * inv_s;
    const float missed = fmaf(q.s, exp2_hw(-l2s), -1.f);
    return LogSum{l2s, fmaf(l2s, kLn2, fmaf((float)(kLog2eRest * kLn2d * kLn2d), mean_y, missed)), mean_y, inv_s};
}
__device__ __forceinline__ float log_prob_f32(const Sums &q, const LogSum &l, float zact) { return q.s == 0.f ? 0.f : (zact - q.m) - l.ls; }
__device__ __forceinline__ float entropy_f32(const Sums &q, const LogSum &l) { return q.s == 0.f ? 0.f : l.ls - kLn2 * l.mean_y; }

// What the gradient of a row is made of: dz_i = -p_i (g_logp + g_H (log p_i + H)), and g_logp more at the
// action.  With y = (z - m) log2 e, p = 2^y / s and log p = ln 2 (y - log2 s) it is 2^y (c + e y),
//   e = -g_H ln 2 / s,  c = -(g_logp + g_H (H - ln 2 log2 s)) / s:
// 1 / s is in the coefficients, not in the exponent, which would be rounded at its size.
struct RowCoef {
    float m, c, e, g, zero;  // zero != 0: the row's gradient is 0
};

// `empty`: no column has a probability.  rest: log s; used with the entropy's gradient only, as H.
__device__ __forceinline__ RowCoef coef_of(float m, bool empty, float inv_s, float rest, float H, float gl, float ge) {
    RowCoef k;
    k.m = shift_of(m);
    k.c = -(gl + (ge != 0.f ? ge * (H - rest) : 0.f)) * inv_s;
    k.e = -ge * kLn2 * inv_s;
    k.g = gl;
    k.zero = empty || (gl == 0.f && ge == 0.f) ? 1.f : 0.f;
    return k;
}

template <bool ENT>
__device__ __forceinline__ float grad_of(const RowCoef &k, float z) {
    const float y = (z - k.m) * kLog2e, e = exp2_hw(y);
    return ENT ? e * fmaf(k.e, fmaxf(y, kYMin), k.c) : e * k.c;
}
__device__ __forceinline__ float grad_any(const RowCoef &k, float z) {
    return k.e != 0.f ? grad_of<true>(k, z) : grad_of<false>(k, z);
}

// One vector's gradient to column i0 of the row dz; `same`: dz has the logits' alignment; STREAM: past the caches.
template <typename T, bool STREAM>
__device__ __forceinline__ void store_vec(T *dz, int i0, const float (&x)[kVec<T>], bool same) {
    if (same) {
        const uint4 v = pack(x);
        u32x4 *to = reinterpret_cast<u32x4 *>(dz + i0);
        if (STREAM) __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, to);
        else *to = u32x4{v.x, v.y, v.z, v.w};
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) store(dz + i0 + i, x[i]);
    }
}
template <typename T, bool STREAM>
__device__ __forceinline__ void grad_vec(T *dz, int i0, const uint4 &raw, const RowCoef &k, bool same) {
    float x[kVec<T>];
    unpack(raw, x);
    if (k.zero != 0.f) {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) x[i] = 0.f;
    } else if (k.e != 0.f) {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) x[i] = grad_of<true>(k, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) x[i] = grad_of<false>(k, x[i]);
    }
    store_vec<T, STREAM>(dz, i0, x, same);
}

// ---- statistics of (row, chunk) items: a chunk is `per` vectors, the first also has the row's edges ----
enum Out : int { kPartial = 0, kLogp = 1, kPartialFine = 2 };

struct StatOut {
    Stat *stat;  // kPartial, kPartialFine: [row][chunk] {m, s, u, z[action]}
    float *logp, *entropy, *lse;
};

__device__ __forceinline__ void put_logp(const StatOut &o, int64_t r, const Sums &q, float zact) {
    const LogSum l = log_sum_f32(q);
    o.logp[r] = log_prob_f32(q, l, zact);
    if (o.entropy) o.entropy[r] = entropy_f32(q, l);
    if (o.lse) {
        o.lse[2 * r] = q.m;
        o.lse[2 * r + 1] = q.s == 0.f ? 0.f : l.ls;
    }
}

// An item by TPR threads (a wave: four items a workgroup, no barrier), NV vectors each in flight, summed four
// at a time so that one change of the maximum serves 32 bf16 columns.  Bound by the reads: 400 MB of bf16 rows in
// 85 us (4.7 TB/s; a bare read of them 6.1), FINE's two more instructions a column 10 us of it; whole rows of 8,192
// vectors in two rounds of workgroups, and without the loads ahead, took 119 us without FINE.
template <typename T, int TPR, int NV, int OUT>
__global__ __launch_bounds__(TPR < kThreads ? kThreads : TPR) void k_stats(Rows q, int chunks, int per, StatOut o) {
    constexpr int WG = TPR < kThreads ? kThreads : TPR, N = kVec<T>, G = NV < 4 ? NV : 4;
    constexpr bool FINE = OUT == kPartialFine;
    __shared__ Sums red[2][16];
    int half = 0;
    const int t = threadIdx.x % TPR;
    const int64_t items = (int64_t)q.M * chunks;
    for (int64_t it = (int64_t)blockIdx.x * (WG / TPR) + threadIdx.x / TPR; it < items; it += (int64_t)gridDim.x * (WG / TPR)) {
        // a wave lies in one item
        const int r = __builtin_amdgcn_readfirstlane(chunks == 1 ? (int)it : (int)(it / chunks));
        const int c = __builtin_amdgcn_readfirstlane((int)(it - (int64_t)r * chunks));
        if (!row_counts(q, r)) continue;
        const T *z = static_cast<const T *>(q.z) + (int64_t)r * q.ld;
        const Parts<T> parts(z, q.a);
        const int act = min(max(q.act[r], 0), q.a - 1);
        const float zact = to_f32(z[act]);
        const int ei = c == 0 ? parts.edge(t) : -1;
        const float ex = ei < 0 ? -INFINITY : to_f32(z[ei]);
        Sums sum{-INFINITY, 0.f, 0.f};
        const int v1 = min((c + 1) * per, parts.full);
        for (int v = c * per; v < v1; v += TPR * NV) {
            const T *from = z + parts.head + (int64_t)v * N;
            const int left = v1 - v;
            uint4 raw[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) raw[j] = load_vec(slice(from, left * 16, TPR * 16 * j), t * 16);
#pragma unroll
            for (int g = 0; g < NV; g += G) {
                if (TPR * g >= left) break;
#pragma unroll
                for (int j = g; j < g + G; ++j)
                    if (TPR * (j + 1) > left && t + TPR * j >= left) raw[j] = all_excluded<T>();
                add_vectors<FINE, N, G>(sum, raw + g);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (c == 0 && parts.head + parts.tail > 0) {
            const float x[1][1] = {{ex}};
            add_values<FINE, 1, 1>(sum, x);
        }
        sum = row_join<TPR, FINE>(sum, red, half);
        if (t == 0) {
            if (OUT == kLogp) put_logp(o, r, sum, zact);
            else o.stat[it] = Stat{sum.m, sum.s, sum.u, zact};
        }
    }
}

// A row's sums from its chunks', by one thread in chunk order, eight loads in flight.
template <bool FINE = false>
__device__ __forceinline__ Sums join_chunks(const Stat *__restrict__ st, int chunks) {
    if (chunks == 1) return Sums{st[0].m, st[0].s, st[0].u};
    Sums q{-INFINITY, 0.f, 0.f};
    for (int c = 0; c < chunks; c += 8) {
        Stat x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = st[min(c + j, chunks - 1)];
        float m = q.m;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_nan(m, x[j].m);
        const float ms = shift_of(m);
        rescale<FINE>(q, m, ms);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            Sums y{x[j].m, x[j].s, x[j].u};
            rescale<FINE>(y, m, ms);
            if (c + j < chunks) {
                q.s += y.s;
                q.u += y.u;
            }
        }
    }
    if (!(q.m < INFINITY)) q.s = q.u = __builtin_nanf("");
    return q;
}

__global__ __launch_bounds__(64) void k_logp_join(const Stat *__restrict__ stat, int M, int chunks, StatOut o) {
    for (int64_t r = (int64_t)blockIdx.x * 64 + threadIdx.x; r < M; r += (int64_t)gridDim.x * 64) {
        const Sums sum = join_chunks(stat + r * chunks, chunks);
        put_logp(o, r, sum, stat[r * chunks].zact);
    }
}

// ---- the clipped loss, a row's logits held in registers between its sums and its gradient ----
struct LossOut {
    void *dz;
    int64_t ld_d;
    float *logp;
    double *terms;  // [workgroup][3]: the sums of its rows' terms, in row order
};

// loss_grad's terms of a log ratio beyond kLargeLog: e^89 is more than fp32 holds, 1e-4 e^89 is not, and 0 e^89 is 0.  The
// weight goes into the terms first, and an exponential is the product of two.  (The branch costs the other rows 0.1% over
// 28 shapes; products in 64 bits for all rows, without it, took up to 8% more, 1.7% over all.)
constexpr float kLargeLog = 30.f;

__device__ __forceinline__ void loss_grad_large(const LossArgs &a, float w, float d, float x, float adv, float &gl,
                                                float &surrogate, float &kl, float &w_left) {
    const auto times_exp = [](float v, float of, float &e) {  // v e^of, and e = e^of; an exponent of 166 is as good as infinite
        const float y = of * kLog2e > 240.f ? 240.f : of * kLog2e, n = y > 120.f ? 120.f : 0.f;
        const float e1 = exp2_hw(y - n), e2 = n > 0.f ? 0x1p120f : 1.f;
        e = e1 * e2;
        return (v * e1) * e2;
    };
    const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high, wa = fabsf(w);
    float ratio, e, dk = 0.f;  // kl comes as of a small x
    const float s1 = times_exp(adv * wa, d, ratio), s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * (adv * wa);
    const bool inside = ratio >= lo && ratio <= hi;
    if (a.logp_ref) {
        const float we = times_exp(wa, x, e);
        kl = x > kLargeLog ? (x < INFINITY ? (we - wa) - x * wa : x) : kl * wa;
        if (a.w_kl != 0.f) dk = a.w_kl * (wa - we);
    }
    w_left = copysignf(1.f, w);
    surrogate = s2 < s1 ? s2 : s1;
    gl = w_left * ((s2 < s1 && !inside ? 0.f : -s1) + dk);
}

// loss_row in fp32, evaluated by every wave of a row: in 64 bits it takes 100 registers beside the row's, and only the
// logarithm, the log ratios and the products in 64 bits still 5% over 28 shapes (0-14% of each).
// e^x - x - 1 near 0 comes from its series, where the difference would cancel.  surrogate and kl have yet to be
// multiplied by w_left.
__device__ __forceinline__ void loss_grad(const LossArgs &a, float w, float old, float ref, float adv, float logp, float &gl,
                                          float &ge, float &surrogate, float &kl, float &w_left) {
    const float d = logp - old, x = a.logp_ref ? ref - logp : 0.f;
    const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
    const float ratio = exp2_hw(d * kLog2e);
    const float s1 = ratio * adv, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
    const bool inside = ratio >= lo && ratio <= hi;
    const float ds = s2 < s1 && !inside ? 0.f : -s1;
    float dk = 0.f;
    kl = 0.f;
    if (a.logp_ref) {
        const float e = exp2_hw(x * kLog2e);
        const float series = x * x * fmaf(x, fmaf(x, fmaf(x, fmaf(x, fmaf(x, 1.f / 5040.f, 1.f / 720.f), 1.f / 120.f), 1.f / 24.f), 1.f / 6.f), 0.5f);
        kl = fabsf(x) < 0.25f ? series : (e - 1.f) - x;
        if (a.w_kl != 0.f) dk = a.w_kl * (1.f - e);
    }
    surrogate = s2 < s1 ? s2 : s1;
    gl = w * (ds + dk);
    ge = -w * a.w_entropy;
    w_left = w;
    if (__builtin_expect(fmaxf(d, x) > kLargeLog, 0)) loss_grad_large(a, w, d, x, adv, gl, surrogate, kl, w_left);
}

// The whole row dz = 0, or (other alignment than the logits') an element at a time from memory.
template <typename T, int TPR>
__device__ __forceinline__ void zero_row(T *dz, int a, int t) {
    const Parts<T> parts(dz, a);
    for (int v = t; v < parts.full; v += TPR) reinterpret_cast<uint4 *>(dz + parts.head)[v] = make_uint4(0, 0, 0, 0);
    const int i = parts.edge(t);
    if (i >= 0) store(dz + i, 0.f);
}
template <typename T, int TPR>
__device__ __forceinline__ void grad_elements(const T *z, T *dz, int a, int act, const RowCoef &k, int t) {
    for (int i = t; i < a; i += TPR) store(dz + i, grad_any(k, to_f32(z[i])) + (i == act ? k.g : 0.f));
}

template <typename T, int TPR, int NV, bool ENT>
__device__ __forceinline__ void grad_slices(const T *dz_body, int full, const uint4 (&raw)[NV], const RowCoef &k, int t) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (TPR * j >= full) continue;  // uniform
        float x[kVec<T>];
        unpack(raw[j], x);
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) x[i] = grad_of<ENT>(k, x[i]);
        put_vec(slice(dz_body, full * 16, TPR * 16 * j), t * 16, pack(x));
        __builtin_amdgcn_sched_barrier(0);
    }
}

// TPR threads a row, NV vectors of it each in registers: 4,096 x 131,072 bf16 rows in 400 us, 1.99 GB at 5.0 TB/s
// (a copy of 2 GB moves 4.9), 1,024 x 65,521 fp32 rows in 110 us (4.6 TB/s).  All loads of a row are issued at
// once and its sums follow them in order; a workgroup of 16 waves holds 131,072 bf16 columns in 64 of its 128
// registers a lane.  Row terms in fp64 and loads under masks took 255 registers and spilled (1,623 us).
//
// Waves a SIMD at least: as many as a row's registers leave.  The fewest columns need them all: 65,536 rows of 256 fp32
// columns fill 8 waves of every SIMD four times (40 us; with 7 waves 45.5).
template <typename T, int TPR, int NV>
constexpr int kLossWaves = NV == 1 ? (sizeof(T) == 4 ? 8 : 7) : NV <= 4 ? (sizeof(T) == 4 ? 7 : TPR == 64 ? 6 : 5)
                         : NV == 8 ? (sizeof(T) == 4 || TPR == 64 ? 5 : 4) : TPR == 1024 ? 4 : 3;

template <typename T, int TPR, int NV, bool GRAD>
__global__ __launch_bounds__(TPR < kThreads ? kThreads : TPR, (kLossWaves<T, TPR, NV>)) void k_loss(Rows q, LossArgs a, LossOut o) {
    constexpr int WG = TPR < kThreads ? kThreads : TPR, N = kVec<T>;
    __shared__ Sums red[2][16];
    __shared__ double part[WG / TPR][3];
    int half = 0;
    const int t = threadIdx.x % TPR;
    double acc[3] = {0.0, 0.0, 0.0};
    for (int64_t r0 = (int64_t)blockIdx.x * (WG / TPR) + threadIdx.x / TPR; r0 < q.M; r0 += (int64_t)gridDim.x * (WG / TPR)) {
        const int64_t r = __builtin_amdgcn_readfirstlane((int)r0);  // a wave lies in one row
        const T *z = static_cast<const T *>(q.z) + r * q.ld;
        T *dz = static_cast<T *>(o.dz) + r * o.ld_d;
        const float w = a.weight ? a.weight[r] : a.inv_m;
        if (w == 0.f) {  // padding
            if (GRAD) zero_row<T, TPR>(dz, q.a, t);
            if (t == 0 && o.logp) o.logp[r] = 0.f;
            continue;
        }
        const Parts<T> parts(z, q.a);
        const int full = parts.full;
        const T *body = z + parts.head;
        uint4 raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = load_vec(slice(body, full * 16, TPR * 16 * j), t * 16);
        const int act = min(max(q.act[r], 0), q.a - 1);
        const float zact = to_f32(z[act]), old = a.logp_old[r], adv = a.adv[r];
        const float ref = a.logp_ref ? a.logp_ref[r] : 0.f;
        const int ei = parts.edge(t);
        const float ex = ei < 0 ? -INFINITY : to_f32(z[ei]);
        Sums sum{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (TPR * j >= full) continue;  // uniform
            if (TPR * (j + 1) > full && t + TPR * j >= full) raw[j] = all_excluded<T>();
            add_vectors<false, N, 1>(sum, raw + j);
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int v = t + TPR * NV; v < full; v += TPR)  // what the registers do not hold
            add_vectors<false, N, 1>(sum, reinterpret_cast<const uint4 *>(body) + v);
        if (parts.head + parts.tail > 0) {
            const float x[1][1] = {{ex}};
            add_values<false, 1, 1>(sum, x);
        }
        sum = row_join<TPR>(sum, red, half);
        const LogSum l = log_sum_f32(sum);
        const float logp = log_prob_f32(sum, l, zact), H = entropy_f32(sum, l);
        float gl, ge, surrogate, kl, w_left;
        loss_grad(a, w, old, ref, adv, logp, gl, ge, surrogate, kl, w_left);
        acc[0] -= (double)w_left * (double)surrogate;
        acc[1] += (double)w_left * (double)kl;
        acc[2] += (double)w * (double)H;
        if (t == 0 && o.logp) o.logp[r] = logp;
        if (!GRAD) continue;
        const RowCoef k = coef_of(sum.m, sum.s == 0.f, l.inv_s, l.ls, H, gl, ge);
        if (k.zero != 0.f) {
            zero_row<T, TPR>(dz, q.a, t);
            continue;
        }
        if ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) {
            grad_elements<T, TPR>(z, dz, q.a, act, k, t);
            continue;
        }
        if (k.e != 0.f) grad_slices<T, TPR, NV, true>(dz + parts.head, full, raw, k, t);
        else grad_slices<T, TPR, NV, false>(dz + parts.head, full, raw, k, t);
        for (int v = t + TPR * NV; v < full; v += TPR)
            grad_vec<T, false>(dz, parts.head + v * N, reinterpret_cast<const uint4 *>(body)[v], k, true);
        if (ei >= 0) store(dz + ei, grad_any(k, ex));
        // the chosen action's column once more, by the thread that wrote it
        const int av = (act - parts.head) / N;
        const bool mine = act < parts.head || act >= parts.head + full * N ? ei == act : av % TPR == t;
        if (mine) store(dz + act, grad_any(k, zact) + k.g);
    }
    if (t == 0)
        for (int c = 0; c < 3; ++c) part[threadIdx.x / TPR][c] = acc[c];
    __syncthreads();
    if (threadIdx.x < 3) {
        double s = 0.0;
        for (int i = 0; i < WG / TPR; ++i) s += part[i][threadIdx.x];
        o.terms[(int64_t)blockIdx.x * 3 + threadIdx.x] = s;
    }
}

// Sums of N terms over n entries by one workgroup: thread-strided in order, then over lanes and waves.
template <int N>
__device__ __forceinline__ void sum_terms(const double *__restrict__ terms, int64_t n, double (&out)[N]) {
    __shared__ double part[N][kThreads / 64];
    double s[N] = {};
#pragma unroll 4
    for (int64_t r = threadIdx.x; r < n; r += kThreads)
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] += terms[r * N + c];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        s[c] = wave_sum(s[c]);
        if (threadIdx.x % 64 == 0) part[c][threadIdx.x / 64] = s[c];
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < N; ++c) {
        out[c] = part[c][0];
        for (int w = 1; w < kThreads / 64; ++w) out[c] += part[c][w];
    }
}

__device__ __forceinline__ void write_loss(const double (&s)[3], float w_kl, float w_entropy, float *loss) {
    loss[0] = (float)(s[0] + (w_kl != 0.f ? (double)w_kl * s[1] : 0.0) - (w_entropy != 0.f ? (double)w_entropy * s[2] : 0.0));
    for (int c = 0; c < 3; ++c) loss[1 + c] = (float)s[c];
}

__global__ __launch_bounds__(kThreads) void k_loss_sum(const double *__restrict__ terms, int64_t n, float w_kl,
                                                       float w_entropy, float *__restrict__ loss) {
    double s[3];
    sum_terms<3>(terms, n, s);
    if (threadIdx.x == 0) write_loss(s, w_kl, w_entropy, loss);
}

// ---- preference loss ----
// A row for the gradient pass of one segment: m, 1 / s and the gradient of its log-probability.
struct RowFin {
    float m, inv_s, g, pad;
};

struct PairArgs {
    const float *logp_ref, *weight;
    const int32_t *seq_ptr;
    int n_rows, chunks, n_pairs;
    float beta, smoothing;
};

// Pair p's terms from its log ratios (written where `put`), and the gradient of the preferred track's.
__device__ __forceinline__ double pair_terms(const PairArgs &a, int64_t p, const double (&R)[2], bool put, double *terms, float *ratio) {
    const double h = (double)a.beta * (R[0] - R[1]);
    // -log sigmoid(h) = log(1 + e^-|h|) + max(-h, 0), -log sigmoid(-h) the same of -h; d/dh of the loss = smoothing -
    // sigmoid(-h).  Each part has a sum of its own: h = -inf gives inf and 0, where their difference h gives NaN.
    const double e = exp(-fabs(h));
    const double down = (h >= 0.0 ? e : 1.0) / (1.0 + e);
    if (put) {
        const double near = log1p(e), lose = near + (h < 0.0 ? -h : 0.0), win = near + (h > 0.0 ? h : 0.0);  // NaN: e is
        terms[p * 4] = a.smoothing != 0.f ? (1.0 - (double)a.smoothing) * lose + (double)a.smoothing * win : lose;
        terms[p * 4 + 1] = lose;
        terms[p * 4 + 2] = h;
        terms[p * 4 + 3] = h > 0.0 ? 1.0 : 0.0;
        if (ratio) {
            ratio[2 * p] = (float)R[0];
            ratio[2 * p + 1] = (float)R[1];
        }
    }
    return (double)a.beta * ((double)a.smoothing - down) / (double)a.n_pairs;
}

// Pair p by workgroup p (stepping over pairs): both tracks' log ratios, the loss terms and every row's
// gradient.  Rows come as `chunks` parts of statistics (one segment; their results go to fin) or as
// weighted log ratios `diff` (several; their gradients go to g_row).
template <int WG>
__global__ __launch_bounds__(WG) void k_pairs(PairArgs a, const Stat *__restrict__ stat, const double *__restrict__ diff,
                                                    RowFin *__restrict__ fin, float *__restrict__ g_row,
                                                    double *__restrict__ terms, float *__restrict__ ratio) {
    __shared__ double part[2][2][WG / 64];
    int half = 0;
    for (int64_t p = blockIdx.x; p < a.n_pairs; p += gridDim.x) {
        // in order these are one run of rows, the rejected track's behind the preferred one's
        const int lo = clamp_row(a.seq_ptr[2 * p], a.n_rows), mid = clamp_row(a.seq_ptr[2 * p + 1], a.n_rows);
        const int hi = clamp_row(a.seq_ptr[2 * p + 2], a.n_rows);
        double s[2] = {0.0, 0.0};
        for (int64_t r = (int64_t)lo + threadIdx.x; r < hi; r += WG) {
            double d;
            if (diff) {
                d = diff[r];
            } else {
                const float w = a.weight ? a.weight[r] : 1.f;
                if (w == 0.f) continue;
                const float ref = a.logp_ref ? a.logp_ref[r] : 0.f;
                const Sums q = join_chunks<true>(stat + r * a.chunks, a.chunks);
                const double ls = log((double)q.s) + kLn2d * (double)q.u / (double)q.s;
                const double lp = q.s == 0.f ? 0.0 : ((double)stat[r * a.chunks].zact - (double)q.m) - ls;
                d = (double)w * (lp - (double)ref);
                if (fin) {
                    fin[r].m = q.s == 0.f ? -INFINITY : q.m;
                    fin[r].inv_s = 1.f / q.s;
                }
            }
            s[r >= mid ? 1 : 0] += d;
        }
        for (int side = 0; side < 2; ++side) {
            const double v = wave_sum(s[side]);
            if (threadIdx.x % 64 == 0) part[half][side][threadIdx.x / 64] = v;
        }
        __syncthreads();
        double R[2];
        for (int side = 0; side < 2; ++side) {
            R[side] = part[half][side][0];
            for (int i = 1; i < WG / 64; ++i) R[side] += part[half][side][i];
        }
        half ^= 1;  // the next pair's sums go to the other half: one barrier a pair
        const double g = pair_terms(a, p, R, threadIdx.x == 0, terms, ratio);
        if (!fin && !g_row) continue;
        for (int64_t r = (int64_t)lo + threadIdx.x; r < hi; r += WG) {
            const float w = a.weight ? a.weight[r] : 1.f;
            const float gr = w == 0.f ? 0.f : (float)((double)w * (r >= mid ? -g : g));
            if (fin) fin[r].g = gr;
            else g_row[r] = gr;
        }
    }
}

// By one workgroup: of 3,000 pairs' preference loss 1.5 of 23 us, of a million pairs' 0.35 of 2.3 ms.
__device__ __forceinline__ void pairs_sum(const double *__restrict__ terms, int n_pairs, float *__restrict__ loss) {
    double s[4];
    sum_terms<4>(terms, n_pairs, s);
    if (threadIdx.x == 0)
        for (int c = 0; c < 4; ++c) loss[c] = (float)(s[c] / (double)n_pairs);
}

__global__ __launch_bounds__(kThreads) void k_pairs_sum(const double *__restrict__ terms, int n_pairs, float *__restrict__ loss) {
    pairs_sum(terms, n_pairs, loss);
}

// ---- the gradient of rows whose sums are known, an item (row, chunk of 1,024 vectors) a workgroup ----
// Bound by the bytes: 400 MB read and 500 MB written in 155 us (5.8 TB/s, some of the reads from the Infinity
// Cache).
enum Src : int { kFromFin = 0, kFromLse = 1, kFromLoss = 2 };

struct GradSrc {
    const RowFin *fin;                                     // kFromFin
    const float *lse, *entropy, *g_logp, *g_entropy;       // kFromLse
    const Stat *stat;                                      // kFromLoss: [row][stat_chunks]
    int stat_chunks;
    LossArgs loss;                                         // kFromLoss
    float *logp;
    // the launch's last workgroup sums the loss: over n_pairs pairs' terms (kFromFin) or over the rows (kFromLoss)
    float *loss_out;
    const double *terms;
    int n_pairs;
    void *dz;
    int64_t ld_d;
};

// kFromLoss: row r's sums from its chunks, by one wave.
__device__ __forceinline__ Sums join_wave(const Stat *__restrict__ st, int chunks, float &zact) {
    const int l = threadIdx.x % 64;
    Sums q{-INFINITY, 0.f, 0.f};
    if (l < chunks) {
        const Stat x = st[l];
        q = Sums{x.m, x.s, x.u};
    }
    zact = st[0].zact;
    q = lanes_join<64>(q);
    if (!(q.m < INFINITY)) q.s = q.u = __builtin_nanf("");
    return q;
}

// Few rows' loss terms by one workgroup: a thread a row where rows have few chunks, else a wave a row.
__device__ void loss_of_rows(const GradSrc &a, int M) {
    __shared__ double part[3][kThreads / 64];
    double acc[3] = {0.0, 0.0, 0.0};
    const bool wave = a.stat_chunks > 16;
    const int step = wave ? kThreads / 64 : kThreads;
    for (int r = wave ? (int)threadIdx.x / 64 : (int)threadIdx.x; r < M; r += step) {
        const float w = a.loss.weight ? a.loss.weight[r] : a.loss.inv_m;
        if (w == 0.f) {
            if (a.logp && (!wave || threadIdx.x % 64 == 0)) a.logp[r] = 0.f;
            continue;
        }
        const Stat *st = a.stat + (int64_t)r * a.stat_chunks;
        float zact = st[0].zact;
        const Sums q = wave ? join_wave(st, a.stat_chunks, zact) : join_chunks(st, a.stat_chunks);
        if (wave && threadIdx.x % 64) continue;
        const double lp = log_prob(q, zact);
        double term[3];
        loss_row(a.loss, r, w, lp, entropy_of(q), term);
        for (int c = 0; c < 3; ++c) acc[c] += term[c];
        if (a.logp) a.logp[r] = (float)lp;
    }
    for (int c = 0; c < 3; ++c) {
        const double v = wave_sum(acc[c]);
        if (threadIdx.x % 64 == 0) part[c][threadIdx.x / 64] = v;
    }
    __syncthreads();
    if (threadIdx.x == 0 && a.loss_out) {
        double s[3] = {};
        for (int c = 0; c < 3; ++c)
            for (int i = 0; i < kThreads / 64; ++i) s[c] += part[c][i];
        write_loss(s, a.loss.w_kl, a.loss.w_entropy, a.loss_out);
    }
}

// TPR threads an item: a wave where a row has at most four vectors a lane (30,000 x 600 bf16 log-probabilities and
// gradient 64 us with a workgroup a row, 41 with a wave).
template <typename T, int SRC, bool STREAM, int TPR>
__global__ __launch_bounds__(kThreads) void k_grad(Rows q, int chunks, int per, GradSrc a) {
    constexpr int N = kVec<T>, NV = 4;
    const int64_t items = (int64_t)q.M * chunks;
    if (SRC != kFromLse && blockIdx.x == gridDim.x - 1) {  // the workgroup behind the items' ones
        if (SRC == kFromLoss) loss_of_rows(a, q.M);
        else if (a.loss_out) pairs_sum(a.terms, a.n_pairs, a.loss_out);
        return;
    }
    const int64_t step = (SRC == kFromLse ? gridDim.x : gridDim.x - 1) * (int64_t)(kThreads / TPR);
    const int t = threadIdx.x % TPR;
    for (int64_t it = (int64_t)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR; it < items; it += step) {
        // a wave lies in one item
        const int r = __builtin_amdgcn_readfirstlane(chunks == 1 ? (int)it : (int)(it / chunks));
        const int c = __builtin_amdgcn_readfirstlane((int)(it - (int64_t)r * chunks));
        if (q.seq_ptr && (r < clamp_row(q.seq_ptr[0], q.M) || r >= clamp_row(q.seq_ptr[q.n_seq], q.M))) continue;
        const T *z = static_cast<const T *>(q.z) + (int64_t)r * q.ld;
        T *dz = static_cast<T *>(a.dz) + (int64_t)r * a.ld_d;
        const Parts<T> parts(z, q.a);
        const T *body = z + parts.head;
        const bool same = ((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(dz)) & 15) == 0;
        const int act = min(max(q.act[r], 0), q.a - 1);
        RowCoef k{};
        float hot = 0.f;  // the gradient at the action
        if (SRC == kFromFin) {
            const RowFin f = a.fin[r];
            k = coef_of(f.m, f.m == -INFINITY, f.inv_s, 0.f, 0.f, f.g, 0.f);
        } else if (SRC == kFromLse) {
            const float m = a.lse[2 * (int64_t)r], rest = a.lse[2 * (int64_t)r + 1], ge = a.g_entropy ? a.g_entropy[r] : 0.f;
            k = coef_of(m, m == -INFINITY, exp2_hw(-rest * kLog2e), rest, ge != 0.f ? a.entropy[r] : 0.f, a.g_logp[r], ge);
        } else {
            const float w = a.loss.weight ? a.loss.weight[r] : a.loss.inv_m;
            k.zero = 1.f;
            if (w != 0.f) {
                float zact;
                const Sums s = join_wave(a.stat + (int64_t)r * a.stat_chunks, a.stat_chunks, zact);
                const LogSum l = log_sum_f32(s);
                const float H = entropy_f32(s, l), logp = log_prob_f32(s, l, zact);
                float gl, ge, surrogate, kl, w_left;
                loss_grad(a.loss, w, a.loss.logp_old[r], a.loss.logp_ref ? a.loss.logp_ref[r] : 0.f, a.loss.adv[r], logp, gl, ge,
                          surrogate, kl, w_left);
                k = coef_of(s.m, s.s == 0.f, l.inv_s, l.ls, H, gl, ge);
                hot = grad_any(k, zact) + k.g;
            }
        }
        const int v1 = min((c + 1) * per, parts.full);
        const int av = act >= parts.head && act < parts.head + parts.full * N ? (act - parts.head) / N : -1;
        for (int v = c * per + t; v < v1; v += TPR * NV) {
            uint4 raw[NV];
            if (k.zero == 0.f) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (v + TPR * j < v1) raw[j] = reinterpret_cast<const uint4 *>(body)[v + TPR * j];
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int vj = v + TPR * j;
                if (vj >= v1) break;
                // kFromFin and kFromLse: the chosen action's logit lies in its own vector
                float za = 0.f;
                if (SRC != kFromLoss && vj == av && k.zero == 0.f) za = to_f32(z[act]);
                grad_vec<T, STREAM>(dz, parts.head + vj * N, raw[j], k, same);
                if (vj == av && k.zero == 0.f) store(dz + act, SRC == kFromLoss ? hot : grad_any(k, za) + k.g);
            }
        }
        if (c == 0) {
            const int e = parts.edge(t);
            if (e >= 0) store(dz + e, k.zero != 0.f ? 0.f : grad_any(k, to_f32(z[e])) + (e == act ? k.g : 0.f));
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Heads of several segments, up to 4,096 columns.  A wave owns up to 64 consecutive rows, staged in LDS
// as fp32; `lanes` lanes share a (row, segment) item.  Everything a row needs stays in its wave, so there
// are no barriers between the steps: stage, sums of every item, a lane a row for the objective, gradients
// of every item in place, write back.  Rows of weight 0 are staged with the others; their gradient is 0.  Bound by
// vector instructions and the waits between the steps where rows are many (8,192 x 1,034 fp32: 23 us, 13 at a copy's
// rate; the vector units issue 60% of the time, LDS 30%, and a wave waits for 55% of its own) and by the chain of the
// steps where they are few (4,096 x 26: 8 us, of which the sums take 0.9, the rows' scalars 0.5, the gradients 0.8 and
// the arguments and first loads 2).
// ------------------------------------------------------------------------------------------------
enum TypesMode : int { kTypesLogp, kTypesDiff, kTypesLoss, kTypesGradLse, kTypesGradPairs, kTypesPairs };

constexpr int kTypesItems = 256;  // (row, segment) items of a wave at most
// Columns of a wave's rows at most, or one row: four workgroups' tiles fit a CU (32,768 x 1,034: 91 us, with 4,096
// columns 111).
constexpr int kTypesTile = 2304;
constexpr int kTypesTable = 2 * HARL_SELECT_MAX_SEGMENTS + 4;  // ints of a wave's copy of the segments' offsets and order

// Segments fall into two classes by length, so that a long segment's lanes do not idle at short ones.
struct TypesClass {
    int n, lanes, magic;  // segments of the class, lanes of an item, ceil(2^16 / n): p / n = p magic >> 16
};

struct TypesShape {
    int rows;             // rows of a wave
    TypesClass cls[2];    // long and short segments
    uint8_t order[HARL_SELECT_MAX_SEGMENTS];  // segments, the long ones first
    uint32_t magic;       // ceil(2^32 / a): e / a = umulhi(e, magic) for the tile's e
    int tile, bytes;      // floats of a wave's tile, bytes of a wave's LDS (a multiple of 16)
};

struct Item {
    double lp;
    float m, inv_s, H, ls;  // m = -inf: an empty segment; ls = log s
    int act, pad;
};

struct TypesIO {
    float *logp, *entropy, *lse;                            // outputs (kTypesLogp; kTypesLoss: logp)
    const float *logp_ref;                                  // kTypesDiff
    double *diff;                                           // [row] weight (logp - logp_ref)
    float2 *norm;                                           // [row][segment] {m, 1 / s}: out of kTypesDiff, into kTypesGradPairs
    LossArgs loss;                                          // kTypesLoss
    double *terms;                                          // [workgroup][3]
    const float *in_lse, *in_entropy, *g_logp, *g_entropy;  // kTypesGradLse
    const float *g_row;                                     // kTypesGradPairs
    float *loss_out;                                        // kTypesGradPairs: summed by the launch's last workgroup
    const double *pair_terms;
    int n_pairs;
    void *dz;
    int64_t ld_d;
};

__device__ __forceinline__ void wave_sync() {  // LDS serves a wave's accesses in order
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// max / sum over groups of L consecutive lanes, in every lane of the group: within 16 lanes by data-parallel
// moves, which cost a tenth of a shuffle
template <int L, typename Op>
__device__ __forceinline__ float group_reduce(float x, float none, Op op) {
    if constexpr (L == 64) return lanes_reduce<64>(x, none, op);
    if constexpr (L > 1) x = op(x, dpp<0xb1, 0xf>(x, none));   // quad_perm 1 0 3 2
    if constexpr (L > 2) x = op(x, dpp<0x4e, 0xf>(x, none));   // quad_perm 2 3 0 1
    if constexpr (L > 4) x = op(x, dpp<0x141, 0xf>(x, none));  // row_half_mirror: the other four of eight
    if constexpr (L > 8) x = op(x, dpp<0x140, 0xf>(x, none));  // row_mirror: the other eight of sixteen
    if constexpr (L > 16) x = op(x, __shfl_xor(x, 16));
    return x;
}

// A long segment [i0, i1) of row x by the wave, four columns a lane from 16-byte aligned places of the
// tile: f(i, values) with -inf in the places of other segments' columns.
template <typename F>
__device__ __forceinline__ void for_vectors(const float *x, const float *tile, int i0, int i1, int lane, F f) {
    const int at = (int)(x - tile);
    for (int i = ((at + i0) & ~3) - at + 4 * lane; i < i1; i += 256) {
        const float4 q = *reinterpret_cast<const float4 *>(x + i);
        float v[4] = {q.x, q.y, q.z, q.w};
        if (i < i0 || i + 4 > i1) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j < i0 || i + j >= i1) v[j] = -INFINITY;
        }
        f(i, v);
    }
}
__device__ __forceinline__ void put_vector(float *x, int from, int i0, int i1, const float (&f)[4]) {
    if (from >= i0 && from + 4 <= i1) {
        *reinterpret_cast<float4 *>(x + from) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (from + j >= i0 && from + j < i1) x[from + j] = f[j];
    }
}

template <typename T>
__device__ __forceinline__ void load_tile(const T *z, int64_t ld, int a, int n, uint32_t magic, int head, float *zs, int lane) {
    constexpr int N = kVec<T>;
    const int total = n * a;
    if (ld == a) {  // one run of columns: vectors behind the first aligned one, which zs was placed for
        if (lane < head && lane < total) zs[lane] = to_f32(z[lane]);
        const int full = max(total - head, 0) / N, last = head + full * N + lane;
        const uint4 *body = reinterpret_cast<const uint4 *>(z + head);
        float tail = 0.f;
        if (last < total) tail = to_f32(z[last]);
        for (int v = lane; v < full; v += 256) {
            uint4 raw[4];  // four loads in flight; beyond the end the last vector again
#pragma unroll
            for (int j = 0; j < 4; ++j) raw[j] = body[min(v + 64 * j, full - 1)];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (v + 64 * j >= full) break;
                float x[N];
                unpack(raw[j], x);
                float4 *d = reinterpret_cast<float4 *>(zs + head + (v + 64 * j) * N);
#pragma unroll
                for (int i = 0; i < N / 4; ++i) d[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            }
        }
        if (last < total) zs[last] = tail;
        return;
    }
    for (int e = lane; e < total; e += 256) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = min(e + 64 * j, total - 1), r = (int)__umulhi((uint32_t)i, magic);
            x[j] = to_f32(z[r * ld + (i - r * a)]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e + 64 * j < total) zs[e + 64 * j] = x[j];
    }
}

template <typename T>
__device__ __forceinline__ void store_tile(T *dz, int64_t ld, int a, int n, uint32_t magic, int head, const float *zs, int lane) {
    constexpr int N = kVec<T>;
    const int total = n * a;
    const int mis = (int)(reinterpret_cast<uintptr_t>(dz) / sizeof(T)) & (N - 1);
    if (ld == a && (mis ? N - mis : 0) == head) {
        if (lane < head && lane < total) store(dz + lane, zs[lane]);
        const int full = max(total - head, 0) / N;
        for (int v = lane; v < full; v += 64) {
            float x[N];
            const float4 *s = reinterpret_cast<const float4 *>(zs + head + v * N);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float4 f = s[i];
                x[4 * i] = f.x, x[4 * i + 1] = f.y, x[4 * i + 2] = f.z, x[4 * i + 3] = f.w;
            }
            reinterpret_cast<uint4 *>(dz + head)[v] = pack(x);
        }
        const int e = head + full * N + lane;
        if (e < total) store(dz + e, zs[e]);
        return;
    }
#pragma unroll 4
    for (int e = lane; e < total; e += 64) {
        const int r = (int)__umulhi((uint32_t)e, magic);
        store(dz + r * ld + (e - r * a), zs[e]);
    }
}

// A wave's rows in LDS.
struct WaveTile {
    float *tile, *zs;  // the tile, and its first row's first column
    Item *item;
    float2 *row;
    const int *off;
    int ns, a, lane;
};

// Sums of a class's items, L lanes each, and what follows from an item alone.  Lanes take four columns L apart
// at a time; places behind a segment read its last column and add 0.
template <int L, int MODE>
__device__ __forceinline__ void types_sums(const WaveTile &w, const TypesIO &io, const TypesClass &tc, const int *segs, int64_t r0, int n) {
    const int gl = w.lane % L;
    for (int i = w.lane / L; i < n * tc.n; i += 64 / L) {
        const int ri = i * tc.magic >> 16, s = segs[i - ri * tc.n], p = ri * w.ns + s, i0 = w.off[s], i1 = w.off[s + 1];
        const float *x = w.zs + ri * w.a;
        float m = -INFINITY;
        if constexpr (L == 64) {
            for_vectors(x, w.tile, i0, i1, w.lane, [&](int, const float (&f)[4]) { m = max_nan(max_nan(m, f[0]), max_nan(f[1], max_nan(f[2], f[3]))); });
        } else {
            for (int c = i0 + gl; c < i1; c += 4 * L)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = max_nan(m, x[min(c + j * L, i1 - 1)]);
        }
        m = group_reduce<L>(m, -INFINITY, [](float b, float c) { return max_nan(b, c); });
        const float ms = shift_of(m);
        Sums sum{m, 0.f, 0.f};
        const auto add_one = [&](float z, bool in) {
            const float y = in ? fmaxf((z - ms) * kLog2e, kYMin) : kYMin, e = exp2_hw(y);
            sum.s += e;
            sum.u = fmaf(e, y, sum.u);
        };
        if constexpr (L == 64) {
            for_vectors(x, w.tile, i0, i1, w.lane, [&](int, const float (&f)[4]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) add_one(f[j], true);
            });
        } else {
            for (int c = i0 + gl; c < i1; c += 4 * L)
#pragma unroll
                for (int j = 0; j < 4; ++j) add_one(x[min(c + j * L, i1 - 1)], c + j * L < i1);
        }
        const auto add = [](float b, float c) { return b + c; };
        sum.s = group_reduce<L>(sum.s, 0.f, add);
        sum.u = group_reduce<L>(sum.u, 0.f, add);
        if (!(m < INFINITY)) sum.s = sum.u = __builtin_nanf("");
        if (gl != 0) continue;
        const float zact = x[min(max(w.item[p].act, i0), i1 - 1)];
        const LogSum l = log_sum_f32(sum);
        const int64_t e = r0 * w.ns + p;
        w.item[p].m = sum.s == 0.f ? -INFINITY : m;
        w.item[p].inv_s = l.inv_s;
        if (MODE == kTypesDiff || MODE == kTypesPairs) {  // long sums of small differences follow: 64 bits
            w.item[p].lp = log_prob(sum, zact);
            if (MODE == kTypesDiff) io.norm[e] = make_float2(sum.s == 0.f ? -INFINITY : m, l.inv_s);
            continue;
        }
        const float H = entropy_f32(sum, l);
        w.item[p].lp = (double)log_prob_f32(sum, l, zact);
        w.item[p].H = H;
        w.item[p].ls = l.ls;
        if (MODE == kTypesLogp && io.entropy) io.entropy[e] = H;
        if (MODE == kTypesLogp && io.lse) {
            io.lse[2 * e] = m;
            io.lse[2 * e + 1] = sum.s == 0.f ? 0.f : l.ls;
        }
    }
}

// Gradients of a class's items in the place of their logits.
template <int L, int MODE>
__device__ __forceinline__ void types_grads(const WaveTile &w, const TypesIO &io, const TypesClass &tc, const int *segs, int64_t r0, int n) {
    const int gl = w.lane % L;
    for (int i = w.lane / L; i < n * tc.n; i += 64 / L) {
        const int ri = i * tc.magic >> 16, s = segs[i - ri * tc.n], p = ri * w.ns + s, i0 = w.off[s], i1 = w.off[s + 1];
        const int64_t e = r0 * w.ns + p;
        float *x = w.zs + ri * w.a;
        const float2 g = w.row[ri];
        float m, inv_s, rest = 0.f, H = 0.f;
        if (MODE == kTypesLoss || MODE == kTypesPairs) {
            m = w.item[p].m, inv_s = w.item[p].inv_s;
            if (MODE == kTypesLoss) H = w.item[p].H, rest = w.item[p].ls;
        } else if (MODE == kTypesGradPairs) {
            m = -INFINITY, inv_s = 1.f;
            if (g.x != 0.f) m = io.norm[e].x, inv_s = io.norm[e].y;
        } else {
            m = io.in_lse[2 * e], rest = io.in_lse[2 * e + 1];
            inv_s = exp2_hw(-rest * kLog2e);
            if (g.y != 0.f) H = io.in_entropy[e];
        }
        const RowCoef k = coef_of(m, m == -INFINITY, inv_s, rest, H, g.x, g.y);
        if (k.zero != 0.f) {
            for (int c = i0 + gl; c < i1; c += L) x[c] = 0.f;
            continue;
        }
        const auto each = [&](auto ent) {
            constexpr bool ENT = decltype(ent)::value;
            if constexpr (L == 64) {
                for_vectors(x, w.tile, i0, i1, w.lane, [&](int from, float (&f)[4]) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = grad_of<ENT>(k, f[j]);
                    put_vector(x, from, i0, i1, f);
                });
            } else {
                for (int c = i0 + gl; c < i1; c += 4 * L) {
                    float f[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = grad_of<ENT>(k, x[min(c + j * L, i1 - 1)]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c + j * L < i1) x[c + j * L] = f[j];
                }
            }
        };
        if (k.e != 0.f) each(std::true_type());
        else each(std::false_type());
        const int act = min(max(w.item[p].act, i0), i1 - 1);
        if (gl == 0) x[act] += k.g;  // behind the group's writes: LDS serves a wave in order
    }
}

// f(lanes of an item, class, its segments) for both classes
template <typename F>
__device__ __forceinline__ void for_classes(const TypesShape &sh, const int *order, F f) {
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
        const TypesClass tc = sh.cls[c];
        const int *segs = order + (c ? sh.cls[0].n : 0);
        if (tc.n == 0) break;
        switch (tc.lanes) {
            case 1: f(std::integral_constant<int, 1>(), tc, segs); break;
            case 2: f(std::integral_constant<int, 2>(), tc, segs); break;
            case 4: f(std::integral_constant<int, 4>(), tc, segs); break;
            case 8: f(std::integral_constant<int, 8>(), tc, segs); break;
            case 16: f(std::integral_constant<int, 16>(), tc, segs); break;
            case 32: f(std::integral_constant<int, 32>(), tc, segs); break;
            default: f(std::integral_constant<int, 64>(), tc, segs); break;
        }
    }
}

template <typename T, int MODE>
__global__ __launch_bounds__(kThreads, 5) void k_types(Rows q, TypesShape sh, TypesIO io) {
    constexpr int N = kVec<T>;
    constexpr bool kGradOnly = MODE == kTypesGradLse || MODE == kTypesGradPairs;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    if (MODE == kTypesGradPairs && io.loss_out && blockIdx.x == gridDim.x - 1) {
        pairs_sum(io.pair_terms, io.n_pairs, io.loss_out);
        return;
    }
    const unsigned groups = gridDim.x - (MODE == kTypesGradPairs && io.loss_out ? 1 : 0);
    const int wv = threadIdx.x / 64, lane = threadIdx.x % 64, ns = q.n_seg, a = q.a;
    const int items_max = sh.rows * ns;
    char *mine = smem + wv * sh.bytes;
    float *tile = reinterpret_cast<float *>(mine);
    Item *item = reinterpret_cast<Item *>(mine + (size_t)sh.tile * 4);
    float2 *row = reinterpret_cast<float2 *>(item + items_max);  // a row's gradients of log-probability and entropy
    int *off = reinterpret_cast<int *>(mine + sh.bytes) - kTypesTable, *order = off + HARL_SELECT_MAX_SEGMENTS + 1;
    const int my_off = lane <= ns ? q.off[lane] : 0, my_order = lane < ns ? sh.order[lane] : 0;
    const int lo = q.seq_ptr ? clamp_row(q.seq_ptr[0], q.M) : 0, hi = q.seq_ptr ? clamp_row(q.seq_ptr[q.n_seq], q.M) : q.M;
    double acc[3] = {0.0, 0.0, 0.0};
    for (int64_t r0 = lo + ((int64_t)blockIdx.x * 4 + wv) * sh.rows; r0 < hi; r0 += (int64_t)groups * 4 * sh.rows) {
        const int n = (int)min((int64_t)sh.rows, hi - r0), items = n * ns;
        const T *z = static_cast<const T *>(q.z) + r0 * q.ld;
        const int mis = (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (N - 1), head = mis ? N - mis : 0;
        float *zs = tile + ((4 - head) & 3);
        // everything else of the rows is loaded beside their logits
        const int act0 = lane < items ? q.act[r0 * ns + lane] : 0;
        const bool own = lane < n;
        const int64_t r = r0 + lane;
        float w = 1.f, old = 0.f, ref = 0.f, adv = 0.f;
        if (own && MODE == kTypesDiff) {
            if (q.weight) w = q.weight[r];
            if (io.logp_ref) ref = io.logp_ref[r];
        }
        if (own && MODE == kTypesLoss) {
            w = io.loss.weight ? io.loss.weight[r] : io.loss.inv_m;
            old = io.loss.logp_old[r];
            adv = io.loss.adv[r];
            if (io.loss.logp_ref) ref = io.loss.logp_ref[r];
        }
        load_tile<T>(z, q.ld, a, n, sh.magic, head, zs, lane);
        if (lane < items) item[lane].act = act0;
        for (int p = lane + 64; p < items; p += 64) item[p].act = q.act[r0 * ns + p];
        if (lane <= ns) off[lane] = my_off;
        if (lane < ns) order[lane] = my_order;
        wave_sync();
        const WaveTile wt{tile, zs, item, row, off, ns, a, lane};
        if (!kGradOnly) {
            for_classes(sh, order, [&](auto L, const TypesClass &tc, const int *segs) { types_sums<decltype(L)::value, MODE>(wt, io, tc, segs, r0, n); });
            wave_sync();
        }
        if (own) {
            double lp = 0.0, H = 0.0;
            if (!kGradOnly)
                for (int s = 0; s < ns; ++s) {
                    lp += item[lane * ns + s].lp;
                    if (MODE == kTypesLoss) H += (double)item[lane * ns + s].H;
                }
            float2 g = make_float2(0.f, 0.f);
            if (MODE == kTypesLogp) io.logp[r] = (float)lp;
            if (MODE == kTypesDiff) io.diff[r] = w == 0.f ? 0.0 : (double)w * (lp - (double)ref);
            if (MODE == kTypesLoss) {
                if (w != 0.f) {
                    float surrogate, kl, w_left;
                    loss_grad(io.loss, w, old, ref, adv, (float)lp, g.x, g.y, surrogate, kl, w_left);
                    acc[0] -= (double)w_left * (double)surrogate;
                    acc[1] += (double)w_left * (double)kl;
                    acc[2] += (double)w * H;
                }
                if (io.logp) io.logp[r] = w != 0.f ? (float)lp : 0.f;
            }
            if (MODE == kTypesGradLse) g = make_float2(io.g_logp[r], io.g_entropy ? io.g_entropy[r] : 0.f);
            if (MODE == kTypesGradPairs) g.x = io.g_row[r];
            row[lane] = g;
        }
        wave_sync();
        if (MODE == kTypesLogp || MODE == kTypesDiff || !io.dz) continue;
        for_classes(sh, order, [&](auto L, const TypesClass &tc, const int *segs) { types_grads<decltype(L)::value, MODE>(wt, io, tc, segs, r0, n); });
        wave_sync();
        store_tile<T>(static_cast<T *>(io.dz) + r0 * io.ld_d, io.ld_d, a, n, sh.magic, head, zs, lane);
        wave_sync();
    }
    if (MODE == kTypesLoss) {
        __shared__ double part[4][3];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const double v = wave_sum(acc[c]);
            if (lane == 0) part[wv][c] = v;
        }
        __syncthreads();
        if (threadIdx.x < 3) {
            double v = 0.0;
            for (int w = 0; w < 4; ++w) v += part[w][threadIdx.x];
            io.terms[(int64_t)blockIdx.x * 3 + threadIdx.x] = v;
        }
    }
}

// The whole preference loss of short tracks: pair p by workgroup p (stepping over pairs), its rows dealt to the
// four waves.  Rows that the waves' tiles hold stay there between their sums and their gradients; longer
// tracks are staged and summed once more for the gradients.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_types_pairs(Rows q, TypesShape sh, PairArgs pa, double *__restrict__ terms,
                                                          float *__restrict__ ratio, T *dz, int64_t ld_d) {
    constexpr int N = kVec<T>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ double part[2][2][4];
    const int wv = threadIdx.x / 64, lane = threadIdx.x % 64, ns = q.n_seg, a = q.a;
    char *mine = smem + wv * sh.bytes;
    float *tile = reinterpret_cast<float *>(mine);
    Item *item = reinterpret_cast<Item *>(mine + (size_t)sh.tile * 4);
    float2 *row = reinterpret_cast<float2 *>(item + sh.rows * ns);
    int *off = reinterpret_cast<int *>(mine + sh.bytes) - kTypesTable, *order = off + HARL_SELECT_MAX_SEGMENTS + 1;
    if (lane <= ns) off[lane] = q.off[lane];
    if (lane < ns) order[lane] = sh.order[lane];
    const TypesIO io{};
    int half = 0;
    for (int64_t p = blockIdx.x; p < pa.n_pairs; p += gridDim.x) {
        const int lo = clamp_row(pa.seq_ptr[2 * p], q.M), mid = clamp_row(pa.seq_ptr[2 * p + 1], q.M);
        const int hi = clamp_row(pa.seq_ptr[2 * p + 2], q.M);
        const int rows = min(max((hi - lo + 3) / 4, 1), sh.rows);  // of a wave's tile
        const bool once = hi - lo <= 4 * rows;
        double s[2] = {0.0, 0.0};
        float w = 0.f;
        const auto stage = [&](int64_t r0, int n) {  // rows r0 .. r0 + n - 1: staged, summed; this lane's weighted log ratio
            const int items = n * ns;
            const T *z = static_cast<const T *>(q.z) + r0 * q.ld;
            const int mis = (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (N - 1), head = mis ? N - mis : 0;
            const WaveTile wt{tile, tile + ((4 - head) & 3), item, row, off, ns, a, lane};
            const int act0 = lane < items ? q.act[r0 * ns + lane] : 0;
            float ref = 0.f;
            w = 0.f;
            if (lane < n) {
                w = pa.weight ? pa.weight[r0 + lane] : 1.f;
                if (pa.logp_ref) ref = pa.logp_ref[r0 + lane];
            }
            load_tile<T>(z, q.ld, a, n, sh.magic, head, wt.zs, lane);
            if (lane < items) item[lane].act = act0;
            for (int i = lane + 64; i < items; i += 64) item[i].act = q.act[r0 * ns + i];
            wave_sync();
            for_classes(sh, order, [&](auto L, const TypesClass &tc, const int *segs) { types_sums<decltype(L)::value, kTypesPairs>(wt, io, tc, segs, r0, n); });
            wave_sync();
            double d = 0.0;
            if (w != 0.f) {
                for (int i = 0; i < ns; ++i) d += item[lane * ns + i].lp;
                d = (double)w * (d - (double)ref);
            }
            return d;
        };
        for (int64_t r0 = lo + (int64_t)wv * rows; r0 < hi; r0 += 4 * rows) {
            const int n = (int)min((int64_t)rows, hi - r0);
            const double d = stage(r0, n);
            s[r0 + lane >= mid ? 1 : 0] += lane < n ? d : 0.0;
        }
        for (int side = 0; side < 2; ++side) {
            const double v = wave_sum(s[side]);
            if (lane == 0) part[half][side][wv] = v;
        }
        __syncthreads();
        double R[2];
        for (int side = 0; side < 2; ++side) R[side] = (part[half][side][0] + part[half][side][1]) + (part[half][side][2] + part[half][side][3]);
        half ^= 1;  // one barrier a pair
        const double g = pair_terms(pa, p, R, threadIdx.x == 0, terms, ratio);
        if (!dz) continue;
        for (int64_t r0 = lo + (int64_t)wv * rows; r0 < hi; r0 += 4 * rows) {
            const int n = (int)min((int64_t)rows, hi - r0);
            if (!once) stage(r0, n);
            const T *z = static_cast<const T *>(q.z) + r0 * q.ld;
            const int mis = (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T)) & (N - 1), head = mis ? N - mis : 0;
            const WaveTile wt{tile, tile + ((4 - head) & 3), item, row, off, ns, a, lane};
            if (lane < n) row[lane] = make_float2(w == 0.f ? 0.f : (float)((double)w * (r0 + lane >= mid ? -g : g)), 0.f);
            wave_sync();
            for_classes(sh, order, [&](auto L, const TypesClass &tc, const int *segs) { types_grads<decltype(L)::value, kTypesPairs>(wt, io, tc, segs, r0, n); });
            wave_sync();
            store_tile<T>(dz + r0 * ld_d, ld_d, a, n, sh.magic, head, wt.zs, lane);
            wave_sync();
        }
    }
}

Rows rows_of(const harl_policy_head *h, const void *z, int64_t ld, int32_t M, const int32_t *act) {
    Rows q{};
    q.z = z;
    q.ld = ld;
    q.M = M;
    q.a = h->a;
    q.n_seg = h->n_seg;
    q.act = act;
    for (int s = 0; s <= h->n_seg; ++s) q.off[s] = h->seg_offsets[s];
    return q;
}

unsigned grid_for(int64_t items) { return (unsigned)std::min<int64_t>(std::max<int64_t>(items, 1), kMaxGrid); }

// Which kernels take a head: several segments go by types, and so does one of few columns, where a wave a row
// leaves lanes idle.  65,536 rows by rows / by types, us:
//                            24 columns  128      192      256      384      512      700
//   clipped loss       fp32  35 / 12   36 / 24  40 / 41  42 / 54  51 / 70  56 / 81
//                      bf16  41 / 12   41 / 22  41 / 32  42 / 42  46 / 54  48 / 65
//   log-probabilities  fp32  56 / 12   59 / 27  64 / 46  69 / 64  79 / 85  90 / 106
//   and gradient       bf16  71 / 12   73 / 22  73 / 35  74 / 45  79 / 58  83 / 73  96 / 107
//   preference loss    fp32  64 / 19   70 / 36  73 / 55  77 / 74  83 / 96  97 / 118
//                      bf16  79 / 19   84 / 30  86 / 44  86 / 56  88 / 68  91 / 83  104 / 120
// bf16 rows cross at 1.3 to 2 times the columns of fp32 ones, so that one number of columns suits one type: fp32 rows of
// 257 to 512 columns lose up to 21% to it, bf16 rows of 129 to 255 in the clipped loss up to 28%.  Rows with columns
// between them are staged an element at a time and cross earlier (log-probabilities and gradient, fp32 192 columns
// 73 / 67, 256 76 / 85, bf16 256 81 / 71, 512 91 / 124).
// (One column has no division by multiplication; it goes by rows.)
constexpr int kTypesLossColumns = 128, kTypesColumns = 512;
bool by_types(const harl_policy_head *h, int most) { return h->n_seg > 1 || (h->a > 1 && h->a <= most); }

// ---- launch shapes of one-segment heads ----
int vec_of(const harl_policy_head *h) { return h->dtype == HARL_BF16 ? 8 : 4; }

constexpr int kSplitItems = 1024;  // items that a launch of few rows is cut into
constexpr int kMaxChunks = 64;     // a wave joins a row's chunks
constexpr int kLossGrid = 8192;    // workgroups of k_loss: its terms
constexpr int kPrefChunk = 2048;   // vectors of a preference row's chunk at most

// Chunks of a row: rows that leave the machine idle are cut until there are about kSplitItems items, none of
// fewer than 512 vectors (two a thread).  The clipped loss then reads its logits twice.  Rows cut / whole in k_loss, us:
// 131,072 bf16 columns, 16 rows 16 / 23, 64 17 / 26, 128 26 / 28, 256 49 / 36, 512 86 / 67, 1,000 176 / 128; 60,000, 128
// rows 17 / 17, 1,000 85 / 69; 20,011 fp32 columns, 16 rows 12 / 10, 256 18 / 14, 1,000 58 / 44: from some 150 rows on
// the cut costs that loss more than it gives, up to 47% (65,521 fp32 columns, 1,000 rows 168 / 115).
int chunks_for(const harl_policy_head *h, int32_t M) {
    const int64_t vecs = h->a / vec_of(h);
    return (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(kSplitItems, M), (int64_t)kMaxChunks, vecs / 512}));
}

// The preference loss joins a row's chunks anyway, so all its rows are cut: whole rows of 8,192 vectors
// leave the machine half empty in the last of two rounds.
int pref_chunks_for(const harl_policy_head *h, int32_t M) {
    return (int)std::min<int64_t>(kMaxChunks, std::max<int64_t>(chunks_for(h, M), ceil_div(h->a / vec_of(h), kPrefChunk)));
}

template <typename T, int OUT>
void launch_stats_as(const Rows &q, int chunks, const StatOut &o, hipStream_t stream) {
    const int per = (int)ceil_div(std::max(q.a / kVec<T>, 1), chunks);
    const int64_t items = (int64_t)q.M * chunks;
    if (chunks == 1 && q.a / kVec<T> <= 512)  // a wave a row: no barrier, four rows a workgroup
        hipLaunchKernelGGL((k_stats<T, 64, 4, OUT>), dim3(grid_for(ceil_div(items, 4))), dim3(kThreads), 0, stream, q, chunks, per, o);
    else
        hipLaunchKernelGGL((k_stats<T, 256, 8, OUT>), dim3(grid_for(items)), dim3(kThreads), 0, stream, q, chunks, per, o);
}

template <int OUT>
int launch_wide_stats(const harl_policy_head *h, const Rows &q, int chunks, const StatOut &o, hipStream_t stream) {
    if (h->dtype == HARL_BF16) launch_stats_as<uint16_t, OUT>(q, chunks, o, stream);
    else launch_stats_as<float, OUT>(q, chunks, o, stream);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

template <int SRC>
int launch_wide_grad(const harl_policy_head *h, const Rows &q, const GradSrc &a, hipStream_t stream) {
    const int vecs = std::max(h->a / vec_of(h), 1);
    const int chunks = (int)ceil_div(vecs, 1024), per = (int)ceil_div(vecs, chunks);
    const bool wave = SRC != kFromLoss && vecs <= 256;  // (few rows' loss has more)
    const unsigned grid = (a.dz ? grid_for(ceil_div((int64_t)q.M * chunks, wave ? 4 : 1)) : 0) + (SRC == kFromLse ? 0 : 1);
    // A large gradient that stays in the caches is written back while the next pass reads its logits: 134 MB
    // take 84 us with it and 74 past them, 500 MB 254 and 229; 42 MB the same either way.
    const bool past = SRC != kFromLoss && (int64_t)q.M * h->a * (h->dtype == HARL_BF16 ? 2 : 4) > ((int64_t)64 << 20);
    constexpr bool kPast = SRC != kFromLoss;
    constexpr int kWave = SRC != kFromLoss ? 64 : kThreads;
    const auto pick = [&](auto like) {
        using T = decltype(like);
        return wave ? (past ? k_grad<T, SRC, kPast, kWave> : k_grad<T, SRC, false, kWave>)
                    : (past ? k_grad<T, SRC, kPast, kThreads> : k_grad<T, SRC, false, kThreads>);
    };
    const auto kernel = h->dtype == HARL_BF16 ? pick(uint16_t()) : pick(float());
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, stream, q, chunks, per, a);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

template <typename T, int TPR, int NV>
unsigned launch_loss_as(const Rows &q, const LossArgs &a, const LossOut &o, hipStream_t stream) {
    constexpr int WG = TPR < kThreads ? kThreads : TPR;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(q.M, WG / TPR), kLossGrid);
    if (o.dz) hipLaunchKernelGGL((k_loss<T, TPR, NV, true>), dim3(grid), dim3(WG), 0, stream, q, a, o);
    else hipLaunchKernelGGL((k_loss<T, TPR, NV, false>), dim3(grid), dim3(WG), 0, stream, q, a, o);
    return grid;
}

// The shape whose registers hold a row; the widest rows go in part through memory twice.
template <typename T>
unsigned launch_loss(const Rows &q, const LossArgs &a, const LossOut &o, hipStream_t stream) {
    const int v = q.a / kVec<T>;
    if (v <= 64) return launch_loss_as<T, 64, 1>(q, a, o, stream);
    if (v <= 128) return launch_loss_as<T, 64, 2>(q, a, o, stream);
    if (v <= 256) return launch_loss_as<T, 64, 4>(q, a, o, stream);
    if (v <= 512) return launch_loss_as<T, 64, 8>(q, a, o, stream);
    if (v <= 1024) return launch_loss_as<T, 256, 4>(q, a, o, stream);
    if (v <= 2048) return launch_loss_as<T, 256, 8>(q, a, o, stream);
    if (v <= 4096) return launch_loss_as<T, 256, 16>(q, a, o, stream);
    if (v <= 8192) return launch_loss_as<T, 512, 16>(q, a, o, stream);
    return launch_loss_as<T, 1024, 16>(q, a, o, stream);
}

// ---- launch shapes of heads of several segments ----
// With `want` a wave's tile holds that many rows, or as many as it may.
TypesShape types_shape(const harl_policy_head *h, int32_t M, int64_t want = 0) {
    TypesShape s{};
    int longest = 1;
    for (int i = 0; i < h->n_seg; ++i) longest = std::max(longest, h->seg_offsets[i + 1] - h->seg_offsets[i]);
    // four waves a SIMD, what their registers allow at once; more rows a wave share its fixed work (8,192 x 1,034:
    // 30.8 us with a row a wave, 25.9 with two, 28.4 with three; 65,536 x 26: 19.7 with 8, 16.1 with 16, 19.0 with 32)
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>({64, kTypesItems / h->n_seg, kTypesTile / h->a}));
    s.rows = (int)std::max<int64_t>(1, std::min<int64_t>(most, want ? want : ceil_div(M, 4096)));
    // long segments: more than a quarter of the longest, where that has more than 64 columns (20,000 rows of 185 and
    // five times 3: 32.1 us in one class, 20.7 in two); below, a second class costs what it gives
    const int split = longest > 64 ? longest : 0;
    int at = 0;
    for (int c = 0; c < 2; ++c) {
        int top = 0;
        for (int i = 0; i < h->n_seg; ++i) {
            const int len = h->seg_offsets[i + 1] - h->seg_offsets[i];
            if ((len * 4 > split) == (c == 1)) continue;
            s.order[at++] = (uint8_t)i;
            ++s.cls[c].n;
            top = std::max(top, len);
        }
        // lanes for about 16 columns each, more where a wave has too few items for its lanes
        const int items = s.rows * s.cls[c].n;
        int lanes = 1;
        while (lanes < 64 && lanes * 16 < top) lanes *= 2;
        while (lanes < 64 && lanes < top && lanes * 2 * items <= 64) lanes *= 2;
        s.cls[c].lanes = lanes;
        s.cls[c].magic = s.cls[c].n ? (65536 + s.cls[c].n - 1) / s.cls[c].n : 0;
    }
    s.magic = (uint32_t)((((uint64_t)1 << 32) + h->a - 1) / h->a);
    s.tile = (int)round_up((int64_t)s.rows * h->a + 4, 4);
    s.bytes = s.tile * 4 + s.rows * h->n_seg * (int)sizeof(Item) + (int)round_up(s.rows * 8, 16) + kTypesTable * 4;
    return s;
}

template <typename T, int MODE>
int launch_types_as(const harl_policy_head *h, const Rows &q, const TypesIO &io, unsigned grid, unsigned extra, const TypesShape &s,
                    hipStream_t stream) {
    const size_t lds = 4 * (size_t)s.bytes;
    if (const int rc = ensure_dynamic_lds(reinterpret_cast<const void *>(k_types<T, MODE>), lds)) return rc;
    hipLaunchKernelGGL((k_types<T, MODE>), dim3(grid + extra), dim3(kThreads), lds, stream, q, s, io);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

unsigned types_grid(const TypesShape &s, int32_t M) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(M, 4 * (int64_t)s.rows), kLossGrid));
}

template <int MODE>
int launch_types(const harl_policy_head *h, const Rows &q, const TypesIO &io, hipStream_t stream) {
    const TypesShape s = types_shape(h, q.M);
    const unsigned grid = types_grid(s, q.M), extra = MODE == kTypesGradPairs && io.loss_out ? 1 : 0;
    return h->dtype == HARL_BF16 ? launch_types_as<uint16_t, MODE>(h, q, io, grid, extra, s, stream)
                                 : launch_types_as<float, MODE>(h, q, io, grid, extra, s, stream);
}

// The workspace: statistics per (row, chunk), what the preference loss keeps of a row, loss terms.
struct Ws {
    Stat *stat;
    RowFin *fin;
    double *diff;
    float2 *norm;
    float *g_row;
    double *terms;
    size_t bytes;
};

struct WsCounts {
    int64_t stat, fin, rows, norm, terms;
};

Ws ws_layout(const WsCounts &n, char *base) {
    Ws w{};
    int64_t off = 0;
    auto take = [&](int64_t bytes) {
        char *p = base ? base + off : nullptr;
        off += round_up(bytes, 256);
        return p;
    };
    w.stat = reinterpret_cast<Stat *>(take(n.stat * (int64_t)sizeof(Stat)));
    w.fin = reinterpret_cast<RowFin *>(take(n.fin * (int64_t)sizeof(RowFin)));
    w.diff = reinterpret_cast<double *>(take(n.rows * 8));
    w.norm = reinterpret_cast<float2 *>(take(n.norm * 8));
    w.g_row = reinterpret_cast<float *>(take(n.rows * 4));
    w.terms = reinterpret_cast<double *>(take(n.terms * 8));
    w.bytes = (size_t)std::max<int64_t>(off, 256);
    return w;
}

// Rows in chunks: at most rows + kSplitItems items, and none in chunks from kSplitItems rows on.
Ws logp_ws(const harl_policy_head *h, int64_t M, char *base) {
    return ws_layout(WsCounts{!by_types(h, kTypesColumns) ? std::min<int64_t>(M, kSplitItems) + kSplitItems : 0, 0, 0, 0, 0}, base);
}
Ws loss_ws(const harl_policy_head *h, int64_t M, char *base) {
    return ws_layout(WsCounts{!by_types(h, kTypesLossColumns) ? std::min<int64_t>(M, kSplitItems) + kSplitItems : 0, 0, 0, 0,
                              3 * std::min<int64_t>(M, kLossGrid)}, base);
}
Ws preference_ws(const harl_policy_head *h, int64_t rows, int64_t pairs, char *base) {
    const int64_t cut = std::min<int64_t>(kMaxChunks, std::max<int64_t>(1, ceil_div(h->a / vec_of(h), kPrefChunk)));
    return ws_layout(!by_types(h, kTypesColumns) ? WsCounts{rows * cut + kSplitItems, rows, 0, 0, 4 * pairs}
                                   : WsCounts{0, 0, rows, rows * h->n_seg, 4 * pairs}, base);
}

}  // namespace

size_t objective_logp_ws_bytes(const harl_policy_head *head, int32_t M) { return logp_ws(head, M, nullptr).bytes; }

size_t objective_loss_ws_bytes(const harl_policy_head *head, int32_t M) { return loss_ws(head, M, nullptr).bytes; }

size_t objective_preference_ws_bytes(const harl_policy_head *head, int32_t n_rows, int32_t n_pairs) {
    return preference_ws(head, n_rows, n_pairs, nullptr).bytes;
}

int policy_logp_launch(const harl_policy_head *head, const void *logits, int64_t ld, int32_t M, const int32_t *actions,
                       float *logp, float *entropy, float *lse, void *ws, hipStream_t stream) {
    const Ws w = logp_ws(head, M, static_cast<char *>(ws));
    const Rows q = rows_of(head, logits, ld, M, actions);
    if (by_types(head, kTypesColumns)) {
        TypesIO io{};
        io.logp = logp;
        io.entropy = entropy;
        io.lse = lse;
        return launch_types<kTypesLogp>(head, q, io, stream);
    }
    const int chunks = chunks_for(head, M);
    const StatOut o{w.stat, logp, entropy, lse};
    // few rows of up to 256 KB: a workgroup of 16 waves reads one in 2 us, less than a second launch takes
    const int vecs = head->a / vec_of(head);
    if (chunks > 1 && vecs <= 16384) {
        if (head->dtype == HARL_BF16)
            hipLaunchKernelGGL((k_stats<uint16_t, 1024, 8, kLogp>), dim3(grid_for(M)), dim3(1024), 0, stream, q, 1, vecs, o);
        else
            hipLaunchKernelGGL((k_stats<float, 1024, 8, kLogp>), dim3(grid_for(M)), dim3(1024), 0, stream, q, 1, vecs, o);
        HARL_HIP_CHECK(hipGetLastError());
        return HARL_OK;
    }
    if (chunks == 1) return launch_wide_stats<kLogp>(head, q, 1, o, stream);
    if (const int rc = launch_wide_stats<kPartial>(head, q, chunks, o, stream)) return rc;
    hipLaunchKernelGGL(k_logp_join, dim3(grid_for(ceil_div(M, 64))), dim3(64), 0, stream, w.stat, M, chunks, o);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

int policy_logp_grad_launch(const harl_policy_head *head, const void *logits, int64_t ld, int32_t M,
                            const int32_t *actions, const float *lse, const float *entropy, const float *g_logp,
                            const float *g_entropy, void *dlogits, int64_t ld_d, hipStream_t stream) {
    const Rows q = rows_of(head, logits, ld, M, actions);
    if (by_types(head, kTypesColumns)) {
        TypesIO io{};
        io.in_lse = lse;
        io.in_entropy = entropy;
        io.g_logp = g_logp;
        io.g_entropy = g_entropy;
        io.dz = dlogits;
        io.ld_d = ld_d;
        return launch_types<kTypesGradLse>(head, q, io, stream);
    }
    GradSrc a{};
    a.lse = lse;
    a.entropy = entropy;
    a.g_logp = g_logp;
    a.g_entropy = g_entropy;
    a.dz = dlogits;
    a.ld_d = ld_d;
    return launch_wide_grad<kFromLse>(head, q, a, stream);
}

int policy_loss_launch(const harl_policy_head *head, const harl_policy_loss_config *cfg, const void *logits, int64_t ld,
                       int32_t M, const int32_t *actions, const float *logp_old, const float *logp_ref,
                       const float *adv, const float *weight, void *dlogits, int64_t ld_d, float *logp, float *loss,
                       void *ws, hipStream_t stream) {
    const Ws w = loss_ws(head, M, static_cast<char *>(ws));
    Rows q = rows_of(head, logits, ld, M, actions);
    q.weight = weight;
    const LossArgs a{logp_old, logp_ref, adv, weight, cfg->clip_low, cfg->clip_high, cfg->w_kl, cfg->w_entropy, 1.f / (float)M};
    int64_t n_terms = 0;
    if (by_types(head, kTypesLossColumns)) {
        TypesIO io{};
        io.loss = a;
        io.logp = logp;
        io.terms = w.terms;
        io.dz = dlogits;
        io.ld_d = ld_d;
        if (const int rc = launch_types<kTypesLoss>(head, q, io, stream)) return rc;
        n_terms = types_grid(types_shape(head, M), M);
    } else {
        const int chunks = chunks_for(head, M);
        if (chunks > 1) {
            const StatOut o{w.stat, nullptr, nullptr, nullptr};
            if (const int rc = launch_wide_stats<kPartial>(head, q, chunks, o, stream)) return rc;
            GradSrc g{};
            g.stat = w.stat;
            g.stat_chunks = chunks;
            g.loss = a;
            g.logp = logp;
            g.loss_out = loss;
            g.dz = dlogits;
            g.ld_d = ld_d;
            return launch_wide_grad<kFromLoss>(head, q, g, stream);
        }
        const LossOut o{dlogits, ld_d, logp, w.terms};
        n_terms = head->dtype == HARL_BF16 ? launch_loss<uint16_t>(q, a, o, stream) : launch_loss<float>(q, a, o, stream);
        HARL_HIP_CHECK(hipGetLastError());
    }
    if (!loss) return HARL_OK;
    hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(kThreads), 0, stream, w.terms, n_terms, cfg->w_kl, cfg->w_entropy, loss);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

int preference_loss_launch(const harl_policy_head *head, const harl_preference_config *cfg, const void *logits,
                           int64_t ld, int32_t n_rows, const int32_t *actions, const float *logp_ref,
                           const float *weight, const int32_t *seq_ptr, int32_t n_pairs, void *dlogits, int64_t ld_d,
                           float *ratio, float *loss, void *ws, hipStream_t stream) {
    const Ws w = preference_ws(head, n_rows, n_pairs, static_cast<char *>(ws));
    Rows q = rows_of(head, logits, ld, n_rows, actions);
    q.weight = weight;
    q.seq_ptr = seq_ptr;
    q.n_seq = 2 * n_pairs;
    const bool grad = dlogits && n_rows > 0, types = by_types(head, kTypesColumns);
    const int chunks = !types && n_rows > 0 ? pref_chunks_for(head, n_rows) : 1;
    const PairArgs a{logp_ref, weight, seq_ptr, n_rows, chunks, n_pairs, cfg->beta, cfg->smoothing};
    if (n_rows > 0 && types) {
        // short tracks, and not more pairs than the machine takes at once: one launch in the place of three (256
        // pairs of 1 to 20 rows of 26 columns 20.9 -> 12.7 us; but 3,000 of them 30 -> 41 us, 30 of up to 100 rows
        // 16.6 -> 20.6).  The tracks' lengths lie on the device: the rule sees their average, and where one pair holds
        // nearly all rows one workgroup does nearly all the work (60,416 rows of 26 columns in 1,024 pairs 8.3 ms, in
        // three launches 0.12, and evenly dealt 24 and 23 us; 7,424 rows in 256 pairs 1.0 ms and 27 us, 12 and 18).
        const TypesShape s = types_shape(head, n_rows, ceil_div(n_rows, 2 * (int64_t)n_pairs));  // twice the average pair
        if (n_pairs <= 1024 && (int64_t)n_rows * head->a <= (int64_t)n_pairs * 1536) {
            const size_t lds = 4 * (size_t)s.bytes;
            const auto launch = [&](auto kernel, auto *dz) -> int {
                if (const int rc = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), lds)) return rc;
                hipLaunchKernelGGL(kernel, dim3(grid_for(n_pairs)), dim3(kThreads), lds, stream, q, s, a, w.terms, ratio, dz, ld_d);
                HARL_HIP_CHECK(hipGetLastError());
                return HARL_OK;
            };
            if (const int rc = head->dtype == HARL_BF16 ? launch(k_types_pairs<uint16_t>, static_cast<uint16_t *>(dlogits))
                                                        : launch(k_types_pairs<float>, static_cast<float *>(dlogits)))
                return rc;
            if (!loss) return HARL_OK;
            hipLaunchKernelGGL(k_pairs_sum, dim3(1), dim3(kThreads), 0, stream, w.terms, n_pairs, loss);
            HARL_HIP_CHECK(hipGetLastError());
            return HARL_OK;
        }
        TypesIO io{};
        io.logp_ref = logp_ref;
        io.diff = w.diff;
        io.norm = w.norm;
        if (const int rc = launch_types<kTypesDiff>(head, q, io, stream)) return rc;
    } else if (n_rows > 0) {
        const StatOut o{w.stat, nullptr, nullptr, nullptr};
        if (const int rc = launch_wide_stats<kPartialFine>(head, q, chunks, o, stream)) return rc;
    }
    // a thread a row of an average pair
    const auto pairs = (int64_t)n_pairs * 256 < n_rows ? k_pairs<1024> : k_pairs<256>;
    const unsigned pair_threads = (int64_t)n_pairs * 256 < n_rows ? 1024 : 256;
    hipLaunchKernelGGL(pairs, dim3(grid_for(n_pairs)), dim3(pair_threads), 0, stream, a, w.stat, types ? w.diff : nullptr,
                       grad && !types ? w.fin : nullptr, grad && types ? w.g_row : nullptr, w.terms, ratio);
    HARL_HIP_CHECK(hipGetLastError());
    if (grad && types) {
        TypesIO io{};
        io.norm = w.norm;
        io.g_row = w.g_row;
        io.loss_out = loss;
        io.pair_terms = w.terms;
        io.n_pairs = n_pairs;
        io.dz = dlogits;
        io.ld_d = ld_d;
        return launch_types<kTypesGradPairs>(head, q, io, stream);
    }
    if (grad) {
        GradSrc g{};
        g.fin = w.fin;
        g.loss_out = loss;
        g.terms = w.terms;
        g.n_pairs = n_pairs;
        g.dz = dlogits;
        g.ld_d = ld_d;
        return launch_wide_grad<kFromFin>(head, q, g, stream);
    }
    if (!loss) return HARL_OK;
    hipLaunchKernelGGL(k_pairs_sum, dim3(1), dim3(kThreads), 0, stream, w.terms, n_pairs, loss);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

}  // namespace harl
