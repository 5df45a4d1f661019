// Policy objectives on the logits of any actor: log-probabilities of chosen actions with their
// gradient, the clipped policy loss with a KL term, and the pairwise preference loss of log ratios.
//
// A row of logits z is cut into segments; of each, with m = max z,
//   s = sum e^(z - m), u = sum e^(z - m) (z - m), lse = m + log s, H = log s - u / s,
// and the row's log-probability is the sum over segments of z[action] - lse.  Every objective reaches
// the logits through the row's two gradients g_logp and g_H:
//   dz_i = g_logp (1[i = action] - p_i) - g_H p_i (log p_i + H_s),  p_i = e^(z_i - m) / s.
// k_row_stats computes {m, s, u, z[action]} per (row, segment); the row kernels turn them into each
// objective's per-row values and gradients; k_row_grad writes the logits' gradient.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

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
    const float *weight;     // rows of weight 0 are skipped, or null
    const int32_t *seq_ptr;  // only rows of [seq_ptr[0], seq_ptr[n_seq]) count, or null
    int n_seq;
    int32_t off[HARL_SELECT_MAX_SEGMENTS + 1];
};

// A (row, segment)'s sums, and one row's gradients of log-probability and entropy.
struct Stat {
    float m, s, u, zact;
};
struct RowGrad {
    float g_logp, g_ent;
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

// Largest value (NaN if any is) and sum over a workgroup of kThreads; the result in every thread.
__device__ __forceinline__ float block_max(float x, float *lds) {
    lds[threadIdx.x] = x;
    __syncthreads();
    for (int h = kThreads / 2; h > 0; h >>= 1) {
        if ((int)threadIdx.x < h) {
            const float a = lds[threadIdx.x], b = lds[threadIdx.x + h];
            lds[threadIdx.x] = b > a || b != b ? b : a;
        }
        __syncthreads();
    }
    const float r = lds[0];
    __syncthreads();
    return r;
}
__device__ __forceinline__ float block_sum(float x, float *lds) {
    lds[threadIdx.x] = x;
    __syncthreads();
    for (int h = kThreads / 2; h > 0; h >>= 1) {
        if ((int)threadIdx.x < h) lds[threadIdx.x] += lds[threadIdx.x + h];
        __syncthreads();
    }
    const float r = lds[0];
    __syncthreads();
    return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_row_stats(Rows q, Stat *__restrict__ stat) {
    __shared__ float lds[kThreads];
    for (int64_t r = blockIdx.x; r < q.M; r += gridDim.x) {
        if (!row_counts(q, (int)r)) continue;
        const T *z = static_cast<const T *>(q.z) + r * q.ld;
        for (int g = 0; g < q.n_seg; ++g) {
            const int lo = q.off[g], hi = q.off[g + 1];
            float m = -INFINITY;
            for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
                const float x = to_f32(z[i]);
                m = x > m || x != x ? x : m;
            }
            m = block_max(m, lds);
            float s = 0.f, u = 0.f;
            if (m > -INFINITY || m != m)
                for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
                    const float d = to_f32(z[i]) - m;
                    const float e = expf(d);
                    s += e;
                    u += e * fmaxf(d, -1000.f);  // an excluded action: 0, not 0 times -inf
                }
            s = block_sum(s, lds);
            u = block_sum(u, lds);
            if (threadIdx.x == 0) {
                const int act = min(max(q.act[r * q.n_seg + g], lo), hi - 1);
                stat[r * q.n_seg + g] = Stat{m, s, u, to_f32(z[act])};
            }
        }
    }
}

// A segment's log-probability and entropy; an empty segment (s = 0) adds nothing.
__device__ __forceinline__ double stat_logp(const Stat &t) {
    return t.s == 0.f ? 0.0 : ((double)t.zact - (double)t.m) - log((double)t.s);
}
__device__ __forceinline__ double stat_entropy(const Stat &t) {
    return t.s == 0.f ? 0.0 : log((double)t.s) - (double)t.u / (double)t.s;
}

__global__ __launch_bounds__(kThreads) void k_logp_rows(const Stat *__restrict__ stat, int M, int n_seg,
                                                        float *__restrict__ logp, float *__restrict__ entropy,
                                                        float *__restrict__ lse) {
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < M; r += (int64_t)gridDim.x * kThreads) {
        double lp = 0.0;
        for (int g = 0; g < n_seg; ++g) {
            const Stat t = stat[r * n_seg + g];
            lp += stat_logp(t);
            if (entropy) entropy[r * n_seg + g] = (float)stat_entropy(t);
            if (lse) {
                lse[(r * n_seg + g) * 2] = t.m;
                lse[(r * n_seg + g) * 2 + 1] = t.s == 0.f ? 0.f : (float)log((double)t.s);
            }
        }
        logp[r] = (float)lp;
    }
}

struct LossArgs {
    const float *logp_old, *logp_ref, *adv, *weight;
    float clip_low, clip_high, w_kl, w_entropy;
    float inv_m;
};

// One row's terms of the clipped loss, weighted, and its gradients.
__device__ __forceinline__ RowGrad loss_row(const LossArgs &a, int64_t r, float w, double logp, double H, double (&term)[3]) {
    const double ratio = exp(logp - (double)a.logp_old[r]);
    const double adv = a.adv[r], lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
    const double s1 = ratio * adv, s2 = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;
    const bool inside = ratio >= lo && ratio <= hi;
    double kl = 0.0, dkl = 0.0;
    if (a.logp_ref) {
        const double x = (double)a.logp_ref[r] - logp;
        dkl = -expm1(x);
        kl = x < INFINITY ? -dkl - x : x;  // x = inf (an excluded action): inf, not inf - inf
    }
    term[0] = (double)w * -(s2 < s1 ? s2 : s1);
    term[1] = (double)w * kl;
    term[2] = (double)w * H;
    const double d_surrogate = s2 < s1 && !inside ? 0.0 : -adv * ratio;
    const double d_kl = a.w_kl != 0.f ? (double)a.w_kl * dkl : 0.0;
    return RowGrad{(float)((double)w * (d_surrogate + d_kl)), -w * a.w_entropy};
}

__global__ __launch_bounds__(kThreads) void k_loss_rows(LossArgs a, const Stat *__restrict__ stat, int M, int n_seg,
                                                        RowGrad *__restrict__ grad, double *__restrict__ terms,
                                                        float *__restrict__ logp_out) {
    for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < M; r += (int64_t)gridDim.x * kThreads) {
        const float w = a.weight ? a.weight[r] : a.inv_m;
        double term[3] = {0.0, 0.0, 0.0}, lp = 0.0, H = 0.0;
        RowGrad g{0.f, 0.f};
        if (w != 0.f) {
            for (int k = 0; k < n_seg; ++k) {
                const Stat t = stat[r * n_seg + k];
                lp += stat_logp(t);
                H += stat_entropy(t);
            }
            g = loss_row(a, r, w, lp, H, term);
        }
        grad[r] = g;
        for (int c = 0; c < 3; ++c) terms[r * 3 + c] = term[c];
        if (logp_out) logp_out[r] = (float)lp;
    }
}

// Sums of N terms per row over n rows by one workgroup: thread-strided in row order, then a tree.
template <int N>
__device__ __forceinline__ void sum_terms(const double *__restrict__ terms, int64_t n, double (&out)[N]) {
    __shared__ double part[N][kThreads];
    double s[N] = {};
    for (int64_t r = threadIdx.x; r < n; r += kThreads)
        for (int c = 0; c < N; ++c) s[c] += terms[r * N + c];
    for (int c = 0; c < N; ++c) part[c][threadIdx.x] = s[c];
    __syncthreads();
    for (int h = kThreads / 2; h > 0; h >>= 1) {
        if ((int)threadIdx.x < h)
            for (int c = 0; c < N; ++c) part[c][threadIdx.x] += part[c][threadIdx.x + h];
        __syncthreads();
    }
    for (int c = 0; c < N; ++c) out[c] = part[c][0];
}

__global__ __launch_bounds__(kThreads) void k_loss_sum(const double *__restrict__ terms, int64_t n, float w_kl,
                                                       float w_entropy, float *__restrict__ loss) {
    double s[3];
    sum_terms<3>(terms, n, s);
    if (threadIdx.x == 0) {
        loss[0] = (float)(s[0] + (w_kl != 0.f ? (double)w_kl * s[1] : 0.0) - (w_entropy != 0.f ? (double)w_entropy * s[2] : 0.0));
        for (int c = 0; c < 3; ++c) loss[1 + c] = (float)s[c];
    }
}

struct PairArgs {
    const float *logp_ref, *weight;
    const int32_t *seq_ptr;
    int n_rows, n_seg, n_pairs;
    float beta, smoothing;
};

// Pair p by workgroup p (stepping over pairs): both tracks' log ratios, the loss terms and, with
// grad, every row's gradient.
__global__ __launch_bounds__(kThreads) void k_pairs(PairArgs a, const Stat *__restrict__ stat, RowGrad *__restrict__ grad,
                                                    double *__restrict__ terms, float *__restrict__ ratio) {
    __shared__ double part[kThreads];
    for (int64_t p = blockIdx.x; p < a.n_pairs; p += gridDim.x) {
        double R[2];
        for (int side = 0; side < 2; ++side) {
            const int lo = clamp_row(a.seq_ptr[2 * p + side], a.n_rows), hi = clamp_row(a.seq_ptr[2 * p + side + 1], a.n_rows);
            double s = 0.0;
            for (int64_t r = (int64_t)lo + threadIdx.x; r < hi; r += kThreads) {
                const float w = a.weight ? a.weight[r] : 1.f;
                if (w == 0.f) continue;
                double lp = a.logp_ref ? -(double)a.logp_ref[r] : 0.0;
                for (int k = 0; k < a.n_seg; ++k) lp += stat_logp(stat[r * a.n_seg + k]);
                s += (double)w * lp;
            }
            part[threadIdx.x] = s;
            __syncthreads();
            for (int h = kThreads / 2; h > 0; h >>= 1) {
                if ((int)threadIdx.x < h) part[threadIdx.x] += part[threadIdx.x + h];
                __syncthreads();
            }
            R[side] = part[0];
            __syncthreads();
        }
        const double h = (double)a.beta * (R[0] - R[1]);
        // -log sigmoid(h) = log(1 + e^-|h|) + max(-h, 0); d/dh of the loss = smoothing - sigmoid(-h)
        const double lose = log1p(exp(-fabs(h))) + (h < 0.0 ? -h : (h == h ? 0.0 : h));
        const double down = h >= 0.0 ? exp(-h) / (1.0 + exp(-h)) : 1.0 / (1.0 + exp(h));
        if (threadIdx.x == 0) {
            terms[p * 4] = a.smoothing != 0.f ? lose + (double)a.smoothing * h : lose;
            terms[p * 4 + 1] = lose;
            terms[p * 4 + 2] = h;
            terms[p * 4 + 3] = h > 0.0 ? 1.0 : 0.0;
            if (ratio) {
                ratio[2 * p] = (float)R[0];
                ratio[2 * p + 1] = (float)R[1];
            }
        }
        if (!grad) continue;
        const double g = (double)a.beta * ((double)a.smoothing - down) / (double)a.n_pairs;
        for (int side = 0; side < 2; ++side) {
            const int lo = clamp_row(a.seq_ptr[2 * p + side], a.n_rows), hi = clamp_row(a.seq_ptr[2 * p + side + 1], a.n_rows);
            for (int64_t r = (int64_t)lo + threadIdx.x; r < hi; r += kThreads) {
                const float w = a.weight ? a.weight[r] : 1.f;
                grad[r] = RowGrad{w == 0.f ? 0.f : (float)((double)w * (side ? -g : g)), 0.f};
            }
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_pairs_sum(const double *__restrict__ terms, int n_pairs, float *__restrict__ loss) {
    double s[4];
    sum_terms<4>(terms, n_pairs, s);
    if (threadIdx.x == 0)
        for (int c = 0; c < 4; ++c) loss[c] = (float)(s[c] / (double)n_pairs);
}

struct GradArgs {
    const Stat *stat;              // {m, s, u, .} per (row, segment), or null: lse and entropy are given
    const float *lse, *entropy;
    const RowGrad *grad;           // per row, or null: g_logp and g_entropy
    const float *g_logp, *g_entropy;
    void *dz;
    int64_t ld_d;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void k_row_grad(Rows q, GradArgs a) {
    for (int64_t r = blockIdx.x; r < q.M; r += gridDim.x) {
        if (q.seq_ptr && (r < clamp_row(q.seq_ptr[0], q.M) || r >= clamp_row(q.seq_ptr[q.n_seq], q.M))) continue;
        const T *z = static_cast<const T *>(q.z) + r * q.ld;
        T *dz = static_cast<T *>(a.dz) + r * a.ld_d;
        const float gl = a.grad ? a.grad[r].g_logp : a.g_logp[r];
        const float ge = a.grad ? a.grad[r].g_ent : a.g_entropy ? a.g_entropy[r] : 0.f;
        for (int g = 0; g < q.n_seg; ++g) {
            const int lo = q.off[g], hi = q.off[g + 1];
            const int act = min(max(q.act[r * q.n_seg + g], lo), hi - 1);
            float m = 0.f, rest = 0.f, H = 0.f;  // log-sum-exp m + rest
            bool empty = gl == 0.f && ge == 0.f;
            if (a.stat) {
                if (!empty) {
                    const Stat t = a.stat[r * q.n_seg + g];
                    empty = t.s == 0.f;
                    m = t.m;
                    rest = (float)log((double)t.s);
                    H = (float)stat_entropy(t);
                }
            } else if (!empty) {
                m = a.lse[(r * q.n_seg + g) * 2];
                rest = a.lse[(r * q.n_seg + g) * 2 + 1];
                empty = m == -INFINITY;
                if (ge != 0.f) H = a.entropy[r * q.n_seg + g];
            }
            for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
                float d = 0.f;
                if (!empty) {
                    const float ls = (to_f32(z[i]) - m) - rest;
                    const float p = expf(ls);
                    d = gl * ((i == act ? 1.f : 0.f) - p);
                    if (ge != 0.f) d -= ge * p * (fmaxf(ls, -1000.f) + H);
                }
                store(dz + i, d);
            }
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

int launch_stats(const harl_policy_head *h, const Rows &q, Stat *stat, hipStream_t stream) {
    if (h->dtype == HARL_BF16)
        hipLaunchKernelGGL(k_row_stats<uint16_t>, dim3(grid_for(q.M)), dim3(kThreads), 0, stream, q, stat);
    else
        hipLaunchKernelGGL(k_row_stats<float>, dim3(grid_for(q.M)), dim3(kThreads), 0, stream, q, stat);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

int launch_grad(const harl_policy_head *h, const Rows &q, const GradArgs &a, hipStream_t stream) {
    if (h->dtype == HARL_BF16)
        hipLaunchKernelGGL(k_row_grad<uint16_t>, dim3(grid_for(q.M)), dim3(kThreads), 0, stream, q, a);
    else
        hipLaunchKernelGGL(k_row_grad<float>, dim3(grid_for(q.M)), dim3(kThreads), 0, stream, q, a);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

// The workspace: stats per (row, segment), gradients per row, loss terms per row or pair.
struct Ws {
    Stat *stat;
    RowGrad *grad;
    double *terms;
    size_t bytes;
};

Ws ws_layout(const harl_policy_head *h, int64_t rows, int64_t n_terms, char *base) {
    Ws w{};
    int64_t off = 0;
    auto take = [&](int64_t bytes) {
        char *p = base ? base + off : nullptr;
        off += round_up(std::max<int64_t>(bytes, 1), 256);
        return p;
    };
    w.stat = reinterpret_cast<Stat *>(take(rows * h->n_seg * (int64_t)sizeof(Stat)));
    w.grad = reinterpret_cast<RowGrad *>(take(rows * (int64_t)sizeof(RowGrad)));
    w.terms = reinterpret_cast<double *>(take(n_terms * 8));
    w.bytes = (size_t)off;
    return w;
}

}  // namespace

size_t objective_logp_ws_bytes(const harl_policy_head *head, int32_t M) { return ws_layout(head, M, 0, nullptr).bytes; }

size_t objective_loss_ws_bytes(const harl_policy_head *head, int32_t M) {
    return ws_layout(head, M, 3 * (int64_t)M, nullptr).bytes;
}

size_t objective_preference_ws_bytes(const harl_policy_head *head, int32_t n_rows, int32_t n_pairs) {
    return ws_layout(head, n_rows, 4 * (int64_t)n_pairs, nullptr).bytes;
}

int policy_logp_launch(const harl_policy_head *head, const void *logits, int64_t ld, int32_t M, const int32_t *actions,
                       float *logp, float *entropy, float *lse, void *ws, hipStream_t stream) {
    const Ws w = ws_layout(head, M, 0, static_cast<char *>(ws));
    const Rows q = rows_of(head, logits, ld, M, actions);
    if (const int rc = launch_stats(head, q, w.stat, stream)) return rc;
    hipLaunchKernelGGL(k_logp_rows, dim3(grid_for(ceil_div(M, kThreads))), dim3(kThreads), 0, stream, w.stat, M,
                       head->n_seg, logp, entropy, lse);
    HARL_HIP_CHECK(hipGetLastError());
    return HARL_OK;
}

int policy_logp_grad_launch(const harl_policy_head *head, const void *logits, int64_t ld, int32_t M,
                            const int32_t *actions, const float *lse, const float *entropy, const float *g_logp,
                            const float *g_entropy, void *dlogits, int64_t ld_d, hipStream_t stream) {
    GradArgs a{};
    a.lse = lse;
    a.entropy = entropy;
    a.g_logp = g_logp;
    a.g_entropy = g_entropy;
    a.dz = dlogits;
    a.ld_d = ld_d;
    return launch_grad(head, rows_of(head, logits, ld, M, actions), a, stream);
}

int policy_loss_launch(const harl_policy_head *head, const harl_policy_loss_config *cfg, const void *logits, int64_t ld,
                       int32_t M, const int32_t *actions, const float *logp_old, const float *logp_ref,
                       const float *adv, const float *weight, void *dlogits, int64_t ld_d, float *logp, float *loss,
                       void *ws, hipStream_t stream) {
    const Ws w = ws_layout(head, M, 3 * (int64_t)M, static_cast<char *>(ws));
    Rows q = rows_of(head, logits, ld, M, actions);
    q.weight = weight;
    if (const int rc = launch_stats(head, q, w.stat, stream)) return rc;
    LossArgs a{logp_old, logp_ref, adv, weight, cfg->clip_low, cfg->clip_high, cfg->w_kl, cfg->w_entropy, 1.f / (float)M};
    hipLaunchKernelGGL(k_loss_rows, dim3(grid_for(ceil_div(M, kThreads))), dim3(kThreads), 0, stream, a, w.stat, M,
                       head->n_seg, w.grad, w.terms, logp);
    HARL_HIP_CHECK(hipGetLastError());
    if (loss) {
        hipLaunchKernelGGL(k_loss_sum, dim3(1), dim3(kThreads), 0, stream, w.terms, (int64_t)M, cfg->w_kl,
                           cfg->w_entropy, loss);
        HARL_HIP_CHECK(hipGetLastError());
    }
    if (!dlogits) return HARL_OK;
    GradArgs g{};
    g.stat = w.stat;
    g.grad = w.grad;
    g.dz = dlogits;
    g.ld_d = ld_d;
    return launch_grad(head, q, g, stream);
}

int preference_loss_launch(const harl_policy_head *head, const harl_preference_config *cfg, const void *logits,
                           int64_t ld, int32_t n_rows, const int32_t *actions, const float *logp_ref,
                           const float *weight, const int32_t *seq_ptr, int32_t n_pairs, void *dlogits, int64_t ld_d,
                           float *ratio, float *loss, void *ws, hipStream_t stream) {
    const Ws w = ws_layout(head, n_rows, 4 * (int64_t)n_pairs, static_cast<char *>(ws));
    Rows q = rows_of(head, logits, ld, n_rows, actions);
    q.weight = weight;
    q.seq_ptr = seq_ptr;
    q.n_seq = 2 * n_pairs;
    const bool grad = dlogits && n_rows > 0;
    if (n_rows > 0)
        if (const int rc = launch_stats(head, q, w.stat, stream)) return rc;
    PairArgs a{logp_ref, weight, seq_ptr, n_rows, head->n_seg, n_pairs, cfg->beta, cfg->smoothing};
    hipLaunchKernelGGL(k_pairs, dim3(grid_for(n_pairs)), dim3(kThreads), 0, stream, a, w.stat, grad ? w.grad : nullptr,
                       w.terms, ratio);
    HARL_HIP_CHECK(hipGetLastError());
    if (loss) {
        hipLaunchKernelGGL(k_pairs_sum, dim3(1), dim3(kThreads), 0, stream, w.terms, n_pairs, loss);
        HARL_HIP_CHECK(hipGetLastError());
    }
    if (!grad) return HARL_OK;
    GradArgs g{};
    g.stat = w.stat;
    g.grad = w.grad;
    g.dz = dlogits;
    g.ld_d = ld_d;
    return launch_grad(head, q, g, stream);
}

}  // namespace harl
