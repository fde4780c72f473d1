// Distillation from a teacher's top logits: the loss of every row and the gradient of the student's logits.
#include "logits.hpp"

namespace rp {
namespace {

struct DistillArgs {
    LogitRows x;
    const unsigned char* value;   // [rows][k] teacher's logits
    const int* entry;             // [rows][k] their actions
    const float* teacher_lse;     // or null
    const float* weight;          // or null
    unsigned int k;
    double inv_tt, inv_ts;        // 1 / temperature of teacher, of student
    float c2;                     // log2(e) / student's temperature
    float* loss;
    unsigned char* grad;
    unsigned long long grad_stride;
};

__device__ __forceinline__ void store_gradient(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_gradient(unsigned short* p, float v) {
    *p = __builtin_bit_cast(unsigned short, (__bf16)v);
}

// exp((x - m) / temperature) for x <= m.  The difference comes first: it is small where the weight is large.
__device__ __forceinline__ float weight_of(float x, float m, float c2) { return __builtin_amdgcn_exp2f((x - m) * c2); }

// A running maximum and the sum of exp((x - max) / temperature) beside it.
struct MaxSum {
    float m;
    double s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c2) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return MaxSum{m, 0.0};
    return MaxSum{m, (a.m == -INFINITY ? 0.0 : a.s * (double)weight_of(a.m, m, c2)) +
                         (b.m == -INFINITY ? 0.0 : b.s * (double)weight_of(b.m, m, c2))};
}

template <int W>
struct DistillShared {
    MaxSum row[W];
    float tmax[W], zmax[W];
    double sums[W][4];
    unsigned int twice;    // some action is in two entries
};

// One workgroup of W wavefronts per row.  LDS behind the arguments: which actions have an entry, a bit each
// [(n + 31) / 32 words], and the entries' actions, teacher logits and student logits [k] each.
template <int W, typename T, typename TT, bool REST, bool GRAD>
__global__ __launch_bounds__(64 * W) void distill_kernel(DistillArgs p) {
    extern __shared__ unsigned int lds[];
    __shared__ DistillShared<W> s;
    const unsigned int n = p.x.n, k = p.k, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const unsigned int words = (n + 31u) / 32u;
    unsigned int* named = lds;
    int* act = reinterpret_cast<int*>(lds + words);
    float* tv = reinterpret_cast<float*>(act + k);
    float* zv = tv + k;
    for (unsigned long long row = blockIdx.x; row < p.x.rows; row += gridDim.x) {
        const T* x = reinterpret_cast<const T*>(p.x.data) + row * p.x.stride;
        T* g = GRAD ? reinterpret_cast<T*>(p.grad) + row * p.grad_stride : nullptr;
        const float weight = p.weight ? p.weight[row] : 1.f;
        __syncthreads();   // (the row before is done with LDS)
        if (weight == 0.f) {
            if (tid == 0) p.loss[row] = 0.f;
            if (GRAD)
                for (unsigned int i = tid; i < n; i += 64 * W) store_gradient(g + i, 0.f);
            continue;
        }
        // entries: mark their actions
        for (unsigned int i = tid; i < words; i += 64 * W) named[i] = 0;
        if (tid == 0) s.twice = 0;
        __syncthreads();
        float tmax = -INFINITY, zmax = -INFINITY;
        bool bad = false;
        for (unsigned int e = tid; e < k; e += 64 * W) {
            const int a = p.entry[row * k + e];
            const bool there = (unsigned int)a < n;
            float t = there ? logit_value(reinterpret_cast<const TT*>(p.value) + row * k + e) : -INFINITY;
            float z = there ? logit_value(x + a) : -INFINITY;
            if (there) {
                const unsigned int bit = 1u << (a & 31);
                if (atomicOr(&named[a >> 5], bit) & bit) s.twice = 1;
            }
            act[e] = there ? a : -1;
            tv[e] = t;
            zv[e] = z;
            bad |= !(t < INFINITY);
            tmax = fmaxf(tmax, t);
            zmax = fmaxf(zmax, z);
        }
        __syncthreads();
        // the row: all of it, or (REST) what has no entry
        MaxSum all{-INFINITY, 0.0};
        for (unsigned int i = tid; i < n; i += 64 * W) {
            const float v = logit_value(x + i);
            bad |= !(v < INFINITY);
            if (REST && (named[i >> 5] >> (i & 31u) & 1u)) continue;
            if (v > all.m) {
                all.s = all.m == -INFINITY ? 1.0 : all.s * (double)weight_of(all.m, v, p.c2) + 1.0;
                all.m = v;
            } else if (v > -INFINITY) {
                all.s += (double)weight_of(v, all.m, p.c2);
            }
        }
        const bool any_bad = __syncthreads_or(bad);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const MaxSum o{__shfl_xor(all.m, off, 64), __shfl_xor(all.s, off, 64)};
            all = join(all, o, p.c2);
            tmax = fmaxf(tmax, __shfl_xor(tmax, off, 64));
            zmax = fmaxf(zmax, __shfl_xor(zmax, off, 64));
        }
        if (lane == 0) {
            s.row[wave] = all;
            s.tmax[wave] = tmax;
            s.zmax[wave] = zmax;
        }
        __syncthreads();
        all = s.row[0];
        tmax = s.tmax[0];
        zmax = s.zmax[0];
        for (int w = 1; w < W; ++w) {
            all = join(all, s.row[w], p.c2);
            tmax = fmaxf(tmax, s.tmax[w]);
            zmax = fmaxf(zmax, s.zmax[w]);
        }
        const float m = REST ? fmaxf(all.m, zmax) : all.m;
        const bool empty = m == -INFINITY || (!REST && tmax == -INFINITY);
        // sums over the entries: a_e = exp((t_e - shift) / tt), a_e (t_e - shift) / tt, a_e (z_e - m) / ts, and the
        // student's weight of each action once
        double sum[4] = {0.0, 0.0, 0.0, 0.0};
        const double shift = REST ? (double)p.teacher_lse[row] : tmax == -INFINITY ? 0.0 : (double)tmax * p.inv_tt;
        const bool twice = s.twice;
        for (unsigned int e = tid; e < k; e += 64 * W) {
            if (act[e] < 0) continue;
            const double d = (double)tv[e] * p.inv_tt - shift;
            const double a = exp(d), zd = ((double)zv[e] - (double)m) * p.inv_ts;
            bool first = true;
            if (twice)
                for (unsigned int f = 0; f < e && first; ++f) first = act[f] != act[e];
            sum[0] += a;
            if (a > 0.0 || a != a) {
                sum[1] += a * d;
                sum[2] += a * zd;
            }
            if (first && !empty) sum[3] += exp(zd);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = wave_reduce(sum[j], SumOp{});
        if (lane == 0)
            for (int j = 0; j < 4; ++j) s.sums[wave][j] = sum[j];
        __syncthreads();
        for (int j = 0; j < 4; ++j) {
            sum[j] = s.sums[0][j];
            for (int w = 1; w < W; ++w) sum[j] += s.sums[w][j];
        }
        // row scalars, the same in every thread.  total = sum of exp((x - m) / ts) over the row.
        const double outer = all.m == -INFINITY ? 0.0 : all.s * exp(((double)all.m - (double)m) * p.inv_ts);
        const double total = REST ? outer + sum[3] : outer;
        const double log_total = log(total);
        double loss, q_scale, inside, outside;
        if (!REST) {
            q_scale = 1.0 / sum[0];
            loss = (sum[1] - sum[2]) * q_scale - log(sum[0]) + log_total;
            inside = outside = 1.0;
        } else {
            const double sum_q = sum[0], sum_p = sum[3] / total, p_rest = outer / total;
            q_scale = 1.0;
            loss = sum[1] - sum[2] + sum_q * log_total;
            inside = outside = sum_q;
            if (sum_q < 1.0 && p_rest > 0.0) {
                loss += (1.0 - sum_q) * (log1p(-sum_q) - (sum_p < 0.5 ? log1p(-sum_p) : log(p_rest)));
                inside = 1.0;
                outside = (sum_q - sum_p) / p_rest;
            }
        }
        if (any_bad) loss = NAN;
        if (tid == 0) p.loss[row] = empty && !any_bad ? 0.f : (float)(loss * (double)weight);
        if (!GRAD) continue;
        const double scale = (double)weight * p.inv_ts;
        const float factor = any_bad ? NAN : empty ? 0.f : (float)(scale * outside / total);
        for (unsigned int i = tid; i < n; i += 64 * W)
            store_gradient(g + i, empty && !any_bad ? 0.f : factor * weight_of(logit_value(x + i), m, p.c2));
        __syncthreads();   // (an action with an entry is written again below)
        if (empty || any_bad) continue;
        for (unsigned int e = tid; e < k; e += 64 * W) {
            if (act[e] < 0) continue;
            double q = exp((double)tv[e] * p.inv_tt - shift) * q_scale;
            if (twice) {   // the first of an action's entries writes, with the sum of all
                bool first = true;
                q = 0.0;
                for (unsigned int f = 0; f < k; ++f)
                    if (act[f] == act[e]) {
                        first &= f >= e;
                        q += exp((double)tv[f] * p.inv_tt - shift) * q_scale;
                    }
                if (!first) continue;
            }
            const double pe = exp(((double)zv[e] - (double)m) * p.inv_ts) / total;
            store_gradient(g + act[e], (float)(scale * (pe * inside - q)));
        }
    }
}

template <typename T, typename TT, bool GRAD>
void launch_distill(const DistillArgs& a, hipStream_t st) {
    const unsigned int blocks = (unsigned int)(a.x.rows < (1ull << 18) ? a.x.rows : (1ull << 18));
    const size_t lds = ((a.x.n + 31u) / 32u + 3u * a.k) * 4u;
    if (a.teacher_lse)
        hipLaunchKernelGGL((distill_kernel<4, T, TT, true, GRAD>), dim3(blocks), dim3(256), lds, st, a);
    else
        hipLaunchKernelGGL((distill_kernel<4, T, TT, false, GRAD>), dim3(blocks), dim3(256), lds, st, a);
}

rp_status distill(const char* what, const rp_rows* logits, const rp_teacher* teacher, float* loss, void* grad,
                  uint64_t grad_stride, bool gradient, void* hip_stream) {
    const char* why = logit_rows_fault(logits);
    RP_REQUIRE(!why, "%s: %s", what, why);
    RP_REQUIRE(teacher, "%s: null teacher", what);
    RP_REQUIRE(teacher->k >= 1 && teacher->k <= kMaxTop, "%s: k = %u, must be 1 .. 1024", what, teacher->k);
    RP_REQUIRE(teacher->dtype == RP_F32 || teacher->dtype == RP_BF16, "%s: the teacher's logits must be RP_F32 or RP_BF16", what);
    RP_REQUIRE(teacher->temperature > 0.0 && std::isfinite(teacher->temperature) && teacher->student_temperature > 0.0 &&
                   std::isfinite(teacher->student_temperature),
               "%s: temperatures must be finite and > 0", what);
    if (logits->rows == 0) return RP_OK;
    why = logit_data_fault(logits);
    RP_REQUIRE(!why, "%s: %s", what, why);
    RP_REQUIRE(teacher->value && teacher->index && loss && (!gradient || grad), "%s: null array", what);
    const size_t e = logits->dtype == RP_BF16 ? 2 : 4;
    if (gradient) {
        RP_REQUIRE(grad_stride <= (1ull << 40) && (logits->rows == 1 || grad_stride >= logits->n),
                   "%s: gradient rows closer than a row's length", what);
        RP_REQUIRE((reinterpret_cast<uintptr_t>(grad) & (e - 1)) == 0, "%s: gradient not aligned to its type", what);
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(logits->data), g0 = reinterpret_cast<uintptr_t>(grad);
        const uintptr_t a1 = a0 + ((logits->rows - 1) * logits->stride + logits->n) * e;
        const uintptr_t g1 = g0 + ((logits->rows - 1) * grad_stride + logits->n) * e;
        RP_REQUIRE(a1 <= g0 || g1 <= a0 || (a0 == g0 && (logits->rows == 1 || logits->stride == grad_stride)),
                   "%s: the gradient overlaps the logits other than in place", what);
    }
    const DistillArgs a{logit_rows(logits), static_cast<const unsigned char*>(teacher->value), teacher->index, teacher->lse,
                        teacher->weight, teacher->k, 1.0 / teacher->temperature, 1.0 / teacher->student_temperature,
                        (float)(1.4426950408889634 / teacher->student_temperature), loss,
                        static_cast<unsigned char*>(grad), grad_stride};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool xb = logits->dtype == RP_BF16, tb = teacher->dtype == RP_BF16;
    typedef unsigned short B;
    if (gradient)
        xb ? (tb ? launch_distill<B, B, true>(a, st) : launch_distill<B, float, true>(a, st))
           : (tb ? launch_distill<float, B, true>(a, st) : launch_distill<float, float, true>(a, st));
    else
        xb ? (tb ? launch_distill<B, B, false>(a, st) : launch_distill<B, float, false>(a, st))
           : (tb ? launch_distill<float, B, false>(a, st) : launch_distill<float, float, false>(a, st));
    RP_CHECK_HIP(hipGetLastError());
    return RP_OK;
}

}  // namespace
}  // namespace rp

extern "C" {

size_t rp_distill_workspace_bytes(const rp_rows* logits, uint32_t k) {
    const char* why = rp::logit_rows_fault(logits);
    if (!why && (k == 0 || k > rp::kMaxTop)) why = "k must be 1 .. 1024";
    if (why) {
        rp::set_error("rp_distill_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return 0;
}

rp_status rp_distill_loss(const rp_rows* logits, const rp_teacher* teacher, float* loss, void* workspace, size_t bytes,
                          void* hip_stream) {
    (void)workspace;
    (void)bytes;
    return rp::distill("rp_distill_loss", logits, teacher, loss, nullptr, 0, false, hip_stream);
}

rp_status rp_distill_grad(const rp_rows* logits, const rp_teacher* teacher, float* loss, void* grad, uint64_t grad_stride,
                          void* workspace, size_t bytes, void* hip_stream) {
    (void)workspace;
    (void)bytes;
    return rp::distill("rp_distill_grad", logits, teacher, loss, grad, grad_stride, true, hip_stream);
}

}  // extern "C"
