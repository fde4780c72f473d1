// Distillation from a teacher's top logits: the loss of every row and the gradient of the student's logits.
//
// With m the row's maximum, w_i = exp((x_i - m) / ts) and their sum S the gradient is w_i times one number per row, but for the
// at most 1024 actions with an entry, which are written again.  So a row needs a maximum, a sum, and for the gradient a second
// exponential per element: HBM bounds it as long as the row is read once and written once, from registers.  Sums over a row
// are held in 64 bits from one load to the next, exponentials in 32; entries and row scalars are in 64, since the loss is a
// small difference of large logarithms.  The teacher's mass outside its entries is set against the sum over the other
// actions, which is made directly (a bit per action in LDS tells which they are), not as a difference.
//
// 4096 x 32768 bf16, k = 64, a tenth of the rows of weight 0: 116 to 121 us, 4.2 to 4.4 TB/s of the 5.1 of a copy (the first kernel,
// three passes over memory: 504).  Variants by wavefronts a row: the fewest that hold it, as rows that wait for memory
// or for their chain of scalars are covered by others: 4096 x 1000 fp32 30 us with four wavefronts, 17 with one.
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
    double scale;                 // of the gradient
    float c2;                     // log2(e) / student's temperature
    float* loss;
    unsigned char* grad;
    unsigned long long grad_stride;
};

__device__ __forceinline__ void store_gradient(Global<float>* p, float v) { *p = v; }
__device__ __forceinline__ void store_gradient(Global<unsigned short>* p, float v) {
    *p = __builtin_bit_cast(unsigned short, (__bf16)v);
}

// exp((x - m) / temperature) for x <= m.  The difference comes first: it is small where the weight is large.
__device__ __forceinline__ float weight_of(float x, float m, float c2) { return __builtin_amdgcn_exp2f((x - m) * c2); }

// exp of a number in 64 bits to 32 bits' precision and 64 bits' range: 2^whole times a 32-bit 2^rest.  For what ends in a
// gradient of 32 bits; what the loss is made of is a small difference of large logarithms and takes exp().
__device__ __forceinline__ double wide_exp(double d) {
    const double t = (d < -1e4 ? -1e4 : d) * 1.4426950408889634, whole = rint(t);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(t - whole)), (int)whole);
}

// A maximum and the sum of exp((. - max) / temperature) beside it.
struct MaxSum {
    float m;
    double s;
};

// What a wavefront knows of the row's entries.
struct EntryPart {
    double tm, a, b, c;   // max of t (REST: unused); sums of q' = exp(d), q' d, q' (z - zm) / ts with d = log_weight(t)
    double z;             // sum of exp((z - zm) / ts), each action once
    float zm;
    unsigned int any;     // some entry is there with a logit above -infinity
};

// What every element's gradient needs, worked out once per row.  An element without an entry has factor exp((x - base) / ts).
// The teacher's rest pulls at such elements with a strength that does not fall with their mass, so `base` is their own maximum
// (REST): from the row's, exp and factor leave the range of 32 bits, to opposite sides, 87 temperatures below.
struct RowScalars {
    float m, base, factor;
    double shift, q_scale, inside, scale, inv_total;
    unsigned int state;   // 0: as computed; 1: nothing to learn, all 0; 2: all NaN
};

template <int W>
struct DistillShared {
    MaxSum row[W];
    EntryPart part[W];
    RowScalars out;
    unsigned int twice;   // some action is in two entries
};

// The entries of a row in LDS, in arrays of k.
struct Entries {
    int* act;       // -1: no entry
    float *t, *z;   // the teacher's and the student's logit
};

// Puts the row's entries into LDS and marks the actions among `begin` .. `end` that have one, a bit each, in `named`
// (cleared before, one word more than the range needs).
template <int W, typename T, typename TT, bool MARK>
__device__ __forceinline__ void load_entries(const DistillArgs& p, unsigned long long row, const Global<T>* x, const float* z_given,
                                             unsigned int begin, unsigned int end, Entries en, unsigned int* named,
                                             DistillShared<W>& s) {
    const unsigned int k = p.k;
#pragma unroll 1
    for (unsigned int e = threadIdx.x; e < k; e += 64 * W) {
        const int a = global_in<int>(p.entry)[row * k + e];
        const bool there = (unsigned int)a < p.x.n;
        en.act[e] = there ? a : -1;
        en.t[e] = there ? logit_value(global_in<TT>(p.value) + row * k + e) : -INFINITY;
        en.z[e] = !there ? -INFINITY : z_given ? global_in<float>(z_given)[row * k + e] : logit_value(x + a);
        if (MARK && there && (unsigned int)a >= begin && (unsigned int)a < end) {
            const unsigned int at = a - begin, bit = 1u << (at & 31u);
            if (atomicOr(&named[at >> 5], bit) & bit) s.twice = 1;
        }
    }
}

// log of an entry's unnormalised weight: over `shift`, the largest of the teacher's logits, or (REST) its log-sum-exp.  The
// difference comes before the division: a product less a product may be fused, and is then not zero for the largest.
template <bool REST>
__device__ __forceinline__ double log_weight(const DistillArgs& p, float t, double shift) {
    return REST ? (double)t * p.inv_tt - shift : ((double)t - shift) * p.inv_tt;
}

// Sums over the wavefront's share of the entries.
template <int W, bool REST>
__device__ __forceinline__ void sum_entries(const DistillArgs& p, unsigned long long row, Entries en, DistillShared<W>& s) {
    const unsigned int tid = threadIdx.x, wave = tid >> 6, k = p.k;
    EntryPart r{-INFINITY, 0.0, 0.0, 0.0, 0.0, -INFINITY, 0};
    if (__builtin_amdgcn_readfirstlane(wave * 64u) < k) {
        float tm = -INFINITY;
        bool bad = false;
#pragma unroll 1
        for (unsigned int e = tid; e < k; e += 64 * W) {
            tm = fmaxf(tm, en.t[e]);
            r.zm = fmaxf(r.zm, en.z[e]);
            bad |= en.act[e] >= 0 && !(en.t[e] < INFINITY);
        }
        tm = wave_reduce(tm, MaxOp{});
        r.zm = wave_reduce(r.zm, MaxOp{});
        r.any = tm > -INFINITY;
        r.tm = (double)tm;
        const double tm0 = REST ? (double)global_in<float>(p.teacher_lse)[row] : r.any ? r.tm : 0.0, zm0 = r.zm > -INFINITY ? (double)r.zm : 0.0;
        const bool twice = s.twice;
#pragma unroll 1
        for (unsigned int e = tid; e < k; e += 64 * W) {
            if (en.act[e] < 0) continue;
            const double d = log_weight<REST>(p, en.t[e], tm0), z = (double)en.z[e];
            bool first = true;
            if (twice)
#pragma unroll 1
                for (unsigned int f = 0; f < e && first; ++f) first = en.act[f] != en.act[e];
            // (one exp after the other: side by side they would take the registers that hold the row)
#pragma unroll 1
            for (int which = 0; which < 2; ++which) {
                const double v = exp(which ? (z - zm0) * p.inv_ts : d);
                if (which) {
                    if (first) r.z += v;
                } else {
                    r.a += v;
                    if (!(v == 0.0)) {
                        r.b += v * d;
                        r.c += v * ((z - zm0) * p.inv_ts);
                    }
                }
            }
        }
        if (bad) r.a = NAN;
        r.a = wave_reduce(r.a, SumOp{});
        r.b = wave_reduce(r.b, SumOp{});
        r.c = wave_reduce(r.c, SumOp{});
        r.z = wave_reduce(r.z, SumOp{});
    }
    if ((tid & 63u) == 0) s.part[wave] = r;
}

// Maximum and sum over what `row` holds, of what has no entry (REST) or all of it, the same in the lanes of a wavefront.
// `named` has a bit for every action from `begin` on; `again`: the same elements, read from memory.
template <bool REST, typename T, typename Row, typename Again>
__device__ __forceinline__ MaxSum sum_row(const Row& row, const Again& again, unsigned int begin, const unsigned int* named,
                                          float c2) {
    constexpr int kN = (int)kPerLoad<T>;
    constexpr unsigned int kAll = (1u << kN) - 1u;
    // which elements of a load do not count here
    auto bits_out = [&](unsigned int i, unsigned int gone) -> unsigned int {
        unsigned int bits = (1u << min(gone, (unsigned int)kN)) - 1u;
        if (REST) {
            const unsigned int at = i - begin;
            const unsigned long long two = (unsigned long long)named[(at >> 5) + 1u] << 32 | named[at >> 5];
            bits |= (unsigned int)(two >> (at & 31u)) & kAll;
        }
        return bits;
    };
    if constexpr (!Row::kHeld) {
        // one pass: a thread's own running maximum, to which its sum is brought when it rises
        float m = -INFINITY;
        double sum = 0.0;
        row.each_load([&](u32x4 raw, unsigned int i, unsigned int gone) {
            const unsigned int bits = bits_out(i, gone);
            float top = -INFINITY, load = 0.f;
            if (bits) {
#pragma unroll
                for (int e = 0; e < kN; ++e) top = fmaxf(top, bits >> e & 1u ? -INFINITY : element<T>(raw, e));
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e) top = fmaxf(top, element<T>(raw, e));
            }
            if (top > m) {
                sum *= (double)weight_of(m, top, c2);
                m = top;
            }
            const float m0 = m > -INFINITY ? m : 0.f;
            if (bits) {
#pragma unroll
                for (int e = 0; e < kN; ++e) load += bits >> e & 1u ? 0.f : weight_of(element<T>(raw, e), m0, c2);
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e) load += weight_of(element<T>(raw, e), m0, c2);
            }
            sum += (double)load;
        });
        const float all = wave_reduce(m, MaxOp{});
        const double back = sum == 0.0 ? 0.0 : sum * (double)(m > -INFINITY ? weight_of(m, all, c2) : 1.f);
        return MaxSum{all, wave_reduce(back, SumOp{})};
    } else {
    // (the sum of a load in 32 bits, sums of those in 64)
    auto sum_to = [&](const auto& r, float m0) {
        double sum = 0.0;
        r.each_load([&](u32x4 raw, unsigned int i, unsigned int gone) {
            const unsigned int bits = bits_out(i, gone);
            float load = 0.f;
            if (bits) {
#pragma unroll
                for (int e = 0; e < kN; ++e) load += bits >> e & 1u ? 0.f : weight_of(element<T>(raw, e), m0, c2);
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e) load += weight_of(element<T>(raw, e), m0, c2);
            }
            sum += (double)load;
        });
        return wave_reduce(sum, SumOp{});
    };
    float m = -INFINITY;
    row.each_load([&](u32x4 raw, unsigned int, unsigned int) {
#pragma unroll
        for (int e = 0; e < kN; ++e) m = fmaxf(m, element<T>(raw, e));
    });
    m = wave_reduce(m, MaxOp{});
    double sum = sum_to(row, m > -INFINITY ? m : 0.f);
    if (REST && sum < 1e-20) {
        // what has no entry lies so far below what has one that 32 bits lose it: once more, from its own maximum
        m = -INFINITY;
        again.each_load([&](u32x4 raw, unsigned int i, unsigned int gone) {
            const unsigned int bits = bits_out(i, gone);
#pragma unroll
            for (int e = 0; e < kN; ++e) m = fmaxf(m, bits >> e & 1u ? -INFINITY : element<T>(raw, e));
        });
        m = wave_reduce(m, MaxOp{});
        sum = sum_to(again, m > -INFINITY ? m : 0.f);
    }
    return MaxSum{m, sum};
    }
}

// Sum over the lanes of each quarter of a wavefront, in all of them.
__device__ __forceinline__ double quarter_sum(double v) {
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// From the parts of the row and of its entries to the loss and what the gradient needs.  Called by one wavefront.  There
// are up to 16 parts of either kind: its quarters bring the sums over the row, over the entries' student weights, over
// the teacher's, and (REST) over the row to its own maximum, with one exp for all, and one log serves for the logarithms too.
template <bool REST>
__device__ __forceinline__ void finish_row(const DistillArgs& p, unsigned long long row, float weight, const EntryPart* part,
                                           unsigned int parts, const MaxSum* rows, unsigned int pieces, RowScalars* out,
                                           bool put_loss = true) {
    const unsigned int lane = threadIdx.x & 63u, quarter = lane >> 4, l = lane & 15u;
    const bool part_here = l < parts, row_here = l < pieces;
    const EntryPart& r = part[part_here ? l : 0u];
    const MaxSum& x = rows[row_here ? l : 0u];
    const float own_z = part_here ? r.zm : -INFINITY, own_x = row_here ? x.m : -INFINITY;
    const bool own_any = part_here && r.any;
    const double own_t = own_any ? r.tm : -INFINITY;
    const float zm = wave_reduce(own_z, MaxOp{}), xm = wave_reduce(own_x, MaxOp{});
    const bool any = __ballot(own_any) != 0;
    const float m = REST ? fmaxf(zm, xm) : xm;
    const double m0 = m > -INFINITY ? (double)m : 0.0;
    const double tm = wave_reduce(own_t, MaxOp{});
    const double shift = REST ? (double)global_in<float>(p.teacher_lse)[row] : any ? tm : 0.0;
    const double x0 = xm > -INFINITY ? (double)xm : 0.0;
    double from = quarter == 0 ? (own_x > -INFINITY ? ((double)own_x - m0) * p.inv_ts : 0.0)
                  : REST && quarter == 3 ? (own_x > -INFINITY ? ((double)own_x - x0) * p.inv_ts : 0.0)
                  : quarter == 1 ? (own_z > -INFINITY ? ((double)own_z - m0) * p.inv_ts : 0.0)
                                 : (!REST && own_any ? (own_t - shift) * p.inv_tt : 0.0);
    const double factor = exp(from);
    double first = quarter == 0 || (REST && quarter == 3) ? (row_here ? x.s : 0.0)
                   : quarter == 1                         ? (part_here ? r.z : 0.0)
                                                          : (part_here ? r.a : 0.0);
    double b = part_here ? r.b : 0.0, c = part_here ? r.c : 0.0;
    // (q' (t - tm) from a wavefront's own maximum to the row's)
    if (!REST && quarter >= 2u) b = first == 0.0 ? 0.0 : (b + first * from) * factor;
    // (and q' (z - zm) from its own student's maximum to the row's)
    c = first == 0.0 ? 0.0 : c + first * (own_z > -INFINITY ? ((double)own_z - m0) * p.inv_ts : 0.0);
    if (!REST) c = factor == 0.0 ? 0.0 : c * factor;
    first = quarter_sum(first == 0.0 ? 0.0 : first * factor);
    b = __shfl(quarter_sum(b), 32, 64);
    c = __shfl(quarter_sum(c), 32, 64);
    const double outer = __shfl(first, 0, 64), inner = __shfl(first, 16, 64), a = __shfl(first, 32, 64);
    const double own = __shfl(first, 48, 64);   // (REST) outer, from its own maximum: 1e-20 or more, or 0 if nothing is in it
    const double total = REST ? outer + inner : outer, p_in = inner / total, p_rest = outer / total;
    // (in 64 bits log(1 - v) is as good as log1p(-v) for what is multiplied by 1 - v and added to the rest; p_rest itself may be
    // below the numbers of 64 bits)
    const double logs = log(lane == 0   ? total
                            : lane == 1 ? (REST ? 1.0 - a : a)
                                        : (p_in < 0.5 ? 1.0 - p_in : own));
    const double log_total = __shfl(logs, 0, 64), log_a = __shfl(logs, 1, 64), log_own = __shfl(logs, 2, 64);
    const double log_rest = p_in < 0.5 ? log_own : log_own + (x0 - m0) * p.inv_ts - log_total;
    const double scale = (double)weight * p.scale * p.inv_ts;
    double loss, q_scale = 1.0, inside = 1.0, share = scale / total;
    if (!REST) {
        q_scale = 1.0 / a;
        loss = (b - c) * q_scale - log_a + log_total;
    } else {
        loss = b - c + a * log_total;
        inside = a;
        double outside = a * p_rest;
        if (a < 1.0 && own > 0.0) {
            loss += (1.0 - a) * (log_a - log_rest);
            inside = 1.0;
            outside = p_in < 0.5 ? a - p_in : p_rest - (1.0 - a);   // (the same number, from its smaller parts)
        }
        share = own > 0.0 ? scale * outside / own : 0.0;
    }
    // (NaN and +infinity anywhere have made one of the sums NaN)
    const bool bad = !(total < INFINITY) || a != a;
    const bool empty = !bad && (m == -INFINITY || (!REST && !any));
    if (bad) loss = NAN;
    if (lane == 0) {
        if (put_loss) p.loss[row] = empty ? 0.f : (float)(loss * (double)weight);
        *out = RowScalars{m > -INFINITY ? m : 0.f, xm > -INFINITY ? xm : 0.f, bad ? NAN : (float)share, shift, q_scale,
                          inside, scale, 1.0 / total, empty ? 1u : bad ? 2u : 0u};
    }
}

__device__ __forceinline__ unsigned int bf16_pair_of(float lo, float hi) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned int, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

// The gradient of what `row` holds as if nothing of it had an entry.  Where two threads' loads share elements, at the row's
// end, both store the same values if the row is held; else, as the gradient may lie over the logits, each element is read
// by the thread that stores it alone.
template <typename T, typename Row>
__device__ __forceinline__ void put_gradient(const Row& row, Global<T>* g, const RowScalars& o, float c2) {
    const float m = o.base, factor = o.state == 1u ? 0.f : o.factor;
    row.each_load([&](u32x4 raw, unsigned int i, unsigned int gone) {
        if constexpr (!Row::kHeld) {
            if (gone) {
                for (unsigned int e = gone; e < kPerLoad<T>; ++e)
                    store_gradient(g + i + e, factor * weight_of(logit_value(row.x + i + e), m, c2));
                return;
            }
        }
        auto value = [&](int e) { return factor * weight_of(element<T>(raw, e), m, c2); };
        u32x4 out;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) out[j] = __float_as_uint(value(j));
            else out[j] = bf16_pair_of(value(2 * j), value(2 * j + 1));
        }
        *(Global<u32x4_any>*)(g + i) = out;
    });
}

// The gradient of the actions among begin .. end that have an entry.
template <int W, typename T, bool REST>
__device__ __forceinline__ void put_entries(const DistillArgs& p, Global<T>* g, Entries en, unsigned int begin, unsigned int end,
                                            const RowScalars& o, bool twice) {
    const unsigned int k = p.k;
#pragma unroll 1
    for (unsigned int e = threadIdx.x; e < k; e += 64 * W) {
        const unsigned int a = (unsigned int)en.act[e];
        if (a < begin || a >= end) continue;   // (-1 is beyond any end)
        double q = wide_exp(log_weight<REST>(p, en.t[e], o.shift)) * o.q_scale;
        if (twice) {   // the first of an action's entries writes, with the sum of all
            bool first = true;
            q = 0.0;
#pragma unroll 1
            for (unsigned int f = 0; f < k; ++f)
                if (en.act[f] == (int)a) {
                    first &= f >= e;
                    q += wide_exp(log_weight<REST>(p, en.t[f], o.shift)) * o.q_scale;
                }
            if (!first) continue;
        }
        const double pe = wide_exp(((double)en.z[e] - (double)o.m) * p.inv_ts) * o.inv_total;
        store_gradient(g + a, (float)(o.scale * (pe * o.inside - q)));
    }
}

template <int W, typename T>
__device__ __forceinline__ void put_zeros(Global<T>* g, unsigned int n) {
    for (unsigned int i = threadIdx.x; i < n; i += 64 * W) store_gradient(g + i, 0.f);
}

// A row of up to 64 NV elements in the registers of one wavefront, element by element: no load is too long for it.
template <int NV, typename T>
struct ShortRow {
    float v[NV];
    __device__ __forceinline__ ShortRow(const Global<T>* x, unsigned int n) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const unsigned int i = threadIdx.x + 64u * j;
            v[j] = i < n ? logit_value(x + i) : -INFINITY;
        }
    }
};

// Rows of up to 64 NV actions: one wavefront each.
template <int NV, typename T, typename TT, bool REST, bool GRAD>
__global__ __launch_bounds__(64) void distill_wave_kernel(DistillArgs p) {
    extern __shared__ unsigned int lds[];
    __shared__ DistillShared<1> s;
    const unsigned int n = p.x.n, k = p.k, lane = threadIdx.x;
    constexpr unsigned int kWords = 2u * NV;
    unsigned int* named = lds;
    const Entries en{reinterpret_cast<int*>(lds + kWords), reinterpret_cast<float*>(lds + kWords + k),
                     reinterpret_cast<float*>(lds + kWords + 2u * k)};
    const unsigned long long row = workgroup_row();
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    Global<T>* g = global_out<T>(p.grad) + row * p.grad_stride;
    const float weight = p.weight ? global_in<float>(p.weight)[row] : 1.f;
    if (weight == 0.f) {
        if (lane == 0) p.loss[row] = 0.f;
        if (GRAD) put_zeros<1, T>(g, n);
        return;
    }
    const ShortRow<NV, T> held(x, n);
    if (lane < kWords) named[lane] = 0;
    if (lane == 0) s.twice = 0;
    __syncthreads();
    load_entries<1, T, TT, true>(p, row, x, nullptr, 0, n, en, named, s);
    __syncthreads();
    sum_entries<1, REST>(p, row, en, s);
    float m = -INFINITY;
    bool out[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const unsigned int i = lane + 64u * j;
        out[j] = REST && (named[i >> 5] >> (i & 31u) & 1u);
        m = fmaxf(m, out[j] ? -INFINITY : held.v[j]);
    }
    m = wave_reduce(m, MaxOp{});
    const float m0 = m > -INFINITY ? m : 0.f;
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) sum += out[j] ? 0.0 : (double)weight_of(held.v[j], m0, p.c2);
    sum = wave_reduce(sum, SumOp{});
    if (lane == 0) s.row[0] = MaxSum{m, sum};
    __syncthreads();
    finish_row<REST>(p, row, weight, s.part, 1, s.row, 1, &s.out);
    if (!GRAD) return;
    __syncthreads();
    const RowScalars o = s.out;
    const float factor = o.state == 1u ? 0.f : o.factor;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const unsigned int i = lane + 64u * j;
        if (i < n) store_gradient(g + i, factor * weight_of(held.v[j], o.base, p.c2));
    }
    __syncthreads();   // (an action with an entry is written again)
    if (o.state == 0) put_entries<1, T, REST>(p, g, en, 0, n, o, s.twice != 0);
}

template <int W, typename T, typename TT, bool REST, bool GRAD, typename Row>
__device__ __forceinline__ void distill_row(const DistillArgs& p, unsigned long long row, float weight, const Global<T>* x,
                                            Global<T>* g, const Row& held, unsigned int* named, unsigned int words,
                                            Entries en, DistillShared<W>& s) {
    const unsigned int tid = threadIdx.x, n = p.x.n;
    for (unsigned int i = tid; i < words; i += 64 * W) named[i] = 0;
    if (tid == 0) s.twice = 0;
    __syncthreads();
    load_entries<W, T, TT, REST || GRAD>(p, row, x, nullptr, 0, n, en, named, s);
    __syncthreads();
    sum_entries<W, REST>(p, row, en, s);
    const MaxSum mine = sum_row<REST, T>(held, ReadRow<W, 1, T, false>(x, 0, n), 0, named, p.c2);
    if ((tid & 63u) == 0) s.row[tid >> 6] = mine;
    __syncthreads();
    if (tid < 64) finish_row<REST>(p, row, weight, s.part, W, s.row, W, &s.out);
    if (!GRAD) return;
    __syncthreads();
    put_gradient<T>(held, g, s.out, p.c2);
    __syncthreads();   // (an action with an entry is written again)
    if (s.out.state == 0) put_entries<W, T, REST>(p, g, en, 0, n, s.out, s.twice != 0);
}

// One workgroup of W wavefronts per row, held in registers (NV > 0) or read again for each of three passes.  LDS
// behind the arguments: the marks, (n + 31) / 32 + 1 words, and the entries.
// Longer than 32,768 / 65,536 actions in 32 / 16 bits a row is read twice (400 x 131072 bf16: 61 us; held by 16 wavefronts of 16
// loads 63).  The loss alone needs one pass with a running maximum and nothing held: 1000 x 50021 bf16 28 to 33 us, 3.1 to
// 3.5 TB/s.
template <int W, int NV, int EU, typename T, typename TT, bool REST, bool GRAD>
__global__ __launch_bounds__(64 * W, EU) void distill_kernel(DistillArgs p) {
    extern __shared__ unsigned int lds[];
    __shared__ DistillShared<W> s;
    const unsigned int n = p.x.n, k = p.k;
    const unsigned int words = (n + 31u) / 32u + 1u;
    const Entries en{reinterpret_cast<int*>(lds + words), reinterpret_cast<float*>(lds + words + k),
                     reinterpret_cast<float*>(lds + words + 2u * k)};
    const unsigned long long row = workgroup_row();
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    Global<T>* g = global_out<T>(p.grad) + row * p.grad_stride;
    const float weight = p.weight ? global_in<float>(p.weight)[row] : 1.f;
    if (weight == 0.f) {
        if (threadIdx.x == 0) p.loss[row] = 0.f;
        if (GRAD) put_zeros<W, T>(g, n);
    } else if constexpr (NV > 0) {
        distill_row<W, T, TT, REST, GRAD>(p, row, weight, x, g, HeldRow<W, NV, T, false>(x, 0, n), lds, words, en, s);
    } else {
        distill_row<W, T, TT, REST, GRAD>(p, row, weight, x, g, ReadRow<W, W == 8 ? 8 : 4, T, false>(x, 0, n), lds, words, en, s);
    }
}

// ------------------------------------------------------------------------------------- few long rows, in pieces
// A row in up to 64 pieces of a workgroup each: one launch for the pieces' maxima and sums, one that joins them and writes
// the pieces' gradients.  The first also fetches the student's logits of the entries, since the second may overwrite them.
struct Pieces {
    unsigned int count, length;   // of a row; the last piece takes what is left
};
struct PieceSum {
    MaxSum sum;
    unsigned int twice, pad_;
};
static_assert(sizeof(PieceSum) == 24, "as the workspace is counted");

Pieces pieces_of(unsigned long long rows, unsigned int n) {
    // Where a workgroup a row leaves most of the 256 compute units idle and a row takes one of them longer than a second launch
    // does (about 5 us): up to 128 rows of more than 32,768 actions, 32 rows of more than 16,384.  One workgroup a
    // row -> pieces, us: 11 x 131071 fp32 44 -> 17, 128 x 50000 fp32 30 -> 27 (its loss alone 27 -> 18), 128 x 100000 bf16
    // 34 -> 30; beyond the limits 64 x 20000 fp32 13 -> 16, 128 x 32768 bf16 16 -> 18, 256 x 100000 bf16 37 -> 45.
    // (no rows, no pieces)
    if (rows == 0 || rows > (n > 32768u ? 128u : 32u) || n <= 16384u) return Pieces{1u, n};
    const unsigned int most = (unsigned int)((1024u + rows - 1u) / rows);
    unsigned int count = n / 2048u;
    count = count > most ? most : count;
    count = count > 64u ? 64u : count;
    const unsigned int length = (n / count + 63u) / 64u * 64u;
    count = n / length;
    return Pieces{count, length};
}
size_t pieces_bytes(unsigned long long rows, unsigned int n, unsigned int k) {
    const Pieces c = pieces_of(rows, n);
    return c.count == 1u ? 0 : align_up(rows * c.count * sizeof(PieceSum), 256) + align_up(rows * k * 4u, 256);
}

template <int W, typename T, typename TT, bool REST>
__global__ __launch_bounds__(64 * W, 4) void distill_piece_kernel(DistillArgs p, Pieces c, PieceSum* sums, float* z) {
    extern __shared__ unsigned int named[];
    __shared__ MaxSum part[W];
    __shared__ unsigned int twice;
    const unsigned int tid = threadIdx.x, k = p.k, piece = blockIdx.x;
    const unsigned long long row = blockIdx.y;
    if ((p.weight ? global_in<float>(p.weight)[row] : 1.f) == 0.f) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const unsigned int begin = piece * c.length, end = piece + 1u == c.count ? p.x.n : begin + c.length;
    for (unsigned int i = tid; i < (end - begin + 31u) / 32u + 1u; i += 64 * W) named[i] = 0;
    if (tid == 0) twice = 0;
    __syncthreads();
    for (unsigned int e = tid; e < k; e += 64 * W) {
        const unsigned int a = (unsigned int)global_in<int>(p.entry)[row * k + e];
        if (a >= begin && a < end) {
            const unsigned int at = a - begin, bit = 1u << (at & 31u);
            if (atomicOr(&named[at >> 5], bit) & bit) twice = 1;
            global_out<float>(z)[row * k + e] = logit_value(x + a);
        }
    }
    __syncthreads();
    const ReadRow<W, 4, T, false> read(x, begin, end);
    const MaxSum mine = sum_row<REST, T>(read, read, begin, named, p.c2);
    if ((tid & 63u) == 0) part[tid >> 6] = mine;
    __syncthreads();
    if (tid == 0) {
        float m = part[0].m;
        for (int w = 1; w < W; ++w) m = fmaxf(m, part[w].m);
        double sum = 0.0;
        for (int w = 0; w < W; ++w)
            if (!(part[w].s == 0.0)) sum += part[w].s * (part[w].m > -INFINITY ? exp(((double)part[w].m - (double)m) * p.inv_ts) : 1.0);
        sums[row * c.count + piece] = PieceSum{MaxSum{m, sum}, twice, 0};
    }
}

template <int W, typename T, typename TT, bool REST, bool GRAD>
__global__ __launch_bounds__(64 * W, 4) void distill_join_kernel(DistillArgs p, Pieces c, const PieceSum* sums, const float* z) {
    extern __shared__ unsigned int lds[];
    __shared__ DistillShared<W> s;
    const unsigned int tid = threadIdx.x, k = p.k, piece = blockIdx.x;
    const unsigned long long row = blockIdx.y;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    Global<T>* g = global_out<T>(p.grad) + row * p.grad_stride;
    const unsigned int begin = piece * c.length, end = piece + 1u == c.count ? p.x.n : begin + c.length;
    const float weight = p.weight ? global_in<float>(p.weight)[row] : 1.f;
    if (weight == 0.f) {
        if (tid == 0 && piece == 0) p.loss[row] = 0.f;
        if (GRAD) put_zeros<W, T>(g + begin, end - begin);
        return;
    }
    const Entries en{reinterpret_cast<int*>(lds), reinterpret_cast<float*>(lds + k), reinterpret_cast<float*>(lds + 2u * k)};
    // (the pieces' sums, a lane each, as one)
    float m = -INFINITY;
    double sum = 0.0;
    unsigned int twice = 0;
    if (tid < c.count) {
        const PieceSum& q = sums[row * c.count + tid];
        m = q.sum.m;
        sum = q.sum.s;
        twice = q.twice;
    }
    load_entries<W, T, TT, false>(p, row, x, z, 0, 0, en, nullptr, s);
    if (tid < 64) {
        const float all = wave_reduce(m, MaxOp{});
        if (!(sum == 0.0) && m > -INFINITY) sum *= exp(((double)m - (double)all) * p.inv_ts);
        sum = wave_reduce(sum, SumOp{});
        twice = __ballot(twice) != 0;
        if (tid == 0) {
            s.row[0] = MaxSum{all, sum};
            s.twice = twice;
        }
    }
    __syncthreads();
    sum_entries<W, REST>(p, row, en, s);
    __syncthreads();
    if (tid < 64) finish_row<REST>(p, row, weight, s.part, W, s.row, 1, &s.out, piece == 0);
    if (!GRAD) return;
    __syncthreads();
    put_gradient<T>(ReadRow<W, 4, T, false>(x, begin, end), g, s.out, p.c2);
    __syncthreads();   // (an action with an entry is written again)
    if (s.out.state == 0) put_entries<W, T, REST>(p, g, en, begin, end, s.out, s.twice != 0);
}

template <typename T, typename TT, bool REST, bool GRAD>
hipError_t launch_rows(const DistillArgs& a, void* workspace, hipStream_t st) {
    const unsigned int n = a.x.n;
    const dim3 blocks = row_grid(a.x.rows);
    const size_t lds = ((n + 31u) / 32u + 1u + 3u * a.k) * 4u;
    const Pieces c = pieces_of(a.x.rows, n);
    if (c.count > 1u) {
        const unsigned int rows = (unsigned int)a.x.rows;
        PieceSum* sums = static_cast<PieceSum*>(workspace);
        float* z = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + align_up(rows * c.count * sizeof(PieceSum), 256));
        const size_t marks = ((n - (c.count - 1u) * c.length + 31u) / 32u + 1u) * 4u;
        distill_piece_kernel<4, T, TT, REST><<<dim3(c.count, rows), 256, marks, st>>>(a, c, sums, z);
        distill_join_kernel<4, T, TT, REST, GRAD><<<dim3(GRAD ? c.count : 1u, rows), 256, 12u * a.k, st>>>(a, c, sums, z);
        return hipGetLastError();
    }
    if (n <= 256u) {
        distill_wave_kernel<4, T, TT, REST, GRAD><<<blocks, 64, (8u + 3u * a.k) * 4u, st>>>(a);
    } else if constexpr (!GRAD) {
        if (n <= 2048u) distill_kernel<1, 0, 4, T, TT, REST, GRAD><<<blocks, 64, lds, st>>>(a);
        else distill_kernel<4, 0, 4, T, TT, REST, GRAD><<<blocks, 256, lds, st>>>(a);
    } else {
        if (n <= HeldRow<1, 4, T>::kMost) distill_kernel<1, 4, 4, T, TT, REST, GRAD><<<blocks, 64, lds, st>>>(a);
        else if (n <= HeldRow<2, 8, T>::kMost) distill_kernel<2, 8, 3, T, TT, REST, GRAD><<<blocks, 128, lds, st>>>(a);
        else if (n <= HeldRow<4, 8, T>::kMost) distill_kernel<4, 8, 4, T, TT, REST, GRAD><<<blocks, 256, lds, st>>>(a);
        else if (n <= HeldRow<4, 16, T>::kMost) distill_kernel<4, 16, 4, T, TT, REST, GRAD><<<blocks, 256, lds, st>>>(a);
        else if (n <= HeldRow<8, 16, T>::kMost) distill_kernel<8, 16, 4, T, TT, REST, GRAD><<<blocks, 512, lds, st>>>(a);
        else distill_kernel<8, 0, 4, T, TT, REST, GRAD><<<blocks, 512, lds, st>>>(a);
    }
    return hipGetLastError();
}
template <typename T, typename TT>
hipError_t launch_distill(const DistillArgs& a, bool gradient, void* ws, hipStream_t st) {
    if (a.teacher_lse) return gradient ? launch_rows<T, TT, true, true>(a, ws, st) : launch_rows<T, TT, true, false>(a, ws, st);
    return gradient ? launch_rows<T, TT, false, true>(a, ws, st) : launch_rows<T, TT, false, false>(a, ws, st);
}

}  // namespace

rp_status distill_rows(const char* what, const rp_rows* logits, const rp_teacher* teacher, float* loss, void* grad,
                       uint64_t grad_stride, bool gradient, double scale, void* workspace, size_t bytes, void* hip_stream) {
    const char* why = logit_rows_fault(logits);
    RP_REQUIRE(!why, "%s: %s", what, why);
    RP_REQUIRE(teacher, "%s: null teacher", what);
    RP_REQUIRE(teacher->k >= 1 && teacher->k <= kMaxTop, "%s: k = %u, must be 1 .. 1024", what, teacher->k);
    RP_REQUIRE(teacher->dtype == RP_F32 || teacher->dtype == RP_BF16, "%s: the teacher's logits must be RP_F32 or RP_BF16", what);
    RP_REQUIRE(temperature_fits(teacher->temperature) && temperature_fits(teacher->student_temperature),
               "%s: temperatures must be 1e-30 .. 1e30", what);
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
    const size_t need = pieces_bytes(logits->rows, logits->n, teacher->k);
    if (const char* fault = workspace_fault(workspace, bytes, need)) {
        set_error("%s: %s (%zu bytes given, %zu needed)", what, fault, bytes, need);
        return RP_ENOMEM;
    }
    const DistillArgs a{logit_rows(logits), static_cast<const unsigned char*>(teacher->value), teacher->index, teacher->lse,
                        teacher->weight, teacher->k, 1.0 / teacher->temperature, 1.0 / teacher->student_temperature, scale,
                        (float)(1.4426950408889634 / teacher->student_temperature), loss,
                        static_cast<unsigned char*>(grad), grad_stride};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool xb = logits->dtype == RP_BF16, tb = teacher->dtype == RP_BF16;
    typedef unsigned short B;
    RP_CHECK_HIP(xb ? (tb ? launch_distill<B, B>(a, gradient, workspace, st) : launch_distill<B, float>(a, gradient, workspace, st))
                    : (tb ? launch_distill<float, B>(a, gradient, workspace, st) : launch_distill<float, float>(a, gradient, workspace, st)));
    return RP_OK;
}

}  // namespace rp

extern "C" {

size_t rp_distill_workspace_bytes(const rp_rows* logits, uint32_t k) {
    const char* why = rp::logit_rows_fault(logits);
    if (!why && (k == 0 || k > rp::kMaxTop)) why = "k must be 1 .. 1024";
    if (why) {
        rp::set_error("rp_distill_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return rp::pieces_bytes(logits->rows, logits->n, k);
}

rp_status rp_distill_loss(const rp_rows* logits, const rp_teacher* teacher, float* loss, void* workspace, size_t bytes,
                          void* hip_stream) {
    return rp::distill_rows("rp_distill_loss", logits, teacher, loss, nullptr, 0, false, 1.0, workspace, bytes, hip_stream);
}

rp_status rp_distill_grad(const rp_rows* logits, const rp_teacher* teacher, float* loss, void* grad, uint64_t grad_stride,
                          void* workspace, size_t bytes, void* hip_stream) {
    return rp::distill_rows("rp_distill_grad", logits, teacher, loss, grad, grad_stride, true, 1.0, workspace, bytes, hip_stream);
}

}  // extern "C"
