// Rows of logits: what the operators on them share on the device and on the host.
#pragma once

#include <cmath>

#include "common.hpp"

namespace rp {

constexpr unsigned int kMaxActions = 1u << 18;   // a row's length
constexpr unsigned int kMaxTop = 1024;           // entries of a teacher's row
constexpr unsigned long long kMaxLogitRows = 1ull << 24;

struct LogitRows {
    const unsigned char* data;
    unsigned long long rows, stride;
    unsigned int n;
};

// Pointers to global memory by their type: a pointer whose memory the compiler has to find out at run time costs a load
// that also counts as one of LDS.
template <typename T>
using Global = T __attribute__((address_space(1)));
template <typename T>
__device__ __forceinline__ const Global<T>* global_in(const void* p) { return (const Global<T>*)p; }
template <typename T>
__device__ __forceinline__ Global<T>* global_out(void* p) { return (Global<T>*)p; }

__device__ __forceinline__ float logit_value(const Global<float>* p) { return *p; }
__device__ __forceinline__ float logit_value(const Global<unsigned short>* p) { return __uint_as_float((unsigned int)*p << 16); }

// What is not allowed (NaN, -infinity) becomes -infinity and -0 becomes +0, so that equal logits have
// equal keys.
__device__ __forceinline__ float clean_logit(float x) { return fmaxf(x, -INFINITY) + 0.f; }

// 16 bytes of a row, at any alignment the row's elements have.
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <typename T>
constexpr unsigned int kPerLoad = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ float element(const u32x4& raw, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[e]);
    else return __uint_as_float(e & 1 ? raw[e >> 1] & 0xFFFF0000u : raw[e >> 1] << 16);
}
// A thread's elements i .. of a row that ends at `end` (and has a load's worth of elements at least): the load
// that would pass the end is moved back to it, and what belongs to the thread before comes as -infinity.
template <typename T>
__device__ __forceinline__ unsigned int load_place(unsigned int i, unsigned int end) { return min(i, end - kPerLoad<T>); }
template <typename T>
__device__ __forceinline__ void mask_moved(u32x4& raw, unsigned int i, unsigned int place) {
    if (place == i) return;
    const unsigned int gone = i - place;   // elements of the load that are not this thread's
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            if ((unsigned int)j < gone) raw[j] = 0xFF800000u;
        } else {
            if (2u * j < gone) raw[j] = (raw[j] & 0xFFFF0000u) | 0xFF80u;
            if (2u * j + 1u < gone) raw[j] = (raw[j] & 0xFFFFu) | 0xFF800000u;
        }
    }
}

// A row, or a piece of one, spread over a workgroup's registers: NV loads of 16 bytes a thread.  `each` hands
// every element to f(value, place in the row, place in its load); what is past the end comes as -infinity.  `each_load` hands
// whole loads to f(16 bytes, place of their first element, how many of them are another thread's): with MASK these
// come as -infinity, without as they are.
template <int W, int NV, typename T, bool MASK = true>
struct HeldRow {
    u32x4 raw[NV];
    static constexpr bool kHeld = true;
    unsigned int begin, first, last;   // the piece's first element and the thread's; where the last load starts
    static constexpr unsigned int kStep = 64u * W * kPerLoad<T>;
    static constexpr unsigned int kMost = NV * kStep;
    __device__ __forceinline__ HeldRow(const Global<T>* x, unsigned int begin_, unsigned int end) {
        begin = begin_;
        first = begin + threadIdx.x * kPerLoad<T>;
        last = end - kPerLoad<T>;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            raw[v] = *(const Global<u32x4_any>*)(x + min(first + v * kStep, last));
        // (a branch that the whole workgroup takes: rows mostly fill their loads)
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (MASK && begin + (v + 1) * kStep > end) mask_moved<T>(raw[v], first + v * kStep, min(first + v * kStep, last));
    }
    template <typename F>
    __device__ __forceinline__ void each_load(F f) const {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v && last + kPerLoad<T> <= begin + v * kStep) continue;   // (nothing of the row)
            u32x4 r = raw[v];
            unsigned int i = first;
            asm volatile("" : "+v"(r), "+v"(i));
            i += v * kStep;
            f(r, min(i, last), i - min(i, last));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            // (each pass decodes the elements, and works out their places, anew: kept from one pass to the next
            // they would fill the registers)
            u32x4 r = raw[v];
            unsigned int at = first;
            asm volatile("" : "+v"(r), "+v"(at));
            at = min(at + v * kStep, last);
#pragma unroll
            for (int e = 0; e < (int)kPerLoad<T>; ++e) f(element<T>(r, e), at + e, e);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// The same interface over memory, for rows that registers do not hold: every pass reads the row again, NV loads a thread at a
// time, all under way before the first is used.
template <int W, int NV, typename T, bool MASK = true>
struct ReadRow {
    static constexpr bool kHeld = false;
    const Global<T>* x;
    unsigned int begin, end;
    __device__ __forceinline__ ReadRow(const Global<T>* x_, unsigned int begin_, unsigned int end_) : x(x_), begin(begin_), end(end_) {}
    template <typename F>
    __device__ __forceinline__ void each_load(F f) const {
#pragma unroll 1
        for (unsigned int at = begin; at < end; at += HeldRow<W, NV, T, MASK>::kMost) HeldRow<W, NV, T, MASK>(x, at, end).each_load(f);
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
        for (unsigned int at = begin; at < end; at += HeldRow<W, NV, T, MASK>::kMost) HeldRow<W, NV, T, MASK>(x, at, end).each(f);
    }
};

// Unsigned integers in the order of the floats.
__device__ __forceinline__ unsigned int order_key(float x) {
    const unsigned int b = __float_as_uint(x);
    return b ^ ((unsigned int)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned int k) {
    return __uint_as_float(k ^ ((unsigned int)((int)~k >> 31) | 0x80000000u));
}
__device__ __forceinline__ unsigned int logit_key(float x) { return order_key(clean_logit(x)); }
constexpr unsigned int kMaskedKey = 0x007FFFFFu;   // order_key(-infinity)

// An action in the order of choice as one number, the first the largest: falling logit, rising index.
__device__ __forceinline__ unsigned long long order_word(unsigned int key, unsigned int index) {
    return (unsigned long long)key << 32 | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ unsigned int word_index(unsigned long long w) { return 0xFFFFFFFFu - (unsigned int)w; }
__device__ __forceinline__ unsigned int word_key(unsigned long long w) { return (unsigned int)(w >> 32); }

// -log of an allowed action's weight: (m - x) / temperature.  The row's maximum m may be +infinity; a logit equal
// to it has weight 1 whatever the temperature, any other is then infinitely far away.
__device__ __forceinline__ double logit_depth(float m, float x, double inv_t) {
    return x == m ? 0.0 : isinf(m) ? (double)INFINITY : ((double)m - (double)x) * inv_t;
}

struct MaxOp {
    template <typename V>
    __device__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct MinOp {
    template <typename V>
    __device__ V operator()(V a, V b) const { return a < b ? a : b; }
};
struct SumOp {
    template <typename V>
    __device__ V operator()(V a, V b) const { return a + b; }
};

template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V v, Op op) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off, 64));
    return v;
}

// The same value in every thread of a workgroup of W wavefronts, combined in a fixed order.  `part` holds W
// values; a barrier has to stand between two uses of it.
template <int W, typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V* part) {
    v = wave_reduce(v, op);
    if (W == 1) return v;
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    V all = part[0];
#pragma unroll
    for (int w = 1; w < W; ++w) all = op(all, part[w]);
    return all;
}

// A workgroup a row, in several rows of workgroups where one would have 2^32 threads.  (A loop over rows in the kernel would
// have the compiler keep what does not change from one to the next in the registers that the row needs.)
__device__ __forceinline__ unsigned long long workgroup_row() { return (unsigned long long)blockIdx.y * gridDim.x + blockIdx.x; }
inline dim3 row_grid(unsigned long long rows) {
    const unsigned long long x = rows < (1ull << 16) ? rows : (1ull << 16);
    return dim3((unsigned int)x, (unsigned int)((rows + x - 1) / x));
}

// Host side: rows that the kernels can be given, or why not.
inline const char* logit_rows_fault(const rp_rows* r) {
    if (!r) return "null rows";
    if (r->dtype != RP_F32 && r->dtype != RP_BF16) return "logits must be RP_F32 or RP_BF16";
    if (r->n == 0 || r->n > kMaxActions) return "a row holds 1 to 262144 actions";
    if (r->rows > kMaxLogitRows) return "more than 2^24 rows";
    if (r->stride > (1ull << 40)) return "row stride beyond 2^40";
    return nullptr;
}
inline const char* logit_data_fault(const rp_rows* r) {
    if (!r->data) return "null logits";
    if (reinterpret_cast<uintptr_t>(r->data) & (r->dtype == RP_BF16 ? 1u : 3u)) return "logits not aligned to their type";
    return nullptr;
}
// Temperatures of losses and log-sum-exps: within these ends 1 / t and log2(e) / t are numbers in 32 bits.
inline bool temperature_fits(double t) { return t >= 1e-30 && t <= 1e30; }
inline const char* workspace_fault(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return nullptr;
    if (!workspace || bytes < need) return "the workspace is too small";
    return reinterpret_cast<uintptr_t>(workspace) & 255u ? "the workspace must be 256-byte aligned" : nullptr;
}
inline LogitRows logit_rows(const rp_rows* r) {
    return LogitRows{static_cast<const unsigned char*>(r->data), r->rows, r->stride, r->n};
}

// rp_distill_loss (gradient false) and rp_distill_grad, the gradient times `scale` as well; `what` names the entry point in
// messages.
rp_status distill_rows(const char* what, const rp_rows* logits, const rp_teacher* teacher, float* loss, void* grad,
                       uint64_t grad_stride, bool gradient, double scale, void* workspace, size_t bytes, void* hip_stream);

}  // namespace rp
