// Choosing actions from rows of logits (temperature, top-k, top-p, min-p, given random numbers) and a
// row's top actions with its log-sum-exp.
#include "logits.hpp"

namespace rp {
namespace {

struct ChooseArgs {
    LogitRows x;
    double temperature, top_p, min_p;
    long long top_k;
    const float *row_temperature, *row_top_p, *row_min_p;
    const int* row_top_k;
    const float* u;
    int* index;
    float* logp;
};

struct TopArgs {
    LogitRows x;
    unsigned int k;
    double inv_t;
    unsigned char* values;
    int* index;
    float* lse;
};

// ------------------------------------------------------------------- one workgroup per row, by search
// A weight as a 64-bit whole number, 2^44 for the best action: sums of them do not depend on their order, and
// the 2^18 weights of the longest row stay below 2^63.
constexpr double kOne = 17592186044416.0;   // 2^44

__device__ __forceinline__ unsigned long long fixed_weight(float m, float x, double inv_t) {
    return x == -INFINITY ? 0ull : (unsigned long long)(exp(-logit_depth(m, x, inv_t)) * kOne + 0.5);
}

template <int W>
struct SearchShared {
    unsigned long long sum[2][W];
    unsigned int count[2][W];
    unsigned int base;
};

// Sums over the row: the weights and the number of the logits that `in` takes.
template <int W, typename T, typename In>
__device__ void search_sum(const T* x, unsigned int n, float m, double inv_t, In in, SearchShared<W>& s, unsigned int& turn,
                           unsigned long long* mass, unsigned int* count) {
    unsigned long long a = 0;
    unsigned int c = 0;
    for (unsigned int i = threadIdx.x; i < n; i += 64 * W) {
        const float v = clean_logit(logit_value(x + i));
        if (!in(order_key(v)) || v == -INFINITY) continue;
        ++c;
        if (mass) a += fixed_weight(m, v, inv_t);
    }
    // (two sets of partial sums in turn: a set is used again only after the barrier of the other's use)
    turn ^= 1u;
    if (mass) *mass = block_reduce<W>(a, SumOp{}, s.sum[turn]);
    if (count) *count = block_reduce<W>(c, SumOp{}, s.count[turn]);
}

// Place of the `c`-th (from 1) logit with key v, by index.
template <int W, typename T>
__device__ unsigned int search_equal(const T* x, unsigned int n, unsigned int v, unsigned int c, SearchShared<W>& s) {
    const unsigned int lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    unsigned int found = 0xFFFFFFFFu, before = 0;
    for (unsigned int i0 = 0; i0 < n; i0 += 64 * W) {
        const unsigned int i = i0 + threadIdx.x;
        const bool hit = i < n && order_key(clean_logit(logit_value(x + i))) == v;
        const unsigned long long hits = __ballot(hit);
        __syncthreads();
        if (lane == 0) s.count[0][wave] = __popcll(hits);
        __syncthreads();
        unsigned int at = before, all = 0;
        for (unsigned int w = 0; w < W; ++w) {
            if (w < wave) at += s.count[0][w];
            all += s.count[0][w];
        }
        at += __popcll(hits & ((1ull << lane) - 1ull)) + 1u;
        if (hit && at == c) s.base = i;
        before += all;
        if (before >= c) break;
    }
    __syncthreads();
    found = s.base;
    return found;
}

// The largest key v in [lo, hi] whose logits and those above it satisfy `enough` (monotone in v; the lowest does).
template <int W, typename Enough>
__device__ unsigned int search_key(unsigned int lo, unsigned int hi, Enough enough) {
    while (lo < hi) {
        const unsigned int mid = lo + (hi - lo) / 2u + ((hi - lo) & 1u);
        if (enough(mid)) lo = mid;
        else hi = mid - 1u;
    }
    return lo;
}

template <int W, typename T>
__device__ void choose_by_search(const ChooseArgs& p, unsigned long long row, SearchShared<W>& s) {
    const T* x = reinterpret_cast<const T*>(p.x.data) + row * p.x.stride;
    const unsigned int n = p.x.n;
    unsigned int turn = 0;
    // the allowed logits' range and number
    unsigned int hi = kMaskedKey, lo = 0xFFFFFFFFu, allowed = 0;
    for (unsigned int i = threadIdx.x; i < n; i += 64 * W) {
        const float v = clean_logit(logit_value(x + i));
        if (v == -INFINITY) continue;
        const unsigned int k = order_key(v);
        hi = max(hi, k);
        lo = min(lo, k);
        ++allowed;
    }
    __syncthreads();
    hi = block_reduce<W>(hi, MaxOp{}, s.count[0]);
    lo = block_reduce<W>(lo, MinOp{}, s.count[1]);
    __syncthreads();
    allowed = block_reduce<W>(allowed, SumOp{}, s.count[0]);
    __syncthreads();
    if (allowed == 0) {
        if (threadIdx.x == 0) {
            p.index[row] = -1;
            if (p.logp) p.logp[row] = 0.f;
        }
        return;
    }
    const double t = p.row_temperature ? (double)p.row_temperature[row] : p.temperature;
    if (!(t > 0.0)) {
        const unsigned int at = search_equal<W>(x, n, hi, 1, s);
        if (threadIdx.x == 0) {
            p.index[row] = (int)at;
            if (p.logp) p.logp[row] = 0.f;
        }
        return;
    }
    const double inv_t = 1.0 / t;
    const float m = key_value(hi);
    const long long k = p.row_top_k ? (long long)p.row_top_k[row] : p.top_k;
    const double top_p = p.row_top_p ? (double)p.row_top_p[row] : p.top_p;
    const double min_p = p.row_min_p ? (double)p.row_min_p[row] : p.min_p;

    // inclusive sum of the first action in order at which the sum reaches `need`
    unsigned int at_key, at_count;
    auto reach = [&](unsigned long long need) {
        at_key = search_key<W>(lo, hi, [&](unsigned int v) {
            unsigned long long a;
            search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return key >= v; }, s, turn, &a, nullptr);
            return a >= need;
        });
        unsigned long long above;
        search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return key > at_key; }, s, turn, &above, nullptr);
        const unsigned long long w = fixed_weight(m, key_value(at_key), inv_t);
        at_count = w ? (unsigned int)((need - above + w - 1) / w) : 1u;
        return above + at_count * w;
    };

    unsigned long long mass;
    if (k > 0 && k < (long long)allowed) {
        const unsigned int v = search_key<W>(lo, hi, [&](unsigned int v) {
            unsigned int c;
            search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return key >= v; }, s, turn, nullptr, &c);
            return c >= (unsigned int)k;
        });
        unsigned int c;
        search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return key > v; }, s, turn, &mass, &c);
        mass += ((unsigned int)k - c) * fixed_weight(m, key_value(v), inv_t);
    } else {
        search_sum<W>(x, n, m, inv_t, [&](unsigned int) { return true; }, s, turn, &mass, nullptr);
    }
    const unsigned long long total = mass;
    if (top_p < 1.0) {
        const double need = ceil(top_p * (double)total);
        mass = reach(need >= 1.0 ? min((unsigned long long)need, total) : 1ull);
    }
    if (min_p > 0.0) {
        unsigned long long a;
        search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return exp(-logit_depth(m, key_value(key), inv_t)) >= min_p; },
                      s, turn, &a, nullptr);
        mass = min(mass, a);
    }
    if (mass < (unsigned long long)kOne) mass = (unsigned long long)kOne;
    const float u = p.u[row];
    const double drawn = u > 0.f ? (double)u * (double)mass : 0.0;
    reach(drawn < (double)mass ? min((unsigned long long)drawn + 1ull, mass) : mass);
    const unsigned int at = search_equal<W>(x, n, at_key, at_count, s);
    if (threadIdx.x == 0) {
        p.index[row] = (int)at;
        if (p.logp) p.logp[row] = (float)(-logit_depth(m, key_value(at_key), inv_t) - log((double)mass / kOne));
    }
}

template <int W, typename T>
__global__ __launch_bounds__(64 * W) void choose_search_kernel(ChooseArgs p) {
    __shared__ SearchShared<W> s;
    for (unsigned long long row = blockIdx.x; row < p.x.rows; row += gridDim.x) {
        choose_by_search<W, T>(p, row, s);
        __syncthreads();
    }
}

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(unsigned short* p, float v) { *p = (unsigned short)(__float_as_uint(v) >> 16); }

// Sorts `count` (a power of two) numbers in LDS, the largest first.
template <int W>
__device__ void sort_words(unsigned long long* w, unsigned int count) {
    for (unsigned int size = 2; size <= count; size <<= 1)
        for (unsigned int gap = size >> 1; gap; gap >>= 1) {
            __syncthreads();
            for (unsigned int t = threadIdx.x; t < count / 2u; t += 64 * W) {
                const unsigned int i = 2u * t - (t & (gap - 1u)), j = i + gap;
                const unsigned long long a = w[i], b = w[j];
                if ((a < b) == ((i & size) == 0)) {
                    w[i] = b;
                    w[j] = a;
                }
            }
        }
    __syncthreads();
}

template <int W, typename T>
__global__ __launch_bounds__(64 * W) void top_search_kernel(TopArgs p) {
    __shared__ SearchShared<W> s;
    __shared__ unsigned long long words[kMaxTop];
    __shared__ unsigned int taken;
    __shared__ double part[2][W];
    const unsigned int n = p.x.n;
    for (unsigned long long row = blockIdx.x; row < p.x.rows; row += gridDim.x) {
        const T* x = reinterpret_cast<const T*>(p.x.data) + row * p.x.stride;
        unsigned int turn = 0, hi = kMaskedKey, allowed = 0;
        for (unsigned int i = threadIdx.x; i < n; i += 64 * W) {
            const unsigned int k = order_key(clean_logit(logit_value(x + i)));
            hi = max(hi, k);
            allowed += k > kMaskedKey;
        }
        __syncthreads();
        hi = block_reduce<W>(hi, MaxOp{}, s.count[0]);
        allowed = block_reduce<W>(allowed, SumOp{}, s.count[1]);
        __syncthreads();
        const float m = key_value(hi);
        if (p.lse) {
            double a = 0.0;
            if (allowed)
                for (unsigned int i = threadIdx.x; i < n; i += 64 * W) {
                    const float v = clean_logit(logit_value(x + i));
                    if (v != -INFINITY) a += exp(-logit_depth(m, v, p.inv_t));
                }
            a = block_reduce<W>(a, SumOp{}, part[0]);
            if (threadIdx.x == 0) p.lse[row] = allowed ? (float)((double)m * p.inv_t + log(a)) : -INFINITY;
        }
        const unsigned int k = min(p.k, allowed);
        unsigned int v = 0, above = 0;
        if (k) {
            v = search_key<W>(kMaskedKey + 1u, hi, [&](unsigned int v) {
                unsigned int c;
                search_sum<W>(x, n, m, 0.0, [&](unsigned int key) { return key >= v; }, s, turn, nullptr, &c);
                return c >= k;
            });
            search_sum<W>(x, n, m, 0.0, [&](unsigned int key) { return key > v; }, s, turn, nullptr, &above);
        }
        // the logits above v in any order, then the first k - above equal to it
        for (unsigned int i = threadIdx.x; i < kMaxTop; i += 64 * W) words[i] = 0;
        if (threadIdx.x == 0) taken = 0;
        __syncthreads();
        const unsigned int lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
        unsigned int equal_before = 0;
        if (k)
            for (unsigned int i0 = 0; i0 < n; i0 += 64 * W) {
                const unsigned int i = i0 + threadIdx.x;
                const unsigned int key = i < n ? order_key(clean_logit(logit_value(x + i))) : 0u;
                if (key > v) words[atomicAdd(&taken, 1u)] = order_word(key, i);
                const unsigned long long hits = __ballot(key == v);
                __syncthreads();
                if (lane == 0) s.count[0][wave] = __popcll(hits);
                __syncthreads();
                unsigned int at = equal_before + __popcll(hits & ((1ull << lane) - 1ull));
                for (unsigned int w = 0; w < W; ++w) {
                    if (w < wave) at += s.count[0][w];
                    equal_before += s.count[0][w];
                }
                if (key == v && above + at < k) words[above + at] = order_word(key, i);
            }
        unsigned int padded = 2;
        while (padded < p.k) padded <<= 1;
        sort_words<W>(words, padded);
        for (unsigned int j = threadIdx.x; j < p.k; j += 64 * W) {
            const unsigned long long at = row * p.k + j;
            store_value(reinterpret_cast<T*>(p.values) + at, j < k ? key_value(word_key(words[j])) : -INFINITY);
            p.index[at] = j < k ? (int)word_index(words[j]) : -1;
        }
        __syncthreads();
    }
}

// Workgroups of one launch: a row each, more rows than that in turn.
unsigned int row_blocks(unsigned long long rows) { return (unsigned int)(rows < (1ull << 18) ? rows : (1ull << 18)); }

}  // namespace
}  // namespace rp

extern "C" {

size_t rp_choose_workspace_bytes(const rp_rows* logits) {
    if (const char* why = rp::logit_rows_fault(logits)) {
        rp::set_error("rp_choose_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return 0;
}

rp_status rp_choose_actions(const rp_rows* logits, const rp_choice* how, const float* u, int32_t* index, float* logp,
                            void* workspace, size_t bytes, void* hip_stream) {
    const char* why = rp::logit_rows_fault(logits);
    RP_REQUIRE(!why, "rp_choose_actions: %s", why);
    RP_REQUIRE(how, "rp_choose_actions: null settings");
    if (logits->rows == 0) return RP_OK;
    why = rp::logit_data_fault(logits);
    RP_REQUIRE(!why, "rp_choose_actions: %s", why);
    RP_REQUIRE(u && index, "rp_choose_actions: null array");
    (void)workspace;
    (void)bytes;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const rp::ChooseArgs a{rp::logit_rows(logits), how->temperature, how->top_p, how->min_p, how->top_k,
                           how->row_temperature, how->row_top_p, how->row_min_p, how->row_top_k, u, index, logp};
    const dim3 grid(rp::row_blocks(logits->rows));
    if (logits->dtype == RP_BF16)
        hipLaunchKernelGGL((rp::choose_search_kernel<4, unsigned short>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((rp::choose_search_kernel<4, float>), grid, dim3(256), 0, st, a);
    RP_CHECK_HIP(hipGetLastError());
    return RP_OK;
}

size_t rp_top_workspace_bytes(const rp_rows* logits, uint32_t k) {
    const char* why = rp::logit_rows_fault(logits);
    if (!why && (k == 0 || k > rp::kMaxTop || k > logits->n)) why = "k must be 1 .. min(n, 1024)";
    if (why) {
        rp::set_error("rp_top_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return 0;
}

rp_status rp_top_actions(const rp_rows* logits, uint32_t k, double temperature, void* values, int32_t* index, float* lse,
                         void* workspace, size_t bytes, void* hip_stream) {
    const char* why = rp::logit_rows_fault(logits);
    RP_REQUIRE(!why, "rp_top_actions: %s", why);
    RP_REQUIRE(k >= 1 && k <= rp::kMaxTop && k <= logits->n, "rp_top_actions: k = %u, must be 1 .. min(n, 1024)", k);
    RP_REQUIRE(temperature > 0.0 && std::isfinite(temperature), "rp_top_actions: the temperature must be finite and > 0");
    if (logits->rows == 0) return RP_OK;
    why = rp::logit_data_fault(logits);
    RP_REQUIRE(!why, "rp_top_actions: %s", why);
    RP_REQUIRE(values && index, "rp_top_actions: null array");
    (void)workspace;
    (void)bytes;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const rp::TopArgs a{rp::logit_rows(logits), k, 1.0 / temperature, static_cast<unsigned char*>(values), index, lse};
    const dim3 grid(rp::row_blocks(logits->rows));
    if (logits->dtype == RP_BF16)
        hipLaunchKernelGGL((rp::top_search_kernel<4, unsigned short>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((rp::top_search_kernel<4, float>), grid, dim3(256), 0, st, a);
    RP_CHECK_HIP(hipGetLastError());
    return RP_OK;
}

}  // extern "C"
