// Choosing actions from rows of logits (temperature, top-k, top-p, min-p, given random numbers) and a
// row's top actions with its log-sum-exp.
//
// Both are about the order of a row by falling logit, of which only the front matters: nothing is sorted but the few
// actions around the places in question.  The least work is one reading of the row (HBM at 5.1 TB/s).  By length and number of
// rows:
//  - up to 64 actions: one wavefront, an action a lane; a lane finds its place by comparing with all (choose_wave_kernel).
//  - up to 16,384 / 32,768 actions in 32 / 16 bits: one workgroup that holds the row in registers, so that it is read once
//    (choose_kernel, top_kernel).
//  - longer rows, and few rows of more than 8192: a launch for pieces of the row, one that joins them.
// Top-k (up to 1024) and the best action: the k-th largest of the maxima of 1024 to 4096 slices of the row is a lower bound of
// the k-th largest logit and close to it; what is not below it is sorted in LDS.  All actions: a histogram of the
// weights, 2048 bins to 40 temperatures below the maximum; only bins where a sum ends are listed.  What these cannot take (more than
// 1024 kept by top-k, more than 2048 actions in a bin where a sum ends or above the bound, +infinity, a random number of 1 or
// more without top-k) is found by binary search over the values, a pass over the row for each step.  Flat rows come to that: a bin
// is 1/51 to 1/26 of a temperature wide and holds more than 2048 of 131,072 normal logits whose deviation is under 0.5 to 1
// temperatures.  1 x 131072 bf16 at a deviation of 0.5, top-p: 4.2 ms (torch 0.5), 256 rows 4.9 (3.7); top 2000 of one
// row 1.8 ms (0.5), of 256 3.4 (3.7).
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
    float c2;             // log2(e) / temperature
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
__device__ void search_sum(const Global<T>* x, unsigned int n, float m, double inv_t, In in, SearchShared<W>& s, unsigned int& turn,
                           unsigned long long* mass, unsigned int* count) {
    unsigned long long a = 0;
    unsigned int c = 0;
#pragma unroll 1
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
__device__ unsigned int search_equal(const Global<T>* x, unsigned int n, unsigned int v, unsigned int c, SearchShared<W>& s) {
    const unsigned int lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    unsigned int found = 0xFFFFFFFFu, before = 0;
#pragma unroll 1
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
#pragma unroll 1
    while (lo < hi) {
        const unsigned int mid = lo + (hi - lo) / 2u + ((hi - lo) & 1u);
        if (enough(mid)) lo = mid;
        else hi = mid - 1u;
    }
    return lo;
}

template <int W, typename T>
__device__ void choose_by_search(const ChooseArgs& p, unsigned long long row, SearchShared<W>& s) {
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const unsigned int n = p.x.n;
    unsigned int turn = 0;
    // the allowed logits' range and number
    unsigned int hi = kMaskedKey, lo = 0xFFFFFFFFu, allowed = 0;
#pragma unroll 1
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

    // the last action that stays, by key and place among equal ones, as each limit has it; kAll: the last one with that key
    constexpr unsigned int kAll = 0xFFFFFFFFu;
    unsigned int last_key = lo, last_count = kAll;
    auto ends = [&](unsigned int key, unsigned int count) {
        if (key > last_key || (key == last_key && count < last_count)) {
            last_key = key;
            last_count = count;
        }
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
        ends(v, (unsigned int)k - c);
    } else {
        search_sum<W>(x, n, m, inv_t, [&](unsigned int) { return true; }, s, turn, &mass, nullptr);
    }
    const unsigned long long total = mass;
    if (top_p < 1.0) {
        const double need = ceil(top_p * (double)total);
        mass = reach(need >= 1.0 ? min((unsigned long long)need, total) : 1ull);
        ends(at_key, at_count);
    }
    if (min_p > 0.0) {
        unsigned long long a;
        unsigned int least = hi;   // of this thread's
        search_sum<W>(x, n, m, inv_t, [&](unsigned int key) {
            const bool stays = exp(-logit_depth(m, key_value(key), inv_t)) >= min_p;
            if (stays) least = min(least, key);
            return stays;
        }, s, turn, &a, nullptr);
        mass = min(mass, a);
        // (the set that the next sums do not use)
        ends(block_reduce<W>(least, MinOp{}, s.count[turn]), min_p <= 1.0 ? kAll : 1u);
    }
    if (mass < (unsigned long long)kOne) mass = (unsigned long long)kOne;
    const float u = p.u[row];
    if (u >= 1.f) {
        at_key = last_key;
        at_count = last_count;
        if (at_count == kAll) search_sum<W>(x, n, m, inv_t, [&](unsigned int key) { return key == at_key; }, s, turn, nullptr, &at_count);
    } else {
        const double drawn = u > 0.f ? (double)u * (double)mass : 0.0;
        reach(min((unsigned long long)drawn + 1ull, mass));
    }
    const unsigned int at = search_equal<W>(x, n, at_key, at_count, s);
    if (threadIdx.x == 0) {
        p.index[row] = (int)at;
        if (p.logp) p.logp[row] = (float)(-logit_depth(m, key_value(at_key), inv_t) - log((double)mass / kOne));
    }
}


__device__ __forceinline__ void store_value(Global<float>* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(Global<unsigned short>* p, float v) { *p = (unsigned short)(__float_as_uint(v) >> 16); }

// ------------------------------------------------------------------- one workgroup per row, by candidates
constexpr unsigned int kBins = 2048;    // of the histogram of weights
constexpr unsigned int kList = 2048;    // actions that are sorted in LDS
constexpr unsigned int kSliceBins = 1024;
constexpr unsigned int kBuckets = 1024, kFine = 256;

template <int W>
struct ChooseShared {
    union {
        unsigned long long hist[kBins];     // 2^-44 of the weight at the bin's middle
        double sums[kBins];                 // inclusive sums over bins, or over a sorted list
        unsigned int slices[kSliceBins];
    };
    unsigned long long words[kList];
    union {
        unsigned int buckets[kBuckets + 1];
        unsigned long long fine[kFine];     // a bin's weights, by parts of the bin
    };
    SearchShared<W> search;
    double part[W];
    unsigned int wave_count[W];
    unsigned long long word;
    unsigned int taken, bin;
    float key;
};

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Sorts the `count` words in LDS, the largest first.  Up to 128: every thread ranks one against all.  More: 1024 buckets
// linear in the value, a count of each, every word to its bucket's place, and there a rank against its bucket.
template <int W>
__device__ void sort_words(ChooseShared<W>& s, unsigned int count) {
    const unsigned int tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    unsigned long long* w = s.words;
    if (count <= 128u) {
        unsigned long long mine = 0;
        unsigned int rank = 0;
        __syncthreads();
        if (tid < count) {
            mine = w[tid];
#pragma unroll 4
            for (unsigned int j = 0; j < count; ++j) rank += w[j] > mine;
        }
        __syncthreads();
        if (tid < count) w[rank] = mine;
        __syncthreads();
        return;
    }
    constexpr int kEach = kList / (64 * W), kPer = kBuckets / (64 * W);
    unsigned long long mine[kEach];
    unsigned int at[kEach];   // bucket << 16 | place in it
    float low = INFINITY, high = -INFINITY;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const unsigned int i = j * 64 * W + tid;
        mine[j] = i < count ? w[i] : 0ull;
        if (i < count) {
            low = fminf(low, key_value(word_key(mine[j])));
            high = fmaxf(high, key_value(word_key(mine[j])));
        }
    }
    low = wave_reduce(low, MinOp{});
    high = wave_reduce(high, MaxOp{});
    float2* ends = reinterpret_cast<float2*>(s.part);
    if (lane == 0) ends[wave] = float2{low, high};
#pragma unroll
    for (int j = 0; j < kPer; ++j) s.buckets[j * 64 * W + tid] = 0;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < W; ++v) {
        low = fminf(low, ends[v].x);
        high = fmaxf(high, ends[v].y);
    }
    const float range = high - low, scale = range > 0.f && range < INFINITY ? (kBuckets - 1) / range : 0.f;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j * 64 * W + tid < count) {
            // (equal logits go by their place in the row, infinite ends share one bucket)
            const unsigned int b = scale > 0.f    ? min((unsigned int)((high - key_value(word_key(mine[j]))) * scale), kBuckets - 1u)
                                   : range == 0.f ? word_index(mine[j]) / (kMaxActions / kBuckets)
                                                  : 0u;
            at[j] = b << 16 | atomicAdd(&s.buckets[b], 1u);
        }
    __syncthreads();
    // counts -> where each bucket starts
    unsigned int c[kPer], run = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        c[j] = run;
        run += s.buckets[tid * kPer + j];
    }
    unsigned int upto = run;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned int o = __shfl_up(upto, off, 64);
        if (lane >= (unsigned int)off) upto += o;
    }
    if (lane == 63u) s.wave_count[wave] = upto;
    __syncthreads();
    unsigned int base = upto - run;
#pragma unroll
    for (int v = 0; v < W; ++v) base += (unsigned int)v < wave ? s.wave_count[v] : 0u;
#pragma unroll
    for (int j = 0; j < kPer; ++j) s.buckets[tid * kPer + j] = base + c[j];
    if (tid == 0) s.buckets[kBuckets] = count;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j * 64 * W + tid < count) w[s.buckets[at[j] >> 16] + (at[j] & 0xFFFFu)] = mine[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j * 64 * W + tid < count) {
            const unsigned int from = s.buckets[at[j] >> 16], to = s.buckets[(at[j] >> 16) + 1u];
            unsigned int rank = from;
#pragma unroll 4
            for (unsigned int i = from; i < to; ++i) rank += w[i] > mine[j];
            at[j] = rank;
        }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j * 64 * W + tid < count) w[at[j]] = mine[j];
    __syncthreads();
}

// The elements that `in` takes, as words in LDS in any order; returns their number, which may pass kList (the
// rest is not kept then).
template <int W, typename Row, typename In>
__device__ __forceinline__ unsigned int gather_words(const Row& row, ChooseShared<W>& s, In in) {
    if (threadIdx.x == 0) s.taken = 0;
    __syncthreads();
    row.each([&](float x, unsigned int i, int) {
        if (in(x)) {
            const unsigned int at = atomicAdd(&s.taken, 1u);
            if (at < kList) s.words[at] = order_word(logit_key(x), i);
        }
    });
    __syncthreads();
    const unsigned int taken = s.taken;
    __syncthreads();
    return taken;
}

// The maximum of each of a thread's slots (its elements at one place of its loads), and the row's.
template <int W, int SLOTS, typename Row>
__device__ __forceinline__ float slot_max(const Row& row, float (&slot)[SLOTS], ChooseShared<W>& s) {
#pragma unroll
    for (int e = 0; e < SLOTS; ++e) slot[e] = -INFINITY;
    row.each([&](float x, unsigned int, int e) { slot[e] = fmaxf(slot[e], x); });
    float m = slot[0];
#pragma unroll
    for (int e = 1; e < SLOTS; ++e) m = fmaxf(m, slot[e]);
    m = wave_reduce(m, MaxOp{});
    float* part = reinterpret_cast<float*>(s.part);
    if (W > 1) {
        if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, part[w]);
        __syncthreads();
    }
    return m + 0.f;
}

// Number of the first of `bins` counts at which their running sum reaches `need` (the last one if it never does).
// Called by one wavefront.
__device__ __forceinline__ unsigned int bin_of_count(const unsigned int* counts, unsigned int bins, unsigned int need) {
    const unsigned int lane = threadIdx.x & 63u, per = bins / 64u;
    unsigned int mine = 0;
    for (unsigned int j = 0; j < per; ++j) mine += counts[lane * per + j];
    unsigned int upto = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned int o = __shfl_up(upto, off, 64);
        if (lane >= (unsigned int)off) upto += o;
    }
    const unsigned long long there = __ballot(upto >= need);
    if (!there) return bins - 1u;
    const unsigned int owner = __ffsll((long long)there) - 1u;
    unsigned int bin = 0, run = upto - mine;
    if (lane == owner)
        for (unsigned int j = 0; j < per; ++j) {
            run += counts[lane * per + j];
            if (run >= need) {
                bin = lane * per + j;
                break;
            }
        }
    return __shfl(bin, (int)owner, 64);
}

// A value that at least k of some numbers between `low` (each thread's own share of them) and m are not below, and not many
// more: the k-th largest to one of 1024 steps.  `each` hands every one of the thread's numbers to what it is given.
template <int W, typename Each>
__device__ float threshold_of(float low, float m, unsigned int k, ChooseShared<W>& s, Each each) {
    const unsigned int tid = threadIdx.x;
    low = wave_reduce(low, MinOp{});
    float* part = reinterpret_cast<float*>(s.part);
    __syncthreads();
    if ((tid & 63u) == 0) part[tid >> 6] = low;
    for (unsigned int i = tid; i < kSliceBins; i += 64 * W) s.slices[i] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) low = fminf(low, part[w]);
    const float range = m - low;
    const float scale = range > 0.f && range < INFINITY ? (kSliceBins - 1) / range : 0.f;
    each([&](float v) { atomicAdd(&s.slices[min((unsigned int)((m - v) * scale), kSliceBins - 1u)], 1u); });
    __syncthreads();
    if (tid < 64) {
        const unsigned int b = bin_of_count(s.slices, kSliceBins, k);
        // (the lower edge, and a little more than its rounding can be off; the last bin takes all that is allowed)
        if (tid == 0) {
            const float t = m - (float)(b + 1u) * (range / (kSliceBins - 1)) * 1.00001f;
            s.key = b + 1u == kSliceBins ? -3.402823466e38f
                    : range == 0.f      ? m
                    : scale > 0.f       ? t - fabsf(t) * 0x1p-22f
                                        : -3.402823466e38f;
        }
    }
    __syncthreads();
    return s.key;
}

// A value that the k largest of a row (maximum m) are not below, and not many more are not, from the slices' maxima.  A slice
// is what a thread holds in one slot, so there are 64 W times 4 or 8 of them, at least 1024.
template <int W, int SLOTS>
__device__ __forceinline__ float top_threshold(const float (&slot)[SLOTS], float m, unsigned int k, ChooseShared<W>& s) {
    float low = INFINITY;
#pragma unroll
    for (int e = 0; e < SLOTS; ++e)
        if (slot[e] > -INFINITY) low = fminf(low, slot[e]);
    return threshold_of<W>(low, m, k, s, [&](auto count) {
#pragma unroll
        for (int e = 0; e < SLOTS; ++e)
            if (slot[e] > -INFINITY) count(slot[e]);
    });
}

// ---------------------------------------------------------------------------------- sums along a sorted list
// Inclusive sums of the weights of words[0 .. count) behind `before`, into sums[].  Called by one wavefront.
__device__ __forceinline__ void list_sums(const unsigned long long* words, unsigned int count, double before, float m,
                                          double inv_t, double* sums) {
    const unsigned int lane = threadIdx.x & 63u;
#pragma unroll 1
    for (unsigned int j0 = 0; j0 < count; j0 += 64) {
        const unsigned int j = j0 + lane;
        double c = j < count ? exp(-logit_depth(m, key_value(word_key(words[j])), inv_t)) : 0.0;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double o = __shfl_up(c, off, 64);
            if (lane >= (unsigned int)off) c += o;
        }
        c += before;
        if (j < count) sums[j] = c;
        before = __shfl(c, 63, 64);
    }
}
// How many of the sums `low` holds for: the sums rise, so they are the first ones.  Called by one wavefront.
template <typename Low>
__device__ __forceinline__ unsigned int list_count(unsigned int count, Low low) {
    unsigned int n = 0;
#pragma unroll 1
    for (unsigned int j0 = 0; j0 < count; j0 += 64) {
        const unsigned int j = j0 + (threadIdx.x & 63u);
        const unsigned int here = __popcll(__ballot(j < count && low(j)));
        n += here;
        if (here < 64u) break;
    }
    return n;
}

struct RowChoice {
    double inv_t, top_p, min_p;
    float u;
    unsigned int k;      // 1 .. 1024: so many; 0: all
    bool greedy, search; // search: more than 1024, or the last of all that stay, which may lie below every bin
};
__device__ __forceinline__ RowChoice row_choice(const ChooseArgs& p, unsigned long long row) {
    RowChoice c;
    const double t = p.row_temperature ? (double)p.row_temperature[row] : p.temperature;
    const long long k = p.row_top_k ? (long long)p.row_top_k[row] : p.top_k;
    c.top_p = p.row_top_p ? (double)p.row_top_p[row] : p.top_p;
    c.min_p = p.row_min_p ? (double)p.row_min_p[row] : p.min_p;
    c.u = p.u[row];
    c.greedy = !(t > 0.0);
    // (beyond these ends the temperature changes no float's weight, and products with it stay finite)
    c.inv_t = c.greedy ? 1.0 : 1.0 / fmin(fmax(t, 1e-250), 1e250);
    c.search = false;
    c.k = c.greedy ? 1u : 0u;
    if (!c.greedy && k > 0 && k < (long long)p.x.n) {
        c.k = k <= (long long)kMaxTop ? (unsigned int)k : 0u;
        c.search = c.k == 0u;
    }
    c.search |= !c.k && c.u >= 1.f;
    return c;
}

__device__ __forceinline__ void put_choice(const ChooseArgs& p, unsigned long long row, int index, float logp) {
    p.index[row] = index;
    if (p.logp) p.logp[row] = logp;
}

// The choice from the row's sorted first actions (at least min(k, allowed) of them).  Called by one wavefront.
__device__ void choose_from_list(const ChooseArgs& p, unsigned long long row, const RowChoice& c,
                                 const unsigned long long* words, unsigned int count, float m, double* sums) {
    const unsigned int lane = threadIdx.x & 63u;
    if (c.greedy) {
        if (lane == 0) put_choice(p, row, (int)word_index(words[0]), 0.f);
        return;
    }
    count = min(count, c.k);
    list_sums(words, count, 0.0, m, c.inv_t, sums);
    wave_lds_fence();
    unsigned int left = count;
    if (c.top_p < 1.0) {
        const double most = c.top_p * sums[count - 1u];
        left = list_count(count - 1u, [&](unsigned int j) { return sums[j] < most; }) + 1u;
    }
    if (c.min_p > 0.0) {
        const unsigned int n = list_count(
            left, [&](unsigned int j) { return exp(-logit_depth(m, key_value(word_key(words[j])), c.inv_t)) >= c.min_p; });
        left = n ? n : 1u;
    }
    const double mass = sums[left - 1u], drawn = c.u > 0.f ? (double)c.u * mass : 0.0;
    const unsigned int at = min(list_count(left, [&](unsigned int j) { return sums[j] <= drawn; }), left - 1u);
    if (lane == 0)
        put_choice(p, row, (int)word_index(words[at]),
                   (float)(-logit_depth(m, key_value(word_key(words[at])), c.inv_t) - log(mass)));
}

// ------------------------------------------------------------------------------- the histogram of a row's weights
// Bins are as wide as a power of two near temperature / 32 and aligned to its multiples: x / width, its whole part and
// what is left are exact in 64 bits, and pieces of a row can be binned on their own.  2048 bins reach
// 40 temperatures below the maximum or further; what lies below has less than 2^18 e^-40 = 1.2e-12 of the best action's
// weight together, where a random number of 24 bits cannot fall.
struct Bins {
    double width, inv_width, slope;   // slope: width / temperature
    double top;                       // number of the maximum's bin, counted from value 0
    __device__ __forceinline__ Bins(float m, double inv_t) {
        // 40 / 2048 = 0.0195 temperatures, rounded up to a power of two
        int e;
        (void)frexp((40.0 / kBins) / inv_t, &e);
        width = ldexp(1.0, e);
        inv_width = ldexp(1.0, -e);
        slope = width * inv_t;
        top = floor((double)m * inv_width);
    }
    // the floats of bin b are lo <= x < hi
    __device__ __forceinline__ float lo(double b) const { return __double2float_ru((top - b) * width); }
    // (nothing is above bin 0; where logits are so large that top + 1 is top, it holds the maximum alone)
    __device__ __forceinline__ float hi(double b) const {
        return b == 0.0 ? INFINITY : __double2float_ru((top - b + 1.0) * width);
    }
    // weight at the middle of bin b
    __device__ __forceinline__ double middle(float m, double b) const {
        return exp(-((double)m * inv_width - (top - b) - 0.5) * slope);
    }
};

// exp(z) 2^44 as a whole number, for z within +- 0.0195: the sixth power's term, which is left out, is below 2^-43.
__device__ __forceinline__ unsigned long long near_units(double z) {
    double w = fma(z, 1.0 / 120.0, 1.0 / 24.0);
    w = fma(w, z, 1.0 / 6.0);
    w = fma(w, z, 0.5);
    w = fma(w, z, 1.0);
    w = fma(w, z, 1.0);
    // (adding 2^52 leaves the whole number in the low bits)
    return __double_as_longlong(fma(w, kOne, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
}

template <int W, typename Row>
__device__ __forceinline__ void bin_weights(const Row& row, const Bins& bins, ChooseShared<W>& s) {
    for (unsigned int i = threadIdx.x; i < kBins; i += 64 * W) s.hist[i] = 0;
    __syncthreads();
    const float least = bins.lo((double)(kBins - 1));
    const double inv_width = bins.inv_width, slope = bins.slope, top = bins.top;
    row.each([&](float x, unsigned int, int) {
        if (x >= least) {
            const double at = (double)x * inv_width, whole = floor(at);
            atomicAdd(&s.hist[(int)(top - whole)], near_units(fma(at - whole, slope, -0.5 * slope)));
        }
    });
    __syncthreads();
}

// hist -> inclusive sums of the weights (the best action's is 1), in place.
template <int W>
__device__ void sum_bins(const Bins& bins, float m, ChooseShared<W>& s) {
    constexpr int kPer = kBins / (64 * W);
    const unsigned int tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    double c[kPer], run = 0.0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned int b = tid * kPer + j;
        const unsigned long long h = s.hist[b];
        if (h) run += (double)h * (1.0 / kOne) * bins.middle(m, (double)b);
        c[j] = run;
    }
    double upto = run;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double o = __shfl_up(upto, off, 64);
        if (lane >= (unsigned int)off) upto += o;
    }
    __syncthreads();
    if (lane == 63u) s.part[wave] = upto;
    __syncthreads();
    double base = 0.0, before = __shfl_up(upto, 1, 64);
    if (lane == 0) before = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) base += (unsigned int)w < wave ? s.part[w] : 0.0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) s.sums[tid * kPer + j] = base + (before + c[j]);
    __syncthreads();
}

// The first bin whose inclusive sum `reached` holds for; kBins - 1 if none.  (Neighbouring sums are made in
// different orders and may fall by a last bit where they should rise: the lowest such bin counts.)
template <int W, typename Reached>
__device__ unsigned int find_bin(ChooseShared<W>& s, Reached reached) {
    constexpr int kPer = kBins / (64 * W);
    if (threadIdx.x == 0) s.bin = kBins - 1;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned int b = threadIdx.x * kPer + j;
        if (reached(s.sums[b]) && (b == 0 || !reached(s.sums[b - 1u]))) atomicMin(&s.bin, b);
    }
    __syncthreads();
    const unsigned int bin = s.bin;
    __syncthreads();
    return bin;
}

// Of the `count` actions of bin b in LDS, the first in order with which the inclusive sum over the row reaches `target` (passes
// it, if `past`), or the last of them if rounding has it otherwise: its word and that sum, in s.word and
// s.part[0].  A bin of a long row holds some hundred actions, up to all that the list takes, so a histogram of its parts comes
// before anything is sorted.
template <int W>
__device__ __forceinline__ void locate(const Bins& bins, unsigned int b, unsigned int count, double target, bool past, float m, double inv_t,
                       ChooseShared<W>& s) {
    const unsigned int tid = threadIdx.x;
    double before = b ? s.sums[b - 1u] : 0.0;
    if (count > 128u) {
        constexpr int kEach = kList / (64 * W);
        unsigned long long mine[kEach];
        unsigned int part[kEach];
        for (unsigned int i = tid; i < kFine; i += 64 * W) s.fine[i] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const unsigned int i = j * 64 * W + tid;
            if (i < count) {
                mine[j] = s.words[i];
                const double at = (double)key_value(word_key(mine[j])) * bins.inv_width, rest = at - floor(at);
                part[j] = min((unsigned int)((1.0 - rest) * kFine), kFine - 1u);
                atomicAdd(&s.fine[part[j]], near_units(fma(rest, bins.slope, -0.5 * bins.slope)));
            }
        }
        __syncthreads();
        if (tid < 64) {
            constexpr int kPer = kFine / 64;
            unsigned long long c[kPer], run = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                c[j] = run;
                run += s.fine[tid * kPer + j];
            }
            unsigned long long upto = run;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const unsigned long long o = __shfl_up(upto, off, 64);
                if (tid >= (unsigned int)off) upto += o;
            }
            const double unit = bins.middle(m, (double)b) * (1.0 / kOne);
            const unsigned long long start = upto - run;
            // the first part that reaches the target, or the last one with anything in it
            unsigned int first = kFine, last = 0;
#pragma unroll
            for (int j = kPer - 1; j >= 0; --j) {
                const unsigned long long f = s.fine[tid * kPer + j];
                const double v = before + (double)(start + c[j] + f) * unit;
                if (f && (past ? v > target : v >= target)) first = tid * kPer + j;
                if (f && !last) last = tid * kPer + j;
            }
            const unsigned int all = wave_reduce(first, MinOp{});
            const unsigned int end = wave_reduce(last, MaxOp{});
            const unsigned int take = all < kFine ? all : end;
            if (tid == take / kPer) {
                unsigned long long sum = start;
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (tid * kPer + j < take) sum += s.fine[tid * kPer + j];
                s.part[0] = before + (double)sum * unit;
                s.bin = take;
                s.taken = 0;
            }
        }
        __syncthreads();
        const unsigned int take = s.bin;
        before = s.part[0];
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (j * 64 * W + tid < count && part[j] == take) s.words[atomicAdd(&s.taken, 1u)] = mine[j];
        __syncthreads();
        count = s.taken;
        __syncthreads();
    }
    sort_words<W>(s, count);
    if (tid < 64) {
        double run = before, sum = before;
        unsigned int at = count - 1u;
        bool found = false;
#pragma unroll 1
        for (unsigned int j0 = 0; j0 < count && !found; j0 += 64) {
            const unsigned int j = j0 + tid;
            double v = j < count ? exp(-logit_depth(m, key_value(word_key(s.words[j])), inv_t)) : 0.0;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double o = __shfl_up(v, off, 64);
                if (tid >= (unsigned int)off) v += o;
            }
            v += run;
            run = __shfl(v, 63, 64);
            const unsigned long long yes = __ballot(j < count && (past ? v > target : v >= target));
            found = yes != 0;
            if (found) at = j0 + __ffsll((long long)yes) - 1u;
            sum = found ? __shfl(v, (int)(at - j0), 64) : run;
        }
        if (tid == 0) {
            s.word = s.words[at];
            s.part[0] = sum;
        }
    }
    __syncthreads();
}

// A row whose whole weight is with `count` equal logits, listed in LDS: sums are whole numbers, and a limit that ends exactly
// at one of them (top-p of 1/2 over an even number) has to be met to the unit.  The choice in s.word; false if they are not
// equal.
template <int W>
__device__ __forceinline__ bool choose_equal(const RowChoice& c, unsigned int count, float m, double* mass, ChooseShared<W>& s) {
    const unsigned int tid = threadIdx.x, key = order_key(m);
    unsigned int others = 0;
    for (unsigned int i = tid; i < count; i += 64 * W) others |= word_key(s.words[i]) ^ key;
    others = block_reduce<W>(others, MaxOp{}, s.search.count[0]);
    __syncthreads();
    if (others) return false;
    double kept = (double)count;
    if (c.top_p < 1.0) kept = fmax(ceil(c.top_p * kept), 1.0);
    if (c.min_p > 1.0) kept = 1.0;
    const unsigned int at = min((unsigned int)(c.u > 0.f ? (double)c.u * kept : 0.0), (unsigned int)kept - 1u);
    sort_words<W>(s, count);
    if (tid == 0) s.word = s.words[at];
    *mass = kept;
    return true;
}

// From the inclusive sums over bins to the choice; false if a bin holds too many actions for LDS, or, by a rounding of the
// sums, none.
template <int W, typename Row>
__device__ __forceinline__ bool choose_from_bins(const Row& row_, const ChooseArgs& p, unsigned long long row, const RowChoice& c,
                                 const Bins& bins, float m, ChooseShared<W>& s) {
    const unsigned int tid = threadIdx.x;
    double mass = s.sums[kBins - 1];
    // the sum over the actions that stay: each limit keeps the first so many, and the shorter one counts
    unsigned int bin_p = kBins, bin_m = kBins;
    // (the best action always stays, and the sum reaches its weight with it)
    const double most = fmax(c.top_p * mass, 0.5);
    if (c.top_p < 1.0) bin_p = find_bin<W>(s, [&](double v) { return v >= most; });
    if (c.min_p > 0.0) {
        const double b = bins.top - floor(((double)m + log(fmin(c.min_p, 1.0)) / c.inv_t) * bins.inv_width);
        bin_m = b < (double)kBins ? (unsigned int)fmax(b, 0.0) : kBins;
    }
    const unsigned int last = min(bin_p, bin_m);
    // (all of it in the first bin)
    const bool one_bin = s.sums[kBins - 1] == s.sums[0];
    bool done = false;
    // first the bin where the actions that stay end, if there is a limit, then the one of the choice
    auto round = [&](int pass) __attribute__((always_inline)) {
        const double target = pass == 0 ? most : c.u > 0.f ? (double)c.u * mass : 0.0;
        const bool past = pass == 1;
        unsigned int bin = last;
        if (pass) bin = find_bin<W>(s, [&](double v) { return past ? v > target : v >= target; });
        const float lo = bins.lo((double)bin), hi = bins.hi((double)bin);
        const unsigned int count = gather_words<W>(row_, s, [&](float x) { return x >= lo && x < hi; });
        const bool find = pass == 1 || bin_p == last;
        if (count > kList || (count == 0 && find)) return false;
        if (one_bin && bin == 0 && choose_equal<W>(c, count, m, &mass, s)) {
            done = true;
            return true;
        }
        if (pass == 0 && bin_m == last) {
            // (whole numbers: their sum does not depend on the order in which the list was filled)
            unsigned long long units = 0;
            for (unsigned int i = tid; i < count; i += 64 * W) {
                const double w = exp(-logit_depth(m, key_value(word_key(s.words[i])), c.inv_t));
                if (w >= c.min_p) units += (unsigned long long)(w * kOne + 0.5);
            }
            units = block_reduce<W>(units, SumOp{}, s.search.sum[0]);
            __syncthreads();
            mass = fmin(mass, fmax((last ? s.sums[last - 1u] : 0.0) + (double)units * (1.0 / kOne), 1.0));
        }
        if (find) {
            locate<W>(bins, bin, count, target, past, m, c.inv_t, s);
            if (pass == 0) mass = fmin(mass, s.part[0]);
            __syncthreads();
        }
        return true;
    };
    if constexpr (W == 8) {
        // (once in the code: twice, the compiler no longer keeps the eight loads of a thread in registers, 42 us instead of 30
        // for 1000 x 32768; the others keep theirs and lose by the loop, 52 us instead of 45 for 4096 x 1000)
#pragma unroll 1
        for (int pass = last < kBins ? 0 : 1; pass < 2 && !done; ++pass)
            if (!round(pass)) return false;
    } else {
        if (last < kBins && !round(0)) return false;
        if (!done && !round(1)) return false;
    }
    if (tid == 0)
        put_choice(p, row, (int)word_index(s.word),
                   (float)(-logit_depth(m, key_value(word_key(s.word)), c.inv_t) - log(mass)));
    return true;
}

// One row, all of it at hand.
template <int W, int SLOTS, typename T, typename Row>
__device__ __forceinline__ void choose_row(const Row& held, const ChooseArgs& p, unsigned long long row, ChooseShared<W>& s) {
    const RowChoice c = row_choice(p, row);
    float slot[SLOTS];
    const float m = slot_max<W, SLOTS>(held, slot, s);
    if (m == -INFINITY) {
        if (threadIdx.x == 0) put_choice(p, row, -1, 0.f);
        return;
    }
    bool done = false;
    if (!c.search && !(m == INFINITY)) {
        if (c.k) {
            const float t = top_threshold<W, SLOTS>(slot, m, c.k, s);
            const unsigned int count = gather_words<W>(held, s, [&](float x) { return x >= t; });
            if (count <= kList) {
                sort_words<W>(s, count);
                if (threadIdx.x < 64) choose_from_list(p, row, c, s.words, count, m, s.sums);
                done = true;
            }
        } else {
            const Bins bins(m, c.inv_t);
            bin_weights<W>(held, bins, s);
            sum_bins<W>(bins, m, s);
            done = choose_from_bins<W>(held, p, row, c, bins, m, s);
        }
    }
    if (!done) {
        __syncthreads();
        choose_by_search<W, T>(p, row, s.search);
    }
}

// Eight wavefronts with eight loads each for long rows: 16 wavefronts of four and 4 of sixteen take 78 and 74 us for 66 at
// 1000 x 32768 bf16 top-p, 38 and 34 for 30 at top-k.  What bounds it is not HBM (2.2 TB/s at top-k) but the instructions per
// element: decoding, comparing, and without top-k some twenty in 64 bits and an LDS atomic for the weight.
template <int W, int NV, int EU, typename T>
__global__ __launch_bounds__(64 * W, EU) void choose_kernel(ChooseArgs p) {
    __shared__ ChooseShared<W> s;
    const unsigned long long row = workgroup_row();
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const HeldRow<W, NV, T> held(x, 0, p.x.n);
    choose_row<W, (int)kPerLoad<T>, T>(held, p, row, s);
}

// -------------------------------------------------------------------------------------------- top actions
template <int W, typename T>
__device__ void put_top(const TopArgs& p, unsigned long long row, const unsigned long long* words, unsigned int count) {
    for (unsigned int j = threadIdx.x; j < p.k; j += 64 * W) {
        const unsigned long long at = row * p.k + j;
        store_value(global_out<T>(p.values) + at, j < count ? key_value(word_key(words[j])) : -INFINITY);
        p.index[at] = j < count ? (int)word_index(words[j]) : -1;
    }
}

// The first k actions by search: those above the k-th value in any order, then the first ones equal to it.
template <int W, typename T>
__device__ unsigned int top_by_search(const Global<T>* x, unsigned int n, unsigned int k, float m, ChooseShared<W>& s) {
    unsigned int turn = 0, allowed, above;
    search_sum<W>(x, n, m, 0.0, [](unsigned int) { return true; }, s.search, turn, nullptr, &allowed);
    k = min(k, allowed);
    const unsigned int v = search_key<W>(kMaskedKey + 1u, order_key(m), [&](unsigned int v) {
        unsigned int c;
        search_sum<W>(x, n, m, 0.0, [&](unsigned int key) { return key >= v; }, s.search, turn, nullptr, &c);
        return c >= k;
    });
    search_sum<W>(x, n, m, 0.0, [&](unsigned int key) { return key > v; }, s.search, turn, nullptr, &above);
    if (threadIdx.x == 0) s.taken = 0;
    __syncthreads();
    const unsigned int lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    unsigned int equal_before = 0;
#pragma unroll 1
    for (unsigned int i0 = 0; i0 < n; i0 += 64 * W) {
        const unsigned int i = i0 + threadIdx.x;
        const unsigned int key = i < n ? logit_key(logit_value(x + i)) : 0u;
        if (key > v) s.words[atomicAdd(&s.taken, 1u)] = order_word(key, i);
        const unsigned long long hits = __ballot(key == v);
        __syncthreads();
        if (lane == 0) s.search.count[0][wave] = __popcll(hits);
        __syncthreads();
        unsigned int at = equal_before + __popcll(hits & ((1ull << lane) - 1ull));
        for (unsigned int w = 0; w < W; ++w) {
            if (w < wave) at += s.search.count[0][w];
            equal_before += s.search.count[0][w];
        }
        if (key == v && above + at < k) s.words[above + at] = order_word(key, i);
    }
    return k;
}

// The sum of exp((x - m) / temperature) over what the workgroup holds, in every thread.  (The sum of a load in 32 bits, sums of
// those in 64.)
template <int W, int SLOTS, typename Row>
__device__ __forceinline__ double exp_sum(const Row& held, float m, float c2, ChooseShared<W>& s) {
    double a = 0.0;
    if (m > -INFINITY && m < INFINITY) {
        float load = 0.f;
        held.each([&](float v, unsigned int, int e) {
            const float w = __builtin_amdgcn_exp2f((fmaxf(v, -INFINITY) - m) * c2);
            load = e ? load + w : w;
            if (e == SLOTS - 1) a += (double)load;
        });
    }
    a = block_reduce<W>(a, SumOp{}, s.part);
    __syncthreads();
    return a;
}
__device__ __forceinline__ void put_lse(const TopArgs& p, unsigned long long row, float m, double total) {
    p.lse[row] = m == INFINITY || m == -INFINITY ? m : (float)((double)m * p.inv_t + log(total));
}

template <int W, int SLOTS, typename T, typename Row>
__device__ __forceinline__ void top_row(const Row& held, const TopArgs& p, unsigned long long row, const Global<T>* x, ChooseShared<W>& s) {
    float slot[SLOTS];
    const float m = slot_max<W, SLOTS>(held, slot, s);
    unsigned int count = 0;
    if (m > -INFINITY) {
        const float t = top_threshold<W, SLOTS>(slot, m, p.k, s);
        count = gather_words<W>(held, s, [&](float v) { return v >= t; });
    }
    if (p.lse) {
        const double total = exp_sum<W, SLOTS>(held, m, p.c2, s);
        if (threadIdx.x == 0) put_lse(p, row, m, total);
    }
    if (m > -INFINITY) {
        if (count > kList) count = top_by_search<W, T>(x, p.x.n, p.k, m, s);
        sort_words<W>(s, count);
    }
    put_top<W, T>(p, row, s.words, min(count, p.k));
}

// 2048 x 32768 bf16, k = 64: 47 us, 2.9 TB/s; four workgroups a compute unit, of which each takes in turn its loads and three passes
// over registers (maxima, candidates, exponentials: about twelve instructions and an exp per element).
template <int W, int NV, int EU, typename T>
__global__ __launch_bounds__(64 * W, EU) void top_kernel(TopArgs p) {
    __shared__ ChooseShared<W> s;
    const unsigned long long row = workgroup_row();
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const HeldRow<W, NV, T> held(x, 0, p.x.n);
    top_row<W, (int)kPerLoad<T>, T>(held, p, row, x, s);
}

// ------------------------------------------------------------------- rows of up to 64 actions: one wavefront each
__device__ __forceinline__ double lane_value(double v, int lane) {
    const unsigned long long b = __double_as_longlong(v);
    const unsigned int lo = __builtin_amdgcn_readlane((int)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}

// Which lanes come before this one in the order of choice, a bit each.
__device__ __forceinline__ unsigned long long lanes_before(unsigned int key, unsigned int n) {
    const unsigned int lane = threadIdx.x & 63u;
    unsigned long long before = 0;
    for (unsigned int j = 0; j < n; ++j) {
        const unsigned int other = __builtin_amdgcn_readlane((int)key, (int)j);
        before |= (unsigned long long)(other > key || (other == key && j < lane)) << j;
    }
    return before;
}

// (5.5 us for one row of 30, 7.4 for 128 with settings of their own: two trips to memory, and the chains of 30 sums, exp and log)
template <typename T>
__global__ __launch_bounds__(256) void choose_wave_kernel(ChooseArgs p) {
    const unsigned int lane = threadIdx.x & 63u, n = p.x.n;
    const unsigned int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned long long row = workgroup_row() * 4u + wave;
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const float v = lane < n ? clean_logit(logit_value(x + lane)) : -INFINITY;
    const RowChoice c = row_choice(p, row);
    const long long k = p.row_top_k ? (long long)p.row_top_k[row] : p.top_k;
    const unsigned long long before_me = lanes_before(order_key(v), n);
    const unsigned int rank = __popcll(before_me);
    const bool allowed = v > -INFINITY;
    const float m = wave_reduce(v, MaxOp{});
    if (m == -INFINITY) {
        if (lane == 0) put_choice(p, row, -1, 0.f);
        return;
    }
    if (c.greedy) {
        if (rank == 0) put_choice(p, row, (int)lane, 0.f);
        return;
    }
    bool stays = allowed && (k <= 0 || (long long)rank < k);
    const double w = stays ? exp(-logit_depth(m, v, c.inv_t)) : 0.0;
    double before = 0.0, total = 0.0;
    for (unsigned int j = 0; j < n; ++j) {
        const double other = lane_value(w, (int)j);
        total += other;
        before += before_me >> j & 1ull ? other : 0.0;
    }
    if (c.top_p < 1.0) stays &= before < c.top_p * total;
    if (c.min_p > 0.0) stays &= w >= c.min_p;
    stays |= rank == 0;
    const double upto = before + w;
    const double mass = wave_reduce(stays ? upto : 0.0, MaxOp{});
    const double drawn = c.u > 0.f ? (double)c.u * mass : 0.0;
    // the first in order whose sum passes the drawn one, else the last that stays
    const bool hit = stays && upto > drawn;
    const unsigned int first = wave_reduce(hit ? rank : 64u, MinOp{});
    const unsigned int at = first < 64u ? first : wave_reduce(stays ? rank : 0u, MaxOp{});
    if (rank == at) put_choice(p, row, (int)lane, (float)(-logit_depth(m, v, c.inv_t) - log(mass)));
}

template <typename T>
__global__ __launch_bounds__(256) void top_wave_kernel(TopArgs p) {
    const unsigned int lane = threadIdx.x & 63u, n = p.x.n;
    const unsigned int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned long long row = workgroup_row() * 4u + wave;
    if (row >= p.x.rows) return;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const float v = lane < n ? clean_logit(logit_value(x + lane)) : -INFINITY;
    const unsigned int rank = __popcll(lanes_before(order_key(v), n));
    const unsigned int allowed = __popcll(__ballot(v > -INFINITY));
    if (rank < p.k && lane < n) {
        const unsigned long long at = row * p.k + rank;
        store_value(global_out<T>(p.values) + at, v);
        p.index[at] = rank < allowed ? (int)lane : -1;
    }
    if (p.lse) {
        const float m = wave_reduce(v, MaxOp{});
        const double w = m > -INFINITY && m < INFINITY ? (double)__builtin_amdgcn_exp2f((v - m) * p.c2) : 0.0;
        const double total = wave_reduce(w, SumOp{});
        if (lane == 0) p.lse[row] = m == INFINITY || m == -INFINITY ? m : (float)((double)m * p.inv_t + log(total));
    }
}

// ------------------------------------------------------------------------------ rows in pieces of a workgroup each
// Long rows, and few ones: a launch brings each piece of a row to its candidates or to its histogram of weights, in the
// workspace; a second one, a workgroup a row, joins them.  The histograms' bins lie on multiples of one width, so a piece needs
// no other's maximum.  us of the two launches: 1 x 131072 bf16 top-k 9 + 8; 37 x 50021 fp32 top-p 8 + 25, 256 x 131072 bf16 with
// settings of their own 30 + 37: where there is no top-k, the join reads its row again for each of the one or two bins it lists,
// on one compute unit.
struct Pieces {
    unsigned int count, length;   // of a row; the last piece takes what is left
};
struct PieceHead {
    double top, sum;      // number of the histogram's first bin; sum of exp((x - m) / temperature)
    float m;
    unsigned int taken;   // candidates; more than kList: they did not fit
    unsigned int pad_[2];
};
static_assert(sizeof(PieceHead) == 32, "as the workspace is counted");
struct PieceSpace {
    PieceHead* heads;                 // [rows][count]
    unsigned long long* words;        // [rows][count][kList]: candidates, or the histogram
};
static_assert(kList == kBins, "candidates and histogram share their place");

// One piece's elements at least a threshold that its k largest reach, as words in memory.
template <int W, int SLOTS, typename Row>
__device__ __forceinline__ unsigned int piece_words(const Row& held, const float (&slot)[SLOTS], float m, unsigned int k,
                                                    unsigned long long* out, ChooseShared<W>& s) {
    const float t = top_threshold<W, SLOTS>(slot, m, k, s);
    if (threadIdx.x == 0) s.taken = 0;
    __syncthreads();
    held.each([&](float x, unsigned int i, int) {
        if (x >= t) {
            const unsigned int at = atomicAdd(&s.taken, 1u);
            if (at < kList) global_out<unsigned long long>(out)[at] = order_word(logit_key(x), i);
        }
    });
    __syncthreads();
    return s.taken;
}

template <int W, int NV, int EU, typename T>
__global__ __launch_bounds__(64 * W, EU) void choose_piece_kernel(ChooseArgs p, Pieces c, PieceSpace ws) {
    constexpr int SLOTS = (int)kPerLoad<T>;
    __shared__ ChooseShared<W> s;
    const unsigned long long row = blockIdx.y, at = row * c.count + blockIdx.x;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const unsigned int begin = blockIdx.x * c.length, end = blockIdx.x + 1u == c.count ? p.x.n : begin + c.length;
    const HeldRow<W, NV, T> held(x, begin, end);
    const RowChoice choice = row_choice(p, row);
    float slot[SLOTS];
    const float m = slot_max<W, SLOTS>(held, slot, s);
    unsigned int taken = 0;
    double top = 0.0;
    if (m > -INFINITY && m < INFINITY && !choice.search) {
        unsigned long long* out = ws.words + at * kList;
        if (choice.k) {
            taken = piece_words<W, SLOTS>(held, slot, m, choice.k, out, s);
        } else {
            const Bins bins(m, choice.inv_t);
            bin_weights<W>(held, bins, s);
            for (unsigned int i = threadIdx.x; i < kBins; i += 64 * W) global_out<unsigned long long>(out)[i] = s.hist[i];
            top = bins.top;
        }
    }
    if (threadIdx.x == 0) ws.heads[at] = PieceHead{top, 0.0, m, taken, {0, 0}};
}

template <int W, int NV, int EU, typename T>
__global__ __launch_bounds__(64 * W, EU) void top_piece_kernel(TopArgs p, Pieces c, PieceSpace ws) {
    constexpr int SLOTS = (int)kPerLoad<T>;
    __shared__ ChooseShared<W> s;
    const unsigned long long row = blockIdx.y, at = row * c.count + blockIdx.x;
    const Global<T>* x = global_in<T>(p.x.data) + row * p.x.stride;
    const unsigned int begin = blockIdx.x * c.length, end = blockIdx.x + 1u == c.count ? p.x.n : begin + c.length;
    const HeldRow<W, NV, T> held(x, begin, end);
    float slot[SLOTS];
    const float m = slot_max<W, SLOTS>(held, slot, s);
    unsigned int taken = 0;
    if (m > -INFINITY) taken = piece_words<W, SLOTS>(held, slot, m, p.k, ws.words + at * kList, s);
    __syncthreads();
    const double sum = p.lse ? exp_sum<W, SLOTS>(held, m, p.c2, s) : 0.0;
    if (threadIdx.x == 0) ws.heads[at] = PieceHead{0.0, sum, m, taken, {0, 0}};
}

// The candidates of a row's pieces (up to 64) as a sorted list in LDS of which the first k are the row's; returns its length, or
// more than kList if they do not fit.  m: the row's maximum.  A wavefront takes every W-th piece, and 64 candidates to a
// register as long as there are some: one trip to memory, then three passes over registers; more are read again.
template <int W>
__device__ unsigned int join_words(const PieceHead* heads, const unsigned long long* words, unsigned int pieces, float m,
                                   unsigned int k, ChooseShared<W>& s) {
    constexpr int kHeld = 8;
    const unsigned int tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned int mine = lane < pieces ? heads[lane].taken : 0u;
    if (__ballot(mine > kList)) return kList + 1u;
    const unsigned int total = wave_reduce(mine, SumOp{});
    const Global<unsigned long long>* in = global_in<unsigned long long>(words);
    unsigned long long held[kHeld];
    unsigned int q = wave, off = 0, held_now = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        held[j] = 0;
        while (q < pieces && off >= __builtin_amdgcn_readlane((int)mine, (int)q)) {
            q += W;
            off = 0;
        }
        if (q < pieces) {
            if (off + lane < (unsigned int)__builtin_amdgcn_readlane((int)mine, (int)q)) held[j] = in[(size_t)q * kList + off + lane];
            off += 64u;
            held_now = j + 1;
        }
    }
    auto each_word = [&](auto f) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            if (j < (int)held_now && held[j]) f(held[j]);
        for (unsigned int r = q, at = off; r < pieces; r += W, at = 0) {
            const unsigned int n = __builtin_amdgcn_readlane((int)mine, (int)r);
            for (unsigned int i = at + lane; i < n; i += 64u) f(in[(size_t)r * kList + i]);
        }
    };
    float t = -3.402823466e38f;
    if (total > 128u && total > k) {
        // the k-th largest to one of 1024 steps between the maximum and the smallest candidate
        float low = INFINITY;
        each_word([&](unsigned long long w) { low = fminf(low, key_value(word_key(w))); });
        t = threshold_of<W>(low, m, k, s, [&](auto count) { each_word([&](unsigned long long w) { count(key_value(word_key(w))); }); });
    }
    if (tid == 0) s.taken = 0;
    __syncthreads();
    each_word([&](unsigned long long w) {
        if (key_value(word_key(w)) >= t) {
            const unsigned int at = atomicAdd(&s.taken, 1u);
            if (at < kList) s.words[at] = w;
        }
    });
    __syncthreads();
    const unsigned int taken = s.taken;
    __syncthreads();
    if (taken <= kList) sort_words<W>(s, taken);
    return taken;
}

template <int W, typename T>
__global__ __launch_bounds__(64 * W, 4) void choose_join_kernel(ChooseArgs p, Pieces c, PieceSpace ws) {
    __shared__ ChooseShared<W> s;
    const unsigned int tid = threadIdx.x, lane = tid & 63u;
    const unsigned long long row = blockIdx.x;
    const PieceHead* heads = ws.heads + row * c.count;
    const unsigned long long* words = ws.words + row * c.count * kList;
    const RowChoice choice = row_choice(p, row);
    const float m = wave_reduce(lane < c.count ? heads[lane].m : -INFINITY, MaxOp{});
    if (m == -INFINITY) {
        if (tid == 0) put_choice(p, row, -1, 0.f);
        return;
    }
    bool done = false;
    if (!choice.search && m < INFINITY) {
        if (choice.k) {
            const unsigned int count = join_words<W>(heads, words, c.count, m, choice.k, s);
            if (count <= kList) {
                if (tid < 64) choose_from_list(p, row, choice, s.words, count, m, s.sums);
                done = true;
            }
        } else {
            const Bins bins(m, choice.inv_t);
            unsigned long long sum[kBins / (64 * W)] = {};
            // bins between the row's first and each piece's, a lane for each
            const double down = lane < c.count && heads[lane].m > -INFINITY ? bins.top - heads[lane].top : (double)kBins;
            const unsigned int from = down < (double)kBins ? (unsigned int)down : kBins;
            constexpr unsigned int kPer = kBins / (64 * W), kAhead = 8;
#pragma unroll 1
            for (unsigned int q0 = 0; q0 < c.count; q0 += kAhead) {
                unsigned long long piece[kAhead][kPer];
#pragma unroll
                for (unsigned int i = 0; i < kAhead; ++i) {
                    // (pieces past the last one are that one again, and not added)
                    const unsigned int q = min(q0 + i, c.count - 1u), d = __builtin_amdgcn_readlane((int)from, (int)q);
#pragma unroll
                    for (unsigned int j = 0; j < kPer; ++j) {
                        const unsigned int bin = j * 64 * W + tid;
                        const bool in = q0 + i < c.count && bin >= d;
                        piece[i][j] = global_in<unsigned long long>(words)[(size_t)q * kBins + (in ? bin - d : 0u)];
                        piece[i][j] = in ? piece[i][j] : 0ull;
                    }
                }
#pragma unroll
                for (unsigned int i = 0; i < kAhead; ++i)
#pragma unroll
                    for (unsigned int j = 0; j < kPer; ++j) sum[j] += piece[i][j];
            }
#pragma unroll
            for (unsigned int j = 0; j < kBins / (64 * W); ++j) s.hist[j * 64 * W + tid] = sum[j];
            __syncthreads();
            sum_bins<W>(bins, m, s);
            done = choose_from_bins<W>(ReadRow<W, 8, T>(global_in<T>(p.x.data) + row * p.x.stride, 0, p.x.n), p, row, choice, bins, m, s);
        }
    }
    if (!done) {
        __syncthreads();
        choose_by_search<W, T>(p, row, s.search);
    }
}

template <int W, typename T>
__global__ __launch_bounds__(64 * W, 4) void top_join_kernel(TopArgs p, Pieces c, PieceSpace ws) {
    __shared__ ChooseShared<W> s;
    const unsigned int lane = threadIdx.x & 63u;
    const unsigned long long row = blockIdx.x;
    const PieceHead* heads = ws.heads + row * c.count;
    const float own = lane < c.count ? heads[lane].m : -INFINITY, m = wave_reduce(own, MaxOp{});
    if (p.lse && threadIdx.x < 64) {
        const double sum = own > -INFINITY && m < INFINITY ? heads[lane].sum * exp(-logit_depth(m, own, p.inv_t)) : 0.0;
        const double total = wave_reduce(sum, SumOp{});
        if (lane == 0) put_lse(p, row, m, total);
    }
    unsigned int count = 0;
    if (m > -INFINITY) {
        count = join_words<W>(heads, ws.words + row * c.count * kList, c.count, m, p.k, s);
        if (count > kList) {
            count = top_by_search<W, T>(global_in<T>(p.x.data) + row * p.x.stride, p.x.n, p.k, m, s);
            sort_words<W>(s, count);
        }
    }
    put_top<W, T>(p, row, s.words, min(count, p.k));
}

// ------------------------------------------------------------------------------------------------ launches
// How a row is cut: not at all where a workgroup's registers hold it and there are enough rows to fill the compute units, or the
// row is too short for a second launch to pay.  (Pieces of 4096 instead of 8192 at least: 9 x 100003 top 500 47 us for the join
// alone, which has to take in twice the candidates.)
template <typename T>
Pieces pieces_of(unsigned long long rows, unsigned int n) {
    const unsigned int held = HeldRow<8, 8, T>::kMost;
    if (n <= held && (rows > 128u || n <= 8192u)) return Pieces{1u, n};
    // pieces as long as a workgroup holds; shorter ones down to 8192 while there are fewer than 512
    unsigned int count = (n + held - 1u) / held;
    const unsigned int fill = (unsigned int)((512u + rows - 1u) / rows), most = n / 8192u;
    if (count < fill) count = fill < most ? fill : most > count ? most : count;
    if (count > 64u) count = 64u;
    // (a row that stays whole is not rounded up: no whole piece of such a length would fit into it)
    if (count == 1u) return Pieces{1u, n};
    const unsigned int length = (n / count + 63u) / 64u * 64u;
    // (the last piece takes what is left, so it must fit too)
    count = n / length;
    if (n - (count - 1u) * length > held) ++count;
    return Pieces{count, length};
}
Pieces pieces_of(const rp_rows* r) {
    return r->dtype == RP_BF16 ? pieces_of<unsigned short>(r->rows, r->n) : pieces_of<float>(r->rows, r->n);
}
// Rows whose pieces are in the workspace at once (more go in several launches).
unsigned long long rows_at_once(const rp_rows* r, const Pieces& c) {
    const unsigned long long most = 8192u / c.count;
    return r->rows < most ? r->rows : most;
}
size_t pieces_bytes(const rp_rows* r) {
    if (r->rows == 0 || r->n <= 64u) return 0;
    const Pieces c = pieces_of(r);
    if (c.count == 1u) return 0;
    const size_t n = rows_at_once(r, c) * c.count;
    return align_up(n * sizeof(PieceHead), 256) + n * kList * 8u;
}
PieceSpace piece_space(void* workspace, unsigned long long rows, const Pieces& c) {
    return PieceSpace{static_cast<PieceHead*>(workspace),
                      reinterpret_cast<unsigned long long*>(static_cast<unsigned char*>(workspace) +
                                                            align_up(rows * c.count * sizeof(PieceHead), 256))};
}

template <typename T>
hipError_t launch_choose(const rp_rows* r, ChooseArgs a, void* workspace, hipStream_t st) {
    const unsigned int n = a.x.n;
    const dim3 blocks = row_grid(a.x.rows);
    if (n <= 64u) {
        choose_wave_kernel<T><<<row_grid((a.x.rows + 3) / 4), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    const Pieces c = pieces_of(r);
    if (c.count == 1u) {
        if (n <= HeldRow<4, 2, T>::kMost) choose_kernel<4, 2, 4, T><<<blocks, 256, 0, st>>>(a);
        else choose_kernel<8, 8, 4, T><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    }
    const unsigned long long rows = a.x.rows, step = rows_at_once(r, c);
    const PieceSpace ws = piece_space(workspace, step, c);
    for (unsigned long long at = 0; at < rows; at += step) {
        const unsigned int part = (unsigned int)(rows - at < step ? rows - at : step);
        choose_piece_kernel<8, 8, 4, T><<<dim3(c.count, part), 512, 0, st>>>(a, c, ws);
        choose_join_kernel<16, T><<<part, 1024, 0, st>>>(a, c, ws);
        a.x.data += part * a.x.stride * sizeof(T);
        a.u += part;
        a.index += part;
        if (a.logp) a.logp += part;
        if (a.row_temperature) a.row_temperature += part;
        if (a.row_top_p) a.row_top_p += part;
        if (a.row_min_p) a.row_min_p += part;
        if (a.row_top_k) a.row_top_k += part;
    }
    return hipGetLastError();
}
template <typename T>
hipError_t launch_top(const rp_rows* r, TopArgs a, void* workspace, hipStream_t st) {
    const unsigned int n = a.x.n;
    const dim3 blocks = row_grid(a.x.rows);
    if (n <= 64u) {
        top_wave_kernel<T><<<row_grid((a.x.rows + 3) / 4), 256, 0, st>>>(a);
        return hipGetLastError();
    }
    const Pieces c = pieces_of(r);
    if (c.count == 1u) {
        if (n <= HeldRow<4, 2, T>::kMost) top_kernel<4, 2, 4, T><<<blocks, 256, 0, st>>>(a);
        else top_kernel<8, 8, 4, T><<<blocks, 512, 0, st>>>(a);
        return hipGetLastError();
    }
    const unsigned long long rows = a.x.rows, step = rows_at_once(r, c);
    const PieceSpace ws = piece_space(workspace, step, c);
    for (unsigned long long at = 0; at < rows; at += step) {
        const unsigned int part = (unsigned int)(rows - at < step ? rows - at : step);
        top_piece_kernel<8, 8, 4, T><<<dim3(c.count, part), 512, 0, st>>>(a, c, ws);
        top_join_kernel<16, T><<<part, 1024, 0, st>>>(a, c, ws);
        a.x.data += part * a.x.stride * sizeof(T);
        a.values += (size_t)part * a.k * sizeof(T);
        a.index += (size_t)part * a.k;
        if (a.lse) a.lse += part;
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace rp

extern "C" {

size_t rp_choose_workspace_bytes(const rp_rows* logits) {
    if (const char* why = rp::logit_rows_fault(logits)) {
        rp::set_error("rp_choose_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return rp::pieces_bytes(logits);
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
    const size_t need = rp::pieces_bytes(logits);
    if (const char* fault = rp::workspace_fault(workspace, bytes, need)) {
        rp::set_error("rp_choose_actions: %s (%zu bytes given, %zu needed)", fault, bytes, need);
        return RP_ENOMEM;
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const rp::ChooseArgs a{rp::logit_rows(logits), how->temperature, how->top_p, how->min_p, how->top_k,
                           how->row_temperature, how->row_top_p, how->row_min_p, how->row_top_k, u, index, logp};
    RP_CHECK_HIP(logits->dtype == RP_BF16 ? rp::launch_choose<unsigned short>(logits, a, workspace, st)
                                           : rp::launch_choose<float>(logits, a, workspace, st));
    return RP_OK;
}

size_t rp_top_workspace_bytes(const rp_rows* logits, uint32_t k) {
    const char* why = rp::logit_rows_fault(logits);
    if (!why && (k == 0 || k > rp::kMaxTop || k > logits->n)) why = "k must be 1 .. min(n, 1024)";
    if (why) {
        rp::set_error("rp_top_workspace_bytes: %s", why);
        return (size_t)-1;
    }
    return rp::pieces_bytes(logits);
}

rp_status rp_top_actions(const rp_rows* logits, uint32_t k, double temperature, void* values, int32_t* index, float* lse,
                         void* workspace, size_t bytes, void* hip_stream) {
    const char* why = rp::logit_rows_fault(logits);
    RP_REQUIRE(!why, "rp_top_actions: %s", why);
    RP_REQUIRE(k >= 1 && k <= rp::kMaxTop && k <= logits->n, "rp_top_actions: k = %u, must be 1 .. min(n, 1024)", k);
    RP_REQUIRE(rp::temperature_fits(temperature), "rp_top_actions: the temperature must be 1e-30 .. 1e30");
    if (logits->rows == 0) return RP_OK;
    why = rp::logit_data_fault(logits);
    RP_REQUIRE(!why, "rp_top_actions: %s", why);
    RP_REQUIRE(values && index, "rp_top_actions: null array");
    const size_t need = rp::pieces_bytes(logits);
    if (const char* fault = rp::workspace_fault(workspace, bytes, need)) {
        rp::set_error("rp_top_actions: %s (%zu bytes given, %zu needed)", fault, bytes, need);
        return RP_ENOMEM;
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const rp::TopArgs a{rp::logit_rows(logits), k, 1.0 / temperature, (float)(1.4426950408889634 / temperature),
                        static_cast<unsigned char*>(values), index, lse};
    RP_CHECK_HIP(logits->dtype == RP_BF16 ? rp::launch_top<unsigned short>(logits, a, workspace, st)
                                           : rp::launch_top<float>(logits, a, workspace, st));
    return RP_OK;
}

}  // extern "C"
