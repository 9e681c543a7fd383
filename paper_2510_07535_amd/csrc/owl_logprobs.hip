// Log probabilities of given tokens, entropy and the top alternatives of rows of logits.
//
// With x = scale * (logit - top), top the row's greatest logit, l = sum e^x, t = sum x e^x:
//     log p = x - ln l,      entropy = ln l - t / l .
// The greatest logit is kept as it is: times the scale it would round, by up to 2^-24 of itself, which every log probability would be
// off by (that of a near-certain token above 0), and at the ends of the type it would be infinite.
// A workgroup reads its logits once, into registers: a whole row of up to 32K, or a slice of 4K of a longer one (or of more rows than
// there are compute units). A second launch, a workgroup a row, joins the slices' (top, l, t),
//     top = max top_s,  x_s = scale * (top_s - top),  w_s = e^x_s,  L = sum w_s l_s,  T = sum w_s (t_s + x_s l_s) .
//
// The greatest n logits: the threads form 64 groups; the n-th greatest of the groups' greatest is a bound that n logits reach, and if
// the great ones lie in no order hardly more do (10: 11, 32: 44).  Those go to LDS, and one's place is the number of greater ones, of
// equal logits those with smaller tokens.  Should more than 512 reach the bound (equal ones), they are taken one after the
// other.  The join bounds the slices' ordered lists likewise.
//
// Bound by the logits' bytes, and by the vector unit: some nine instructions and an exponential a logit, 250 instructions a wavefront
// for the selection.  us, in a graph: 120 rows of 128K in fp32 18.5 (3.3 TB/s; without alternatives 14.5, 4.2 TB/s; the join 4 of them),
// 400 rows of 200K in bf16 54.7, 1 row of 32K in bf16 6.6 and of 128K 8.3.  The greatest one after the other, each a reduction of the
// workgroup: 67 and 21 instead of 18.5 and 6.6.  Slices of 2K / 8K / 16K: 24.0 / 18.8 / 21.5 (more selections, or fewer loads in
// flight).
#include <float.h>

#include <type_traits>

#include "owl_device.h"

namespace owl {

constexpr int kJoinThreads = 512, kSliceWaves = 4, kRowWaves = 16;
constexpr int kSliceHeld = 16, kSlice = 64 * kSliceWaves * kSliceHeld;
constexpr int kGroups = 64;                                  // of a slice's threads, 4 or 16 of them each
constexpr int kLogFound = 512;                               // candidates for a slice's greatest
constexpr int kLogTop = 32;                                  // the most alternatives asked for
constexpr float kLog2e = 1.4426950408889634f;
// Below this e^x is 0, and x stands for -infinity: what is excluded adds 0, not 0 times infinity.
constexpr float kFloor = -1.0e4f;

// Logits as integers of the same order, 0 standing for what is no number with a sign; -0 and +0 are equal.
__device__ __forceinline__ uint32_t logit_order(float x)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, x + 0.0f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float order_logit(uint32_t order)
{
    return __builtin_bit_cast(float, order & 0x80000000u ? order & 0x7FFFFFFFu : ~order);
}

// A logit and its token in one number that orders them: greater logits first, smaller tokens first among equals.  0: none.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t token)
{
    if (!(x > -INFINITY)) return 0;
    return ((uint64_t)logit_order(x) << 32) | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ float key_logit(uint64_t key)
{
    return order_logit((uint32_t)(key >> 32));
}
__device__ __forceinline__ int key_token(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

__device__ __forceinline__ float wave_fmax(float v)
{
#define OWL_DPP_FMAX(ctrl, rows)                                                                                             \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), ctrl, rows, 0xf, false)))
    OWL_DPP_FMAX(0x111, 0xf);
    OWL_DPP_FMAX(0x112, 0xf);
    OWL_DPP_FMAX(0x114, 0xf);
    OWL_DPP_FMAX(0x118, 0xf);
    OWL_DPP_FMAX(0x142, 0xa);
    OWL_DPP_FMAX(0x143, 0xc);
#undef OWL_DPP_FMAX
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = ((uint64_t)__shfl_xor((uint32_t)(v >> 32), d) << 32) | __shfl_xor((uint32_t)v, d);
        v = o > v ? o : v;
    }
    return v;
}

// The greatest of 4 or 16 neighbouring lanes.
template <int kLanes>
__device__ __forceinline__ float lanes_fmax(float v)
{
#define OWL_DPP_FMAX(ctrl) \
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, false)))
    OWL_DPP_FMAX(0xB1);
    OWL_DPP_FMAX(0x4E);
    if constexpr (kLanes == 16) {
        OWL_DPP_FMAX(0x141);
        OWL_DPP_FMAX(0x140);
    }
#undef OWL_DPP_FMAX
    return v;
}
template <int kLanes>
__device__ __forceinline__ int lanes_sum(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);
    if constexpr (kLanes == 16) {
        v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);
        v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);
    }
    return v;
}

// Both sums, in turn: a step that reads other lanes waits for what was written just before it.
__device__ __forceinline__ void wave_sums(float &a, float &b)
{
#define OWL_DPP_ADD(v, ctrl, rows) \
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, rows, 0xf, false))
#define OWL_DPP_ADDS(ctrl, rows) OWL_DPP_ADD(a, ctrl, rows); OWL_DPP_ADD(b, ctrl, rows)
    OWL_DPP_ADDS(0x111, 0xf);
    OWL_DPP_ADDS(0x112, 0xf);
    OWL_DPP_ADDS(0x114, 0xf);
    OWL_DPP_ADDS(0x118, 0xf);
    OWL_DPP_ADDS(0x142, 0xa);
    OWL_DPP_ADDS(0x143, 0xc);
#undef OWL_DPP_ADDS
#undef OWL_DPP_ADD
    a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, a), 63));
    b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, b), 63));
}

// The number of keys of a list in LDS that are greater than `key`.
__device__ __forceinline__ int greater_keys(const uint64_t *list, int count, uint64_t key)
{
    int place = 0;
#pragma unroll 8
    for (int o = 0; o < count; ++o) place += list[o] > key ? 1 : 0;
    return place;
}

template <typename T>
__device__ __forceinline__ float to_float(T x) { return (float)x; }

// scale * (x - y) for y >= x.  Of logits more than the greatest number apart the difference is formed of their halves.
__device__ __forceinline__ float scaled_difference(float x, float y, float scale)
{
    const float d = x - y;
    return d > -INFINITY ? d * scale : (0.5f * x - 0.5f * y) * scale * 2.0f;
}

// What a slice leaves: its statistics; top is +infinity where it met a logit that is +infinity or no number.
struct SliceStats {
    float top, l, t, unused;
};

template <typename T>
struct LogArgs {
    const T *logits;
    const int32_t *tokens;
    float *logprob, *entropy, *top_logprobs;
    int32_t *top_ids;
    uint32_t *status;
    SliceStats *stats;                               // [rows][slices]
    uint64_t *keys;                                  // [rows][slices][n_top]
    int64_t row_stride;
    int vocab, n_given, n_top, slices;
    float scale;
};

// A thread's given token and its logit, asked for before anything else: the logit's address is known one load later than the rest.
struct Given {
    int token;
    bool known;
    float x;
};
template <typename T>
__device__ __forceinline__ Given take_given(const LogArgs<T> &p, int r, int tid)
{
    Given g{-1, false, 0.f};
    if (tid < p.n_given) {
        g.token = p.tokens[(int64_t)r * p.n_given + tid];
        g.known = g.token >= 0 && g.token < p.vocab;
        if (g.known) g.x = to_float(p.logits[(int64_t)r * p.row_stride + g.token]);
    }
    return g;
}

// Row r once its sums are known (all threads of the workgroup hold them): what does not depend on the greatest logits is written here,
// and put(j, key) writes the j-th of those.
template <typename T>
struct Row {
    const LogArgs<T> &p;
    int r;
    float top, log_l;
    bool bad;

    __device__ Row(const LogArgs<T> &args, int row, int tid, float top_, float l, float t, const Given &given) : p(args), r(row), top(top_)
    {
        bad = top == INFINITY;
        log_l = logf(l);
        if (tid == 0) {
            if (bad) flag_status(p.status, OWL_DEV_BAD_LOGIT);
            if (p.entropy) p.entropy[r] = bad ? __builtin_nanf("") : (top == -INFINITY ? 0.f : log_l - t / l);
        }
        if (tid < p.n_given) {
            if (!given.known && given.token != -1) flag_status(p.status, OWL_DEV_BAD_TOKEN);
            p.logprob[(int64_t)r * p.n_given + tid] = given.known ? logp(given.x) : (given.token == -1 ? 0.f : __builtin_nanf(""));
        }
    }
    __device__ float logp(float x) const
    {
        if (bad) return __builtin_nanf("");
        return x > -INFINITY ? scaled_difference(x, top, p.scale) - log_l : -INFINITY;
    }
    __device__ void put(int j, uint64_t key) const
    {
        const int64_t o = (int64_t)r * p.n_top + j;
        if (p.top_ids) p.top_ids[o] = key && !bad ? key_token(key) : -1;
        if (p.top_logprobs) p.top_logprobs[o] = key ? logp(key_logit(key)) : (bad ? __builtin_nanf("") : -INFINITY);
    }
};

// kWhole: the slice is the row, and nothing is left to join.
template <typename T, int kWaves, int kHeld, bool kWhole>
__global__ void __launch_bounds__(64 * kWaves) logprob_slice_kernel(const LogArgs<T> p)
{
    constexpr int kThreads = 64 * kWaves, kLanes = kThreads / kGroups, E = 16 / sizeof(T), kLoads = kHeld / E;
    __shared__ float s_m[kWaves], s_l[kWaves], s_t[kWaves];
    __shared__ __align__(16) float s_group[kGroups];
    __shared__ uint32_t s_bound;
    __shared__ int s_found;
    __shared__ uint64_t s_key[kWaves];
    __shared__ __align__(16) uint64_t s_keys[kLogFound];
    fetch_args<void(LogArgs<T>)>();
    const int r = blockIdx.x, slice = kWhole ? 0 : blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_top = p.n_top, vocab = p.vocab;
    const T *row = p.logits + (int64_t)r * p.row_stride;
    [[maybe_unused]] Given given{};
    if constexpr (kWhole) given = take_given(p, r, tid);
    // 16-byte pieces at aligned addresses: piece 0 begins `skew` logits before the row
    const int skew = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    const T *pieces = row - skew;
    float x[kHeld];
    auto token_of = [&](int k) -> int { return slice * (kThreads * kHeld) + ((k / E) * kThreads + tid) * E + k % E - skew; };
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int first = token_of(k * E);
        if (first >= 0 && first + E <= vocab) {
            typedef T Vec __attribute__((ext_vector_type(E)));
            const Vec *at = reinterpret_cast<const Vec *>(pieces + (first + skew));
            // (slices are read as a stream, non-temporal: 120 rows of 128K 19.8 -> 18.5 us; whole rows are often still in L2: 64 rows
            // of 32K in fp16 7.8 -> 7.0 without)
            const Vec v = kWhole ? *at : __builtin_nontemporal_load(at);
#pragma unroll
            for (int e = 0; e < E; ++e) x[k * E + e] = to_float(v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[k * E + e] = first + e >= 0 && first + e < vocab ? to_float(row[first + e]) : -INFINITY;
        }
    }
    float piece_top[kLoads], top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        piece_top[k] = x[k * E];
#pragma unroll
        for (int e = 1; e < E; ++e) piece_top[k] = fmaxf(piece_top[k], x[k * E + e]);
        top = fmaxf(top, piece_top[k]);
    }
    const float group_top = lanes_fmax<kLanes>(top), wm = wave_fmax(group_top);
    if (tid % kLanes == 0) s_group[tid / kLanes] = group_top;
    if (tid == 0) {
        s_bound = 0xFFFFFFFFu;
        s_found = 0;
    }
    if (lane == 0) s_m[wave] = wm;
    __syncthreads();
    float m = s_m[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w]);
    // (halves: their difference is finite, and rounded as the whole one)
    const float to_log2 = fminf(p.scale * (2.0f * kLog2e), FLT_MAX), half_base = m > -INFINITY ? 0.5f * m : 0.f;
    float l = 0.f, t = 0.f;
#pragma unroll
    for (int k = 0; k < kHeld; k += 4) {             // (four at a time: an exponential's result is waited for)
        float y[4], e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (maximum keeps what is no number, and the sums tell)
            y[i] = __builtin_elementwise_maximum(__builtin_fmaf(x[k + i], 0.5f, -half_base) * to_log2, kFloor);
            e[i] = __builtin_amdgcn_exp2f(y[i]);
        }
        l += (e[0] + e[1]) + (e[2] + e[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __builtin_fmaf(y[i], e[i], t);
    }
    wave_sums(l, t);
    if (lane == 0) {
        s_l[wave] = l;
        s_t[wave] = t;
    }
    if (n_top > 0) {
        // A bound that n_top logits of the slice reach: the n_top-th of the groups' greatest.  Little more than n_top do, if the
        // great ones are not all in a few groups.
        const float own = s_group[tid / kLanes];
        int above = 0;
#pragma unroll
        for (int o = 0; o < kGroups / kLanes; o += 4) {
            const float4 x4 = *reinterpret_cast<const float4 *>(&s_group[tid % kLanes * (kGroups / kLanes) + o]);
            above += (x4.x > own ? 1 : 0) + (x4.y > own ? 1 : 0) + (x4.z > own ? 1 : 0) + (x4.w > own ? 1 : 0);
        }
        above = lanes_sum<kLanes>(above);
        if (above < n_top && tid % kLanes == 0) atomicMin(&s_bound, logit_order(own));
        __syncthreads();
        const float least = fmaxf(order_logit(s_bound), -FLT_MAX);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (__builtin_amdgcn_ballot_w64(piece_top[k] >= least) == 0) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (x[k * E + e] >= least) {
                    const int place = atomicAdd(&s_found, 1);
                    if (place < kLogFound) s_keys[place] = rank_key(x[k * E + e], (uint32_t)token_of(k * E + e));
                }
            }
        }
    }
    __syncthreads();
    l = t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        l += s_l[w];
        t += s_t[w];
    }
    t *= 1.0f / kLog2e;
    if (!(l < INFINITY)) m = INFINITY;               // (one that is infinite less itself is no number either)
    auto list = [&](auto &&put) {                    // put(j, key): the slice's j-th greatest, in any order of j
        if (n_top == 0) return;
        const int found = s_found;
        if (found <= kLogFound) {
            for (int i = tid; i < found; i += kThreads) {
                const uint64_t key = s_keys[i];
                const int place = greater_keys(s_keys, found, key);
                if (place < n_top) put(place, key);
            }
            for (int j = found + tid; j < n_top; j += kThreads) put(j, 0);
            return;
        }
        // many equal logits: one after the other
        uint64_t last = ~(uint64_t)0;
        for (int j = 0; j < n_top; ++j) {
            uint64_t best = 0;
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const uint64_t key = rank_key(x[k], (uint32_t)token_of(k));
                if (key < last && key > best) best = key;
            }
            best = wave_max64(best);
            if (lane == 0) s_key[wave] = best;
            __syncthreads();
            last = s_key[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) last = s_key[w] > last ? s_key[w] : last;
            __syncthreads();
            if (tid == 0) put(j, last);
        }
    };
    if constexpr (kWhole) {
        const Row<T> out(p, r, tid, m, l, t, given);
        list([&](int j, uint64_t key) { out.put(j, key); });
    } else {
        const int64_t at = (int64_t)r * p.slices + slice;
        if (tid == 0) p.stats[at] = SliceStats{m, l, t, 0.f};
        list([&](int j, uint64_t key) { p.keys[at * n_top + j] = key; });
    }
}

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) logprob_join_kernel(const LogArgs<T> p)
{
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ float s_l[kWaves], s_t[kWaves], s_m[kWaves];
    __shared__ unsigned long long s_least;
    __shared__ int s_count;
    __shared__ uint64_t s_keys[kLogTop * kLogTop];   // (keys that reach the bound are those of n_top lists at most)
    fetch_args<void(LogArgs<T>)>();
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, slices = p.slices, n_top = p.n_top;
    // A thread a slice; and a thread a key of the lists' first columns.
    const SliceStats mine = tid < slices ? p.stats[(int64_t)r * slices + tid] : SliceStats{-INFINITY, 0.f, 0.f, 0.f};
    const uint64_t *all = p.keys + (int64_t)r * slices * n_top;
    const int count = slices * n_top, columns = min(n_top, kJoinThreads / slices), column = tid / slices;
    const bool holds = column < columns;
    const uint64_t column_key = holds ? all[(tid - column * slices) * n_top + column] : 0;
    const uint64_t first_key = tid < count ? all[tid] : 0;
    const Given given = take_given(p, r, tid);
    const float wm = wave_fmax(mine.top);
    if (lane == 0) s_m[wave] = wm;
    if (tid == 0) {
        s_least = 1;
        s_count = 0;
    }
    s_keys[tid] = column_key;
    __syncthreads();
    float m = s_m[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w]);
    // (of rows without any logit, or with bad ones, the sums are not used)
    const float d = m > -INFINITY ? fmaxf(scaled_difference(mine.top, m, p.scale), kFloor) : 0.f, weight = __builtin_amdgcn_exp2f(d * kLog2e);
    float l = weight * mine.l, t = weight * __builtin_fmaf(d, mine.l, mine.t);
    wave_sums(l, t);
    if (lane == 0) {
        s_l[wave] = l;
        s_t[wave] = t;
    }
    // The slices' lists are ordered.  What i + 1 of their first reach in ceil(n_top / (i + 1)) lists, n_top keys reach: the
    // greatest such bound, of the first columns, leaves little more than the answer.
    if (holds && column_key) {
        const int lists = (n_top + column) / (column + 1);
        const int place = greater_keys(s_keys + column * slices, slices, column_key);
        if (place == lists - 1) atomicMax(&s_least, (unsigned long long)column_key);
    }
    __syncthreads();
    l = t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        l += s_l[w];
        t += s_t[w];
    }
    const Row<T> out(p, r, tid, m, l, t, given);
    if (n_top == 0) return;
    const uint64_t least = s_least;
    for (int k = tid; k < count; k += kJoinThreads) {
        const uint64_t key = k == tid ? first_key : all[k];
        if (key >= least) s_keys[atomicAdd(&s_count, 1)] = key;
    }
    __syncthreads();
    const int kept = s_count;
    for (int k = tid; k < kept; k += kJoinThreads) {
        const uint64_t key = s_keys[k];
        const int place = greater_keys(s_keys, kept, key);
        if (place < n_top) out.put(place, key);
    }
    for (int j = kept + tid; j < n_top; j += kJoinThreads) out.put(j, 0);
}

// How a row is cut; it may begin up to seven logits into a piece.  One launch serves rows up to 32K where they all find a compute unit: us,
// two launches -> one, 1 / 120 / 400 rows of 32K 8.2 -> 6.5 / 10.7 -> 8.2 / 17.3 -> 18.4; rows of 64K, with 64 logits a thread, 8.1 -> 9.2 /
// 14.0 -> 12.4 / 26.5 -> 32.1.
struct LogPlan {
    int held, slices;                                // logits of a thread; one slice: no second launch
};
static LogPlan plan_of(const owl_logprob_desc &d, int cus)
{
    const int64_t n = (int64_t)d.vocab + 7;
    if (n <= 64 * kRowWaves * 8) return LogPlan{8, 1};
    if (n <= 64 * kRowWaves * 32 && d.rows <= cus) return LogPlan{32, 1};
    return LogPlan{kSliceHeld, (int)((n + kSlice - 1) / kSlice)};
}

size_t logprob_scratch_bytes(const owl_logprob_desc &d, int cus)
{
    const LogPlan plan = plan_of(d, cus);
    return plan.slices == 1 ? 256 : (size_t)d.rows * plan.slices * (sizeof(SliceStats) + (size_t)d.n_top * sizeof(uint64_t));
}

int64_t logprob_threads(const owl_logprob_desc &d, int cus)
{
    return (int64_t)d.rows * (plan_of(d, cus).slices == 1 ? 64 * kRowWaves : kJoinThreads);
}

template <typename T>
static hipError_t launch_logprobs_as(const owl_logprob_desc &d, const void *logits, const int32_t *tokens, float *logprob, float *entropy,
                                     int32_t *top_ids, float *top_logprobs, void *scratch, uint32_t *status, int cus, hipStream_t s)
{
    const LogPlan plan = plan_of(d, cus);
    LogArgs<T> p{};
    p.logits = static_cast<const T *>(logits);
    p.tokens = tokens;
    p.logprob = logprob;
    p.entropy = entropy;
    p.top_ids = top_ids;
    p.top_logprobs = top_logprobs;
    p.status = status;
    p.stats = static_cast<SliceStats *>(scratch);
    p.keys = reinterpret_cast<uint64_t *>(p.stats + (size_t)d.rows * plan.slices);
    p.row_stride = d.row_stride;
    p.vocab = d.vocab;
    p.n_given = d.n_given;
    p.n_top = top_ids || top_logprobs ? d.n_top : 0;
    p.slices = plan.slices;
    p.scale = d.scale;
    if (plan.slices == 1) {
        auto kernel = plan.held == 8 ? &logprob_slice_kernel<T, kRowWaves, 8, true> : &logprob_slice_kernel<T, kRowWaves, 32, true>;
        hipLaunchKernelGGL(kernel, dim3(d.rows), dim3(64 * kRowWaves), 0, s, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((logprob_slice_kernel<T, kSliceWaves, kSliceHeld, false>), dim3(d.rows, plan.slices), dim3(64 * kSliceWaves), 0, s, p);
    hipLaunchKernelGGL((logprob_join_kernel<T>), dim3(d.rows), dim3(kJoinThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_logprobs(const owl_logprob_desc &d, const void *logits, const int32_t *tokens, float *logprob, float *entropy,
                           int32_t *top_ids, float *top_logprobs, void *scratch, uint32_t *status, int cus, hipStream_t s)
{
    auto launch = d.dtype == OWL_F32 ? &launch_logprobs_as<float> : d.dtype == OWL_BF16 ? &launch_logprobs_as<__bf16> : &launch_logprobs_as<_Float16>;
    return launch(d, logits, tokens, logprob, entropy, top_ids, top_logprobs, scratch, status, cus, s);
}

}  // namespace owl
