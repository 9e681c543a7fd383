// Log probabilities of given tokens, entropy and the top alternatives of rows of logits.
//
// With x = scale * logit, m = max x, l = sum e^(x - m), t = sum (x - m) e^(x - m):
//     log p = x - m - ln l,      entropy = ln l - t / l .
// Two launches.  The first cuts every row into slices, a workgroup each, which reads its logits once into registers
// and leaves (m, l, t) and the slice's greatest logits in the scratch; the second, a workgroup a row, joins them with
//     M = max m_s,  w_s = e^(m_s - M),  L = sum w_s l_s,  T = sum w_s (t_s + (m_s - M) l_s)
// and picks the greatest of the slices' greatest.
#include <float.h>

#include <type_traits>

#include "owl_device.h"

namespace owl {

typedef _Float16 l_f16x2 __attribute__((ext_vector_type(2)));

constexpr int kLogThreads = 256, kLogWaves = kLogThreads / 64;
constexpr int kLogHeld = 32;                                 // logits a thread holds
constexpr int kLogFound = 64;                                // candidates of a wavefront for the slice's greatest
constexpr int kLogTop = 32;                                  // the most alternatives asked for
constexpr int kSlice = kLogThreads * kLogHeld;
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

// A number that at least `want` (<= 64) of the lanes' numbers reach, the wavefront's greatest being that of `most`: the
// interval is halved until hardly more than `want` of them do.
__device__ __forceinline__ uint32_t reached_by(uint32_t order, float most, int want)
{
    uint32_t lo = 0, hi = __builtin_amdgcn_readfirstlane(logit_order(most)) + 1;     // (all reach lo, none hi)
    // the first step goes down from the greatest by a quarter, an octave and a half for a number of the usual size
    uint32_t step = 3u << 22;
    while (hi - lo > 1) {
        const uint32_t mid = step && hi - lo > step ? hi - step : lo + (hi - lo) / 2;
        const int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(order >= mid));
        if (count >= want) {
            lo = mid;
            step = 0;
            if (count <= want + want / 8) break;
        } else {
            hi = mid;
            step *= 2;
        }
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ float to_float(T x) { return (float)x; }

// What a slice leaves: its statistics, and whether it met a logit that is +infinity or no number.
struct SliceStats {
    float m, l, t;
    uint32_t bad;
};

template <typename T>
__global__ void __launch_bounds__(kLogThreads) logprob_slice_kernel(const T *logits, int vocab, int64_t row_stride, float scale,
                                                                   int n_top, int slices, SliceStats *stats, uint64_t *keys)
{
    constexpr int E = 16 / sizeof(T), kLoads = kLogHeld / E;
    __shared__ float s_m[kLogWaves], s_l[kLogWaves], s_t[kLogWaves];
    __shared__ uint32_t s_all[kLogWaves], s_some[kLogWaves];
    __shared__ int s_own[kLogWaves];
    __shared__ uint64_t s_key[kLogWaves], s_found[kLogWaves][kLogFound];
    const int r = blockIdx.x, slice = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *row = logits + (int64_t)r * row_stride;
    // 16-byte pieces at aligned addresses: piece 0 begins `skew` logits before the row
    const int skew = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    const T *pieces = row - skew;
    float x[kLogHeld];
    auto token_of = [&](int k) -> int { return slice * kSlice + ((k / E) * kLogThreads + tid) * E + k % E - skew; };
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int first = token_of(k * E);
        if (first >= 0 && first + E <= vocab) {
            struct alignas(16) Vec { T v[E]; };
            const Vec v = *reinterpret_cast<const Vec *>(pieces + (first + skew));
#pragma unroll
            for (int e = 0; e < E; ++e) x[k * E + e] = to_float(v.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[k * E + e] = first + e >= 0 && first + e < vocab ? to_float(row[first + e]) : -INFINITY;
        }
    }
    float top = x[0];
#pragma unroll
    for (int k = 1; k < kLogHeld; ++k) top = fmaxf(top, x[k]);
    const float wm = wave_fmax(top);
    if (n_top > 0) {
        // Two bounds that n_top logits of the slice reach: those of n_top threads of one wavefront, and of a quarter of
        // them in each.  The greater one is the better: with the logits in no order the second, and where one wavefront
        // has all the great ones the first.
        const uint32_t order = logit_order(top);
        const uint32_t all = reached_by(order, wm, n_top), some = reached_by(order, wm, (n_top + kLogWaves - 1) / kLogWaves);
        if (lane == 0) {
            s_all[wave] = all;
            s_some[wave] = some;
        }
    }
    if (lane == 0) s_m[wave] = wm;
    __syncthreads();
    float m = s_m[0];
#pragma unroll
    for (int w = 1; w < kLogWaves; ++w) m = fmaxf(m, s_m[w]);
    const float to_log2 = fminf(scale * kLog2e, FLT_MAX), base = m > -INFINITY ? m : 0.f;
    m *= scale;
    float l = 0.f, t = 0.f;
#pragma unroll
    for (int k = 0; k < kLogHeld; ++k) {
        // (maximum keeps what is no number, and the sums tell)
        const float y = __builtin_elementwise_maximum((x[k] - base) * to_log2, kFloor);
        const float e = __builtin_amdgcn_exp2f(y);
        l += e;
        t = __builtin_fmaf(y, e, t);
    }
    l = wave_sum(l);
    t = wave_sum(t);
    if (lane == 0) {
        s_l[wave] = l;
        s_t[wave] = t;
    }
    int own = 0;
    if (n_top > 0) {
        uint32_t all = s_all[0], some = s_some[0];
#pragma unroll
        for (int w = 1; w < kLogWaves; ++w) {
            all = max(all, s_all[w]);
            some = min(some, s_some[w]);
        }
        const float least = fmaxf(order_logit(max(all, some)), -FLT_MAX);
#pragma unroll
        for (int k = 0; k < kLogHeld; ++k) {
            const uint64_t hit = __builtin_amdgcn_ballot_w64(x[k] >= least);
            if (hit) {                               // (uniform)
                const int place = own + __builtin_amdgcn_mbcnt_hi((uint32_t)(hit >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0));
                if (x[k] >= least && place < kLogFound) s_found[wave][place] = rank_key(x[k], (uint32_t)token_of(k));
                own += __builtin_popcountll(hit);
            }
        }
        if (lane == 0) s_own[wave] = own;
    }
    __syncthreads();
    if (tid == 0) {
        float ls = 0.f, ts = 0.f;
#pragma unroll
        for (int w = 0; w < kLogWaves; ++w) {
            ls += s_l[w];
            ts += s_t[w];
        }
        const bool bad = !(ls < INFINITY) || m == INFINITY;
        stats[(int64_t)r * slices + slice] = SliceStats{bad ? INFINITY : m, ls, ts * (1.0f / kLog2e), bad ? 1u : 0u};
    }
    if (n_top == 0) return;
    uint64_t *out = keys + ((int64_t)r * slices + slice) * n_top;
    int found = 0;
    bool fits = true;
#pragma unroll
    for (int w = 0; w < kLogWaves; ++w) {
        found += s_own[w];
        fits &= s_own[w] <= kLogFound;
    }
    if (fits) {
        for (int i = lane; i < s_own[wave]; i += 64) {
            const uint64_t key = s_found[wave][i];
            int place = 0;                           // the number of greater ones
#pragma unroll
            for (int w = 0; w < kLogWaves; ++w)
                for (int o = 0; o < s_own[w]; ++o) place += s_found[w][o] > key ? 1 : 0;
            if (place < n_top) out[place] = key;
        }
        for (int j = found + tid; j < n_top; j += kLogThreads) out[j] = 0;
        return;
    }
    // many equal logits: one after the other
    uint64_t last = ~(uint64_t)0;
    for (int j = 0; j < n_top; ++j) {
        uint64_t best = 0;
#pragma unroll
        for (int k = 0; k < kLogHeld; ++k) {
            const uint64_t key = rank_key(x[k], (uint32_t)token_of(k));
            if (key < last && key > best) best = key;
        }
        best = wave_max64(best);
        if (lane == 0) s_key[wave] = best;
        __syncthreads();
        last = s_key[0];
#pragma unroll
        for (int w = 1; w < kLogWaves; ++w) last = s_key[w] > last ? s_key[w] : last;
        __syncthreads();
        if (tid == 0) out[j] = last;
    }
}

template <typename T>
__global__ void __launch_bounds__(kLogThreads) logprob_join_kernel(const T *logits, int vocab, int64_t row_stride, float scale,
                                                                  int n_given, int n_top, int slices, const SliceStats *stats,
                                                                  const uint64_t *keys, const int32_t *tokens, float *logprob,
                                                                  float *entropy, int32_t *top_ids, float *top_logprobs,
                                                                  uint32_t *status)
{
    __shared__ float s_l[kLogWaves], s_t[kLogWaves], s_m[kLogWaves];
    __shared__ unsigned long long s_least;
    __shared__ int s_count;
    __shared__ uint64_t s_keys[kLogTop * kLogTop];   // (keys that reach the bound are those of n_top lists at most)
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const SliceStats *mine = stats + (int64_t)r * slices;
    float m = -INFINITY;
    for (int s = tid; s < slices; s += kLogThreads) m = fmaxf(m, mine[s].m);
    m = wave_fmax(m);
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kLogWaves; ++w) m = fmaxf(m, s_m[w]);
    const bool bad = m == INFINITY, none = m == -INFINITY;
    float l = 0.f, t = 0.f;
    if (!bad && !none) {
        for (int s = tid; s < slices; s += kLogThreads) {
            const SliceStats x = mine[s];
            const float d = fmaxf(x.m - m, kFloor), w = __builtin_amdgcn_exp2f(d * kLog2e);
            l = __builtin_fmaf(w, x.l, l);
            t = __builtin_fmaf(w, __builtin_fmaf(d, x.l, x.t), t);
        }
    }
    l = wave_sum(l);
    t = wave_sum(t);
    if (lane == 0) {
        s_l[wave] = l;
        s_t[wave] = t;
    }
    __syncthreads();
    l = t = 0.f;
#pragma unroll
    for (int w = 0; w < kLogWaves; ++w) {
        l += s_l[w];
        t += s_t[w];
    }
    const float log_l = logf(l), nan = __builtin_nanf("");
    if (tid == 0) {
        if (bad) flag_status(status, OWL_DEV_BAD_LOGIT);
        if (entropy) entropy[r] = bad ? nan : (none ? 0.f : log_l - t / l);
    }
    auto logp = [&](float x) -> float {
        if (bad) return nan;
        return x > -INFINITY ? __builtin_fmaf(x, scale, -m) - log_l : -INFINITY;
    };
    for (int j = tid; j < n_given; j += kLogThreads) {
        const int token = tokens[(int64_t)r * n_given + j];
        const bool known = token >= 0 && token < vocab;
        if (!known && token != -1) flag_status(status, OWL_DEV_BAD_TOKEN);
        logprob[(int64_t)r * n_given + j] = known ? logp(to_float(logits[(int64_t)r * row_stride + token])) : (token == -1 ? 0.f : nan);
    }
    if (n_top == 0) return;
    // The slices' lists are ordered.  What i + 1 of their first reach in ceil(n_top / (i + 1)) lists, n_top keys reach: the
    // greatest such bound, of the first columns (a thread a key), leaves little more than the answer.
    const uint64_t *all = keys + (int64_t)r * slices * n_top;
    const int count = slices * n_top, columns = min(n_top, kLogThreads / slices);
    if (tid == 0) {
        s_least = 1;
        s_count = 0;
    }
    const int i = tid / slices;
    const bool holds = i < columns;
    const uint64_t mine_key = holds ? all[(tid - i * slices) * n_top + i] : 0;
    s_keys[tid] = mine_key;
    __syncthreads();
    if (holds && mine_key) {
        const int lists = (n_top + i) / (i + 1);
        int place = 0;
        for (int o = 0; o < slices; ++o) place += s_keys[i * slices + o] > mine_key ? 1 : 0;
        if (place == lists - 1) atomicMax(&s_least, (unsigned long long)mine_key);
    }
    __syncthreads();
    const uint64_t least = s_least;
    for (int k = tid; k < count; k += kLogThreads) {
        const uint64_t key = all[k];
        if (key >= least) s_keys[atomicAdd(&s_count, 1)] = key;
    }
    __syncthreads();
    const int kept = s_count;
    auto put = [&](int j, uint64_t key) {
        const int64_t o = (int64_t)r * n_top + j;
        if (top_ids) top_ids[o] = key && !bad ? key_token(key) : -1;
        if (top_logprobs) top_logprobs[o] = key ? logp(key_logit(key)) : (bad ? nan : -INFINITY);
    };
    for (int k = tid; k < kept; k += kLogThreads) {
        const uint64_t key = s_keys[k];
        int place = 0;                               // the number of greater ones
        for (int o = 0; o < kept; ++o) place += s_keys[o] > key ? 1 : 0;
        if (place < n_top) put(place, key);
    }
    for (int j = kept + tid; j < n_top; j += kLogThreads) put(j, 0);
}

static int slices_of(const owl_logprob_desc &d)
{
    return (int)(((int64_t)d.vocab + 7 + kSlice - 1) / kSlice);          // a row may begin up to seven logits into a piece
}

size_t logprob_scratch_bytes(const owl_logprob_desc &d, int)
{
    return (size_t)d.rows * slices_of(d) * (sizeof(SliceStats) + (size_t)d.n_top * sizeof(uint64_t));
}

template <typename T>
static hipError_t launch_logprobs_as(const owl_logprob_desc &d, const void *logits, const int32_t *tokens, float *logprob, float *entropy,
                                     int32_t *top_ids, float *top_logprobs, void *scratch, uint32_t *status, hipStream_t s)
{
    const int slices = slices_of(d);
    SliceStats *stats = static_cast<SliceStats *>(scratch);
    uint64_t *keys = reinterpret_cast<uint64_t *>(stats + (size_t)d.rows * slices);
    const T *x = static_cast<const T *>(logits);
    const int n_top = top_ids || top_logprobs ? d.n_top : 0;
    hipLaunchKernelGGL((logprob_slice_kernel<T>), dim3(d.rows, slices), dim3(kLogThreads), 0, s, x, d.vocab, d.row_stride, d.scale, n_top,
                       slices, stats, keys);
    hipLaunchKernelGGL((logprob_join_kernel<T>), dim3(d.rows), dim3(kLogThreads), 0, s, x, d.vocab, d.row_stride, d.scale, d.n_given,
                       n_top, slices, stats, keys, tokens, logprob, entropy, top_ids, top_logprobs, status);
    return hipGetLastError();
}

hipError_t launch_logprobs(const owl_logprob_desc &d, const void *logits, const int32_t *tokens, float *logprob, float *entropy,
                           int32_t *top_ids, float *top_logprobs, void *scratch, uint32_t *status, int, hipStream_t s)
{
    auto launch = d.dtype == OWL_F32 ? &launch_logprobs_as<float> : d.dtype == OWL_BF16 ? &launch_logprobs_as<__bf16> : &launch_logprobs_as<_Float16>;
    return launch(d, logits, tokens, logprob, entropy, top_ids, top_logprobs, scratch, status, s);
}

}  // namespace owl
