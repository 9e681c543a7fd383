// New rows of the paged cache: appending keys and values with the rotary position embedding on the way, to a cache of
// 16- or 32-bit numbers or of 8-bit blocks, and the commit of accepted rows in a cache of 8-bit blocks.
#include <type_traits>

#include "owl_device.h"

namespace owl {

typedef __bf16 a_bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 a_f16x2 __attribute__((ext_vector_type(2)));
typedef float a_f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// The rotation, in 64 bits.  Angles grow with the position: at 128K a product in 32 bits is off by up to 4e-3 and a
// key by half a bf16 step; t * inv_freq is exact in 64 bits for positions up to 2^29 (24 bits of the one, 29 of the other; beyond, it is off
// by 2^-53 of itself).  What the turned channels are rounded to is then the number nearest to the formula's, but for one in some 10^9.
// ---------------------------------------------------------------------------
// scale * sin a and scale * cos a, to about 1e-16 of it: the nearest multiple k of pi/2 is taken off (pi/2 in two parts; with fused products the
// rest is exact to its last place for |k| < 2^52), and on the rest, at most pi/4, the Taylor series end where the next term
// is below 5e-17.
__device__ __forceinline__ double2 cos_sin(double a, double scale)
{
    const double k = __builtin_rint(a * 0.63661977236758134308);
    double r = __builtin_fma(-k, 1.57079632679489655800, a);
    r = __builtin_fma(-k, 6.12323399573676603587e-17, r);
    const double z = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = __builtin_fma(s, z, 1.0 / 6227020800.0);
    s = __builtin_fma(s, z, -1.0 / 39916800.0);
    s = __builtin_fma(s, z, 1.0 / 362880.0);
    s = __builtin_fma(s, z, -1.0 / 5040.0);
    s = __builtin_fma(s, z, 1.0 / 120.0);
    s = __builtin_fma(s, z, -1.0 / 6.0);
    s = __builtin_fma(s * z, r, r);
    c = __builtin_fma(c, z, -1.0 / 87178291200.0);
    c = __builtin_fma(c, z, 1.0 / 479001600.0);
    c = __builtin_fma(c, z, -1.0 / 3628800.0);
    c = __builtin_fma(c, z, 1.0 / 40320.0);
    c = __builtin_fma(c, z, -1.0 / 720.0);
    c = __builtin_fma(c, z, 1.0 / 24.0);
    c = __builtin_fma(c, z, -0.5);
    c = __builtin_fma(c, z, 1.0);
    const int quarter = (int)(k - 4.0 * __builtin_floor(k * 0.25));
    const double x = (quarter & 1 ? s : c) * scale, y = (quarter & 1 ? c : s) * scale;
    return make_double2(quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y);
}

// 64 bits -> 32 bits such that rounding the result to 16 bits rounds the 64-bit number correctly: what 32 bits cannot hold
// is cut off and leaves a one in the last place (round to odd).
__device__ __forceinline__ float to_odd(double d)
{
    const float f = (float)d;
    const double back = (double)f;
    uint32_t bits = __builtin_bit_cast(uint32_t, f);
    if (__builtin_fabs(back) > __builtin_fabs(d)) --bits;
    if (back != d) bits |= 1u;
    return __builtin_bit_cast(float, bits);
}

// The numbers of a 16-byte piece, and back.
template <typename T> struct Piece {
    static constexpr int E = 16 / sizeof(T);
    float v[E];
};

template <typename T>
__device__ __forceinline__ Piece<T> unpack(const uint4 &x)
{
    Piece<T> p;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (std::is_same<T, float>::value) {
            p.v[k] = __builtin_bit_cast(float, w[k]);
        } else if constexpr (std::is_same<T, __bf16>::value) {
            p.v[2 * k] = __builtin_bit_cast(float, w[k] << 16);
            p.v[2 * k + 1] = __builtin_bit_cast(float, w[k] & 0xFFFF0000u);
        } else {
            const a_f16x2 h = __builtin_bit_cast(a_f16x2, w[k]);
            p.v[2 * k] = (float)h[0];
            p.v[2 * k + 1] = (float)h[1];
        }
    }
    return p;
}

template <typename T>
__device__ __forceinline__ uint4 pack(const Piece<T> &p)
{
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (std::is_same<T, float>::value) {
            w[k] = __builtin_bit_cast(uint32_t, p.v[k]);
        } else {
            const a_f32x2 x = {p.v[2 * k], p.v[2 * k + 1]};
            if constexpr (std::is_same<T, __bf16>::value) w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, a_bf16x2));
            else w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, a_f16x2));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What both append kernels need, passed by value.
struct AppendArgs {
    const unsigned char *q, *k, *v;
    const float *inv_freq;
    const int32_t *pos_ids, *page_table, *ctx_lens, *n_new_seq;
    unsigned char *q_out, *k_cache, *v_cache;
    uint8_t *k_scale, *v_scale;
    uint32_t *status;
    int64_t q_stride, k_stride, v_stride;                    // bytes between tokens
    int64_t stride_page, stride_head, stride_token, n_pool_pages;      // bytes; pages
    int32_t n, Hq, Hkv, rot_dim, max_pages, max_ctx_len;
    float rot_scale;
};

// An item is two 16-byte pieces of a head that are turned together (or copied): item i < rot_dim / 2E holds the frequencies
// E i .. E i + E - 1.  Where its pieces begin, in channels:
template <int E, bool kPairs>
__device__ __forceinline__ int2 item_at(int i, int rot_dim)
{
    if (kPairs || 2 * E * i >= rot_dim) return make_int2(2 * E * i, 2 * E * i + E);
    return make_int2(E * i, rot_dim / 2 + E * i);
}

// Turns an item.  The cosine and sine of frequency E i + e, times the scale, are at cs[e * step].
template <typename T, bool kPairs>
__device__ __forceinline__ void turn(Piece<T> &a, Piece<T> &b, const double2 *cs, int step)
{
    constexpr int E = Piece<T>::E;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const double2 w = cs[e * step];
        float &x = kPairs ? (2 * e < E ? a.v[(2 * e) % E] : b.v[(2 * e) % E]) : a.v[e];
        float &y = kPairs ? (2 * e < E ? a.v[(2 * e + 1) % E] : b.v[(2 * e + 1) % E]) : b.v[e];
        const double xd = x, yd = y;
        const double p = xd * w.x - yd * w.y, q = yd * w.x + xd * w.y;
        x = std::is_same<T, float>::value ? (float)p : to_odd(p);
        y = std::is_same<T, float>::value ? (float)q : to_odd(q);
    }
}

__device__ __forceinline__ uint4 load16(const unsigned char *p) { return *reinterpret_cast<const uint4 *>(p); }
__device__ __forceinline__ void store16(unsigned char *p, const uint4 &x) { *reinterpret_cast<uint4 *>(p) = x; }

// Prefix length of sequence b, forced into range for the mapping; *good says whether it was in it.
__device__ __forceinline__ int append_len(const AppendArgs &p, int b, bool report, bool *good)
{
    const int L = load_uniform(p.ctx_lens, b);
    *good = L >= 0 && L <= p.max_ctx_len;
    if (!*good && report) flag_status(p.status, OWL_DEV_BAD_CTX_LEN);
    return *good ? L : (L < 0 ? 0 : p.max_ctx_len);
}

// Page under logical page lp of sequence b, or -1 (reported) where there is none.
__device__ __forceinline__ int append_page(const AppendArgs &p, int b, int lp, bool report)
{
    int page = lp;
    if (p.page_table) page = lp < p.max_pages ? load_uniform(p.page_table + (int64_t)b * p.max_pages, lp) : -1;
    if (page >= 0 && page < p.n_pool_pages) return page;
    if (report) flag_status(p.status, OWL_DEV_BAD_PAGE);
    return -1;
}

// ---------------------------------------------------------------------------
// Append to a cache in the rows' own type: one workgroup per token, an item a thread.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256;

template <typename T, int D, bool kPairs>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs p)
{
    constexpr int E = Piece<T>::E, kItems = D / (2 * E), ES = sizeof(T);
    __shared__ double2 s_cs[D / 2];                          // [e][item]
    fetch_args<void(AppendArgs)>();
    const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n_b = load_n_draft(p.n_new_seq, b, p.n, tid == 0 ? p.status : nullptr);
    if (i >= n_b) return;
    bool good;
    const int L = append_len(p, b, tid == 0, &good), at = L + i;
    const int page = good ? append_page(p, b, at / kPage, tid == 0) : -1;
    const int64_t token = (int64_t)b * p.n + i;
    const int turned = p.rot_dim / (2 * E);                  // items of a head that are turned
    if (tid < p.rot_dim / 2) {
        const int t = p.pos_ids ? p.pos_ids[token] : at;
        s_cs[tid % E * turned + tid / E] = cos_sin((double)t * (double)p.inv_freq[tid], (double)p.rot_scale);
    }
    __syncthreads();
    const int q_heads = p.q ? p.Hq : 0, heads = q_heads + 2 * p.Hkv;
    const int64_t row = (int64_t)page * p.stride_page + at % kPage * p.stride_token;
    for (int id = tid; id < heads * kItems; id += kAppendThreads) {
        const int item = id % kItems, head = id / kItems;
        const int2 c = item_at<E, kPairs>(item, p.rot_dim);
        const unsigned char *from;
        unsigned char *to;
        bool rotate = item < turned;
        if (head < q_heads) {
            from = p.q + token * p.q_stride + head * (D * ES);
            to = p.q_out + (token * p.Hq + head) * (D * ES);
        } else if (head < q_heads + p.Hkv) {
            from = p.k + token * p.k_stride + (head - q_heads) * (D * ES);
            to = p.k_cache + row + (head - q_heads) * p.stride_head;
        } else {
            from = p.v + token * p.v_stride + (head - q_heads - p.Hkv) * (D * ES);
            to = p.v_cache + row + (head - q_heads - p.Hkv) * p.stride_head;
            rotate = false;
        }
        if (head >= q_heads && page < 0) continue;
        uint4 x = load16(from + c.x * ES), y = load16(from + c.y * ES);
        if (rotate) {
            Piece<T> a = unpack<T>(x), z = unpack<T>(y);
            turn<T, kPairs>(a, z, s_cs + item, turned);
            x = pack<T>(a);
            y = pack<T>(z);
        }
        store16(to + c.x * ES, x);
        store16(to + c.y * ES, y);
    }
}

// ---------------------------------------------------------------------------
// 8-bit blocks
// ---------------------------------------------------------------------------
template <typename T> struct BlockRange;                     // what a block of numbers of type T may hold (owl.h)
template <> struct BlockRange<__bf16> {
    static constexpr int least = -117;
    static constexpr float top = 0x1.ep127f;
};
template <> struct BlockRange<_Float16> {
    static constexpr int least = -15;
    static constexpr float top = 0x1.ep15f;
};

// A number as it enters a block: within the range, or no number.
template <typename T>
__device__ __forceinline__ float admit(float v)
{
    const float c = fminf(fmaxf(v, -BlockRange<T>::top), BlockRange<T>::top);
    return __builtin_isfinite(v) ? c : __builtin_nanf("");
}

// The least e of the type's range with big <= 448 * 2^e = 1.75 * 2^(e + 8), for the bits of a finite big >= 0.
template <typename T>
__device__ __forceinline__ int block_exponent(uint32_t bits)
{
    return max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), BlockRange<T>::least);
}

__device__ __forceinline__ float two_to(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// Four numbers, times a power of two, as e4m3 (nearest even) in one word; the block's exponent keeps them within 448.
__device__ __forceinline__ uint32_t narrow4(const float *v, float scale)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * scale, v[1] * scale, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * scale, v[3] * scale, w, true);
}

__device__ __forceinline__ void widen4(uint32_t bytes, float scale, float *v)
{
    const a_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)bytes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)bytes, true);
    v[0] = lo[0] * scale;
    v[1] = lo[1] * scale;
    v[2] = hi[0] * scale;
    v[3] = hi[1] * scale;
}

// Greatest magnitude among n numbers, as bits; what is no number does not count.
template <int n>
__device__ __forceinline__ uint32_t greatest(const float *v)
{
    float m = 0.f;
#pragma unroll
    for (int k = 0; k < n; ++k) m = fmaxf(m, fabsf(v[k]));   // (of a NaN and a number: the number)
    return __builtin_bit_cast(uint32_t, m);
}

// ---------------------------------------------------------------------------
// Append to 8-bit blocks: one workgroup per (16-token block, KV head, sequence).  Its first half takes the block of K, its second that
// of V, an item a thread; then all of it turns the query heads of the group.  A block's scale depends on all its rows, so the
// old ones are read again and the block is written whole; positions that lie side by side cost each block once.
// Long chunks are bound by memory: 4 prompts' chunks of 2501 tokens, 389 MB, 82 us (4.8 TB/s, what a large copy reaches).  Trees are
// bound by one workgroup's chain, lengths -> page -> old block, angles and products in 64 bits -> greatest magnitude -> block: 16
// sequences with up to 26 tokens 8.0 us in a graph (8.8 with the queries read behind the block and angles one after the other; 8.4 with
// 512 threads, with which chunks take 87.7).  By counters a wavefront waits for 60 % of its cycles there and issues for 33 %, 730 vector
// instructions of it, most of them in 64 bits.
// ---------------------------------------------------------------------------
template <typename T, int D, bool kPairs>
__global__ void __launch_bounds__(kAppendThreads) append_quant_kernel(const AppendArgs p)
{
    constexpr int E = 8, kItems = D / (2 * E), ES = 2;
    __shared__ double2 s_cs[kPage * (D / 2 + 8)];            // [token][e][item], a token's 128 bytes further than they need
    __shared__ uint32_t s_big[2];
    fetch_args<void(AppendArgs)>();
    const int g = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const bool teller = tid == 0 && g == 0;
    const int n_b = load_n_draft(p.n_new_seq, b, p.n, teller ? p.status : nullptr);
    bool good;
    const int L = append_len(p, b, teller, &good), block = L / kPage + (int)blockIdx.x;
    const int first = block * kPage - L;                     // new token of slot 0; negative: rows before the context's end
    if (first >= n_b || n_b == 0) return;                    // (no new row: the block stays as it is)
    const int page = good ? append_page(p, b, block, teller) : -1;
    const int half = p.rot_dim / 2, turned = p.rot_dim / (2 * E);
    if (tid < 2) s_big[tid] = 0;
    // a thread a frequency, of every fourth (eighth) token: the chains of its angles run side by side
    constexpr int kAtOnce = kAppendThreads / (D / 2), kAngles = kPage / kAtOnce;
    const int f = tid % (D / 2);
    double angle[kAngles];
    {
        const double freq = f < half ? (double)p.inv_freq[f] : 0.0;
#pragma unroll
        for (int k = 0; k < kAngles; ++k) {
            const int i = first + tid / (D / 2) + k * kAtOnce;
            const int t = p.pos_ids && i >= 0 && i < n_b ? p.pos_ids[(int64_t)b * p.n + i] : L + i;
            angle[k] = (double)t * freq;
        }
    }
    // this thread's 16 numbers of the block
    const int tensor = tid / (kAppendThreads / 2), own = tid % (kAppendThreads / 2);
    const int slot = own / kItems, item = own % kItems, i = first + slot;
    const bool mine = own < kPage * kItems && page >= 0 && i < n_b;
    const int2 c = item_at<E, kPairs>(item, p.rot_dim);
    uint8_t *scale_at = (tensor ? p.v_scale : p.k_scale) + (int64_t)page * p.Hkv + g;
    unsigned char *to = (tensor ? p.v_cache : p.k_cache) + (int64_t)page * p.stride_page + g * p.stride_head + slot * p.stride_token;
    uint4 x{}, y{};
    float old_scale = 0.f;
    if (mine && i >= 0) {
        const unsigned char *from = (tensor ? p.v + ((int64_t)b * p.n + i) * p.v_stride : p.k + ((int64_t)b * p.n + i) * p.k_stride) + g * (D * ES);
        x = load16(from + c.x * ES);
        y = load16(from + c.y * ES);
    } else if (mine) {
        const uint2 u = *reinterpret_cast<const uint2 *>(to + c.x), w = *reinterpret_cast<const uint2 *>(to + c.y);
        x = make_uint4(u.x, u.y, 0, 0);
        y = make_uint4(w.x, w.y, 0, 0);
        old_scale = __builtin_bit_cast(float, (uint32_t)*scale_at << 23);
    }
    // and its first two items of the queries: all that is read is asked for before the angles are formed
    const int group = p.Hq / p.Hkv, q_items = p.q ? kPage * group * kItems : 0;
    struct Query {
        int item, slot;                                      // slot -1: none
        int64_t row;
        uint4 x, y;
    };
    auto query = [&](int id) -> Query {
        Query r;
        r.item = id % kItems;
        const int rest = id / kItems, s = (int)(((float)rest + 0.5f) * __builtin_amdgcn_rcpf((float)group));     // rest / group, exactly
        const int tok = first + s;
        const bool is = id < q_items && tok >= 0 && tok < n_b;
        r.slot = is ? s : -1;
        if (!is) return r;
        const int head = g * group + rest - s * group;
        const int64_t token = (int64_t)b * p.n + tok;
        const int2 at = item_at<E, kPairs>(r.item, p.rot_dim);
        r.row = token * p.Hq + head;
        const unsigned char *from = p.q + token * p.q_stride + head * (D * ES);
        r.x = load16(from + at.x * ES);
        r.y = load16(from + at.y * ES);
        return r;
    };
    auto answer = [&](const Query &r) {
        if (r.slot < 0) return;
        const int2 at = item_at<E, kPairs>(r.item, p.rot_dim);
        uint4 u = r.x, w = r.y;
        if (r.item < turned) {
            Piece<T> a = unpack<T>(u), z = unpack<T>(w);
            turn<T, kPairs>(a, z, s_cs + r.slot * (D / 2 + 8) + r.item, turned);
            u = pack<T>(a);
            w = pack<T>(z);
        }
        unsigned char *out = p.q_out + r.row * (D * ES);
        store16(out + at.x * ES, u);
        store16(out + at.y * ES, w);
    };
    Query q0 = query(tid), q1 = query(tid + kAppendThreads);
#pragma unroll
    for (int k = 0; k < kAngles; ++k)
        if (f < half) s_cs[(tid / (D / 2) + k * kAtOnce) * (D / 2 + 8) + f % E * turned + f / E] = cos_sin(angle[k], (double)p.rot_scale);
    __syncthreads();
    float v[2 * E] = {};
    if (mine && i >= 0) {
        Piece<T> a = unpack<T>(x), z = unpack<T>(y);
        if (tensor == 0 && item < turned) {
            turn<T, kPairs>(a, z, s_cs + slot * (D / 2 + 8) + item, turned);
            a = unpack<T>(pack<T>(a));                       // what a 16-bit cache would hold
            z = unpack<T>(pack<T>(z));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = a.v[e];
            v[E + e] = z.v[e];
        }
    } else if (mine) {
        widen4(x.x, old_scale, v);
        widen4(x.y, old_scale, v + 4);
        widen4(y.x, old_scale, v + 8);
        widen4(y.y, old_scale, v + 12);
    }
#pragma unroll
    for (int e = 0; e < 2 * E; ++e) v[e] = admit<T>(v[e]);
    const int big = wave_max((int)greatest<2 * E>(v));
    if ((tid & 63) == 0) atomicMax(&s_big[tensor], (uint32_t)big);
    for (int id = tid; id < q_items; id += 2 * kAppendThreads) {
        answer(q0);
        answer(q1);
        q0 = query(id + 2 * kAppendThreads);
        q1 = query(id + 3 * kAppendThreads);
    }
    __syncthreads();
    if (mine) {
        const int e = block_exponent<T>(s_big[tensor]);
        const float scale = two_to(-e);
        *reinterpret_cast<uint2 *>(to + c.x) = make_uint2(narrow4(v, scale), narrow4(v + 4, scale));
        *reinterpret_cast<uint2 *>(to + c.y) = make_uint2(narrow4(v + 8, scale), narrow4(v + 12, scale));
        if (own == 0) *scale_at = (uint8_t)(e + 127);
    }
}

template <typename T, int D>
static hipError_t launch_append_as(const AppendArgs &p, int B, bool pairs, bool quant, hipStream_t s)
{
    if constexpr (!std::is_same<T, float>::value) {
        if (quant) {
            // blocks from the one that holds the context's end to the one that holds the last new token, wherever it begins
            const dim3 grid((p.n + 2 * kPage - 2) / kPage, p.Hkv, B);
            if (pairs) hipLaunchKernelGGL((append_quant_kernel<T, D, true>), grid, dim3(kAppendThreads), 0, s, p);
            else hipLaunchKernelGGL((append_quant_kernel<T, D, false>), grid, dim3(kAppendThreads), 0, s, p);
            return hipGetLastError();
        }
    }
    const dim3 grid(p.n, B);
    if (pairs) hipLaunchKernelGGL((append_kernel<T, D, true>), grid, dim3(kAppendThreads), 0, s, p);
    else hipLaunchKernelGGL((append_kernel<T, D, false>), grid, dim3(kAppendThreads), 0, s, p);
    return hipGetLastError();
}

int64_t append_threads(int64_t n_tokens, bool quant)
{
    return (quant ? (n_tokens + 2 * kPage - 2) / kPage : n_tokens) * kAppendThreads;
}

hipError_t launch_append(const owl_verify_desc &d, const owl_append_desc &a, const void *q, const void *k_new, const void *v_new,
                         const float *inv_freq, const int32_t *pos_ids, void *q_out, void *k_cache, void *v_cache,
                         uint8_t *k_scale, uint8_t *v_scale, const int32_t *page_table, const int32_t *ctx_lens,
                         const int32_t *n_new_seq, uint32_t *status, hipStream_t s)
{
    const int64_t es = d.qkv_dtype == OWL_F32 ? 4 : 2, cb = k_scale ? 1 : es;
    AppendArgs p;
    p.q = static_cast<const unsigned char *>(q);
    p.k = static_cast<const unsigned char *>(k_new);
    p.v = static_cast<const unsigned char *>(v_new);
    p.inv_freq = inv_freq;
    p.pos_ids = pos_ids;
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.n_new_seq = n_new_seq;
    p.q_out = static_cast<unsigned char *>(q_out);
    p.k_cache = static_cast<unsigned char *>(k_cache);
    p.v_cache = static_cast<unsigned char *>(v_cache);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.status = status;
    p.q_stride = a.q_stride * es;
    p.k_stride = a.k_stride * es;
    p.v_stride = a.v_stride * es;
    p.stride_page = d.kv_stride_page * cb;
    p.stride_head = d.kv_stride_head * cb;
    p.stride_token = d.kv_stride_token * cb;
    p.n_pool_pages = d.n_pool_pages;
    p.n = a.n_tokens;
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.rot_dim = a.rot_dim;
    p.max_pages = d.max_pages_per_seq;
    p.max_ctx_len = d.max_ctx_len;
    p.rot_scale = a.rot_scale;
    const bool pairs = a.rot_style == OWL_ROT_PAIRS, quant = k_scale != nullptr;
    const bool wide = d.head_dim == 128;
    switch (d.qkv_dtype) {
    case OWL_BF16: return wide ? launch_append_as<__bf16, 128>(p, d.batch, pairs, quant, s) : launch_append_as<__bf16, 64>(p, d.batch, pairs, quant, s);
    case OWL_F16: return wide ? launch_append_as<_Float16, 128>(p, d.batch, pairs, quant, s) : launch_append_as<_Float16, 64>(p, d.batch, pairs, quant, s);
    default: return wide ? launch_append_as<float, 128>(p, d.batch, pairs, false, s) : launch_append_as<float, 64>(p, d.batch, pairs, false, s);
    }
}

// ---------------------------------------------------------------------------
// KV commit in 8-bit blocks: one workgroup per (KV head, sequence, tensor).  The rows of the path land in at most five blocks,
// from the one that holds position ctx_lens[b] on; a piece is 16 bytes of a row, and the 64 pieces of a
// wavefront belong to one block.  All that the new blocks consist of is read, with the scales of the pages it
// comes from, before the barrier; the blocks' greatest magnitudes meet in LDS there, and everything is written behind
// it.  Checks as in the commit of a 16-bit cache.
// ---------------------------------------------------------------------------
constexpr int kCommitQuantThreads = 256, kCommitBlocks = (64 + 2 * kPage - 2) / kPage;

template <typename T, int D>
__global__ void __launch_bounds__(kCommitQuantThreads) commit_quant_kernel(
    unsigned char *k_cache, unsigned char *v_cache, uint8_t *k_scale, uint8_t *v_scale, const int32_t *page_table,
    const int32_t *ctx_lens, const int32_t *accepted, const int32_t *n_accept, int N, int Hkv, int max_pages, int max_ctx_len,
    int64_t n_pool_pages, int64_t stride_page, int64_t stride_head, int64_t stride_token, int32_t *new_ctx_lens, uint32_t *status)
{
    constexpr int PPR = D / 16, kPieces = kPage * PPR;       // pieces of a row, of a block
    constexpr int kHeld = (kCommitBlocks * kPieces + kCommitQuantThreads - 1) / kCommitQuantThreads;
    __shared__ uint32_t s_big[kCommitBlocks];
    const int g = blockIdx.x, b = blockIdx.y;
    unsigned char *cache = (blockIdx.z ? v_cache : k_cache) + g * stride_head;
    uint8_t *scales = (blockIdx.z ? v_scale : k_scale) + g;
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < kCommitBlocks) s_big[tid] = 0;
    const int a = accepted[(int64_t)b * N + min(lane, N - 1)];
    int na = load_uniform(n_accept, b), L = load_uniform(ctx_lens, b);
    if (L < 0 || L > max_ctx_len) {
        if (tid == 0) flag_status(status, OWL_DEV_BAD_CTX_LEN);
        L = L < 0 ? 0 : max_ctx_len;
    }
    if (na < 0 || na > N) {
        if (tid == 0) flag_status(status, OWL_DEV_BAD_ACCEPT);
        na = 0;
    }
    // row `lane` of the path: physical pages of its source and destination, unchecked ids
    const int before = __shfl_up(a, 1), from = L + min(max(a, 0), N - 1), to = L + lane;
    const int from_lp = from / kPage, to_lp = to / kPage, base_lp = L / kPage;
    int from_page = from_lp, to_page = to_lp, base_page = base_lp;
    if (page_table) {
        const int32_t *pages = page_table + (int64_t)b * max_pages;
        from_page = pages[min(from_lp, max_pages - 1)];
        to_page = pages[min(to_lp, max_pages - 1)];
        base_page = pages[min(base_lp, max_pages - 1)];      // of the rows before the context's end, as of row 0
    }
    const bool bad_page = (page_table && max(from_lp, to_lp) >= max_pages) || min(from_page, to_page) < 0 || max(from_page, to_page) >= n_pool_pages;
    const bool mine = lane < na, bad = a < 0 || a >= N || (lane > 0 && a <= before);
    const bool any_bad = __builtin_amdgcn_ballot_w64(mine && bad) != 0;
    if (any_bad || __builtin_amdgcn_ballot_w64(mine && bad_page) != 0) {
        if (tid == 0) flag_status(status, any_bad ? OWL_DEV_BAD_ACCEPT : OWL_DEV_BAD_PAGE);
        na = 0;
    }
    if (g == 0 && blockIdx.z == 0 && tid == 0 && new_ctx_lens) new_ctx_lens[b] = L + na;
    const int64_t src = (int64_t)from_page * stride_page + from % kPage * stride_token;
    const int64_t dst = (int64_t)to_page * stride_page + to % kPage * stride_token;
    const uint64_t moved = __builtin_amdgcn_ballot_w64(lane < na && src != dst);      // rows of the path that change places
    if (moved == 0) return;                                  // uniform over the workgroup

    const int kept = L % kPage, total = kept + na;           // rows of the blocks, from slot 0 of the first one on
    auto shfl64 = [](int64_t v, int from_lane) -> int64_t {
        const uint32_t lo = __shfl((uint32_t)v, from_lane), hi = __shfl((uint32_t)((uint64_t)v >> 32), from_lane);
        return (int64_t)(((uint64_t)hi << 32) | lo);
    };
    float v[kHeld][16];
    int64_t at[kHeld];                                       // where a piece goes, -1: nowhere
    int page_of[kHeld];                                      // and in which page
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const int id = tid + h * kCommitQuantThreads, blk = id / kPieces, slot = id % kPieces / PPR, piece = id % PPR;
        const int r = blk * kPage + slot, i = r - kept;      // row of the path; negative: in place
        const int il = min(max(i, 0), 63);
        const int64_t s = shfl64(src, il), d = shfl64(dst, il);
        const int s_page = __shfl(from_page, il), d_page = __shfl(to_page, il);
        // rows of the path that fall into this block, and whether one of them moves
        const int lo = max(blk * kPage - kept, 0), hi = min((blk + 1) * kPage - kept, na);
        const uint64_t rows = hi > lo ? (~(uint64_t)0 >> (64 - (hi - lo))) << lo : 0;
        const bool wanted = blk < kCommitBlocks && r < total && (moved & rows) != 0;
        const int64_t here = i < 0 ? (int64_t)base_page * stride_page + slot * stride_token : s;
        at[h] = wanted ? (i < 0 ? here : d) + piece * 16 : -1;
        page_of[h] = i < 0 ? base_page : d_page;
#pragma unroll
        for (int e = 0; e < 16; ++e) v[h][e] = 0.f;
        if (wanted) {
            const uint4 x = load16(cache + here + piece * 16);
            const float scale = __builtin_bit_cast(float, (uint32_t)scales[(int64_t)(i < 0 ? base_page : s_page) * Hkv] << 23);
            widen4(x.x, scale, v[h]);
            widen4(x.y, scale, v[h] + 4);
            widen4(x.z, scale, v[h] + 8);
            widen4(x.w, scale, v[h] + 12);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[h][e] = admit<T>(v[h][e]);
        }
    }
    __syncthreads();                                         // s_big is clear (and all reads done, as the values below are used)
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const int blk = (tid + h * kCommitQuantThreads) / kPieces;
        const int big = wave_max((int)greatest<16>(v[h]));
        if (lane == 0 && blk < kCommitBlocks) atomicMax(&s_big[blk], (uint32_t)big);
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        if (at[h] < 0) continue;
        const int id = tid + h * kCommitQuantThreads, blk = id / kPieces;
        const int e = block_exponent<T>(s_big[blk]);
        const float scale = two_to(-e);
        store16(cache + at[h], make_uint4(narrow4(v[h], scale), narrow4(v[h] + 4, scale), narrow4(v[h] + 8, scale), narrow4(v[h] + 12, scale)));
        if (id % kPieces == 0) scales[(int64_t)page_of[h] * Hkv] = (uint8_t)(e + 127);      // slot 0 of a block is always one of its rows
    }
}

template <typename T, int D>
static hipError_t launch_commit_quant_as(const owl_verify_desc &d, void *k_cache, void *v_cache, uint8_t *k_scale, uint8_t *v_scale,
                                         const int32_t *page_table, const int32_t *ctx_lens, const int32_t *accepted,
                                         const int32_t *n_accept, int32_t *new_ctx_lens, uint32_t *status, hipStream_t s)
{
    hipLaunchKernelGGL((commit_quant_kernel<T, D>), dim3(d.n_kv_heads, d.batch, 2), dim3(kCommitQuantThreads), 0, s,
                       static_cast<unsigned char *>(k_cache), static_cast<unsigned char *>(v_cache), k_scale, v_scale, page_table,
                       ctx_lens, accepted, n_accept, d.n_draft, d.n_kv_heads, d.max_pages_per_seq, d.max_ctx_len, d.n_pool_pages,
                       d.kv_stride_page, d.kv_stride_head, d.kv_stride_token, new_ctx_lens, status);
    return hipGetLastError();
}

hipError_t launch_commit_quant(const owl_verify_desc &d, void *k_cache, void *v_cache, uint8_t *k_scale, uint8_t *v_scale,
                               const int32_t *page_table, const int32_t *ctx_lens, const int32_t *accepted,
                               const int32_t *n_accept, int32_t *new_ctx_lens, uint32_t *status, hipStream_t s)
{
    auto launch = d.qkv_dtype == OWL_BF16 ? (d.head_dim == 128 ? &launch_commit_quant_as<__bf16, 128> : &launch_commit_quant_as<__bf16, 64>)
                                          : (d.head_dim == 128 ? &launch_commit_quant_as<_Float16, 128> : &launch_commit_quant_as<_Float16, 64>);
    return launch(d, k_cache, v_cache, k_scale, v_scale, page_table, ctx_lens, accepted, n_accept, new_ctx_lens, status, s);
}

}  // namespace owl
