// New rows of the paged cache: appending keys and values with the norms of the heads and the rotary position embedding on the
// way, to a cache of 16- or 32-bit numbers, of 8-bit blocks or of 4-bit groups, and the commit of accepted rows in a cache of
// 8-bit blocks.
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
    float rot_scale, eps;
    const float *q_gain, *k_gain;                            // norms: a gain a channel, or null = ones
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

// ---------------------------------------------------------------------------
// The norm of a head, in 64 bits like the rotation behind it, so that a row is rounded once, when it is stored.  A head's items lie in
// neighbouring lanes, whose squares meet by DPP, no LDS.
// ---------------------------------------------------------------------------
template <int ctrl>
__device__ __forceinline__ double lane_of(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, ctrl, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), ctrl, 0xf, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over n = 4, 8 or 16 neighbouring lanes, all of them active; each gets it, and the same one.
template <int n>
__device__ __forceinline__ double lanes_sum(double v)
{
    v += lane_of<0xB1>(v);                                   // lane ^ 1
    v += lane_of<0x4E>(v);                                   // lane ^ 2
    if constexpr (n > 4) v += lane_of<0x141>(v);             // the other four of eight, mirrored
    if constexpr (n > 8) v += lane_of<0x140>(v);             // the other eight of sixteen
    return v;
}

// 1 / sqrt(x), to about 1e-16 of it: the instruction's 2^-26 or so and two Newton steps.  0 and infinity, for which the steps are
// no numbers, keep what the instruction gives, infinity and 0.
__device__ __forceinline__ double inverse_root(double x)
{
    const double y0 = __builtin_amdgcn_rsq(x);
    double y = y0;
#pragma unroll
    for (int k = 0; k < 2; ++k) y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
    return x > 0.0 && x < __builtin_inf() ? y : y0;
}

// An item of a head of q or k: normalised with the head's gains (of channels at.x .. and at.y ..), then turned if `rotate` says so,
// and rounded once.  kItems lanes that hold the same head call this together.
template <typename T, bool kPairs, int kItems>
__device__ __forceinline__ void normalise(Piece<T> &a, Piece<T> &b, const float *gain, int2 at, double eps, bool rotate, const double2 *cs, int step)
{
    constexpr int E = Piece<T>::E;
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) sum = __builtin_fma((double)a.v[e], (double)a.v[e], __builtin_fma((double)b.v[e], (double)b.v[e], sum));
    const double r = inverse_root(lanes_sum<kItems>(sum) * (1.0 / (2 * E * kItems)) + eps);
    auto rounded = [](double d) -> float { return std::is_same<T, float>::value ? (float)d : to_odd(d); };
#pragma unroll
    for (int e = 0; e < E; ++e) {
        // the two channels that frequency E i + e turns, or channels e of the two pieces
        float &x = kPairs ? (2 * e < E ? a.v[(2 * e) % E] : b.v[(2 * e) % E]) : a.v[e];
        float &y = kPairs ? (2 * e < E ? a.v[(2 * e + 1) % E] : b.v[(2 * e + 1) % E]) : b.v[e];
        const int cx = kPairs ? (2 * e < E ? at.x : at.y) + (2 * e) % E : at.x + e, cy = kPairs ? cx + 1 : at.y + e;
        const double xd = (double)x * r * (double)gain[cx], yd = (double)y * r * (double)gain[cy];
        double p = xd, q = yd;
        if (rotate) {
            const double2 w = cs[e * step];
            p = xd * w.x - yd * w.y;
            q = yd * w.x + xd * w.y;
        }
        x = rounded(p);
        y = rounded(q);
    }
}

// The gains of q, then of k, into LDS.
template <int D, int kThreads>
__device__ __forceinline__ void take_gains(const AppendArgs &p, float *s_gain)
{
    for (int c = threadIdx.x; c < 2 * D; c += kThreads) {
        const float *from = c < D ? p.q_gain : p.k_gain;
        s_gain[c] = from ? from[c % D] : 1.0f;
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

__device__ __forceinline__ float two_to(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// ---------------------------------------------------------------------------
// 4-bit groups
// ---------------------------------------------------------------------------
template <typename T> struct GroupRange;                     // exponents of a group of numbers of type T (owl.h)
template <> struct GroupRange<__bf16> { static constexpr int least = -125, most = 125; };
template <> struct GroupRange<_Float16> { static constexpr int least = -23, most = 13; };

// The least e of the type's range with big <= 7 * 2^e = 1.75 * 2^(e + 2), for the bits of a finite big >= 0.
template <typename T>
__device__ __forceinline__ int group_exponent(uint32_t bits)
{
    const int e = (int)(bits >> 23) - 127 - 2 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(e, GroupRange<T>::least), GroupRange<T>::most);
}

// Greatest magnitude of a piece, as bits; infinity and what is no number lie above all others.
template <typename T>
__device__ __forceinline__ uint32_t greatest_bits(const Piece<T> &p)
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < Piece<T>::E; ++e) m = max(m, __builtin_bit_cast(uint32_t, p.v[e]) & 0x7FFFFFFFu);
    return m;
}

// Greatest of n = 4 or 8 neighbouring lanes' numbers, all of them active.
template <int n>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));
    if constexpr (n > 4) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));
    return v;
}

// Eight numbers of a group with exponent e as codes, nearest even, the first in the lowest four bits; beyond 6 * 2^e they are 6 * 2^e.
__device__ __forceinline__ uint32_t codes8(const float *v, int e)
{
    const float s = two_to(e);
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
}

// An item of a row on its way into a cache of 4-bit groups: `row` and `scales` are where the row's codes and scale bytes go.  A piece
// lies in one group, a group's pieces in neighbouring lanes; D / 16 lanes that hold the same row call this together.
template <typename T, int D>
__device__ __forceinline__ void store_groups(const Piece<T> &a, const Piece<T> &b, int2 at, unsigned char *row, uint8_t *scales)
{
    constexpr int kGroups = D / 32;
    const int ga = at.x / 32, gb = at.y / 32;
    const uint32_t own_a = greatest_bits(a), own_b = greatest_bits(b);
    uint32_t big_a = 0, big_b = 0;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
        const uint32_t m = lanes_max<D / 16>(max(ga == k ? own_a : 0u, gb == k ? own_b : 0u));
        if (ga == k) big_a = m;
        if (gb == k) big_b = m;
    }
    const bool none_a = big_a >= 0x7F800000u, none_b = big_b >= 0x7F800000u;         // infinity or no number among them: no numbers
    const int ea = group_exponent<T>(big_a), eb = group_exponent<T>(big_b);
    *reinterpret_cast<uint32_t *>(row + at.x / 2) = none_a ? 0u : codes8(a.v, ea);
    *reinterpret_cast<uint32_t *>(row + at.y / 2) = none_b ? 0u : codes8(b.v, eb);
    if (at.x % 32 == 0) scales[ga] = none_a ? 255 : (uint8_t)(ea + 127);
    if (at.y % 32 == 0) scales[gb] = none_b ? 255 : (uint8_t)(eb + 127);
}

// ---------------------------------------------------------------------------
// Append to a cache in the rows' own type, or (kFour) of 4-bit groups, which ask nothing of other tokens either: one workgroup per
// token, an item a thread.  kNorm: with the norms of the heads.
// Many tokens are bound by memory: a prompt of 8K in fp16, 201 MB, 43 us with the norms and 40 without (4.7 and 5.0 TB/s), in fp32 78 (5.2 TB/s), with the norms into 4 bits
// 45 (3.9); four chunks of 2501 into 4 bits, 380 MB, 75 us (5.1 TB/s).  Few are bound by a workgroup's chain, lengths -> page, angles and products in 64 bits, of which an
// item with the norm has some 200: with 384 threads, which 48 heads of 128 channels are in one pass, a tree of 60 tokens takes 4.3 us
// and 16 trees of up to 26 into 4 bits 6.3; with 256 5.2 and 6.9.  Where 256 threads take more than one pass, 384 / 256, us, of 700, 1024 and 2048 tokens: 48 heads 7.4 / 7.7, 8.6 / 9.1,
// 14.4 / 13.4, into 4 bits 7.6 / 8.1, 9.9 / 9.5, 16.3 / 14.3; 80 heads 10.1 / 10.6, 12.3 / 12.2, 23.4 / 22.1; fp32, 48 heads, 8.2 / 8.4, 10.6 / 10.4, 22.6 / 23.1.  Where they take one, 18 heads,
// 4.0 / 3.9 of 60, 5.5 / 5.2 of 700.  (With the rows asked for before the lengths, 5.5 and 7.0: they wait for nothing that the angles do not take as long as.)
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256, kNormThreads = 384, kNormTokens = 768;

template <typename T, int D, bool kPairs, bool kNorm, bool kFour, int kThreads>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendArgs p)
{
    constexpr int E = Piece<T>::E, kItems = D / (2 * E), ES = sizeof(T);
    __shared__ double2 s_cs[D / 2];                          // [e][item]
    __shared__ float s_gain[kNorm ? 2 * D : 1];
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
    if constexpr (kNorm) take_gains<D, kThreads>(p, s_gain);
    __syncthreads();
    const int q_heads = p.q ? p.Hq : 0, heads = q_heads + 2 * p.Hkv;
    const int64_t row = (int64_t)page * p.stride_page + at % kPage * p.stride_token;
    for (int id = tid; id < heads * kItems; id += kThreads) {
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
        if (head >= q_heads && page < 0) continue;           // (the same for all items of a head)
        uint4 x = load16(from + c.x * ES), y = load16(from + c.y * ES);
        if constexpr (kNorm) {
            if (head < q_heads + p.Hkv) {
                Piece<T> a = unpack<T>(x), z = unpack<T>(y);
                normalise<T, kPairs, kItems>(a, z, s_gain + (head < q_heads ? 0 : D), c, (double)p.eps, rotate, s_cs + item, turned);
                x = pack<T>(a);
                y = pack<T>(z);
            }
        } else if (rotate) {
            Piece<T> a = unpack<T>(x), z = unpack<T>(y);
            turn<T, kPairs>(a, z, s_cs + item, turned);
            x = pack<T>(a);
            y = pack<T>(z);
        }
        if constexpr (kFour) {
            if (head >= q_heads) {
                const bool is_v = head >= q_heads + p.Hkv;
                const int h = head - q_heads - (is_v ? p.Hkv : 0);
                uint8_t *scales = (is_v ? p.v_scale : p.k_scale) + (((int64_t)page * p.Hkv + h) * kPage + at % kPage) * (D / 32);
                store_groups<T, D>(unpack<T>(x), unpack<T>(y), c, to, scales);       // what a 16-bit cache would hold
                continue;
            }
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
template <typename T, int D, bool kPairs, bool kNorm>
__global__ void __launch_bounds__(kAppendThreads) append_quant_kernel(const AppendArgs p)
{
    constexpr int E = 8, kItems = D / (2 * E), ES = 2;
    __shared__ double2 s_cs[kPage * (D / 2 + 8)];            // [token][e][item], a token's 128 bytes further than they need
    __shared__ float s_gain[kNorm ? 2 * D : 1];
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
    if constexpr (kNorm) take_gains<D, kAppendThreads>(p, s_gain);
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
        if (kNorm || r.item < turned) {
            Piece<T> a = unpack<T>(u), z = unpack<T>(w);
            const double2 *cs = s_cs + r.slot * (D / 2 + 8) + r.item;
            if constexpr (kNorm) normalise<T, kPairs, kItems>(a, z, s_gain, at, (double)p.eps, r.item < turned, cs, turned);
            else turn<T, kPairs>(a, z, cs, turned);
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
        if (tensor == 0 && (kNorm || item < turned)) {
            const double2 *cs = s_cs + slot * (D / 2 + 8) + item;
            if constexpr (kNorm) normalise<T, kPairs, kItems>(a, z, s_gain + D, c, (double)p.eps, item < turned, cs, turned);
            else turn<T, kPairs>(a, z, cs, turned);
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

template <typename T, int D, bool kPairs, bool kNorm, bool kFour>
static void launch_append_tokens(const AppendArgs &p, int B, hipStream_t s)
{
    const int64_t items = ((int64_t)(p.q ? p.Hq : 0) + 2 * (int64_t)p.Hkv) * (D / (2 * Piece<T>::E));
    if constexpr (kNorm)
        if (items > kAppendThreads && (int64_t)p.n * B <= kNormTokens) {
            hipLaunchKernelGGL((append_kernel<T, D, kPairs, kNorm, kFour, kNormThreads>), dim3(p.n, B), dim3(kNormThreads), 0, s, p);
            return;
        }
    hipLaunchKernelGGL((append_kernel<T, D, kPairs, kNorm, kFour, kAppendThreads>), dim3(p.n, B), dim3(kAppendThreads), 0, s, p);
}

template <typename T, int D, bool kPairs, bool kNorm>
static void launch_append_rows(const AppendArgs &p, int B, Cached cached, hipStream_t s)
{
    if constexpr (!std::is_same<T, float>::value) {
        if (cached == Cached::kBlocks8) {
            // blocks from the one that holds the context's end to the one that holds the last new token, wherever it begins
            const dim3 grid((p.n + 2 * kPage - 2) / kPage, p.Hkv, B);
            hipLaunchKernelGGL((append_quant_kernel<T, D, kPairs, kNorm>), grid, dim3(kAppendThreads), 0, s, p);
            return;
        }
        if (cached == Cached::kGroups4) {
            launch_append_tokens<T, D, kPairs, kNorm, true>(p, B, s);
            return;
        }
    }
    launch_append_tokens<T, D, kPairs, kNorm, false>(p, B, s);
}

template <typename T, int D>
static hipError_t launch_append_as(const AppendArgs &p, int B, bool pairs, bool norm, Cached cached, hipStream_t s)
{
    if (pairs) norm ? launch_append_rows<T, D, true, true>(p, B, cached, s) : launch_append_rows<T, D, true, false>(p, B, cached, s);
    else norm ? launch_append_rows<T, D, false, true>(p, B, cached, s) : launch_append_rows<T, D, false, false>(p, B, cached, s);
    return hipGetLastError();
}

int64_t append_threads(int64_t n_tokens, Cached cached)
{
    return (cached == Cached::kBlocks8 ? (n_tokens + 2 * kPage - 2) / kPage : n_tokens) * kAppendThreads;
}

hipError_t launch_append(const owl_verify_desc &d, const owl_append_desc &a, const owl_norm_desc *norm, Cached cached, const void *q,
                         const void *k_new, const void *v_new, const float *q_gain, const float *k_gain, const float *inv_freq,
                         const int32_t *pos_ids, void *q_out, void *k_cache, void *v_cache,
                         uint8_t *k_scale, uint8_t *v_scale, const int32_t *page_table, const int32_t *ctx_lens,
                         const int32_t *n_new_seq, uint32_t *status, hipStream_t s)
{
    const int64_t es = d.qkv_dtype == OWL_F32 ? 4 : 2, cb = cached == Cached::kOwnType ? es : 1;
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
    p.eps = norm ? norm->eps : 0.f;
    p.q_gain = q_gain;
    p.k_gain = k_gain;
    const bool pairs = a.rot_style == OWL_ROT_PAIRS, normed = norm != nullptr;
    const bool wide = d.head_dim == 128;
    switch (d.qkv_dtype) {
    case OWL_BF16: return wide ? launch_append_as<__bf16, 128>(p, d.batch, pairs, normed, cached, s) : launch_append_as<__bf16, 64>(p, d.batch, pairs, normed, cached, s);
    case OWL_F16: return wide ? launch_append_as<_Float16, 128>(p, d.batch, pairs, normed, cached, s) : launch_append_as<_Float16, 64>(p, d.batch, pairs, normed, cached, s);
    default: return wide ? launch_append_as<float, 128>(p, d.batch, pairs, normed, cached, s) : launch_append_as<float, 64>(p, d.batch, pairs, normed, cached, s);
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
