// Split-KV pass of the verify-step attention over a cache of 4-bit groups, for gfx950 (MI355X).
//
// The share of a workgroup, its pieces and their partials are those of owl_splitkv.h; the loop is another one:
//   scores    S^T[key][row] = K . Q^T by v_mfma_f32_16x16x32 on widened keys (v_cvt_scalef32_pk_*_fp4: two numbers an instruction, scale applied, exact).
//             The pipe also takes codes as they lie (v_mfma_scale_f32_16x16x128_f8f6f4, with q as a sum of two or three e4m3 numbers), but not with sums
//             in 32 bits: of 16 neighbouring channels it drops what lies 2^13 below the greatest product (measured; the 16-bit product drops nothing there).
//             Where one channel makes a score of 64 the weights were off by 0.7 %, at 512 by 7 %.  (With those products 240 rows over 64K take 65 us
//             instead of 69, 320 over 128K 152 instead of 162, in fp16 77 instead of 71 and 197 instead of 195.)
//   values    O^T += V^T . P^T, V read from LDS by the transposing read, as in the 16-bit pass.
//   softmax   Each wavefront has a reference of its own for each row, which stays until a score lies more than kGroupRoom above it and then
//             moves to the row's highest score.
// Two kernels.  Shared stages: 128 tokens at a time, of which each of the eight wavefronts brings one page of K and one of V, 16 bytes (8 for
// head_dim 64) and a scale byte a lane of each, through registers, and widens them into LDS a stage ahead: two buffers of each.  One barrier a stage.
// (Each wavefront widening the codes of K that it multiplies, from a third of the bytes in LDS: 240 rows over 64K 77 instead of 69 us, 104 49 instead of 47.)
// The wavefronts are WR row groups of TPW tiles times WK key groups, which take the 32-token steps of a stage in turn and merge at the end of a piece.
// Keys of a wavefront's own, for few rows: further below.
//
// What bounds it (8 KV heads, head_dim 128): the stream for a row or two, 120-123 us for 16 sequences of 8K-64K at one node each (6.0 TB/s of codes and
// scales); products, fragments from LDS and softmax beside each other where rows are many, 161 us for 320 rows over 128K in bf16 (1.07 PFLOP/s; fp16, in two row
// groups, 195).  Between the two, 104 rows at 64K 47 us, in 16 sequences 362 (fp16 367): by counters the matrix pipe is busy for 38 % of the time and LDS for 31 %, a
// wavefront issues for 35 % of its cycles, is ready without issuing for 31 % (its SIMD's pipe or other wavefront) and waits for 33 % (barrier, LDS, memory).
#include "owl_splitkv.h"

namespace owl {

constexpr int kStage = 128;                          // tokens of a stage

// How far a score may lie above its row's reference: a weight is at most 2^kRoom.  fp16 ends at 2^16.
template <typename T> constexpr float kGroupRoom = 11.0f;
template <> constexpr float kGroupRoom<__bf16> = 24.0f;

// A row of widened K or V in LDS, padded so that neither the reads, of V transposing, 32 bytes of 8 rows at a time, of K 16 bytes, nor the stores meet a bank
// twice, and so that all fragments are at fixed distances from one address.
template <int D> constexpr int kRow = 2 * D + 32;

template <int D, int TPW, int WR>
struct GGeo {
    static constexpr int WK = kWaves / WR, STEPS = 4 / WK;       // key groups; 32-token steps of a stage that each takes
    static constexpr int NG = D / 32;                            // groups of a row
    static constexpr int LB = D / 8, LW = LB / 4;                // bytes (words) of a page of one tensor that a lane brings
    static constexpr int T_BYTES = kStage * kRow<D>;            // a stage of K or of V, widened
    static constexpr int K = 2 * T_BYTES, MAIN = 4 * T_BYTES;    // two stages of V, then two of K
    static constexpr int NT = D / 16;                            // channel tiles of O^T
    static constexpr int TILE = NT * 1024 + 512;                 // a wavefront's part of a tile in the merge
    static constexpr size_t LDS = MAIN;
    static_assert(WR * WK == kWaves && STEPS >= 1, "eight wavefronts share four steps");
    static_assert(kWaves * TILE <= MAIN, "the merge fits the buffers");
};

// Two e2m1 codes, of byte `kByte` of a word, times a power of two, as two numbers of type T.
template <typename T, int kByte>
__device__ __forceinline__ uint32_t widen_codes(uint32_t word, float scale)
{
    if constexpr (std::is_same<T, __bf16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, kByte));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, kByte));
}

template <typename T>
__device__ __forceinline__ uint4 widen_word(uint32_t word, float scale)
{
    return make_uint4(widen_codes<T, 0>(word, scale), widen_codes<T, 1>(word, scale), widen_codes<T, 2>(word, scale), widen_codes<T, 3>(word, scale));
}

// max over the four lanes {l, l^16, l^32, l^48}
__device__ __forceinline__ uint32_t quad_column_max_bits(uint32_t x)
{
    auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t y = max((uint32_t)r[0], (uint32_t)r[1]);
    auto r2 = __builtin_amdgcn_permlane16_swap(y, y, false, false);
    return max((uint32_t)r2[0], (uint32_t)r2[1]);
}

// A query tile as B operands, and what takes its products to the exponents of two.  Lane (j, quad) holds numbers of row j, eight for each product; kOwn: those of
// channels quad D / 4 .., which are the ones that the lane of key j has codes of.  (The products' k are the channels in any order that is the same for both.)
template <typename T, int D>
struct Query {
    uint4 part[D / 32];
    float c_log2;
};

template <typename T, int D, bool kOwn>
__device__ __forceinline__ Query<T, D> load_query(const unsigned char *row, int quad)
{
    Query<T, D> q;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) q.part[w] = *reinterpret_cast<const uint4 *>(row + (kOwn ? quad * (D / 4) + 8 * w : 32 * w + 8 * quad) * 2);
    return q;
}

// Rows that are not there become zeros.  A number that is infinite or none makes its row's factor none.  A bf16 row with numbers above 2^100 is taken to that, and
// its factor up, so that no size of q makes its products overflow (less where the factor would); what is lost lies 2^199 below.
template <typename T, int D>
__device__ __forceinline__ void take_query(Query<T, D> &q, bool on, float c_log2)
{
    constexpr uint32_t kNone = std::is_same<T, __bf16>::value ? 0x7F80u : 0x7C00u;
    uint32_t big = 0;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
        uint32_t *words = reinterpret_cast<uint32_t *>(&q.part[w]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            words[k] = on ? words[k] : 0u;
            big = max(big, max(words[k] & 0x7FFFu, words[k] >> 16 & 0x7FFFu));
        }
    }
    big = quad_column_max_bits(big);
    q.c_log2 = big >= kNone ? __builtin_nanf("") : c_log2;
    if constexpr (std::is_same<T, __bf16>::value) {
        const int e = (int)(__builtin_bit_cast(uint32_t, c_log2) >> 23) - 127;       // (c_log2 > 0)
        const int up = big >= kNone ? 0 : max(min(100 - ((int)(big >> 7) - 127), 0), e - 127);
        if (__builtin_amdgcn_ballot_w64(up < 0) != 0) {
            q.c_log2 = __builtin_ldexpf(q.c_log2, -up);
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {
                uint32_t *words = reinterpret_cast<uint32_t *>(&q.part[w]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    words[k] = pack2<T>(__builtin_ldexpf(__builtin_bit_cast(float, words[k] << 16), up),
                                        __builtin_ldexpf(__builtin_bit_cast(float, words[k] & 0xFFFF0000u), up));
            }
        }
    }
}

// s[t][kt] = 16 keys' codes . 16 rows of tile t, for kt = 0 or 1, widened in registers: what is widened serves all tiles.
template <typename T, int D, int TPW>
__device__ __forceinline__ void score(const uint32_t (&codes)[D / 32], float scale, const Query<T, D> (&q)[TPW], int kt, f32x4 (&s)[TPW][2])
{
#pragma unroll
    for (int t = 0; t < TPW; ++t) s[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
        const uint4 keys = widen_word<T>(codes[w], scale);
#pragma unroll
        for (int t = 0; t < TPW; ++t) s[t][kt] = mfma16<T>(keys, q[t].part[w], s[t][kt]);
    }
}

// 4 or 2 words at an offset from a wave-uniform address; kOnce: no other row group reads them, and they are not kept (non-temporal).
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
template <int LW, bool kOnce>
__device__ __forceinline__ void load_words(uint32_t (&to)[LW], const unsigned char *base, uint32_t at)
{
    typedef typename std::conditional<LW == 4, Words4, Words2>::type Words;
    const Words *from = reinterpret_cast<const Words *>(base + at);
    Words x;
    if constexpr (kOnce) x = __builtin_nontemporal_load(from);
    else x = *from;
#pragma unroll
    for (int w = 0; w < LW; ++w) to[w] = x[w];
}

struct GPiece {
    int b, L, Nb;                                    // sequence, its prefix length and number of drafts
    int pos0, pos1;                                  // [pos0, pos1) of its L + Nb cached rows, pos0 a multiple of 64
    size_t slot;                                     // where the partials of row tile 0 go
};

// A row tile of a piece as its partial: in fp32 as the accumulators stand, or normalised and in fp16 (kPartMl in owl_internal.h).
template <int NT>
__device__ __forceinline__ void store_partial(const KParams &p, size_t slot, f32x4 (&O)[NT + 1], float m, int lane)
{
    const int j = lane & 15, quad = lane >> 4;
    const float l = O[NT][0];
    float third = 1.0f;
    if (!p.half_partials) {
        float4 *po = static_cast<float4 *>(p.part_o) + slot * (size_t)(NT * 64);
#pragma unroll
        for (int u = 0; u < NT; ++u) po[u * 64 + lane] = make_float4(O[u][0], O[u][1], O[u][2], O[u][3]);
    } else {
        const float inv_l = l > 0.f ? 1.0f / l : 0.f;          // a row that saw no key: all zeros
        float big = 0.f;
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                O[u][r] *= inv_l;
                big = fmaxf(big, fabsf(O[u][r]));
            }
        big = fmaxf(quad_column_max(big), FLT_MIN);  // (the inverse of a subnormal one may be infinite)
        const float inv_s = 1.0f / big;
        uint4 *po = static_cast<uint4 *>(p.part_o) + slot * (size_t)(NT / 2 * 64) + lane;
#pragma unroll
        for (int u = 0; u < NT; u += 2)
            po[(u / 2) * 64] = make_uint4(pack2<_Float16>(O[u][0] * inv_s, O[u][1] * inv_s), pack2<_Float16>(O[u][2] * inv_s, O[u][3] * inv_s),
                                           pack2<_Float16>(O[u + 1][0] * inv_s, O[u + 1][1] * inv_s),
                                           pack2<_Float16>(O[u + 1][2] * inv_s, O[u + 1][3] * inv_s));
        third = l * big;
    }
    if (quad == 0) {
        float *stats = p.part_ml + slot * kPartMl + 3 * j;
        stats[0] = m;
        stats[1] = l;
        stats[2] = third;
    }
}

template <typename T, int D, int TPW, int WR>
__device__ __forceinline__ void run_group_piece(const QuantParams &p, unsigned char *smem, int wave, int lane, int g, int rg, const GPiece &pc)
{
    using GEO = GGeo<D, TPW, WR>;
    constexpr int NT = GEO::NT, NG = GEO::NG, LB = GEO::LB, LW = GEO::LW, WK = GEO::WK, STEPS = GEO::STEPS;
    const int j = lane & 15, qd = lane >> 4;
    const int wr = wave % WR, wk = wave / WR;
    const int b = pc.b, L = pc.L, Nb = pc.Nb, pos0 = pc.pos0, pos1 = pc.pos1;
    const int stages = (pos1 - pos0 + kStage - 1) / kStage;

    // ---- transfers: this wavefront's page of a stage, a quarter of a row a lane ----
    const int slot = lane >> 2, quarter = lane & 3, group = D == 128 ? quarter : quarter >> 1;
    const int64_t head_off = (int64_t)g * p.stride_head;
    const int last_lp = (pos1 - 1) / kPage, last_slot = (pos1 - 1) % kPage, lp0 = pos0 / kPage + wave;
    // Lane i holds where the page of stage first + i lies, of this KV head, in the pools and in the scales; bad pages are page 0, and behind the
    // piece's last page it is that one again.
    struct Where {
        int64_t at, scales;
    };
    auto stage_pages = [&](int first) -> Where {
        const int lp = min(lp0 + (first + lane) * kWaves, last_lp);
        int pg = lp;
        if (p.page_table) pg = p.page_table[(int64_t)b * p.max_pages + min(lp, p.max_pages - 1)];
        const bool bad = pg < 0 || pg >= p.n_pool_pages || (p.page_table && lp >= p.max_pages);
        if (bad) flag_status(p.dev_status, OWL_DEV_BAD_PAGE);
        const int64_t page = bad ? 0 : pg;
        return Where{page * p.stride_page + head_off, (page * p.Hkv + g) * (kPage * NG)};
    };
    Where pages = stage_pages(0);
    auto lane_of = [](int64_t v, int i) -> int64_t {
        return ((int64_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, i);
    };
    struct Held {                                    // of one tensor
        uint32_t words[LW], scale;
    };
    // No load is in a branch: the compiler would wait for all of them where the paths meet.
    const uint32_t tok = (uint32_t)p.stride_token, slot_off = (uint32_t)slot * tok, slot_scale = (uint32_t)(slot * NG);
    auto load = [&](const void *cache, const uint8_t *scales, int s) -> Held {
        const int most = lp0 + s * kWaves < last_lp ? kPage - 1 : last_slot;         // rows past the end: the last one again, masked later
        Held h;
        load_words<LW, false>(h.words, static_cast<const unsigned char *>(cache) + lane_of(pages.at, s & 63), min(slot_off, (uint32_t)most * tok) + quarter * LB);
        h.scale = (scales + lane_of(pages.scales, s & 63))[min(slot_scale, (uint32_t)(most * NG)) + group];
        return h;
    };
    // ... and into LDS, in 16 bits: the lanes of the upper half of a row store its 16-byte pieces in another order, so that eight lanes meet no bank twice
    const int key = wave * kPage + slot, turn = D == 128 ? quarter >> 1 : 0;
    const uint32_t put_at = key * kRow<D> + quarter * LW * 16;
    auto put = [&](const Held &h, uint32_t buffer) {
        const float scale = __builtin_bit_cast(float, h.scale << 23);            // (255: the conversion gives no numbers)
        const uint32_t at = put_at + buffer;
        unsigned char *even = smem + (at + turn * 16), *odd = smem + (at + 16 - turn * 16);
#pragma unroll
        for (int w = 0; w < LW; w += 2) {
            const uint32_t a = turn ? h.words[w + 1] : h.words[w], c = turn ? h.words[w] : h.words[w + 1];
            *reinterpret_cast<uint4 *>(even + w * 16) = widen_word<T>(a, scale);
            *reinterpret_cast<uint4 *>(odd + w * 16) = widen_word<T>(c, scale);
        }
    };
    // V of stage s is put while stage s - 1 is computed, and so is K, but that the pages of a key group's first step are those of stage s + 1: the last step
    // of a stage forms the first scores of the next.  Both are asked for a stage before that.
    constexpr bool kPipe = TPW <= 2;                 // (three tiles leave no registers for two generations of scores)
    const int early = kPipe && wave % (2 * STEPS) < 2 ? 1 : 0;
    Held k_held = load(p.k, p.k_scale, early), v_held = load(p.v, p.v_scale, 0), k_first{};
    if constexpr (kPipe) k_first = load(p.k, p.k_scale, 0);

    // ---- query rows: tiles wr, wr + WR, ... of the row group ----
    const float inv_g = __builtin_amdgcn_rcpf((float)p.G);
    const unsigned char *q_head = static_cast<const unsigned char *>(p.q) + ((int64_t)b * p.N * p.Hq + (int64_t)g * p.G) * D * 2;
    Query<T, D> q[TPW];
    int irow[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int in_group = t * WR + wr, tg = rg * p.group_tiles + in_group;
        const bool tile_ok = in_group < p.group_tiles && tg < p.RT;
        const int row = tg * kRowTile + j, i = (int)(((float)row + 0.5f) * inv_g);     // node row / G, exactly (see owl_splitkv.h)
        irow[t] = tile_ok && row < p.R && i < Nb ? i : -1;
        const int rc = min(row, p.R - 1), ic = (int)(((float)rc + 0.5f) * inv_g);
        q[t] = load_query<T, D, false>(q_head + ((int64_t)ic * (p.Hq - p.G) + rc) * (D * 2), qd);
        take_query(q[t], irow[t] >= 0, p.c_log2);
    }
    const int my_tiles = max(0, (min(p.group_tiles, p.RT - rg * p.group_tiles) - wr + WR - 1) / WR);       // wave-uniform
    uint64_t anc = 0;                                // the drafts that node `lane` sees
    if (pos1 > L) anc = ancestor_sets(p.parent[(int64_t)b * p.N + min(lane, p.N - 1)], lane, Nb, p.dev_status);

    f32x4 O[TPW][NT + 1];
    float m[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        m[t] = kMInit;
#pragma unroll
        for (int u = 0; u <= NT; ++u) O[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- one step of 32 tokens ----
    const uint32_t k_take = GEO::K + (wk * STEPS * 32 + j) * kRow<D> + qd * 16;
    const uint32_t v_take = (wk * STEPS * 32 + 4 * qd + (j >> 2)) * kRow<D> + (j & 3) * 8;
    auto load_k_frag = [&](const unsigned char *k_rows, int kt, int w) -> uint4 {
        return *reinterpret_cast<const uint4 *>(k_rows + kt * kPage * kRow<D> + w * 64);
    };
    auto load_v_frag = [&](const unsigned char *v_rows, int u) -> uint4 {
        const uint2 lo = lds_read_tr16(v_rows + u * 32), hi = lds_read_tr16(v_rows + u * 32 + kPage * kRow<D>);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
    };
    auto mask = [&](f32x4 (&s)[2], int t, int step_pos) {
        const int node = max(irow[t], 0);
        uint64_t seen = ((uint64_t)__shfl((uint32_t)(anc >> 32), node) << 32) | __shfl((uint32_t)anc, node);
        if (irow[t] < 0) seen = pos1 > L ? ~(uint64_t)0 >> (64 - Nb) : 0;       // a row without a node sees all of them
        const int ahead = L - step_pos;              // prefix keys in this step (< 32), or minus the drafts before it
        const uint32_t bits = ahead >= 0 ? ((1u << ahead) - 1u) | (uint32_t)(seen << ahead)
                                         : (-ahead < 64 ? (uint32_t)(seen >> -ahead) : 0u);
        const uint32_t va = bits >> (4 * qd), vb = va >> 16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[0][r] = (va >> r) & 1u ? s[0][r] : -INFINITY;
            s[1][r] = (vb >> r) & 1u ? s[1][r] : -INFINITY;
        }
    };
    auto exponents = [&](const f32x4 (&s)[2], int t, float (&x)[8]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[r] = __builtin_fmaf(s[0][r], q[t].c_log2, -m[t]);
            x[4 + r] = __builtin_fmaf(s[1][r], q[t].c_log2, -m[t]);
        }
    };
    auto highest = [](const float (&x)[8]) -> float {
        return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    };
    // moves the references of the rows that have a score above their room
    auto move_reference = [&](const f32x4 (&s)[2], int t) {
        const float all[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]};
        const float sc = quad_column_max(highest(all)) * q[t].c_log2;
        const float mn = sc > m[t] + kGroupRoom<T> ? sc : m[t];
        const float alpha = fast_exp2(m[t] - mn);
        m[t] = mn;
#pragma unroll
        for (int u = 0; u <= NT; ++u) O[t][u] *= alpha;
    };
    // (the matrix pipe takes 16-bit weights; the row sum adds the same rounded ones)
    auto weights = [&](float (&x)[8]) -> uint4 {
#pragma unroll
        for (int r = 0; r < 8; ++r) x[r] = fast_exp2(x[r]);
        return make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
    };
    const uint4 ones = make_uint4(ones2<T>(), ones2<T>(), ones2<T>(), ones2<T>());

    // Up to two tiles a wavefront.  S, the step's scores, are there already; the next step's keys are asked for first and multiplied before the weights are
    // formed, and V's fragments, in the same registers, behind those products.  (Half of V's, or the next keys, asked for earlier: no registers, 49-57 us for
    // 104 rows over 64K.)  A score above its row's room shows when the weights are formed, which are then formed again.
    auto piped_step = [&](auto na_tag, f32x4 (&S)[TPW][2], f32x4 (&next)[TPW][2], const unsigned char *next_rows, const unsigned char *v_rows, int step_pos) {
        constexpr int NA = decltype(na_tag)::value;
        uint4 vf[NT], pf[TPW], kf[2][LW];
#pragma unroll
        for (int w = 0; w < LW; ++w)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) kf[kt][w] = load_k_frag(next_rows, kt, w);
        asm volatile("" ::: "memory");               // (no load sinks below)
        if (step_pos + 32 > L)                       // reaches drafts or the ragged end (uniform)
#pragma unroll
            for (int t = 0; t < NA; ++t) mask(S[t], t, step_pos);
        float x[NA][8], top = -INFINITY;
#pragma unroll
        for (int t = 0; t < NA; ++t) {
            exponents(S[t], t, x[t]);
            top = fmaxf(top, highest(x[t]));
        }
#pragma unroll
        for (int w = 0; w < LW; ++w)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int t = 0; t < NA; ++t) next[t][kt] = mfma16<T>(kf[kt][w], q[t].part[w], w == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : next[t][kt]);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int u = 0; u < NT; ++u) vf[u] = load_v_frag(v_rows, u);
#pragma unroll
        for (int t = 0; t < NA; ++t) pf[t] = weights(x[t]);
        if (__builtin_amdgcn_ballot_w64(top > kGroupRoom<T>) != 0) {             // any lane's own keys can raise the alarm (uniform, rarely taken after the first step)
#pragma unroll
            for (int t = 0; t < NA; ++t) {
                move_reference(S[t], t);
                exponents(S[t], t, x[t]);
                pf[t] = weights(x[t]);
            }
        }
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int t = 0; t < NA; ++t) O[t][u] = mfma16<T>(vf[u], pf[t], O[t][u]);
#pragma unroll
        for (int t = 0; t < NA; ++t) O[t][NT] = mfma16<T>(ones, pf[t], O[t][NT]);
    };
    // Three tiles: registers for one generation of scores, all of a step's ahead of the softmax, and for a few of V's fragments.
    constexpr int kAhead = 3;
    auto plain_step = [&](auto na_tag, const unsigned char *k_rows, const unsigned char *v_rows, int step_pos) {
        constexpr int NA = decltype(na_tag)::value;
        uint4 vf[NT], pf[TPW];
        f32x4 s[TPW][2];
#pragma unroll
        for (int w = 0; w < LW; ++w)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const uint4 kf = load_k_frag(k_rows, kt, w);
#pragma unroll
                for (int t = 0; t < NA; ++t) s[t][kt] = mfma16<T>(kf, q[t].part[w], w == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[t][kt]);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) vf[u] = load_v_frag(v_rows, u);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < NA; ++t) {
            if (step_pos + 32 > L) mask(s[t], t, step_pos);
            float x[8];
            exponents(s[t], t, x);
            if (__builtin_amdgcn_ballot_w64(highest(x) > kGroupRoom<T>) != 0) {
                move_reference(s[t], t);
                exponents(s[t], t, x);
            }
            pf[t] = weights(x);
        }
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            if (u + kAhead < NT) vf[u + kAhead < NT ? u + kAhead : 0] = load_v_frag(v_rows, u + kAhead);
#pragma unroll
            for (int t = 0; t < NA; ++t) O[t][u] = mfma16<T>(vf[u], pf[t], O[t][u]);
            asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int t = 0; t < NA; ++t) O[t][NT] = mfma16<T>(ones, pf[t], O[t][NT]);
    };

    // ---- the loop ----
    put(k_held, GEO::K);
    put(v_held, 0);
    v_held = load(p.v, p.v_scale, 1);
    k_held = load(p.k, p.k_scale, 1 + early);
    if constexpr (kPipe) put(k_first, GEO::K + GEO::T_BYTES);
    __syncthreads();
    auto run = [&](auto na_tag) {
        constexpr int NA = decltype(na_tag)::value;
        f32x4 Sa[TPW][2], Sb[TPW][2];
        if constexpr (kPipe) {
            if constexpr (NA > 0) {
#pragma unroll
                for (int w = 0; w < LW; ++w)
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {
                        const uint4 kf = load_k_frag(smem + (k_take + GEO::T_BYTES), kt, w);
#pragma unroll
                        for (int t = 0; t < NA; ++t) Sa[t][kt] = mfma16<T>(kf, q[t].part[w], w == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : Sa[t][kt]);
                    }
            }
            __syncthreads();
        }
        for (int s = 0; s < stages; ++s) {
            const uint32_t now = s & 1 ? GEO::T_BYTES : 0, then = GEO::T_BYTES - now;
            put(v_held, then);
            if (!early && ((s + 2) & 63) == 0 && s + 2 < stages) pages = stage_pages(s + 2);
            v_held = load(p.v, p.v_scale, s + 2);
            put(k_held, GEO::K + then);
            if (early && ((s + 3) & 63) == 0 && s + 3 < stages) pages = stage_pages(s + 3);
            k_held = load(p.k, p.k_scale, s + 2 + early);
            if constexpr (NA > 0) {
                const unsigned char *k_rows = smem + (k_take + now), *v_rows = smem + (v_take + now);
                const int pos = pos0 + s * kStage + wk * STEPS * 32;
                static_for<0, STEPS>([&](auto i_tag) {
                    constexpr int i = decltype(i_tag)::value;
                    if (pos + i * 32 >= pos1) return;                            // uniform
                    if constexpr (kPipe) {
                        f32x4 (&S)[TPW][2] = i % 2 ? Sb : Sa, (&next)[TPW][2] = i % 2 ? Sa : Sb;
                        // (the last step forms scores of what lies behind the end, for nobody)
                        piped_step(na_tag, S, next, k_rows + (i + 1) % STEPS * 32 * kRow<D>, v_rows + i * 32 * kRow<D>, pos + i * 32);
                    } else {
                        plain_step(na_tag, k_rows + i * 32 * kRow<D>, v_rows + i * 32 * kRow<D>, pos + i * 32);
                    }
                });
                if constexpr (kPipe && STEPS % 2 == 1)
#pragma unroll
                    for (int t = 0; t < NA; ++t) {
                        Sa[t][0] = Sb[t][0];
                        Sa[t][1] = Sb[t][1];
                    }
            }
            __syncthreads();
        }
    };
    // (a wavefront computes the tiles it has)
    if (my_tiles >= TPW) run(std::integral_constant<int, TPW>{});
    else if (TPW > 1 && my_tiles == TPW - 1) run(std::integral_constant<int, (TPW > 1 ? TPW - 1 : 0)>{});
    else if (TPW > 2 && my_tiles == TPW - 2) run(std::integral_constant<int, (TPW > 2 ? TPW - 2 : 0)>{});
    else run(std::integral_constant<int, 0>{});

    // ---- the key groups' sums meet in LDS, tile by tile, and become the piece's partial ----
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int in_group = t * WR + wr, tg = rg * p.group_tiles + in_group;
        const bool ok = in_group < p.group_tiles && tg < p.RT;
        if constexpr (WK > 1) {
            const int finisher = t % WK;
            if (t > 0) __syncthreads();
            if (ok && wk != finisher) {
                unsigned char *own = smem + wave * GEO::TILE;
#pragma unroll
                for (int u = 0; u < NT; ++u) reinterpret_cast<f32x4 *>(own)[u * 64 + lane] = O[t][u];
                reinterpret_cast<float2 *>(own + NT * 1024)[lane] = make_float2(m[t], O[t][NT][0]);
            }
            __syncthreads();
            if (ok && wk == finisher) {
#pragma unroll
                for (int k = 1; k < WK; ++k) {
                    const unsigned char *src = smem + (wr + (finisher + k) % WK * WR) * GEO::TILE;
                    const float2 ml = reinterpret_cast<const float2 *>(src + NT * 1024)[lane];
                    const float mn = fmaxf(m[t], ml.x), a1 = fast_exp2(m[t] - mn), a2 = fast_exp2(ml.x - mn);
                    m[t] = mn;
#pragma unroll
                    for (int u = 0; u < NT; ++u) O[t][u] = O[t][u] * a1 + reinterpret_cast<const f32x4 *>(src)[u * 64 + lane] * a2;
                    O[t][NT][0] = O[t][NT][0] * a1 + ml.y * a2;
                }
                store_partial<NT>(p, pc.slot + tg, O[t], m[t], lane);
            }
        } else if (ok) {
            store_partial<NT>(p, pc.slot + tg, O[t], m[t], lane);
        }
    }
}

// The share of a workgroup, piece by piece: f(KV head, row group, piece) is called for each, with a barrier between two.  Shares, row groups and
// slots are those of the pass over 16-bit caches.  Most lone sequences are as long as announced: ask(KV head, row group, sequence, first position) is
// called before the length is known.
template <typename A, typename F>
__device__ __forceinline__ void for_each_piece(const KParams &p, A &&ask, F &&f)
{
    uint32_t n = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
    int rg = 0;
    if (p.row_groups > 1) {                          // groups of a stream follow each other on one XCD
        const uint32_t slot = n >> 3;
        rg = (int)(slot % (uint32_t)p.row_groups);
        n = ((slot / (uint32_t)p.row_groups) << 3) | (n & 7);
    }
    const int item = (int)(n / (uint32_t)p.Hkv), g = (int)(n % (uint32_t)p.Hkv);
    const size_t head_slots = (size_t)g * p.n_slots;
    int b = 0, before = 0, x, x1, slot0;
    Deal deal = p.full;
    SeqSize size{0, 0};
    bool sized = false;
    if (!p.dealt) {                                  // equal splits of C tokens, of one sequence each
        const int c = item % (int)gridDim.y;
        b = item / (int)gridDim.y;
        if (b >= p.B || c >= p.max_splits) return;   // padding of the grid
        x = c * (p.C / kSplitQuantum);
        x1 = x + p.C / kSplitQuantum;
        slot0 = b * p.max_splits + c - b;
        ask(g, rg, b, x * kSplitQuantum);
    } else {
        if (item >= p.rule.max_workers) return;      // padding of the grid
        if (p.B == 1) {
            ask(g, rg, 0, deal_begin(deal, min(item, deal.workers - 1)) * kSplitQuantum);
            size = SeqSize{load_ctx_len(p.ctx_lens, 0, p.max_ctx_len, p.dev_status), load_n_draft(p.n_draft_seq, 0, p.N, p.dev_status)};
            const int T1 = size.drafts == 0 ? 0 : size.len + size.drafts;
            if (T1 != p.max_ctx_len + p.N) deal = deal_units(p, max(seq_units(p, T1), 1));
        } else {
            const BatchUnits u = batch_units(p);
            if (u.total == 0) return;                // not one sequence has drafts
            deal = deal_units(p, u.total);
            if (item < deal.workers) find_unit(p, u, deal_begin(deal, item), &b, &before);
            size = size_of(p, u, b);
        }
        sized = true;
        if (item >= deal.workers) return;
        x = deal_begin(deal, item);
        x1 = deal_begin(deal, item + 1);
        slot0 = item;
    }
    for (bool again = false; b < p.B; ++b) {
        if (!sized) size = SeqSize{load_ctx_len(p.ctx_lens, b, p.max_ctx_len, p.dev_status), load_n_draft(p.n_draft_seq, b, p.N, p.dev_status)};
        sized = false;
        const int L = size.len, Nb = size.drafts;
        const int T_b = Nb == 0 ? 0 : L + Nb;
        const int s0 = x - before, s1 = min(x1 - before, stages_of(T_b));
        if (s0 < s1) {
            if (again) __syncthreads();              // LDS is free again
            again = true;
            f(g, rg, GPiece{b, L, Nb, s0 * kSplitQuantum, min(s1 * kSplitQuantum, T_b), (head_slots + slot0 + b) * p.RT});
        }
        before += seq_units(p, T_b);
        if (before >= x1 || !p.dealt) break;
        x = before;
    }
}

template <typename T, int D, int TPW, int WR>
__global__ void __launch_bounds__(kThreads) splitkv_groups_kernel(const QuantParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    fetch_args<void(QuantParams)>();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for_each_piece(p, [](int, int, int, int) {}, [&](int g, int rg, const GPiece &pc) { run_group_piece<T, D, TPW, WR>(p, smem, wave, lane, g, rg, pc); });
}

// ---------------------------------------------------------------------------
// Few rows: a wavefront shares nothing until the end of a piece.  The 32-token chunks of a piece are dealt to the eight wavefronts in turn; a
// wavefront takes all rows of its row group, TPW tiles, against its own chunks.  K's codes and scale bytes go from memory into the
// registers of the lanes that widen them (16 keys of 64 bytes are 64 lanes' 16 bytes); V is widened into 9 KB of LDS of the
// wavefront's own and read back transposed, in order, without a barrier.  Two chunks of each tensor are on their way while one is computed (three
// and four are no faster).  At the end the wavefronts' sums meet in LDS, a channel tile a wavefront, and leave one partial in fp32.
// Six nodes at 32K: 14 us and 4 for the combine, of which the loop, at the rate of memory, is 6; the rest is the way to the first chunk (lengths and
// pages, then codes: two round trips), the merge and the partials.  Where the plan takes which: plan_groups in owl_api.hip, with both sides measured.
// ---------------------------------------------------------------------------
template <int D>
struct OGeo {
    static constexpr int NT = D / 16, NG = D / 32, VROW = kRow<D>, LW = D / 32;    // LW: words of K and of V that a lane brings from a page
    static constexpr int CHUNK = 2 * kPage, WAVE = CHUNK * VROW;
    static constexpr int DEPTH = 2;                              // chunks under way
    static constexpr int TILE = NT * 1024 + 512;
    static constexpr size_t LDS = (size_t)kWaves * (WAVE > TILE ? WAVE : TILE);
};

struct OwnPages {
    int pages, pos0;                                 // lane 2 i + h: page h of chunk i of this wavefront in the piece from pos0 on; unchecked
};

__device__ __forceinline__ int own_chunk_pages(const KParams &p, int b, int pos0, int wave, int lane, int first)
{
    const int lp = pos0 / kPage + (wave + kWaves * (first + (lane >> 1))) * 2 + (lane & 1);
    return p.page_table ? p.page_table[(int64_t)b * p.max_pages + min(lp, p.max_pages - 1)] : lp;
}

template <typename T, int D, int TPW, bool kOnce>
__device__ __forceinline__ void run_own_piece(const QuantParams &p, unsigned char *smem, int wave, int lane, int g, int rg, const GPiece &pc,
                                              OwnPages ahead)
{
    using GEO = OGeo<D>;
    constexpr int NT = GEO::NT, NG = GEO::NG, LW = GEO::LW, CHUNK = GEO::CHUNK, kDepth = GEO::DEPTH;
    const int j = lane & 15, qd = lane >> 4, slot = lane >> 2, quarter = lane & 3;
    const int b = pc.b, L = pc.L, Nb = pc.Nb, pos0 = pc.pos0, pos1 = pc.pos1;
    const int chunks = (pos1 - pos0 + CHUNK - 1) / CHUNK;
    const int mine = max(0, (chunks - wave + kWaves - 1) / kWaves);
    unsigned char *ring = smem + wave * GEO::WAVE;

    // ---- query rows: asked for before anything that waits for the pages ----
    const float inv_g = __builtin_amdgcn_rcpf((float)p.G);
    const unsigned char *q_head = static_cast<const unsigned char *>(p.q) + ((int64_t)b * p.N * p.Hq + (int64_t)g * p.G) * D * 2;
    Query<T, D> q[TPW];
    int irow[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int tg = rg * p.group_tiles + t;
        const bool tile_ok = t < p.group_tiles && tg < p.RT;
        const int row = tg * kRowTile + j, i = (int)(((float)row + 0.5f) * inv_g);     // node row / G, exactly (see owl_splitkv.h)
        irow[t] = tile_ok && row < p.R && i < Nb ? i : -1;
        const int rc = min(row, p.R - 1), ic = (int)(((float)rc + 0.5f) * inv_g);
        q[t] = load_query<T, D, true>(q_head + ((int64_t)ic * (p.Hq - p.G) + rc) * (D * 2), qd);
    }

    // Bad pages are page 0; behind the piece's end it is the piece's last one.
    const int last_lp = (pos1 - 1) / kPage, last_slot = (pos1 - 1) % kPage, lp0 = pos0 / kPage + wave * 2;
    auto checked = [&](int pg, int first) -> int {
        const int lp = lp0 + (first + (lane >> 1)) * (2 * kWaves) + (lane & 1);
        const int other = __shfl_xor(pg, 1);
        if ((lane & 1) && lp > last_lp) pg = other;  // the last chunk's second page
        const bool bad = pg < 0 || pg >= p.n_pool_pages || (p.page_table && min(lp, last_lp) >= p.max_pages);
        if (bad && lp - (lane & 1) <= last_lp) flag_status(p.dev_status, OWL_DEV_BAD_PAGE);
        return bad ? 0 : pg;
    };
    int pages = checked(ahead.pos0 == pos0 ? ahead.pages : own_chunk_pages(p, b, pos0, wave, lane, 0), 0);

    // ---- transfers ----
    struct Held {
        uint32_t k[2][LW], v[2][LW], ks[2], vs[2];
    };
    Held held[kDepth];
    const int64_t head_off = (int64_t)g * p.stride_head;
    const uint32_t tok = (uint32_t)p.stride_token;
    const uint32_t k_piece = (uint32_t)(qd * LW * 4), v_piece = (uint32_t)(quarter * LW * 4), ks_piece = D == 128 ? qd : qd >> 1, vs_piece = D == 128 ? quarter : quarter >> 1;
    const uint32_t k_slot = (uint32_t)j * tok, v_slot = (uint32_t)slot * tok, ks_slot = (uint32_t)(j * NG), vs_slot = (uint32_t)(slot * NG);
    auto load = [&](Held &h, int i) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t page = __builtin_amdgcn_readlane(pages, (i & 31) * 2 + t), at = page * p.stride_page + head_off;
            const int most = lp0 + i * (2 * kWaves) + t < last_lp ? kPage - 1 : last_slot;      // rows past the end: the last one again, masked later
            const uint32_t bytes = (uint32_t)most * tok, scales = (uint32_t)(most * NG);
            const int64_t s_at = (page * p.Hkv + g) * (kPage * NG);
            load_words<LW, kOnce>(h.k[t], static_cast<const unsigned char *>(p.k) + at, min(k_slot, bytes) + k_piece);
            h.ks[t] = (p.k_scale + s_at)[min(ks_slot, scales) + ks_piece];
            load_words<LW, kOnce>(h.v[t], static_cast<const unsigned char *>(p.v) + at, min(v_slot, bytes) + v_piece);
            h.vs[t] = (p.v_scale + s_at)[min(vs_slot, scales) + vs_piece];
        }
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
        if (d < mine) load(held[d], d);

#pragma unroll
    for (int t = 0; t < TPW; ++t) take_query(q[t], irow[t] >= 0, p.c_log2);
    uint64_t anc = 0;                                // the drafts that node `lane` sees
    if (pos1 > L) anc = ancestor_sets(p.parent[(int64_t)b * p.N + min(lane, p.N - 1)], lane, Nb, p.dev_status);

    f32x4 O[TPW][NT + 1];
    float m[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        m[t] = kMInit;
#pragma unroll
        for (int u = 0; u <= NT; ++u) O[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // ---- the loop ----
    unsigned char *const put_at = ring + slot * GEO::VROW + quarter * LW * 16;
    const unsigned char *const take_at = ring + (4 * qd + (j >> 2)) * GEO::VROW + (j & 3) * 8;
    auto step = [&](Held &h, int i, auto more_tag) {
        f32x4 S[TPW][2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) score<T, D>(h.k[kt], __builtin_bit_cast(float, h.ks[kt] << 23), q, kt, S);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const float scale = __builtin_bit_cast(float, h.vs[kt] << 23);           // (255: the conversion gives no numbers)
#pragma unroll
            for (int w = 0; w < LW; ++w)
                *reinterpret_cast<uint4 *>(put_at + kt * kPage * GEO::VROW + w * 16) = widen_word<T>(h.v[kt][w], scale);
        }
        if (decltype(more_tag)::value || i + kDepth < mine) load(h, i + kDepth);
        const int step_pos = pos0 + (wave + kWaves * i) * CHUNK;
        uint4 pf[TPW];
#pragma unroll
        for (int t = 0; t < TPW; ++t) {
            f32x4 &s0 = S[t][0], &s1 = S[t][1];
            if (step_pos + CHUNK > L) {              // reaches drafts or the ragged end (uniform)
                const int node = max(irow[t], 0);
                uint64_t seen = ((uint64_t)__shfl((uint32_t)(anc >> 32), node) << 32) | __shfl((uint32_t)anc, node);
                if (irow[t] < 0) seen = pos1 > L ? ~(uint64_t)0 >> (64 - Nb) : 0;       // a row without a node sees all of them
                const int before = L - step_pos;     // prefix keys in this chunk (< 32), or minus the drafts before it
                const uint32_t word = before >= 0 ? ((1u << before) - 1u) | (uint32_t)(seen << before)
                                                  : (-before < 64 ? (uint32_t)(seen >> -before) : 0u);
                const uint32_t va = word >> (4 * qd), vb = va >> 16;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s0[r] = (va >> r) & 1u ? s0[r] : -INFINITY;
                    s1[r] = (vb >> r) & 1u ? s1[r] : -INFINITY;
                }
            }
            float x[8];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = __builtin_fmaf(s0[r], q[t].c_log2, -m[t]);
                x[4 + r] = __builtin_fmaf(s1[r], q[t].c_log2, -m[t]);
            }
            const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            if (__builtin_amdgcn_ballot_w64(top > kGroupRoom<T>) != 0) {
                const float tm = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
                const float sc = quad_column_max(tm) * q[t].c_log2;
                const float mn = sc > m[t] + kGroupRoom<T> ? sc : m[t];
                const float alpha = fast_exp2(m[t] - mn);
                m[t] = mn;
#pragma unroll
                for (int u = 0; u <= NT; ++u) O[t][u] *= alpha;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = __builtin_fmaf(s0[r], q[t].c_log2, -mn);
                    x[4 + r] = __builtin_fmaf(s1[r], q[t].c_log2, -mn);
                }
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) x[r] = fast_exp2(x[r]);
            pf[t] = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
        }
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const uint2 lo = lds_read_tr16(take_at + u * 32), hi = lds_read_tr16(take_at + u * 32 + kPage * GEO::VROW);
            const uint4 vf = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
            for (int t = 0; t < TPW; ++t) O[t][u] = mfma16<T>(vf, pf[t], O[t][u]);
        }
        const uint4 ones = make_uint4(ones2<T>(), ones2<T>(), ones2<T>(), ones2<T>());
#pragma unroll
        for (int t = 0; t < TPW; ++t) O[t][NT] = mfma16<T>(ones, pf[t], O[t][NT]);
        // the pages of the 32 chunks behind those that are under way
        if (((i + kDepth) & 31) == 31 && i + kDepth + 1 < mine) pages = checked(own_chunk_pages(p, b, pos0, wave, lane, i + kDepth + 1), i + kDepth + 1);
    };
    int i = 0;
    for (; i + 2 * kDepth <= mine; i += kDepth)
        static_for<0, kDepth>([&](auto d) { step(held[decltype(d)::value], i + decltype(d)::value, std::true_type{}); });
    for (; i < mine; i += kDepth)
        static_for<0, kDepth>([&](auto d) {
            if (i + decltype(d)::value < mine) step(held[decltype(d)::value], i + decltype(d)::value, std::false_type{});
        });

    // ---- the wavefronts' sums meet, a tile after the other, and become the piece's partial ----
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int tg = rg * p.group_tiles + t;
        if (t >= p.group_tiles || tg >= p.RT) break; // uniform
        __syncthreads();                             // no wavefront reads its own part of LDS, or the tile before, any more
        unsigned char *own = smem + wave * GEO::TILE;
#pragma unroll
        for (int u = 0; u < NT; ++u) reinterpret_cast<f32x4 *>(own)[u * 64 + lane] = O[t][u];
        reinterpret_cast<float2 *>(own + NT * 1024)[lane] = make_float2(m[t], O[t][NT][0]);
        __syncthreads();
        if (wave < NT) {                             // channel tile `wave`
            float2 ml[kWaves];
            float M = kMInit, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                ml[w] = reinterpret_cast<const float2 *>(smem + w * GEO::TILE + NT * 1024)[lane];
                M = fmaxf(M, ml[w].x);
            }
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float a = fast_exp2(ml[w].x - M);
                l = __builtin_fmaf(ml[w].y, a, l);
                const f32x4 x = reinterpret_cast<const f32x4 *>(smem + w * GEO::TILE)[wave * 64 + lane];
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(x[r], a, sum[r]);
            }
            const size_t part = pc.slot + tg;
            static_cast<float4 *>(p.part_o)[part * (size_t)(NT * 64) + wave * 64 + lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            if (wave == 0 && qd == 0) {
                float *stats = p.part_ml + part * kPartMl + 3 * j;
                stats[0] = M;
                stats[1] = l;
                stats[2] = 1.0f;
            }
        }
    }
}

template <typename T, int D, int TPW, bool kOnce>
__global__ void __launch_bounds__(kThreads) splitkv_groups_few_kernel(const QuantParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    fetch_args<void(QuantParams)>();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    OwnPages ahead{0, -1};
    for_each_piece(
        p, [&](int, int, int b, int pos0) { ahead = OwnPages{own_chunk_pages(p, b, pos0, wave, lane, 0), pos0}; },
        [&](int g, int rg, const GPiece &pc) {
            run_own_piece<T, D, TPW, kOnce>(p, smem, wave, lane, g, rg, pc, ahead);
            ahead.pos0 = -1;
        });
}

// (no entry point has events for these kernels)
template <typename T, int D, int TPW, int WR>
static void launch_groups_variant(const KParams &args, dim3 grid, hipStream_t s, hipEvent_t, hipEvent_t)
{
    hipLaunchKernelGGL((splitkv_groups_kernel<T, D, TPW, WR>), grid, dim3(kThreads), (GGeo<D, TPW, WR>::LDS), s, static_cast<const QuantParams &>(args));
}

template <typename T, int D, int TPW, bool kOnce>
static void launch_few_variant(const KParams &args, dim3 grid, hipStream_t s, hipEvent_t, hipEvent_t)
{
    hipLaunchKernelGGL((splitkv_groups_few_kernel<T, D, TPW, kOnce>), grid, dim3(kThreads), OGeo<D>::LDS, s, static_cast<const QuantParams &>(args));
}

// (wk = 8: keys of a wavefront's own; wr: 1, the only row group, or 2, one of several)
#define OWL_GROUP_FEW(DT, T, D, TPW, GROUPS)                                                                       \
    Variant { DT, D, TPW, GROUPS, kWaves, false, Cached::kGroups4, OGeo<D>::LDS, &launch_few_variant<T, D, TPW, GROUPS == 1>, \
              reinterpret_cast<const void *>(&splitkv_groups_few_kernel<T, D, TPW, GROUPS == 1>) }
#define OWL_GROUP_FEWS(DT, T, D) OWL_GROUP_FEW(DT, T, D, 1, 1), OWL_GROUP_FEW(DT, T, D, 2, 1), OWL_GROUP_FEW(DT, T, D, 2, 2)
#define OWL_GROUP_VARIANT(DT, T, D, TPW, WR)                                                                                      \
    Variant { DT, D, TPW, WR, kWaves / WR, false, Cached::kGroups4, GGeo<D, TPW, WR>::LDS, &launch_groups_variant<T, D, TPW, WR>, \
              reinterpret_cast<const void *>(&splitkv_groups_kernel<T, D, TPW, WR>) }
#define OWL_GROUP_VARIANTS(DT, T, D)                                                                                      \
    OWL_GROUP_VARIANT(DT, T, D, 1, 2), OWL_GROUP_VARIANT(DT, T, D, 2, 2), OWL_GROUP_VARIANT(DT, T, D, 2, 4), OWL_GROUP_VARIANT(DT, T, D, 2, 8)

static const Variant kGroupVariants[] = {
    OWL_GROUP_VARIANTS(OWL_BF16, __bf16, 128), OWL_GROUP_VARIANT(OWL_BF16, __bf16, 128, 3, 8),
    OWL_GROUP_VARIANTS(OWL_BF16, __bf16, 64), OWL_GROUP_VARIANT(OWL_BF16, __bf16, 64, 3, 8),
    OWL_GROUP_VARIANTS(OWL_F16, _Float16, 128), OWL_GROUP_VARIANTS(OWL_F16, _Float16, 64),
    OWL_GROUP_FEWS(OWL_BF16, __bf16, 128), OWL_GROUP_FEWS(OWL_BF16, __bf16, 64), OWL_GROUP_FEWS(OWL_F16, _Float16, 128), OWL_GROUP_FEWS(OWL_F16, _Float16, 64),
};

VariantList group_variants() { return VariantList{kGroupVariants, (int)(sizeof kGroupVariants / sizeof kGroupVariants[0])}; }

}  // namespace owl
