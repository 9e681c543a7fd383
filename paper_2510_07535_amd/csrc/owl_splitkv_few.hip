// Split-KV pass of the verify-step attention over a cache of 8-bit blocks for few query rows, or short contexts, for gfx950
// (MI355X); which calls come here is the plan's to say.
//
// The share of a workgroup, its pieces, their partials, and how 8 bits become operands of 16 are those of owl_splitkv.h; the loop
// is another one.  Half the bytes arrive in half the time, so what bounds the shared ring beside its stream, eight wavefronts that
// read every fragment for their own rows and meet at a barrier every 64 tokens, would be the whole cost here.
// Here a wavefront shares nothing until the end of a piece:
//   keys      The 32-token chunks of a piece are dealt to the eight wavefronts in turn.  A wavefront streams its own
//             chunks, two of each tensor in flight, into its own part of LDS, waits for nothing but its own transfers, and
//             reads every fragment once; no barrier in the loop, and the two wavefronts of a SIMD drift apart by
//             themselves, so that one's products overlap the other's softmax.
//   rows      It takes all rows of its row group, one or two tiles, against each fragment: what turning 8 bits
//             into 16 costs is paid once for them.  More tiles are further row groups, other workgroups that
//             find the chunks in their XCD's L2.  (Three tiles a wavefront leave no registers to read ahead, and were slower than
//             more groups; four wavefronts of 512 registers with up to five tiles, products and softmax of a tile woven by hand,
//             were slower than the shared ring, 99.5 us with 15 tiles at 64K against 76.)
//   softmax   Each wavefront has a reference of its own for each row.  It stays until a score lies more than `kRoom` above it;
//             the row then moves to its highest score.
//   merge     At the end of a piece the wavefronts' sums meet in LDS, a tile after the other, a channel tile a wavefront, and
//             leave one partial, in fp32 (rounded to fp16 it would cost half of what the answer's own rounding does).
// us, shared ring -> here, 8 KV heads, head_dim 128, bf16 queries: 1 node (4 rows) at 64K 39.0 -> 27.7 (4.9 TB/s), 6 nodes
// (24 rows) at 32K 25.1 -> 20.7, at 128K 68.7 -> 51.9 (5.2 TB/s), 16 sequences of 8K-64K with 4 rows 302 -> 211 (6.3 TB/s: the stream is the
// bound), 16 nodes (64 rows, 2 groups) at 64K 41.9 -> 40.9, 60 nodes (240 rows, 8 groups) on 5K in fp16 22.7 -> 19.0.  From two groups on the chunks' way from L2 and their conversion, once a
// group, are the bound.
//
// The scores of a chunk come out with the keys of its first page in one accumulator and those of its second in the other.
#include "owl_splitkv.h"

namespace owl {

constexpr int kChunk = 2 * kPage;                    // tokens of a chunk

// One byte a lane, of the first four lanes, from global memory into consecutive 32-bit LDS words, zeros above it.  All lanes
// of the wavefront are active where this is called.
__device__ __forceinline__ void dma_scales(const uint8_t *gptr, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, 15\n\tglobal_load_lds_ubyte %1, off\n\ts_mov_b64 exec, -1\n"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(gptr)
                 : "memory", "m0");
}

// 16 bytes a lane, from a wave-uniform base and a 32-bit offset of the lane to LDS, lane-linear from lds_addr (wave-uniform) on.
// kOnce: no other row group reads them, and they are not kept (non-temporal): 6 nodes at 128K 55.4 -> 51.4 us; where several groups
// read them it would be 296 -> 342 (48 rows, 16 sequences of 8K-64K).
template <bool kOnce>
__device__ __forceinline__ void dma16s_to(uint64_t sbase, uint32_t voff, uint32_t lds_addr)
{
    if constexpr (kOnce) {
        dma16s(sbase, voff, __builtin_amdgcn_readfirstlane(lds_addr));
    } else {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n"
                     :
                     : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(sbase)
                     : "memory", "m0");
    }
}

// At most N of this wavefront's loads are in flight, and what they brought is seen from here on.
template <int N>
__device__ __forceinline__ void arrived()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    wait_vmcnt<N>();
    asm volatile("" ::: "memory");
}

// This wavefront's LDS reads are done: what they read may be overwritten.
__device__ __forceinline__ void reads_done()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Transposing 64-bit LDS read of bytes: in a block of 16 lanes, lane i receives byte i % 8 of what lanes 2e + i / 8 (e = 0..7) point at,
// one after the other.  With lane 2e + c pointing at channels 8c .. 8c + 7 of key e, lane i ends up with channel i of eight keys.
__device__ __forceinline__ uint2 lds_read_tr8(const unsigned char *p)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3))) *)(p));
    return __builtin_bit_cast(uint2, v);
}

// Geometry of one instantiation.
template <int D>
struct QGeo {
    static constexpr int PPR = D / 16;               // 16-byte pieces of a cached row
    static constexpr int RPI = 1024 / D;             // rows a DMA instruction brings
    static constexpr int PAGE_DMAS = kPage / RPI;    // instructions for a page of one tensor
    static constexpr int DMAS = 2 * PAGE_DMAS;       // for a chunk of one tensor
    static constexpr int NT = D / 16, KQ = D / 32;   // channel tiles of O^T, k-steps of a score
    static constexpr int TENSOR = kChunk * D;        // bytes of a chunk of one tensor
    static constexpr int WAVE = 4 * TENSOR;          // two slots of K, two of V
    static constexpr int TILE = NT * 1024 + 512;     // a wavefront's part of a tile in the merge: O^T fragments, (m, l) of each lane
    static constexpr int MERGE = kWaves * TILE;
    static constexpr size_t MAIN = (size_t)(kWaves * WAVE > 2 * MERGE ? kWaves * WAVE : 2 * MERGE);
    static constexpr size_t SCALES = MAIN, LDS = SCALES + kWaves * 2 * 16;
    // The piece in which piece 0 of a row sits (XOR), so that the fragment reads meet no bank twice.  The 16 rows that 16 lanes read at
    // a time are, of K, those of a page, and of V slots 0-7 (or 8-15) of the two pages; 256 / D rows share a round of the banks.
    static constexpr int k_turn(int slot) { return slot / (256 / D) & (PPR - 1); }
    static constexpr int v_turn(int slot, int page) { return (slot / (256 / D) & (PPR / 2 - 1)) | page * (PPR / 2); }
};

// How far a score may lie above its row's reference: a weight is at most 2^kRoom.  fp16 ends at 2^16.
template <typename T> constexpr float kRoom = 11.0f;
template <> constexpr float kRoom<__bf16> = 24.0f;

struct QPiece {
    int b, L, Nb;                                    // sequence, its prefix length and number of drafts
    int pos0, pos1;                                  // [pos0, pos1) of its L + Nb cached rows, pos0 a multiple of 64
    size_t slot;                                     // where the partials of row tile 0 go
};

// Pages of the chunks first .. first + 31 of this wavefront in the piece that begins at pos0, lane 2 i + h holding page h of chunk
// first + i; unchecked, and past the table its last entry again.
__device__ __forceinline__ int load_chunk_pages(const KParams &p, int b, int pos0, int wave, int lane, int first)
{
    const int lp = pos0 / kPage + (wave + kWaves * (first + (lane >> 1))) * 2 + (lane & 1);
    return p.page_table ? p.page_table[(int64_t)b * p.max_pages + min(lp, p.max_pages - 1)] : lp;
}

template <typename T, int D, int TPW, bool kOnce>
__device__ __forceinline__ void run_quant_piece(const QuantParams &p, unsigned char *smem, int wave, int lane, int g, int rg, const QPiece &pc,
                                               int pages, bool have_pages)
{
    using GEO = QGeo<D>;
    constexpr int NT = GEO::NT, KQ = GEO::KQ, PPR = GEO::PPR, RPI = GEO::RPI, DMAS = GEO::DMAS, TENSOR = GEO::TENSOR;
    const int j = lane & 15, qd = lane >> 4;
    const int b = pc.b, L = pc.L, Nb = pc.Nb, pos0 = pc.pos0, pos1 = pc.pos1;
    const int chunks = (pos1 - pos0 + kChunk - 1) / kChunk;
    const int mine = max(0, (chunks - wave + kWaves - 1) / kWaves);
    const int last_lp = (pos1 - 1) / kPage, last_slot = (pos1 - 1) % kPage;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    unsigned char *ring = smem + wave * GEO::WAVE;
    const uint32_t ring_lds = lds0 + wave * GEO::WAVE;
    const uint32_t scale_off = (uint32_t)GEO::SCALES + wave * 32;

    if (!have_pages) pages = load_chunk_pages(p, b, pos0, wave, lane, 0);
    // Entries past the end of the piece become the chunk's first page, which is one of its pages; bad ones page 0.
    auto checked = [&](int pg, int first) -> int {
        const int chunk = first + (lane >> 1), lp = pos0 / kPage + (wave + kWaves * chunk) * 2 + (lane & 1);
        const int other = __shfl_xor(pg, 1);
        if ((lane & 1) && lp > last_lp) pg = other;
        const bool bad = pg < 0 || pg >= p.n_pool_pages || (p.page_table && min(lp, last_lp) >= p.max_pages);
        if (bad && chunk < mine) flag_status(p.dev_status, OWL_DEV_BAD_PAGE);
        return bad ? 0 : pg;
    };
    pages = checked(pages, 0);

    // ---- transfers ----
    // A page is brought by PAGE_DMAS instructions of 1 KB: a scalar base, which changes from page to page, and fixed offsets of the lanes.
    // The last page of the piece is clamped: rows past the end re-read the last one, finite, and masked later.
    const int64_t head_off = (int64_t)g * p.stride_head;
    const uint32_t tok_bytes = (uint32_t)p.stride_token;
    auto lane_offset = [&](int tensor, int h, int it, int most) -> uint32_t {
        const int row = it * RPI + lane / PPR, turn = tensor ? GEO::v_turn(row, h) : GEO::k_turn(row);
        return (uint32_t)min(row, most) * tok_bytes + (uint32_t)((lane % PPR ^ turn) << 4);
    };
    uint32_t k_off[GEO::PAGE_DMAS], v_off[2][GEO::PAGE_DMAS];
#pragma unroll
    for (int it = 0; it < GEO::PAGE_DMAS; ++it) {
        k_off[it] = lane_offset(0, 0, it, kPage - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) v_off[h][it] = lane_offset(1, h, it, kPage - 1);
    }
    const uint64_t scale_base = (uint64_t)(uintptr_t)(lane & 2 ? p.v_scale : p.k_scale) + (uint32_t)g;
    // The chunk that is being asked for: byte offsets of its pages, and whether it holds the piece's last one.
    uint64_t page_at[2] = {0, 0};
    bool ends = false;
    auto issue_pages = [&](auto tensor_tag, auto slot_tag) {
        constexpr int tensor = decltype(tensor_tag)::value, slot = decltype(slot_tag)::value;
        const uint64_t cache = (uint64_t)(uintptr_t)(tensor ? p.v : p.k);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t sbase = uniform64(cache + page_at[h]);
#pragma unroll
            for (int it = 0; it < GEO::PAGE_DMAS; ++it)
                dma16s_to<kOnce>(sbase, tensor ? v_off[h][it] : k_off[it], ring_lds + (tensor * 2 + slot) * TENSOR + (h * GEO::PAGE_DMAS + it) * 1024);
        }
    };
    auto issue_last = [&](int tensor, int slot, int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int lp = pos0 / kPage + (wave + kWaves * i) * 2 + h;
            const uint64_t sbase = uniform64((uint64_t)(uintptr_t)(tensor ? p.v : p.k) + page_at[h]);
#pragma unroll
            for (int it = 0; it < GEO::PAGE_DMAS; ++it)
                dma16s_to<kOnce>(sbase, lane_offset(tensor, h, it, lp >= last_lp ? last_slot : kPage - 1),
                                 ring_lds + (tensor * 2 + slot) * TENSOR + (h * GEO::PAGE_DMAS + it) * 1024);
        }
    };
    // K of chunk i, the four scales of the chunk with it; then V of the same chunk
    auto issue_k = [&](auto slot_tag, int i) {
        constexpr int slot = decltype(slot_tag)::value;
        const int p0 = __builtin_amdgcn_readlane(pages, (i & 31) * 2), p1 = __builtin_amdgcn_readlane(pages, (i & 31) * 2 + 1);
        page_at[0] = (uint64_t)((int64_t)p0 * p.stride_page + head_off);
        page_at[1] = (uint64_t)((int64_t)p1 * p.stride_page + head_off);
        ends = pos0 / kPage + (wave + kWaves * i) * 2 + 1 >= last_lp;
        if (!ends) issue_pages(std::integral_constant<int, 0>{}, slot_tag);
        else issue_last(0, slot, i);
        const uint32_t pg = lane & 1 ? (uint32_t)p1 : (uint32_t)p0;
        dma_scales(reinterpret_cast<const uint8_t *>(scale_base + (uint64_t)pg * (uint32_t)p.Hkv), lds0 + scale_off + slot * 16);
    };
    auto issue_v = [&](auto slot_tag, int i) {
        if (!ends) issue_pages(std::integral_constant<int, 1>{}, slot_tag);
        else issue_last(1, decltype(slot_tag)::value, i);
    };
    using Slot0 = std::integral_constant<int, 0>;
    using Slot1 = std::integral_constant<int, 1>;
    if (mine > 0) {
        issue_k(Slot0{}, 0);
        issue_v(Slot0{}, 0);
    }
    if (mine > 1) {
        issue_k(Slot1{}, 1);
        issue_v(Slot1{}, 1);
    }

    // ---- query rows: tiles 0 .. TPW - 1 of the row group ----
    const float inv_g = __builtin_amdgcn_rcpf((float)p.G);
    const unsigned char *q_head = static_cast<const unsigned char *>(p.q) + ((int64_t)b * p.N * p.Hq + (int64_t)g * p.G) * D * 2;
    uint4 qf[TPW][KQ];
    int irow[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int tg = rg * p.group_tiles + t;
        const bool tile_ok = t < p.group_tiles && tg < p.RT;
        const int row = tg * kRowTile + j, i = (int)(((float)row + 0.5f) * inv_g);     // node row / G, exactly (see owl_splitkv.h)
        irow[t] = tile_ok && row < p.R && i < Nb ? i : -1;
        const int rc = min(row, p.R - 1), ic = (int)(((float)rc + 0.5f) * inv_g);
        const unsigned char *src = q_head + ((int64_t)ic * (p.Hq - p.G) + rc) * (D * 2);
#pragma unroll
        for (int kk = 0; kk < KQ; ++kk) {            // channels 64 (kk / 2) + 16 quad + 8 (kk % 2) .. + 7, as a 16-byte read of K brings them
            const uint4 x = *reinterpret_cast<const uint4 *>(src + (8 * (kk / 2) + 2 * qd + kk % 2) * 16);
            qf[t][kk] = irow[t] >= 0 ? x : make_uint4(0, 0, 0, 0);
        }
    }
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
    const float c_log2 = p.c_log2;

    // ---- the loop ----
    // Fragments are read from LDS half a step ahead: K of the next chunk before V^T P of this one, V before the scores' products; then
    // the slot is free and takes the chunk after the next one.  In flight, oldest first: V of this chunk, K and scales and V of the
    // next one, those of the one that this step asks for.
    uint4 kr[2][KQ / 2], scales;
    auto read_k = [&](auto slot_tag, int jj, int qq) {
        constexpr int slot = decltype(slot_tag)::value;
        scales = *reinterpret_cast<const uint4 *>(smem + scale_off + slot * 16);
        const uint32_t at = (uint32_t)(slot * TENSOR + jj * D + ((qq ^ GEO::k_turn(jj)) << 4));
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int c = 0; c < KQ / 2; ++c) kr[kt][c] = *reinterpret_cast<const uint4 *>(ring + (at ^ (c << 6)) + kt * kPage * D);
    };
    auto step = [&](auto slot_tag, int i) {
        constexpr int slot = decltype(slot_tag)::value;
        const int step_pos = pos0 + (wave + kWaves * i) * kChunk;
        const bool more = i + 1 < mine, refill = i + 2 < mine;
        // the pages of the 32 chunks behind the two that are under way
        if ((i & 31) == 30 && refill) pages = checked(load_chunk_pages(p, b, pos0, wave, lane, i + 2), i + 2);
        if (more) arrived<2 * DMAS + 1>();
        else arrived<0>();
        int jj = j, qq = qd;                         // (formed anew in each step: kept, what follows from them takes 20 registers)
        asm volatile("" : "+v"(jj), "+v"(qq));
        // lane 2e + c of block `quad`: key 4 quad + e of the first page, from e = 4 on 4 quad + e - 4 of the second, as the scores
        // lie; channels 16 u + 8 c .. + 7
        const int v_slot = 4 * qq + ((jj >> 1) & 3), v_page = jj >> 3;
        const uint32_t v_at = (uint32_t)((2 + slot) * TENSOR + (v_page * kPage + v_slot) * D + (GEO::v_turn(v_slot, v_page) << 4) + (jj & 1) * 8);
        uint2 vr[NT];
#pragma unroll
        for (int u = 0; u < NT; ++u) vr[u] = lds_read_tr8(ring + (v_at ^ (u << 4)));
        const float ks[2] = {__builtin_bit_cast(float, scales.x << 23), __builtin_bit_cast(float, scales.y << 23)};
        const float vs[2] = {__builtin_bit_cast(float, scales.z << 23), __builtin_bit_cast(float, scales.w << 23)};
        f32x4 S[TPW][2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            uint4 kf[KQ];
#pragma unroll
            for (int c = 0; c < KQ / 2; ++c) {
                kf[2 * c] = widen8<T>(make_uint2(kr[kt][c].x, kr[kt][c].y), ks[kt], ks[kt]);
                kf[2 * c + 1] = widen8<T>(make_uint2(kr[kt][c].z, kr[kt][c].w), ks[kt], ks[kt]);
            }
#pragma unroll
            for (int t = 0; t < TPW; ++t) S[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KQ; ++kk)
#pragma unroll
                for (int t = 0; t < TPW; ++t) S[t][kt] = mfma16<T>(kf[kk], qf[t][kk], S[t][kt]);
        }
        reads_done();                                // (K of this chunk and V)
        if (refill) {
            issue_k(slot_tag, i + 2);
            issue_v(slot_tag, i + 2);
        }
        uint4 pf[TPW];
#pragma unroll
        for (int t = 0; t < TPW; ++t) {
            f32x4 &s0 = S[t][0], &s1 = S[t][1];
            if (step_pos + kChunk > L) {             // reaches drafts or the ragged end (uniform)
                const int node = max(irow[t], 0);
                uint64_t seen = ((uint64_t)__shfl((uint32_t)(anc >> 32), node) << 32) | __shfl((uint32_t)anc, node);
                if (irow[t] < 0) seen = pos1 > L ? ~(uint64_t)0 >> (64 - Nb) : 0;       // a row without a node sees all of them
                const int ahead = L - step_pos;      // prefix keys in this chunk (< 32), or minus the drafts before it
                const uint32_t word = ahead >= 0 ? ((1u << ahead) - 1u) | (uint32_t)(seen << ahead)
                                                 : (-ahead < 64 ? (uint32_t)(seen >> -ahead) : 0u);
                const uint32_t va = word >> (4 * qd), vb = va >> 16;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s0[r] = (va >> r) & 1u ? s0[r] : -INFINITY;
                    s1[r] = (vb >> r) & 1u ? s1[r] : -INFINITY;
                }
            }
            const float tm = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
            // any lane's own keys can raise the alarm (uniform branch, rarely taken after the first chunk)
            if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(tm, c_log2, -m[t]) > kRoom<T>) != 0) {
                const float sc = quad_column_max(tm) * c_log2;
                const float mn = sc > m[t] + kRoom<T> ? sc : m[t];
                const float alpha = fast_exp2(m[t] - mn);
                m[t] = mn;
#pragma unroll
                for (int u = 0; u <= NT; ++u) O[t][u] *= alpha;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s0[r] = fast_exp2(__builtin_fmaf(s0[r], c_log2, -m[t]));
                s1[r] = fast_exp2(__builtin_fmaf(s1[r], c_log2, -m[t]));
            }
            // (the matrix pipe takes 16-bit weights; the row sum adds the same rounded ones)
            pf[t] = make_uint4(pack2<T>(s0[0], s0[1]), pack2<T>(s0[2], s0[3]), pack2<T>(s1[0], s1[1]), pack2<T>(s1[2], s1[3]));
        }
        if (more) {
            if (refill) arrived<DMAS + 2 * DMAS + 1>();
            else arrived<DMAS>();
            read_k(std::integral_constant<int, 1 - slot>{}, jj, qq);
        }
        const uint4 ones = make_uint4(ones2<T>(), ones2<T>(), ones2<T>(), ones2<T>());
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const uint4 vf = widen8<T>(vr[u], vs[0], vs[1]);
#pragma unroll
            for (int t = 0; t < TPW; ++t) O[t][u] = mfma16<T>(vf, pf[t], O[t][u]);
        }
#pragma unroll
        for (int t = 0; t < TPW; ++t) O[t][NT] = mfma16<T>(ones, pf[t], O[t][NT]);
    };
    if (mine > 0) {
        if (mine > 1) arrived<DMAS + 2 * DMAS + 1>();
        else arrived<DMAS>();
        read_k(Slot0{}, j, qd);
    }
    for (int i = 0; i < mine; i += 2) {
        step(Slot0{}, i);
        if (i + 1 < mine) step(Slot1{}, i + 1);
    }

    // ---- the wavefronts' sums meet, a tile after the other in two buffers by turns, and become the piece's partial ----
    __syncthreads();                                 // no wavefront reads its ring any more
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
        const int tg = rg * p.group_tiles + t;
        if (t >= p.group_tiles || tg >= p.RT) break; // uniform
        unsigned char *buf = smem + (t & 1) * GEO::MERGE;
        unsigned char *own = buf + wave * GEO::TILE;
#pragma unroll
        for (int u = 0; u < NT; ++u) reinterpret_cast<f32x4 *>(own)[u * 64 + lane] = O[t][u];
        reinterpret_cast<float2 *>(own + NT * 1024)[lane] = make_float2(m[t], O[t][NT][0]);
        __syncthreads();
        if (wave < NT) {                             // channel tile `wave`
            float2 ml[kWaves];
            float M = kMInit, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                ml[w] = reinterpret_cast<const float2 *>(buf + w * GEO::TILE + NT * 1024)[lane];
                M = fmaxf(M, ml[w].x);
            }
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float a = fast_exp2(ml[w].x - M);
                l = __builtin_fmaf(ml[w].y, a, l);
                const f32x4 x = reinterpret_cast<const f32x4 *>(buf + w * GEO::TILE)[wave * 64 + lane];
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(x[r], a, sum[r]);
            }
            const size_t slot = pc.slot + tg;
            static_cast<float4 *>(p.part_o)[slot * (size_t)(NT * 64) + wave * 64 + lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            if (wave == 0 && qd == 0) {
                float *stats = p.part_ml + slot * kPartMl + 3 * j;
                stats[0] = M;
                stats[1] = l;
                stats[2] = 1.0f;
            }
        }
    }
}

template <typename T, int D, int TPW, bool kOnce>
__global__ void __launch_bounds__(kThreads) splitkv_few_kernel(const QuantParams p)
{
    extern __shared__ __align__(16) unsigned char smem[];
    fetch_args<void(QuantParams)>();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Which share of which (KV head, row group): as in the pass over 16-bit caches.
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
    if (!p.dealt) {                                  // equal splits of C tokens, of one sequence each
        const int c = item % (int)gridDim.y;
        b = item / (int)gridDim.y;
        if (b >= p.B || c >= p.max_splits) return;   // padding of the grid
        x = c * (p.C / kSplitQuantum);
        x1 = x + p.C / kSplitQuantum;
        slot0 = b * p.max_splits + c - b;
    } else {
        if (item >= p.rule.max_workers) return;      // padding of the grid
        x = deal_begin(deal, min(item, deal.workers - 1));
    }
    // Most lone sequences are as long as announced: their pages are asked for along with the length.
    int pages = 0, pages_pos = -1;
    if (!p.dealt || p.B == 1) {
        pages_pos = x * kSplitQuantum;
        pages = load_chunk_pages(p, b, pages_pos, wave, lane, 0);
    }
    SeqSize size{0, 0};
    bool sized = false;
    if (p.dealt) {
        if (p.B == 1) {
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
            const QPiece pc{b, L, Nb, s0 * kSplitQuantum, min(s1 * kSplitQuantum, T_b), (head_slots + slot0 + b) * p.RT};
            run_quant_piece<T, D, TPW, kOnce>(p, smem, wave, lane, g, rg, pc, pages, pages_pos == pc.pos0);
            pages_pos = -1;
        }
        before += seq_units(p, T_b);
        if (before >= x1 || !p.dealt) break;
        x = before;
    }
}

template <typename T, int D, int TPW, bool kOnce>
static void launch_few_variant(const KParams &args, dim3 grid, hipStream_t s, hipEvent_t start, hipEvent_t stop)
{
    const QuantParams &p = static_cast<const QuantParams &>(args);
    if (start || stop)
        hipExtLaunchKernelGGL((splitkv_few_kernel<T, D, TPW, kOnce>), grid, dim3(kThreads), QGeo<D>::LDS, s, start, stop, 0, p);
    else
        hipLaunchKernelGGL((splitkv_few_kernel<T, D, TPW, kOnce>), grid, dim3(kThreads), QGeo<D>::LDS, s, p);
}

// (wr: 1, the only row group, or 2, one of several)
#define OWL_FEW_VARIANT(DT, T, D, TPW, GROUPS) \
    Variant { DT, D, TPW, GROUPS, kWaves, false, Cached::kBlocks8, QGeo<D>::LDS, &launch_few_variant<T, D, TPW, GROUPS == 1>, \
              reinterpret_cast<const void *>(&splitkv_few_kernel<T, D, TPW, GROUPS == 1>) }
#define OWL_FEW_VARIANTS(DT, T, D) OWL_FEW_VARIANT(DT, T, D, 1, 1), OWL_FEW_VARIANT(DT, T, D, 2, 1), OWL_FEW_VARIANT(DT, T, D, 2, 2)

static const Variant kFewTileVariants[] = {
    OWL_FEW_VARIANTS(OWL_BF16, __bf16, 128), OWL_FEW_VARIANTS(OWL_BF16, __bf16, 64),
    OWL_FEW_VARIANTS(OWL_F16, _Float16, 128), OWL_FEW_VARIANTS(OWL_F16, _Float16, 64),
};

VariantList few_tile_variants() { return VariantList{kFewTileVariants, (int)(sizeof kFewTileVariants / sizeof kFewTileVariants[0])}; }

}  // namespace owl
