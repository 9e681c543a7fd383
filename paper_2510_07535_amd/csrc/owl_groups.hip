// Caches of 4-bit groups: the commit of accepted rows, and reading rows back as 16-bit numbers.  (Appending: owl_append.hip; the
// attention: owl_splitkv_groups.hip.)
#include <type_traits>

#include "owl_device.h"

namespace owl {

// ---------------------------------------------------------------------------
// KV commit: one workgroup per (KV head, sequence, tensor).  A row keeps its codes and its scales wherever it lies, so rows move as
// they are: 16 bytes of codes a thread, which covers 64 rows, and a row's scales in one word.  All is read before the barrier and
// stored behind it.  Checks as in the commit of a 16-bit cache.
// ---------------------------------------------------------------------------
constexpr int kCommitGroupThreads = 256;

template <int D>
__global__ void __launch_bounds__(kCommitGroupThreads) commit_groups_kernel(
    unsigned char *k_cache, unsigned char *v_cache, uint8_t *k_scale, uint8_t *v_scale, const int32_t *page_table,
    const int32_t *ctx_lens, const int32_t *accepted, const int32_t *n_accept, int N, int Hkv, int max_pages, int max_ctx_len,
    int64_t n_pool_pages, int64_t stride_page, int64_t stride_head, int64_t stride_token, int32_t *new_ctx_lens, uint32_t *status)
{
    constexpr int kPieces = D / 32;                          // 16-byte pieces of a row's codes, and bytes of its scales
    static_assert(64 * kPieces <= kCommitGroupThreads, "a piece a thread");
    typedef typename std::conditional<kPieces == 4, uint32_t, uint16_t>::type Scales;
    typedef uint32_t Piece __attribute__((ext_vector_type(4)));
    fetch_args<decltype(commit_groups_kernel<D>)>();
    const int g = blockIdx.x, b = blockIdx.y;
    unsigned char *cache = (blockIdx.z ? v_cache : k_cache) + g * stride_head;
    uint8_t *scales = (blockIdx.z ? v_scale : k_scale) + (int64_t)g * kPage * kPieces;
    const int tid = threadIdx.x, lane = tid & 63;
    const int a = accepted[(int64_t)b * N + min(lane, N - 1)];
    int na = load_uniform(n_accept, b), L = load_uniform(ctx_lens, b);
    asm volatile("" : "+s"(na), "+s"(L));                    // (both asked for before either is looked at)
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
    const int from_lp = from / kPage, to_lp = to / kPage;
    int from_page = from_lp, to_page = to_lp;
    if (page_table) {
        const int32_t *pages = page_table + (int64_t)b * max_pages;
        from_page = pages[min(from_lp, max_pages - 1)];
        to_page = pages[min(to_lp, max_pages - 1)];
    }
    const bool bad_page = (page_table && max(from_lp, to_lp) >= max_pages) || min(from_page, to_page) < 0 || max(from_page, to_page) >= n_pool_pages;
    const bool mine = lane < na, bad = a < 0 || a >= N || (lane > 0 && a <= before);
    const bool any_bad = __builtin_amdgcn_ballot_w64(mine && bad) != 0;          // the same in every wavefront
    if (any_bad || __builtin_amdgcn_ballot_w64(mine && bad_page) != 0) {
        if (tid == 0) flag_status(status, any_bad ? OWL_DEV_BAD_ACCEPT : OWL_DEV_BAD_PAGE);
        na = 0;
    }
    if (g == 0 && blockIdx.z == 0 && tid == 0 && new_ctx_lens) new_ctx_lens[b] = L + na;
    const bool moves = lane < na && (from_page != to_page || from % kPage != to % kPage);
    if (__builtin_amdgcn_ballot_w64(moves) == 0) return;     // uniform over the workgroup

    // piece tid % kPieces of row tid / kPieces; of rows that stay where they are, nothing
    const int r = tid / kPieces, rl = min(r, 63);
    const int f_page = __shfl(from_page, rl), f_slot = __shfl(from, rl) % kPage, t_page = __shfl(to_page, rl), t_slot = __shfl(to, rl) % kPage;
    const bool move = r < 64 && __shfl((int)moves, rl) != 0;
    Piece held{};
    Scales word{};
    if (move) held = *reinterpret_cast<const Piece *>(cache + (int64_t)f_page * stride_page + f_slot * stride_token + tid % kPieces * 16);
    const bool word_too = tid < 64 && moves;                 // the scales of row `lane`
    if (word_too) word = *reinterpret_cast<const Scales *>(scales + ((int64_t)from_page * Hkv * kPage + from % kPage) * kPieces);
    __syncthreads();                                         // all reads done before the first write
    if (move) *reinterpret_cast<Piece *>(cache + (int64_t)t_page * stride_page + t_slot * stride_token + tid % kPieces * 16) = held;
    if (word_too) *reinterpret_cast<Scales *>(scales + ((int64_t)to_page * Hkv * kPage + to % kPage) * kPieces) = word;
}

hipError_t launch_commit_groups(const owl_verify_desc &d, void *k_cache, void *v_cache, uint8_t *k_scale, uint8_t *v_scale,
                                const int32_t *page_table, const int32_t *ctx_lens, const int32_t *accepted,
                                const int32_t *n_accept, int32_t *new_ctx_lens, uint32_t *status, hipStream_t s)
{
    const dim3 grid(d.n_kv_heads, d.batch, 2), block(kCommitGroupThreads);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, s, static_cast<unsigned char *>(k_cache), static_cast<unsigned char *>(v_cache), k_scale,
                           v_scale, page_table, ctx_lens, accepted, n_accept, d.n_draft, d.n_kv_heads, d.max_pages_per_seq, d.max_ctx_len,
                           d.n_pool_pages, d.kv_stride_page, d.kv_stride_head, d.kv_stride_token, new_ctx_lens, status);
    };
    if (d.head_dim == 128) launch(commit_groups_kernel<128>);
    else launch(commit_groups_kernel<64>);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Rows back as 16-bit numbers, exactly what the groups stand for.  A workgroup takes a page: what it holds of a KV head is 16 D / 8 units of
// 8 channels, 4 bytes of codes in and 16 bytes out, a unit a thread, so that a wavefront reads and writes whole lines; the loads of
// four heads (of head_dim 64 eight) are in flight together.  Bound by what it writes: 80 % of its bytes.
// ---------------------------------------------------------------------------
constexpr int kGatherGroupThreads = 256;

template <typename T, int D>
__global__ void __launch_bounds__(kGatherGroupThreads) gather_groups_kernel(const unsigned char *cache, const uint8_t *scale,
                                                                            const int32_t *page_table, int seq, int max_pages,
                                                                            int64_t n_pool_pages, int Hkv, int64_t stride_page,
                                                                            int64_t stride_head, int64_t stride_token, int64_t first,
                                                                            int64_t n, int64_t n_pages, unsigned char *dst, uint32_t *status)
{
    constexpr int kUnits = kPage * D / 8, kHeads = kGatherGroupThreads / kUnits, kGroups = D / 32, kAtOnce = 4;
    const int unit = threadIdx.x % kUnits, slot = unit / (D / 8), piece = unit % (D / 8), h0 = threadIdx.x / kUnits;
    for (int64_t i = blockIdx.x; i < n_pages; i += gridDim.x) {
        const int64_t lp = first / kPage + i, t = lp * kPage + slot - first;
        const int64_t page = load_page(page_table, seq, max_pages, n_pool_pages, (int)lp, threadIdx.x == 0 ? status : nullptr);
        if (t < 0 || t >= n) continue;
        const unsigned char *codes = cache + page * stride_page + slot * stride_token + piece * 4;
        const uint8_t *scales = scale + (page * Hkv * kPage + slot) * kGroups + piece / 4;
        unsigned char *to = dst + (t * Hkv * D + piece * 8) * 2;
        for (int g = h0; g < Hkv; g += kAtOnce * kHeads) {
            uint32_t w[kAtOnce];
            uint8_t e[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int gk = min(g + k * kHeads, Hkv - 1);
                w[k] = *reinterpret_cast<const uint32_t *>(codes + gk * stride_head);
                e[k] = scales[(int64_t)gk * kPage * kGroups];
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (g + k * kHeads >= Hkv) continue;
                const float s = __builtin_bit_cast(float, (uint32_t)e[k] << 23);         // (255: infinity, which the conversion takes for none)
                uint4 x;
                if constexpr (std::is_same<T, __bf16>::value) {
                    x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s, 0));
                    x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s, 1));
                    x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s, 2));
                    x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s, 3));
                } else {
                    x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[k], s, 0));
                    x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[k], s, 1));
                    x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[k], s, 2));
                    x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[k], s, 3));
                }
                *reinterpret_cast<uint4 *>(to + (int64_t)(g + k * kHeads) * D * 2) = x;
            }
        }
    }
}

hipError_t launch_gather_groups(const owl_verify_desc &d, const void *cache, const uint8_t *scale, const int32_t *page_table, int seq,
                                int64_t first, int64_t n, void *dst, uint32_t *status, hipStream_t s)
{
    if (n == 0) return hipSuccess;
    const int64_t n_pages = (first + n - 1) / kPage - first / kPage + 1;
    const dim3 grid((unsigned)(n_pages < (1 << 20) ? n_pages : 1 << 20)), block(kGatherGroupThreads);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, s, static_cast<const unsigned char *>(cache), scale, page_table, seq, d.max_pages_per_seq,
                           d.n_pool_pages, d.n_kv_heads, d.kv_stride_page, d.kv_stride_head, d.kv_stride_token, first, n, n_pages,
                           static_cast<unsigned char *>(dst), status);
    };
    if (d.qkv_dtype == OWL_BF16) d.head_dim == 128 ? launch(gather_groups_kernel<__bf16, 128>) : launch(gather_groups_kernel<__bf16, 64>);
    else d.head_dim == 128 ? launch(gather_groups_kernel<_Float16, 128>) : launch(gather_groups_kernel<_Float16, 64>);
    return hipGetLastError();
}

}  // namespace owl
