// What the kernels of the paged cache share: its geometry as the kernels see it, and the workspace's layout.
#pragma once
#include "common.cuh"
#include "paged_plan.cuh"

namespace pafu {

// Workspace of the paged entry points: status header (256 bytes), tickets (zero between calls), partial results.
constexpr int kStatusWordPaged = 1;            // a pafu_status that a kernel of the paged cache found on the device
constexpr int kPaTicketRow = 1024;             // CTAs of the attention kernel, at most
constexpr int kPagedTickets = 3 * kPaTicketRow + 64;      // 32-bit words behind the header: three a CTA of the attention, the last one the tables' own
constexpr size_t kPagedPartOffset = kWsHeaderBytes + kPagedTickets * 4;
constexpr int kPagedCtasPerSm = 4;             // most CTAs of the attention kernel on an SM
constexpr int kPagedRows = 16;                 // query heads that one item handles (rows of a tensor-core tile)
static_assert(kPagedCtasPerSm * kMaxPersistentGrid <= kPaTicketRow, "a ticket for every CTA");
static_assert(kPagedPartOffset % 256 == 0 && kPagedPartOffset == PAFU_PAGED_HEADER_BYTES, "the part of the workspace that starts at zero");

// The pools, with strides in 16-byte units.
struct PagedPool {
    const char* K;
    const char* V;
    const int32_t* table;
    uint32_t n_pages;
    int32_t max_pages;
    FastDiv page;
    uint32_t page_u, token_u, head_u;
};

// Partial results of split items: two a CTA, each the rows' numerators, maxima and sums
inline size_t paged_part_bytes(int32_t d_head) {
    return (size_t)kPagedCtasPerSm * device_sm_count() * 2 * kPagedRows * (d_head + 2) * sizeof(float);
}
pafu_status launch_paged_attn(const pafu_paged_cache& c, const void* Q, int64_t q_token, int64_t q_head, const int32_t* lens,
                              int64_t n_sink, int64_t n_recent, float scale, void* O, float* LSE, void* ws, cudaStream_t stream);
pafu_status launch_paged_append(const pafu_paged_cache& c, const void* Kn, const void* Vn, int64_t ld_token, int64_t ld_head,
                                const int64_t* slots, int64_t n_tokens, void* ws, cudaStream_t stream);
pafu_status launch_paged_tables(const pafu_paged_cache& c, const int32_t* len_old, const int32_t* len_new, int32_t* free_list,
                                const int32_t* n_free, int32_t* n_free_out, int32_t* len_out, int64_t* slots, int64_t n_slots,
                                int32_t* cu_new, void* ws, cudaStream_t stream);

inline int type_bytes(int32_t t) { return t == PAFU_TYPE_E4M3 ? 1 : 2; }

inline PagedPool pool_of(const pafu_paged_cache& c) {
    const int64_t es = type_bytes(c.cache_type);
    PagedPool p;
    p.K = static_cast<const char*>(c.K);
    p.V = static_cast<const char*>(c.V);
    p.table = c.table;
    p.n_pages = (uint32_t)c.n_pages;
    p.max_pages = c.max_pages;
    p.page = fast_div((uint32_t)c.page_size);
    p.page_u = c.n_pages > 1 ? (uint32_t)(c.page_stride * es / 16) : 0u;
    p.token_u = c.page_size > 1 ? (uint32_t)(c.token_stride * es / 16) : 0u;
    p.head_u = c.n_kv_heads > 1 ? (uint32_t)(c.head_stride * es / 16) : 0u;
    return p;
}

}  // namespace pafu
