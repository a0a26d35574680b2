// Block tables, slot map and rows of the paged cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"

namespace pafu {

namespace {

// ---------------------------------------------------------------------------------- tables
// From the lengths before and after a step: which pages each request gives back and gets, where its new tokens go.
// All of it follows from three prefix sums over the requests (pages needed, pages given back, new tokens), so every CTA computes
// them for itself - each thread sums a stretch of requests, one scan of the threads' sums - and then takes its part of
// the entries to write; an entry finds its request by a binary search in the threads' sums and a walk through one stretch.
// That keeps a step one launch: nothing a CTA reads is written by another (a request that grows only gets table
// entries behind those that are read, the free list only entries above its top), apart from the lengths and the free count,
// which may be updated in place; the CTA that counts itself out last writes those.  A step moves a few KB to MB: the
// trips to memory that follow one another bound it, so a thread issues its loads before it uses the first, and in a
// long step takes eight neighbouring tokens, which mostly share a request and a page.
constexpr int kTabThreads = 512;

struct TablesArgs {
    int32_t* table;
    int32_t max_pages, n_requests;
    uint32_t n_pages;
    FastDiv page;
    const int32_t* len_old;
    const int32_t* len_new;
    int32_t* free_list;
    const int32_t* n_free;
    int32_t* n_free_out;
    int32_t* len_out;
    int64_t* slots;
    int64_t n_slots;
    int32_t* cu_new;
    int32_t* status;
    int32_t* ticket;
};

struct Lens {
    int32_t old_len, new_len, have, want;      // tokens and pages before and after
    __device__ int32_t need() const { return max(want - have, 0); }
    __device__ int32_t back() const { return max(have - want, 0); }
    __device__ int32_t tokens() const { return max(new_len - old_len, 0); }
};

struct Sums {
    int64_t need, back, tokens;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return Sums{a.need + b.need, a.back + b.back, a.tokens + b.tokens}; }

__device__ __forceinline__ int32_t pages_of(const FastDiv& page, int32_t len) {
    return len <= 0 ? 0 : (int32_t)div_by((uint32_t)(len - 1), page) + 1;
}

// PER: neighbouring tokens a thread
template <int PER>
__global__ void __launch_bounds__(kTabThreads) paged_tables_kernel(const TablesArgs a) {
    __shared__ int64_t s_need[kTabThreads + 1], s_back[kTabThreads + 1], s_tok[kTabThreads + 1];
    __shared__ Sums s_warp[kTabThreads / 32];
    __shared__ int32_t s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dep_wait();
    const int per = (a.n_requests + kTabThreads - 1) / kTabThreads;
    auto lens_of = [&](int32_t before, int32_t after) {
        return Lens{before, after, pages_of(a.page, before), pages_of(a.page, after)};
    };
    auto lens = [&](int r) { return lens_of(ld_index(a.len_old + r), ld_index(a.len_new + r)); };
    const int32_t F = ld_index(a.n_free);
    const int r0 = min(tid * per, a.n_requests), r1 = min(r0 + per, a.n_requests);
    Sums mine{0, 0, 0};
    bool bad = F < 0 || (uint32_t)F > a.n_pages;
    for (int r = r0; r < r1; r += 4) {
        int32_t before[4], after[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            before[i] = r + i < r1 ? ld_index(a.len_old + r + i) : 0;
            after[i] = r + i < r1 ? ld_index(a.len_new + r + i) : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Lens x = lens_of(before[i], after[i]);
            bad |= x.old_len < 0 || x.new_len < 0 || x.have > a.max_pages || x.want > a.max_pages;
            mine = mine + Sums{x.need(), x.back(), x.tokens()};
        }
    }
    Sums inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums v{__shfl_up_sync(0xffffffffu, inc.need, o), __shfl_up_sync(0xffffffffu, inc.back, o), __shfl_up_sync(0xffffffffu, inc.tokens, o)};
        if (lane >= o) inc = inc + v;
    }
    if (lane == 31) s_warp[warp] = inc;
    bad = __syncthreads_or(bad);
    Sums all{0, 0, 0}, before{inc.need - mine.need, inc.back - mine.back, inc.tokens - mine.tokens};
    for (int w = 0; w < kTabThreads / 32; ++w) {
        if (w < warp) before = before + s_warp[w];
        all = all + s_warp[w];
    }
    s_need[tid] = before.need;
    s_back[tid] = before.back;
    s_tok[tid] = before.tokens;
    __syncthreads();
    // all or nothing: every page must exist, every token have a place in the slot map
    const int64_t height = (int64_t)F + all.back;               // of the stack, with what is given back on top
    const bool short_of = all.need > height || all.tokens > a.n_slots;
    const bool ok = !bad && !short_of && height - all.need <= (int64_t)a.n_pages;
    if (!ok && blockIdx.x == 0 && tid == 0) *a.status = bad || !short_of ? PAFU_ERR_BAD_PAGE : PAFU_ERR_NO_PAGES;

    // request that holds number i of a sum; returns i's place among the request's own
    auto find = [&](const int64_t* sums, int64_t i, auto value, int* request, Lens* x) {
        int lo = 0, hi = kTabThreads - 1;                        // last thread whose sum is <= i
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (sums[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        int64_t at = sums[lo];
        int r = lo * per;
        *x = lens(r);
        while (i >= at + value(*x)) {
            at += value(*x);
            *x = lens(++r);
        }
        *request = r;
        return i - at;
    };
    auto need_of = [](const Lens& x) { return x.need(); };
    auto back_of = [](const Lens& x) { return x.back(); };
    auto tokens_of = [](const Lens& x) { return x.tokens(); };
    // where entry v of the stack lies: in the free list, then the pages given back in the order of requests and columns
    auto stack = [&](int64_t v) -> const int32_t* {
        if (v < F) return a.free_list + v;
        int r;
        Lens x;
        const int64_t i = find(s_back, v - F, back_of, &r, &x);
        return a.table + (int64_t)r * a.max_pages + x.want + i;
    };
    // table entries, entries of the free list, and the slot map side by side: no thread does one after the other
    const int64_t pages = ok ? all.need : 0, pushed = ok ? max(height - all.need - F, (int64_t)0) : 0;
    const int64_t jobs = pages + pushed + (a.n_slots + PER - 1) / PER;
    for (int64_t job = (int64_t)blockIdx.x * kTabThreads + tid; job < jobs; job += (int64_t)gridDim.x * kTabThreads) {
        if (job < pages) {
            int r;
            Lens x;
            const int64_t c = find(s_need, job, need_of, &r, &x);
            a.table[(int64_t)r * a.max_pages + x.have + c] = ld_index(stack(height - 1 - job));
        } else if (job < pages + pushed) {
            const int64_t v = F + job - pages;
            a.free_list[v] = ld_index(stack(v));
        } else {
            const int64_t j0 = (job - pages - pushed) * PER;
            const int32_t* from[PER];                            // the tokens' pages
            int32_t place[PER];
            int r = 0;
            Lens x{0, 0, 0, 0};
            int64_t pos = 0, needed = 0;
            if (ok && j0 < all.tokens) {
                pos = find(s_tok, j0, tokens_of, &r, &x) + x.old_len;
                needed = s_need[r / per];                        // pages needed by the requests before r
                for (int q = r / per * per; q < r; ++q) needed += lens(q).need();
            }
            int32_t last = -1;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (!ok || j0 + k >= all.tokens) {
                    from[k] = nullptr;
                    place[k] = 0;
                    continue;
                }
                while (pos >= x.new_len) {                       // the next request with new tokens
                    needed += x.need();
                    x = lens(++r);
                    pos = x.old_len;
                    last = -1;
                }
                const int32_t p = (int32_t)div_by((uint32_t)pos, a.page);
                if (k > 0 && p == last) from[k] = from[k - 1];
                else if (p < x.have) from[k] = a.table + (int64_t)r * a.max_pages + p;
                else from[k] = stack(height - 1 - (needed + p - x.have));
                last = p;
                place[k] = (int32_t)(pos - (int64_t)p * a.page.d);
                ++pos;
            }
            int32_t page[PER];
#pragma unroll
            for (int k = 0; k < PER; ++k) page[k] = from[k] != nullptr ? ld_index(from[k]) : 0;
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (j0 + k < a.n_slots) a.slots[j0 + k] = from[k] != nullptr ? (int64_t)page[k] * a.page.d + place[k] : -1;
        }
    }
    if (blockIdx.x == 0) {
        int64_t at = before.tokens;
        for (int r = r0; r < r1; ++r) {
            a.cu_new[r] = ok ? (int32_t)at : 0;
            at += lens(r).tokens();
        }
        if (tid == 0) a.cu_new[a.n_requests] = ok ? (int32_t)all.tokens : 0;
    }
    // what may be updated in place, once every CTA has read it
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0) {
            __threadfence();
            s_last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
            if (s_last) *a.ticket = 0;
        }
        __syncthreads();
        if (!s_last) return;
    }
    for (int r = tid; r < a.n_requests; r += kTabThreads) {
        const int32_t o = ld_index(a.len_old + r), n = ld_index(a.len_new + r);
        a.len_out[r] = ok ? n : o;
    }
    if (tid == 0) *a.n_free_out = ok ? (int32_t)(height - all.need) : F;
}

// ---------------------------------------------------------------------------------- append
// Copies rows to their slots, 16 bytes of the cache a lane; 8-bit caches take 16 values (32 bytes of the row), multiplied by the
// reciprocal of their head's scale, rounded to nearest even and saturated.  Bound by the bytes; for a few tokens by latency.
struct AppendArgs {
    char* K;
    char* V;
    const char* Kn;
    const char* Vn;
    int64_t ld_token, ld_head;        // of the new rows, in bytes
    const int64_t* slots;
    uint32_t n_rows;                  // new tokens times heads, below 2^31
    int64_t n_slots;                  // of the pool
    FastDiv page, heads;
    uint32_t page_u, token_u, head_u;
    const float* k_scale;
    const float* v_scale;
    int32_t* status;
};

constexpr int kAppThreads = 256;

template <bool F16>
__device__ __forceinline__ uint32_t narrow4(uint32_t lo, uint32_t hi, float inv) {
    float2 a, b;
    if (F16) {
        a = __half22float2(*reinterpret_cast<__half2*>(&lo));
        b = __half22float2(*reinterpret_cast<__half2*>(&hi));
    } else {
        a = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&lo));
        b = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&hi));
    }
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(r) : "f"(a.x * inv), "f"(a.y * inv), "f"(b.x * inv), "f"(b.y * inv));
    return r;
}

template <int D, bool F16, bool E4M3>
__global__ void __launch_bounds__(kAppThreads) paged_append_kernel(const AppendArgs a) {
    constexpr int LANES = D * (E4M3 ? 1 : 2) / 16;       // lanes a row
    constexpr int IN = E4M3 ? 32 : 16;                   // bytes of the new row a lane
    grid_dep_wait();
    const uint32_t stride = gridDim.x * (kAppThreads / LANES);
    const int part = threadIdx.x % LANES;
    for (uint32_t i = blockIdx.x * (kAppThreads / LANES) + threadIdx.x / LANES; i < a.n_rows; i += stride) {
        const uint32_t token = div_by(i, a.heads), h = i - token * a.heads.d;
        int64_t slot;
        asm volatile("ld.global.s64 %0, [%1];" : "=l"(slot) : "l"(a.slots + token) : "memory");
        if (slot < 0) continue;
        if (slot >= a.n_slots) {                          // not a place of the pool: left out, and reported
            *a.status = PAFU_ERR_BAD_PAGE;
            continue;
        }
        const uint32_t page = div_by((uint32_t)slot, a.page);
        const uint32_t to = page * a.page_u + ((uint32_t)slot - page * a.page.d) * a.token_u + h * a.head_u;
        const int64_t from = (int64_t)token * a.ld_token + (int64_t)h * a.ld_head + part * IN;
        const uint4 k0 = *reinterpret_cast<const uint4*>(a.Kn + from), v0 = *reinterpret_cast<const uint4*>(a.Vn + from);
        uint4 k = k0, v = v0;
        if (E4M3) {
            const uint4 k1 = *reinterpret_cast<const uint4*>(a.Kn + from + 16), v1 = *reinterpret_cast<const uint4*>(a.Vn + from + 16);
            const float ki = a.k_scale != nullptr ? 1.f / a.k_scale[h] : 1.f, vi = a.v_scale != nullptr ? 1.f / a.v_scale[h] : 1.f;
            k = make_uint4(narrow4<F16>(k0.x, k0.y, ki), narrow4<F16>(k0.z, k0.w, ki), narrow4<F16>(k1.x, k1.y, ki), narrow4<F16>(k1.z, k1.w, ki));
            v = make_uint4(narrow4<F16>(v0.x, v0.y, vi), narrow4<F16>(v0.z, v0.w, vi), narrow4<F16>(v1.x, v1.y, vi), narrow4<F16>(v1.z, v1.w, vi));
        }
        *reinterpret_cast<uint4*>(a.K + (uint64_t)to * 16 + part * 16) = k;
        *reinterpret_cast<uint4*>(a.V + (uint64_t)to * 16 + part * 16) = v;
    }
}

template <int D, bool F16, bool E4M3>
pafu_status append(const AppendArgs& a, cudaStream_t stream) {
    constexpr int ROWS = kAppThreads / (D * (E4M3 ? 1 : 2) / 16);
    const int64_t blocks = ((int64_t)a.n_rows + ROWS - 1) / ROWS;
    const int64_t most = 16ll * device_sm_count();
    return cuda_ok(launch_dependent(paged_append_kernel<D, F16, E4M3>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kAppThreads), 0,
                                    stream, 1, a));
}

}  // namespace

pafu_status launch_paged_tables(const pafu_paged_cache& c, const int32_t* len_old, const int32_t* len_new, int32_t* free_list,
                                const int32_t* n_free, int32_t* n_free_out, int32_t* len_out, int64_t* slots, int64_t n_slots,
                                int32_t* cu_new, void* ws, cudaStream_t stream) {
    TablesArgs a;
    a.table = c.table;
    a.max_pages = c.max_pages;
    a.n_requests = c.n_requests;
    a.n_pages = (uint32_t)c.n_pages;
    a.page = fast_div((uint32_t)c.page_size);
    a.len_old = len_old;
    a.len_new = len_new;
    a.free_list = free_list;
    a.n_free = n_free;
    a.n_free_out = n_free_out;
    a.len_out = len_out;
    a.slots = slots;
    a.n_slots = n_slots;
    a.cu_new = cu_new;
    a.status = static_cast<int32_t*>(ws) + kStatusWordPaged;
    a.ticket = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + kWsHeaderBytes) + kPagedTickets - 1;
    // Eight tokens a thread once one each would take more than 32 CTAs: a step of 2000 requests and 360000 tokens takes 9 us so
    // and 19 with one, one of 256 single tokens 4.3 and 5.5.
    const bool runs = n_slots > 32 * kTabThreads;
    const int64_t jobs = (runs ? n_slots / 8 : n_slots) + c.n_requests / 4, want = (jobs + kTabThreads - 1) / kTabThreads;
    const int64_t most = device_sm_count(), grid = want < 1 ? 1 : want < most ? want : most;
    return cuda_ok(launch_dependent(runs ? paged_tables_kernel<8> : paged_tables_kernel<1>, dim3((unsigned)grid), dim3(kTabThreads), 0, stream, 1, a));
}

pafu_status launch_paged_append(const pafu_paged_cache& c, const void* Kn, const void* Vn, int64_t ld_token, int64_t ld_head,
                                const int64_t* slots, int64_t n_tokens, void* ws, cudaStream_t stream) {
    const PagedPool p = pool_of(c);
    AppendArgs a;
    a.K = static_cast<char*>(c.K);
    a.V = static_cast<char*>(c.V);
    a.Kn = static_cast<const char*>(Kn);
    a.Vn = static_cast<const char*>(Vn);
    a.ld_token = ld_token * 2;
    a.ld_head = ld_head * 2;
    a.slots = slots;
    a.n_rows = (uint32_t)(n_tokens * c.n_kv_heads);
    a.n_slots = c.n_pages * c.page_size;
    a.page = p.page;
    a.heads = fast_div((uint32_t)c.n_kv_heads);
    a.page_u = p.page_u;
    a.token_u = p.token_u;
    a.head_u = p.head_u;
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.status = static_cast<int32_t*>(ws) + kStatusWordPaged;
    const bool f16 = c.type == PAFU_TYPE_F16, e4m3 = c.cache_type == PAFU_TYPE_E4M3;
    if (c.d_head == 128) {
        if (e4m3) return f16 ? append<128, true, true>(a, stream) : append<128, false, true>(a, stream);
        return append<128, false, false>(a, stream);            // 16-bit rows are copied as they are
    }
    if (e4m3) return f16 ? append<64, true, true>(a, stream) : append<64, false, true>(a, stream);
    return append<64, false, false>(a, stream);
}

}  // namespace pafu
