// Block tables, slot map and rows of the paged cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "paged.cuh"

namespace pafu {

namespace {

// ---------------------------------------------------------------------------------- tables
// From the lengths before and after a step: which pages each request gives back and gets, where its new tokens go.
// All of it follows from prefix sums over the requests (pages needed, pages given back, new tokens, and the runs below), so every
// CTA computes them for itself - each thread sums a stretch of requests, one scan of the threads' sums - and then takes its part of
// what there is to write.  The unit is a run: new tokens of a request that lie in the same stretch of sixteen places of a page.  A
// thread finds its run by a binary search in the threads' sums and a walk through one stretch of requests, looks up the page once,
// writes the run's slots, and the table entry where the run begins a new page.
// That keeps a step one launch: nothing a CTA reads is written by another (a request that grows only gets table
// entries behind those that are read, the free list only entries above its top), apart from the lengths and the free count,
// which may be updated in place; the CTA that counts itself out last writes those.  A step moves a few KB to MB: the
// trips to memory and the searches that follow one another bound it.  2000 requests with 360000 new tokens: 11.9 us, 19 with a search
// and a lookup for every token; 256 requests with one token each: 4.5 us, of which 1.9 are the lengths and the scan.
constexpr int kTabThreads = 512;
constexpr int kTabRun = 16;           // tokens of a run, at most

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
    int64_t need, back, tokens, runs;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
    return Sums{a.need + b.need, a.back + b.back, a.tokens + b.tokens, a.runs + b.runs};
}

__device__ __forceinline__ int32_t pages_of(const FastDiv& page, int32_t len) {
    return len <= 0 ? 0 : (int32_t)div_by((uint32_t)(len - 1), page) + 1;
}

__global__ void __launch_bounds__(kTabThreads) paged_tables_kernel(const TablesArgs a) {
    __shared__ uint32_t s_back[kTabThreads], s_runs[kTabThreads], s_need[kTabThreads], s_tok[kTabThreads];
    __shared__ Sums s_warp[kTabThreads / 32];
    __shared__ int32_t s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int32_t per_page = (int32_t)((a.page.d + kTabRun - 1) / kTabRun);         // runs of a full page
    grid_dep_wait();
    const int per = (a.n_requests + kTabThreads - 1) / kTabThreads;
    auto lens_of = [&](int32_t before, int32_t after) {
        return Lens{before, after, pages_of(a.page, before), pages_of(a.page, after)};
    };
    auto lens = [&](int r) { return lens_of(ld_index(a.len_old + r), ld_index(a.len_new + r)); };
    // number of the run that position `pos` is in, counted from the request's first position
    auto run_at = [&](int32_t pos) {
        const int32_t p = (int32_t)div_by((uint32_t)pos, a.page);
        return p * per_page + (pos - p * (int32_t)a.page.d) / kTabRun;
    };
    auto runs_of = [&](const Lens& x) { return x.tokens() > 0 ? run_at(x.new_len - 1) - run_at(x.old_len) + 1 : 0; };
    const int32_t F = ld_index(a.n_free);
    const int r0 = min(tid * per, a.n_requests), r1 = min(r0 + per, a.n_requests);
    Sums mine{0, 0, 0, 0};
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
            const bool wrong = x.old_len < 0 || x.new_len < 0 || x.have > a.max_pages || x.want > a.max_pages;
            bad |= wrong;
            if (!wrong) mine = mine + Sums{x.need(), x.back(), x.tokens(), runs_of(x)};
        }
    }
    Sums inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums v{__shfl_up_sync(0xffffffffu, inc.need, o), __shfl_up_sync(0xffffffffu, inc.back, o),
                     __shfl_up_sync(0xffffffffu, inc.tokens, o), __shfl_up_sync(0xffffffffu, inc.runs, o)};
        if (lane >= o) inc = inc + v;
    }
    if (lane == 31) s_warp[warp] = inc;
    bad = __syncthreads_or(bad);
    Sums all{0, 0, 0, 0}, before{inc.need - mine.need, inc.back - mine.back, inc.tokens - mine.tokens, inc.runs - mine.runs};
    for (int w = 0; w < kTabThreads / 32; ++w) {
        if (w < warp) before = before + s_warp[w];
        all = all + s_warp[w];
    }
    s_need[tid] = (uint32_t)before.need;
    s_back[tid] = (uint32_t)before.back;
    s_tok[tid] = (uint32_t)before.tokens;
    s_runs[tid] = (uint32_t)before.runs;
    __syncthreads();
    // all or nothing: every page must exist, every token have a place in the slot map
    const int64_t height = (int64_t)F + all.back;               // of the stack, with what is given back on top
    const bool short_of = all.need > height || all.tokens > a.n_slots;
    // (a step that passes gives back fewer than 2^32 pages and has fewer than 2^31 of everything else)
    const bool ok = !bad && !short_of && height - all.need <= (int64_t)a.n_pages;
    if (!ok && blockIdx.x == 0 && tid == 0) *a.status = bad || !short_of ? PAFU_ERR_BAD_PAGE : PAFU_ERR_NO_PAGES;

    // the last thread whose sum is <= i
    auto stretch = [&](const uint32_t* sums, uint32_t i) {
        int lo = 0, hi = kTabThreads - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (sums[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    };
    // where entry v of the stack lies: in the free list, then the pages given back in the order of requests and columns
    auto stack = [&](int64_t v) -> const int32_t* {
        if (v < F) return a.free_list + v;
        const int at = stretch(s_back, (uint32_t)(v - F));
        uint32_t i = (uint32_t)(v - F) - s_back[at];
        int r = at * per;
        Lens x = lens(r);
        while (i >= (uint32_t)x.back()) {
            i -= x.back();
            x = lens(++r);
        }
        return a.table + (int64_t)r * a.max_pages + x.want + i;
    };
    // what is no page of the pool is handed on as it stands, and reported
    auto is_page = [&](int32_t page) {
        const bool yes = (uint32_t)page < a.n_pages;
        if (!yes) *a.status = PAFU_ERR_BAD_PAGE;
        return yes;
    };
    // runs, entries of the free list, and the slot map's end side by side: no thread does one after the other
    const int64_t runs = ok ? all.runs : 0, pushed = ok ? max(height - all.need - F, (int64_t)0) : 0;
    const int64_t filled = ok ? all.tokens : 0, jobs = runs + pushed + (a.n_slots - filled + kTabRun - 1) / kTabRun;
    for (int64_t job = (int64_t)blockIdx.x * kTabThreads + tid; job < jobs; job += (int64_t)gridDim.x * kTabThreads) {
        if (job < runs) {
            const int at = stretch(s_runs, (uint32_t)job);
            int32_t i = (int32_t)((uint32_t)job - s_runs[at]);
            uint32_t needed = s_need[at], token = s_tok[at];
            int r = at * per;
            Lens x = lens(r);
            while (i >= runs_of(x)) {
                i -= runs_of(x);
                needed += x.need();
                token += x.tokens();
                x = lens(++r);
            }
            const int32_t run = run_at(x.old_len) + i, p = run / per_page, first = p * (int32_t)a.page.d + (run - p * per_page) * kTabRun;
            const int32_t last = min(min(first + kTabRun, (p + 1) * (int32_t)a.page.d), x.new_len), pos = max(first, x.old_len);
            int32_t* entry = a.table + (int64_t)r * a.max_pages + p;
            const int32_t page = ld_index(p < x.have ? entry : stack(height - 1 - ((int64_t)needed + p - x.have)));
            if (p >= x.have && first == p * (int32_t)a.page.d) *entry = page;
            const bool place = is_page(page);                 // -1 otherwise: no slot, and not one that the append would take for padding unseen
            const int64_t slot = (int64_t)page * a.page.d + (pos - p * (int32_t)a.page.d);
            int64_t* to = a.slots + token + (pos - x.old_len);
            for (int k = 0; k < last - pos; ++k) to[k] = place ? slot + k : -1;
        } else if (job < runs + pushed) {
            const int64_t v = F + job - runs;
            const int32_t page = ld_index(stack(v));
            is_page(page);
            a.free_list[v] = page;
        } else {
            const int64_t first = filled + (job - runs - pushed) * kTabRun;
            for (int64_t k = first; k < min(first + kTabRun, a.n_slots); ++k) a.slots[k] = -1;
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
    // What may be updated in place, once every CTA has read it.  (No fence, which would wait for the slots' stores to arrive, 4 us: what was
    // read has been used, and what the other CTAs wrote is not looked at.)
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0) {
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
// Copies rows to their slots, 16 bytes of the cache a lane; 8-bit caches take 16 values (32 bytes of the row), divided by their
// head's scale, rounded to nearest even and saturated.  Bound by the bytes (28080 rows of 12 x 128, bf16 to e4m3: 37 to 39 us, 6.1 to 5.8 TB/s; 4680 of
// 40 x 128 copied: 27 us, 6.2 TB/s); for a few tokens by latency.
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

constexpr int kAppThreads = 128;

// x / scale, as far as rounding to e4m3 goes.  The product with the reciprocal is within 2 ulp of the quotient, so the two can only round
// apart where the product is within 4 ulp of a border between e4m3 values (five significant bits at most: 19 zeros follow); there
// the sign of x - border * scale, which one fused operation gives exactly, says on which side the quotient lies.
__device__ __forceinline__ uint32_t beside_border(float q) { return (__float_as_uint(q) << 13) + (4u << 13); }
constexpr uint32_t kBeside = 8u << 13;             // at most that: it is
__device__ __forceinline__ float quotient(float x, float q, float scale) {
    if (beside_border(q) > kBeside || !(fabsf(q) < INFINITY)) return q;
    const float border = __uint_as_float((__float_as_uint(q) + 4u) & ~0x7ffffu), rest = fmaf(-border, scale, x);
    if (rest == 0.f) return border;
    return border * ((rest > 0.f) == (border > 0.f) ? 1.f + 0x1p-20f : 1.f - 0x1p-20f);
}

template <bool F16>
__device__ __forceinline__ float2 widen16(uint32_t v) {
    if (F16) return __half22float2(*reinterpret_cast<__half2*>(&v));
    return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&v));
}

// Sixteen values.  (The test is made once for them: with a scale of full mantissa one value in 60000 is beside a border.  28080 rows: 35.0 us without
// it, 37.0 with it, 39.3 with a test for each.  Without a scale, or with a power of two, one bf16 value in 8 and one fp16 value in 64 lies
// on that grid, and zeros always do: every warp then takes the second loop, for quotients that were exact.  66 us for bf16 rows, 52 for fp16.)
template <bool F16>
__device__ __forceinline__ uint4 narrow16(const uint4& x, const uint4& y, float scale) {
    const uint32_t in[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    const float inv = 1.f / scale;
    float q[16];
    uint32_t nearest = ~0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 v = widen16<F16>(in[i]);
        q[2 * i] = v.x * inv;
        q[2 * i + 1] = v.y * inv;
        nearest = __vimin3_u32(nearest, beside_border(q[2 * i]), beside_border(q[2 * i + 1]));
    }
    if (nearest <= kBeside) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 v = widen16<F16>(in[i]);
            q[2 * i] = quotient(v.x, q[2 * i], scale);
            q[2 * i + 1] = quotient(v.y, q[2 * i + 1], scale);
        }
    }
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("{\n\t.reg .b16 l, h;\n\t"
            "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
            : "=r"(r[i]) : "f"(q[4 * i]), "f"(q[4 * i + 1]), "f"(q[4 * i + 2]), "f"(q[4 * i + 3]));
    return make_uint4(r[0], r[1], r[2], r[3]);
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
            k = narrow16<F16>(k0, k1, a.k_scale != nullptr ? a.k_scale[h] : 1.f);
            v = narrow16<F16>(v0, v1, a.v_scale != nullptr ? a.v_scale[h] : 1.f);
        }
        *reinterpret_cast<uint4*>(a.K + (uint64_t)to * 16 + part * 16) = k;
        *reinterpret_cast<uint4*>(a.V + (uint64_t)to * 16 + part * 16) = v;
    }
}

template <int D, bool F16, bool E4M3>
pafu_status append(const AppendArgs& a, cudaStream_t stream) {
    constexpr int ROWS = kAppThreads / (D * (E4M3 ? 1 : 2) / 16);
    const int64_t blocks = ((int64_t)a.n_rows + ROWS - 1) / ROWS;
    const int64_t most = 64ll * device_sm_count();       // four times what runs at once: 2 % quicker than one round
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
    // A CTA for every 192 jobs that the slots and requests may make, where one does not do; jobs are runs, mostly.  Jobs go to the CTAs 512 at a
    // time, so the first ones take 512 each and the others none where there are fewer: with 360000 new tokens 48 of 148 work.  Pages given back are not
    // in the count: 64 requests of 200000 tokens that end, 800000 pages, take 1340 us beside a slot map of 16 places, one CTA, and 19 us beside one
    // of 200000.
    const int64_t jobs = n_slots / (kTabRun / 2) + c.n_requests, want = jobs <= kTabThreads ? 1 : (jobs + 191) / 192;
    const int64_t most = device_sm_count(), grid = want < most ? want : most;
    return cuda_ok(launch_dependent(paged_tables_kernel, dim3((unsigned)grid), dim3(kTabThreads), 0, stream, 1, a));
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
