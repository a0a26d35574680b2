// Attention of one new token a request over a paged cache: for request r and query head n
//   o = sum_j softmax_j(scale * q . k_j) v_j,   j over the kept positions [0, n_sink) U [T - n_recent, T).
//
// Every key is used by the n_heads / n_kv_heads query heads of its group, 2 flop a byte and head: the cache's bytes bound
// the call, and what a kernel has to do is keep enough of them on their way.  So nothing is staged: a warp's lanes load
// 16-byte pieces of the rows straight into the registers in which mma.sync wants them.  Keys are the rows of S^T = K Q^T and
// the d_head components the rows of O^T = V^T P^T, heads the columns, eight a product: the accumulators of O^T then take half the registers
// that O with 16 rows for at most eight heads would.  The order of the contraction index is free as long as both
// operands follow it, so a lane's 16 contiguous bytes of a key row serve as parts of two (8 bits: four) fragments, and the
// queries are loaded in the same order; the order of O^T's rows is free too, so eight neighbouring lanes read a 128-byte line of a
// value row and a byte permute pairs the rows of two keys.  P goes from S^T's layout to the other product's by 8 x 8 transposes
// in registers.  The rows' addresses come from the page table one tile ahead, so pages of any length, order and
// stride cost the same and may end inside a tile.
// Probabilities p <= 1 enter the product as 16-bit values.  For bf16 what that rounding leaves over follows in a second product
// (2^-17 of a probability is lost then).  fp16 (fp16 and 8-bit pages) rounds 2^15 p, so that its whole exponent range counts: at most 2^-11 of p is
// lost, as rounding an fp16 output loses, or 2^-40 of the largest probability where p is below 2^-29 of it.  (p itself would be a subnormal below
// 2^-14 and nothing below 2^-25: beside a first token that draws the attention that is every other one.)  A second product for fp16 pages,
// measured: 0.3 to 0.7 % longer for up to 8 heads a key head, 5 % for 16, against errors that mostly cancel over the keys: left out.
// 8-bit caches are widened to fp16, which holds every e4m3 value; bf16 queries are scaled by a power of two a row so that
// their largest component lies in [2^14, 2^15) and fp16 holds them to 2^-39 of it.
// Measured: 64 requests of up to 8192 tokens, 32 heads over 8 key heads, 128, bf16 (1.15 GB): 179 us, 6.4 TB/s; 8 bits (0.57 GB, 40 over 8
// heads): 96 us, 5.9 TB/s, where widening takes 42 % of the ALU pipe (37 % of the issue slots are used).  The tensor cores are 14 to 18 % busy, so mma.sync's rate does
// not bound it, and tcgen05 would need its rows in shared memory and P's transpose through tensor memory.  Staging the rows in
// shared memory by cp.async instead (built: fragments from there, 8 and 16 KB a warp under way): 185 us with 12 warps an SM and 8 KB, 243 with 16 KB, since
// what is left of L1 no longer holds tables and spills, 181 with 8 warps and 16 KB; 8 bits 105, 151, 99.
//
// Split over the length: every (request, group of heads) is an item of ceil(kept / step) steps (a step is one tile for each of
// the four warps) and a fixed cost.  All items laid end to end are cut into equal shares, one a CTA, by arithmetic that every
// CTA does for itself from the lengths on the device: the grid does not depend on the lengths, and a captured launch follows
// them.  A cut that would leave few steps of an item on one side moves to the item's end.  A share's first and last
// item may continue in other CTAs: their fp32 partial results go to the workspace, and the CTA that arrives last
// (a counter; nothing waits) joins them in a fixed order, so results do not depend on timing; more than 16 pieces are joined
// in groups of 16 first, by as many CTAs.
// Where no item has more than two tiles and there are more items than CTAs, a warp takes whole items by itself ("solo"): nothing is
// joined, no warp is idle on an item of few keys.  12000 items of up to 10 keys of 128: 66.8 us with four warps an item, 24.2 so.  From four
// tiles on (2400 items of up to 64 keys) both take 24 us, and with fewer items than CTAs four warps are quicker.  (One longer request is enough to have
// four warps an item again: 300 requests of up to 10 tokens, 40 heads, and one of 1000: 83 us.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "paged.cuh"

namespace pafu {

namespace {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = kPaWarps * 32;
constexpr int kPaJoin = 16;           // pieces that are joined at once
constexpr float kPaLift = 15.f;       // power of two that lifts fp16 probabilities, and with them numerators and a lane's sums
static_assert(3 * kPaTicketRow < kPagedTickets, "three counters a CTA, and the tables' own");

struct PagedAttnArgs {
    PagedPool pool;
    const char* Q;
    int64_t q_token, q_head;          // bytes
    const int32_t* lens;
    int32_t n_requests, n_heads, n_kv, group, parts;      // parts: items that share a key head (16 query heads each)
    int32_t sink, recent;             // recent < 0: every position
    float scale;                      // scale * log2(e)
    const float* k_scale;
    const float* v_scale;
    char* O;
    float* LSE;
    int32_t* status;
    int32_t* tickets;
    float* part;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 16 (8) bytes of a row, or zeros.  Not through the read-only path: the append ahead may still write these rows while this kernel is
// already resident (the times are the same).  Predicated in one piece: as a branch, or with a second copy of the loads for whole tiles, the loop
// over the keys runs 4 to 8 % longer.  Rows of 64 bytes are fetched as such: two heads of a token share a 128-byte line, but
// come at different times (16 heads of 64 in 8 bits, 1.08 GB: 365 us with whole lines, 343 so).
#define PAFU_LD_ROW(HINT)                                                                                       \
    __device__ __forceinline__ void ld_row##HINT(uint32_t (&w)[4], const char* p, bool ok) {                    \
        w[0] = w[1] = w[2] = w[3] = 0u;                                                                         \
        asm volatile("{\n\t.reg .pred P;\n\tsetp.ne.b32 P, %5, 0;\n\t"                                          \
                     "@P ld.global.L1::no_allocate.L2::" #HINT "B.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"       \
                     : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]) : "l"(p), "r"((int)ok) : "memory");       \
    }                                                                                                           \
    __device__ __forceinline__ void ld_row##HINT(uint32_t (&w)[2], const char* p, bool ok) {                    \
        w[0] = w[1] = 0u;                                                                                       \
        asm volatile("{\n\t.reg .pred P;\n\tsetp.ne.b32 P, %3, 0;\n\t"                                          \
                     "@P ld.global.L1::no_allocate.L2::" #HINT "B.v2.u32 {%0, %1}, [%2];\n\t}"               \
                     : "+r"(w[0]), "+r"(w[1]) : "l"(p), "r"((int)ok) : "memory");                               \
    }
PAFU_LD_ROW(64)
PAFU_LD_ROW(128)
#undef PAFU_LD_ROW
template <int ROW, int N>
__device__ __forceinline__ void ld_row(uint32_t (&w)[N], const char* p, bool ok) {
    if (ROW <= 64) ld_row64(w, p, ok);
    else ld_row128(w, p, ok);
}

template <bool F16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (F16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// an 8 x 8 matrix of 16-bit values, a row of four lanes' pairs each, transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// two fp32 values as a pair of 16-bit ones, the first in the low half
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
    if (F16) {
        __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<uint32_t*>(&h);
    }
    __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<uint32_t*>(&h);
}
template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
    if (F16) return __half22float2(*reinterpret_cast<__half2*>(&v));
    return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&v));
}

// four e4m3 values as two pairs of fp16 ones
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
}

// Position of the kept keys of a request and their number.
struct Kept {
    int32_t n, sink, shift;
};
__device__ __forceinline__ Kept kept_of(const PagedAttnArgs& a, int32_t T) {
    const int64_t most = (int64_t)a.pool.max_pages * a.pool.page.d;
    if (T < 0 || T > most) {                       // a length that the table cannot hold: its part is used, and reported
        *a.status = PAFU_ERR_BAD_PAGE;
        T = T < 0 ? 0 : (int32_t)most;
    }
    const int64_t window = (int64_t)a.sink + a.recent;
    Kept k;
    k.n = a.recent < 0 || window > T ? T : (int32_t)window;
    k.sink = a.sink;
    k.shift = T - k.n;
    return k;
}

template <int D, bool F16Q, bool E4M3, int HG>
struct Tile {
    static constexpr int ES = E4M3 ? 1 : 2;
    // Keys of a warp's tile: 4 to 8 KB of K and V in flight a warp.  (Half as many: no difference at rows of 256 bytes, which the bytes
    // bound; 6 to 28 % longer at the others, which issue more instructions a byte.)
    static constexpr int KT = D * ES >= 256 ? 16 : 32;
    static constexpr int KR = KT / 8;                             // key rows that a lane has a part of
    static constexpr int KW = D * ES / 16;                        // words of each
    static constexpr int VR = KT / 4;                             // value rows
    static constexpr int VB = D * ES / 8 < 16 ? 8 : 16;           // bytes of a value load
    static constexpr int VC = D * ES / 8 / VB;                    // loads a value row
    static constexpr int VE = VB / ES;                            // elements of a value load
    static constexpr int NT = D / 16;                             // row tiles of O^T
    static constexpr int STEP = KT * kPaWarps;
    static constexpr bool F16 = F16Q || E4M3;                     // type of the products
    static constexpr int ROWS = HG * 8;
    static constexpr int LD = D + 4;
    static constexpr int CTAS = HG * D <= 128 ? 3 : 2;            // an SM: 168 or 255 registers a thread
    static constexpr size_t SMEM = sizeof(float) * (kPaWarps * ROWS * LD + 2 * kPaWarps * ROWS);
    static_assert(KT % 16 == 0 && VE % 4 == 0, "fragments");
};

// Address of a key: its row of the pools in 16-byte units (head included), or ~0
struct KeyAt {
    int32_t page;          // table entry, still to be looked at
    uint32_t in_page;      // 16-byte units within the page; ~0: no such key
};
__device__ __forceinline__ KeyAt key_at(const PagedAttnArgs& a, const Kept& k, const int32_t* row, int32_t j, uint32_t head_u) {
    KeyAt x{0, ~0u};
    if (j < k.n) {
        const uint32_t pos = (uint32_t)(j < k.sink ? j : j + k.shift);
        const uint32_t pg = div_by(pos, a.pool.page);
        x.page = ld_index(row + pg);
        x.in_page = (pos - pg * a.pool.page.d) * a.pool.token_u + head_u;
    }
    return x;
}
__device__ __forceinline__ uint32_t key_offset(const PagedAttnArgs& a, const KeyAt& x) {
    if (x.in_page == ~0u) return ~0u;
    if ((uint32_t)x.page >= a.pool.n_pages) {      // not a page: the key is left out, and reported
        *a.status = PAFU_ERR_BAD_PAGE;
        return ~0u;
    }
    return (uint32_t)x.page * a.pool.page_u + x.in_page;
}

// Where a CTA begins or ends: a position on the line of all items, and the request and item it lies in.
struct Cut {
    uint64_t at, item_at;     // the position; where its item begins
    int32_t r, item;
};
// A CTA's part of an item: steps [lo, hi) of `steps`; pos: where the item begins, seen from the CTA's first position.  Solo: a warp's
// item, hi tiles from 0.
struct Work {
    int32_t r, item, pos, steps, lo, hi;
    Kept kept;
};

// Where an item's heads go, and how
template <int D, bool F16Q>
struct Rows {
    char* O;
    float* LSE;
    int32_t lse_stride;
    float v_scale;
    template <int PER>
    __device__ __forceinline__ void store(int row, int d, const float (&x)[PER], float top, float sum) const {
        const float inv = sum == 0.f ? 0.f : v_scale / sum;
        uint32_t w[PER / 2];
#pragma unroll
        for (int i = 0; i < PER / 2; ++i) w[i] = pack2<F16Q>(x[2 * i] * inv, x[2 * i + 1] * inv);
        char* to = O + ((int64_t)row * D + d) * 2;
        if (PER == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[PER / 2 - 1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
        if (LSE != nullptr && d == 0) LSE[(int64_t)row * lse_stride] = top * 0.6931471805599453f + logf(sum);
    }
};
// A piece's results in the workspace: numerators, maxima, sums
template <int D>
constexpr size_t kPartWords = (size_t)kPagedRows * (D + 2);
template <int D, int PER>
__device__ __forceinline__ void put_part(float* part, int row, int d, const float (&x)[PER], float top, float sum) {
    if (PER == 4) *reinterpret_cast<float4*>(part + row * D + d) = make_float4(x[0], x[1], x[PER - 2], x[PER - 1]);
    else *reinterpret_cast<float2*>(part + row * D + d) = make_float2(x[0], x[1]);
    if (d == 0) {
        part[kPagedRows * D + row] = top;
        part[kPagedRows * D + kPagedRows + row] = sum;
    }
}

// Pieces p0, p0 + by, ... (count <= kPaJoin) of the item whose first piece is CTA `first`'s, joined by the whole CTA: to the output, or in
// place of piece p0.  One trip to L2 for a warp's rows: everything is requested before anything is used.  A call, so that its registers do not
// count in the loop over the keys.
template <int D, bool F16Q>
__device__ __noinline__ void join_pieces(float* parts, int first, int p0, int by, int count, int rows, const Rows<D, F16Q>* out) {
    constexpr int PER = D / 32;                              // columns a lane: a warp has a row
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = lane * PER;
    auto piece = [&](int i) { const int p = p0 + i * by; return parts + (2 * (size_t)(first + p) + (p == 0)) * kPartWords<D>; };
    for (int row = warp; row < rows; row += kPaWarps) {
        float y[kPaJoin][PER], m[kPaJoin], l[kPaJoin];
#pragma unroll
        for (int p = 0; p < kPaJoin; ++p) {
            m[p] = -INFINITY;
            l[p] = 0.f;
#pragma unroll
            for (int k = 0; k < PER; ++k) y[p][k] = 0.f;
            if (p < count) {
                const float* q = piece(p);
                m[p] = __ldcg(q + kPagedRows * D + row);
                l[p] = __ldcg(q + kPagedRows * D + kPagedRows + row);
                if (PER == 4) {
                    const float4 v = __ldcg(reinterpret_cast<const float4*>(q + row * D + d));
                    y[p][0] = v.x, y[p][1] = v.y, y[p][PER - 2] = v.z, y[p][PER - 1] = v.w;
                } else {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(q + row * D + d));
                    y[p][0] = v.x, y[p][1] = v.y;
                }
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int p = 0; p < kPaJoin; ++p) top = fmaxf(top, m[p]);
        const float base = top == -INFINITY ? 0.f : top;
        float x[PER] = {}, sum = 0.f;
#pragma unroll
        for (int p = 0; p < kPaJoin; ++p) {
            const float f = ex2(m[p] - base);
            sum += f * l[p];
#pragma unroll
            for (int k = 0; k < PER; ++k) x[k] += f * y[p][k];
        }
        if (out != nullptr) {
            out->store(row, d, x, top, sum);
        } else {
            __syncwarp();                                    // every lane has read piece p0's maximum and sum, which lane 0 overwrites
            put_part<D>(piece(0), row, d, x, top, sum);
        }
    }
}

// The CTA's items (SOLO: the warp's), one after the other.
template <int D, bool F16Q, bool E4M3, int HG, bool SOLO>
__device__ __forceinline__ void attend(const PagedAttnArgs& a, const PagedCuts& plan, const Cut (&cuts)[2], float* sm, int32_t& last_flag) {
    using C = Tile<D, F16Q, E4M3, HG>;
    constexpr bool solo = SOLO;
    float* sO = sm;                                   // [warp][row][LD]
    float* sM = sm + kPaWarps * C::ROWS * C::LD;      // [warp][row]
    float* sL = sM + kPaWarps * C::ROWS;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int H = a.n_kv * a.parts;                   // items a request
    auto kept_at = [&](int r) { return kept_of(a, ld_index(a.lens + r)); };
    auto steps_of = [](const Kept& k) { return max((k.n + C::STEP - 1) / C::STEP, 1); };
    auto tiles_of = [](const Kept& k) { return (k.n + C::KT - 1) / C::KT; };
    const int n_items = a.n_requests * H, workers = kPaWarps * gridDim.x, worker = warp * gridDim.x + blockIdx.x;
    const int length = solo ? 0 : (int)((int64_t)cuts[1].at - (int64_t)cuts[0].at);
    if (solo ? worker >= n_items : length <= 0) return;

    auto enter = [&](Work& w) {
        if (solo) {
            w.lo = 0;
            w.hi = w.steps = max(tiles_of(w.kept), 1);
            return;
        }
        w.steps = steps_of(w.kept);
        w.lo = max(-w.pos, 0);
        w.hi = min(w.steps, length - w.pos);
    };
    auto advance = [&](const Work& w, Work& x) {
        x = w;
        if (solo) {
            if (workers >= n_items - (w.r * H + w.item)) return false;
            const int i = w.r * H + w.item + workers;
            x.r = i / H;
            x.item = i - x.r * H;
            x.kept = kept_at(x.r);
            enter(x);
            return true;
        }
        x.pos = w.pos + w.steps + kPaItemCost;
        if (x.pos >= length) return false;
        if (++x.item == H) {
            x.item = 0;
            if (++x.r == a.n_requests) return false;
            x.kept = kept_at(x.r);
        }
        enter(x);
        return true;
    };
    Work w;
    w.r = solo ? worker / H : cuts[0].r;
    w.item = solo ? worker % H : cuts[0].item;
    w.pos = solo ? 0 : (int)((int64_t)cuts[0].item_at - (int64_t)cuts[0].at);
    w.kept = kept_at(w.r);
    enter(w);

    // ---- rows and queries on their way
    uint32_t K[C::KR][C::KW / 4][4], V[C::VR][C::VC][C::VB / 4], qf[HG][D / 16][2];
    auto load_K = [&](uint32_t off) {
#pragma unroll
        for (int i = 0; i < C::KR; ++i) {
            const uint32_t o = __shfl_sync(0xffffffffu, off, i * 8 + g);
            const char* p = a.pool.K + (uint64_t)o * 16 + t * 16;
#pragma unroll
            for (int c = 0; c < C::KW / 4; ++c) {
                ld_row<D * C::ES>(K[i][c], p + c * 64, o != ~0u);
            }
        }
    };
    auto load_V = [&](uint32_t off) {
#pragma unroll
        for (int i = 0; i < C::VR; ++i) {
            const uint32_t o = __shfl_sync(0xffffffffu, off, (i >> 2) * 16 + ((i >> 1) & 1) * 8 + 2 * t + (i & 1));
            const char* p = a.pool.V + (uint64_t)o * 16 + g * C::VB;
#pragma unroll
            for (int c = 0; c < C::VC; ++c) {
                ld_row<D * C::ES>(V[i][c], p + c * 8 * C::VB, o != ~0u);
            }
        }
    };
    constexpr uint32_t kFull = C::KT == 32 ? ~0u : (1u << C::KT % 32) - 1u;
    auto valid_of = [&](uint32_t off) { return __ballot_sync(0xffffffffu, off != ~0u) & kFull; };
    // key `j` of the item's kept ones, if it is one of this CTA's
    auto ask = [&](const Work& w, int32_t j) {
        return key_at(a, w.kept, a.pool.table + (int64_t)w.r * a.pool.max_pages, solo || j < w.hi * C::STEP ? j : 0x7fffffff,
                      (uint32_t)(w.item / a.parts) * a.pool.head_u);
    };
    const int stride = solo ? C::KT : C::STEP;
    auto first_key = [&](const Work& w) { return (solo ? 0 : (w.lo * kPaWarps + warp) * C::KT) + (lane & (C::KT - 1)); };
    // the item's first query head, and how many heads it has
    auto head0_of = [&](const Work& w) { const int kv = w.item / a.parts; return kv * a.group + (w.item - kv * a.parts) * kPagedRows; };
    auto rows_of = [&](const Work& w) { return min(kPagedRows, (w.item / a.parts + 1) * a.group - head0_of(w)); };
    // queries: head g (and g + 8), in the order in which the lane's key words come
    auto load_Q = [&](const Work& w) {
        const int head0 = head0_of(w), rows = rows_of(w);
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            const bool have = hg * 8 + g < rows;
            const char* qp = a.Q + w.r * a.q_token + (int64_t)(head0 + hg * 8 + g) * a.q_head;
#pragma unroll
            for (int c = 0; c < C::KW / 4; ++c) {
                constexpr int PER = 16 / C::ES;       // elements of 16 bytes of a key row
                const char* p = qp + (c * 4 * PER + t * PER) * 2;
#pragma unroll
                for (int h = 0; h < PER / 8; ++h) {
                    uint32_t q[4];
                    ld_row<D * 2>(q, p + h * 16, have);
                    const int ks = c * (PER / 4) + h * 2;
                    qf[hg][ks][0] = q[0];
                    qf[hg][ks][1] = q[1];
                    qf[hg][ks + 1][0] = q[2];
                    qf[hg][ks + 1][1] = q[3];
                }
            }
        }
    };

    int32_t j = first_key(w);
    uint32_t off = key_offset(a, ask(w, j));
    KeyAt next = ask(w, j + stride);
    uint32_t valid = valid_of(off);
    load_K(off);
    load_V(off);
    load_Q(w);

    while (true) {
        // the next item's first rows are looked up now and requested behind this item's last ones
        Work x;
        const bool another = advance(w, x);
        const KeyAt x_key = another ? ask(x, first_key(x)) : KeyAt{0, ~0u};

        float c_col[HG][2];                           // factor of the logits of heads 2t, 2t + 1
        const int kv = w.item / a.parts;
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) {
            float c_row = a.scale;
            if (E4M3 && a.k_scale != nullptr) c_row *= a.k_scale[kv];
            if (E4M3 && !F16Q) {
                float top = 0.f;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 v = unpack2<false>(qf[hg][ks][i]);
                        top = fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y)));
                    }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^(14 - e) with e the exponent of the largest component; rows of zeros or with infinities stay
                const int e = (int)(__float_as_uint(top) >> 23);
                const int up = e == 0 || e == 255 ? 0 : min(14 + 127 - e, 100);
                const float f = __uint_as_float((uint32_t)(up + 127) << 23);
                c_row *= __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 v = unpack2<false>(qf[hg][ks][i]);
                        qf[hg][ks][i] = pack2<true>(v.x * f, v.y * f);
                    }
            }
            c_row = fmaxf(c_row, 1e-37f);             // -inf times it stays -inf: a scale of 0 makes all logits equal
            c_col[hg][0] = __shfl_sync(0xffffffffu, c_row, 8 * t);
            c_col[hg][1] = __shfl_sync(0xffffffffu, c_row, 8 * t + 4);
        }

        float o[C::NT][HG][4];
        float m[HG][2], l[HG][2];                     // of heads 2t and 2t + 1; l of this lane's keys
#pragma unroll
        for (int n = 0; n < C::NT; ++n)
#pragma unroll
            for (int hg = 0; hg < HG; ++hg) o[n][hg][0] = o[n][hg][1] = o[n][hg][2] = o[n][hg][3] = 0.f;
#pragma unroll
        for (int hg = 0; hg < HG; ++hg) m[hg][0] = m[hg][1] = -INFINITY, l[hg][0] = l[hg][1] = 0.f;

        for (int s = w.lo; s < w.hi; ++s) {
            const uint32_t off_next = key_offset(a, next);
            j += stride;
            next = ask(w, j + stride);
            const uint32_t valid_next = valid_of(off_next);
            const bool more = s + 1 < w.hi;
            if (valid == 0u) {                        // a short item: nothing for this warp
                if (more) {
                    load_K(off_next);
                    load_V(off_next);
                }
                valid = valid_next;
                continue;
            }
            // S^T = K Q^T: rows are keys, columns heads
            float S[C::KT / 16][HG][4];
#pragma unroll
            for (int i = 0; i < C::KT / 16; ++i) {
#pragma unroll
                for (int hg = 0; hg < HG; ++hg) S[i][hg][0] = S[i][hg][1] = S[i][hg][2] = S[i][hg][3] = 0.f;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t a0, a1, a2, a3;
                    if (E4M3) {
                        widen4(K[2 * i][ks / 4][ks % 4], a0, a2);
                        widen4(K[2 * i + 1][ks / 4][ks % 4], a1, a3);
                    } else {
                        a0 = K[2 * i][ks / 2][ks % 2 * 2];
                        a1 = K[2 * i + 1][ks / 2][ks % 2 * 2];
                        a2 = K[2 * i][ks / 2][ks % 2 * 2 + 1];
                        a3 = K[2 * i + 1][ks / 2][ks % 2 * 2 + 1];
                    }
#pragma unroll
                    for (int hg = 0; hg < HG; ++hg) mma<C::F16>(S[i][hg], a0, a1, a2, a3, qf[hg][ks][0], qf[hg][ks][1]);
                }
            }
            if (more) load_K(off_next);

            if (valid != kFull) {
#pragma unroll
                for (int i = 0; i < C::KT / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (!(valid >> (i * 16 + (k >> 1) * 8 + g) & 1u)) {
#pragma unroll
                            for (int hg = 0; hg < HG; ++hg) S[i][hg][k] = -INFINITY;
                        }
            }
            float f[HG][2];
            bool moved = false;
#pragma unroll
            for (int hg = 0; hg < HG; ++hg)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float top = m[hg][k];
#pragma unroll
                    for (int i = 0; i < C::KT / 16; ++i) top = fmaxf(top, fmaxf(S[i][hg][k], S[i][hg][k + 2]));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                    const float c = c_col[hg][k], ref = top == -INFINITY ? 0.f : top, base = __fmul_rn(ref, c);
                    // bf16: the old maximum rounded as it was when the sums were taken relative to it: exactly 1 where it stays, since o is
                    // left alone then.  As one fused operation it is 2 to the power of what rounding base lost, a tile after the other.
                    // fp16: relative to the maximum itself, for the rounding of a large one would leave fp16's range.
                    f[hg][k] = C::F16 ? ex2((m[hg][k] - ref) * c) : ex2(__fmul_rn(m[hg][k], c) - base);
                    moved |= top != m[hg][k];
                    m[hg][k] = top;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < C::KT / 16; ++i) {
                        S[i][hg][k] = ex2(C::F16 ? fmaf(S[i][hg][k] - ref, c, kPaLift) : fmaf(S[i][hg][k], c, -base));
                        S[i][hg][k + 2] = ex2(C::F16 ? fmaf(S[i][hg][k + 2] - ref, c, kPaLift) : fmaf(S[i][hg][k + 2], c, -base));
                        sum += S[i][hg][k] + S[i][hg][k + 2];
                    }
                    l[hg][k] = l[hg][k] * f[hg][k] + sum;
                }
            // P^T as the second operand: keys along the contraction
            uint32_t ph[C::KT / 16][HG][2], pl[C::KT / 16][HG][2];
#pragma unroll
            for (int i = 0; i < C::KT / 16; ++i)
#pragma unroll
                for (int hg = 0; hg < HG; ++hg)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float x = S[i][hg][2 * h], y = S[i][hg][2 * h + 1];
                        const uint32_t p = pack2<C::F16>(x, y);
                        ph[i][hg][h] = transpose8(p);
                        if (!C::F16) {
                            const float2 back = unpack2<C::F16>(p);
                            pl[i][hg][h] = transpose8(pack2<C::F16>(x - back.x, y - back.y));
                        }
                    }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int n = 0; n < C::NT; ++n)
#pragma unroll
                    for (int hg = 0; hg < HG; ++hg)
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[n][hg][k] *= f[hg][k & 1];
            }
            // O^T += V^T P^T
#pragma unroll
            for (int i = 0; i < C::KT / 16; ++i)
#pragma unroll
                for (int c = 0; c < C::VC; ++c)
#pragma unroll
                    for (int e = 0; e < C::VE; e += 2) {
                        uint32_t a0, a1, a2, a3;
                        if (E4M3) {
                            const uint32_t sel = e % 4 ? 0x7362u : 0x5140u;
                            widen4(__byte_perm(V[i * 4][c][e / 4], V[i * 4 + 1][c][e / 4], sel), a0, a1);
                            widen4(__byte_perm(V[i * 4 + 2][c][e / 4], V[i * 4 + 3][c][e / 4], sel), a2, a3);
                        } else {
                            a0 = __byte_perm(V[i * 4][c][e / 2], V[i * 4 + 1][c][e / 2], 0x5410u);
                            a1 = __byte_perm(V[i * 4][c][e / 2], V[i * 4 + 1][c][e / 2], 0x7632u);
                            a2 = __byte_perm(V[i * 4 + 2][c][e / 2], V[i * 4 + 3][c][e / 2], 0x5410u);
                            a3 = __byte_perm(V[i * 4 + 2][c][e / 2], V[i * 4 + 3][c][e / 2], 0x7632u);
                        }
#pragma unroll
                        for (int hg = 0; hg < HG; ++hg) {
                            float (&acc)[4] = o[(c * C::VE + e) / 2][hg];
                            mma<C::F16>(acc, a0, a1, a2, a3, ph[i][hg][0], ph[i][hg][1]);
                            if (!C::F16) mma<C::F16>(acc, a0, a1, a2, a3, pl[i][hg][0], pl[i][hg][1]);
                        }
                    }
            if (more) load_V(off_next);
            valid = valid_next;
        }

        auto request = [&] {
            off = key_offset(a, x_key);
            valid = valid_of(off);
            load_K(off);
            load_V(off);
            load_Q(x);
            j = first_key(x);
            next = ask(x, j + stride);
        };
        const bool whole = w.lo == 0 && w.hi == w.steps;
        if (another && whole) request();              // (not across the call that joins pieces)

        const int head0 = head0_of(w), rows = rows_of(w);
        constexpr float unlift = C::F16 ? 0x1p-15f : 1.f;     // sums are put right as they leave the registers, numerators at the end
        static_assert(kPaLift == 15.f, "unlift");
        const float v_scale = (E4M3 && a.v_scale != nullptr ? a.v_scale[kv] : 1.f) * unlift;
        if (solo) {
            // the rows as they lie in registers: neighbouring components of heads 2t and 2t + 1
#pragma unroll
            for (int hg = 0; hg < HG; ++hg)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float sum = l[hg][k];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                    sum *= unlift;
                    const int row = hg * 8 + 2 * t + k;
                    if (row < rows) {
                        const float inv = sum == 0.f ? 0.f : v_scale / sum;
                        char* to = a.O + (((int64_t)w.r * a.n_heads + head0 + row) * D + g * C::VE) * 2;
#pragma unroll
                        for (int c = 0; c < C::VC; ++c)
#pragma unroll
                            for (int e = 0; e < C::VE; e += 8) {
                                uint32_t v[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float (&acc)[4] = o[(c * C::VE + e) / 2 + i][hg];
                                    v[i] = pack2<F16Q>(acc[k] * inv, acc[k + 2] * inv);
                                }
                                *reinterpret_cast<uint4*>(to + (c * 8 * C::VE + e) * 2) = make_uint4(v[0], v[1], v[2], v[3]);
                            }
                        if (a.LSE != nullptr && g == 0)
                            a.LSE[(int64_t)(head0 + row) * a.n_requests + w.r] = m[hg][k] * c_col[hg][k] * 0.6931471805599453f + logf(sum);
                    }
                }
            if (!another) break;
            w = x;
            continue;
        }
        // ---- the four warps' results, joined through shared memory
#pragma unroll
        for (int hg = 0; hg < HG; ++hg)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float sum = l[hg][k];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                const int row = hg * 8 + 2 * t + k;
                if (g == 0) {
                    sM[warp * C::ROWS + row] = __fmul_rn(m[hg][k], c_col[hg][k]);
                    sL[warp * C::ROWS + row] = sum * unlift;
                }
                if (row < rows) {
                    float* to = sO + (warp * C::ROWS + row) * C::LD + g * C::VE;
#pragma unroll
                    for (int c = 0; c < C::VC; ++c)
#pragma unroll
                        for (int e = 0; e < C::VE; e += 4) {
                            const int n = (c * C::VE + e) / 2;
                            *reinterpret_cast<float4*>(to + c * 8 * C::VE + e) =
                                make_float4(o[n][hg][k], o[n][hg][k + 2], o[n + 1][hg][k], o[n + 1][hg][k + 2]);
                        }
                }
            }
        __syncthreads();

        constexpr int PER = 4;                             // neighbouring columns a thread
        constexpr size_t kPart = kPartWords<D>;
        const Rows<D, F16Q> out{a.O + ((int64_t)w.r * a.n_heads + head0) * D * 2,
                                a.LSE == nullptr ? nullptr : a.LSE + (int64_t)head0 * a.n_requests + w.r, a.n_requests, v_scale};
        float* my_part = a.part + (2 * blockIdx.x + (w.lo == 0)) * kPart;
        for (int i = tid; i < rows * (D / PER); i += kPaThreads) {
            const int row = i / (D / PER), d = i % (D / PER) * PER;
            float top = -INFINITY;
#pragma unroll
            for (int i4 = 0; i4 < kPaWarps; ++i4) top = fmaxf(top, sM[i4 * C::ROWS + row]);
            const float base = top == -INFINITY ? 0.f : top;
            float x[PER] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
            for (int i4 = 0; i4 < kPaWarps; ++i4) {
                const float fw = ex2(sM[i4 * C::ROWS + row] - base);
                const float4 y = *reinterpret_cast<const float4*>(sO + (i4 * C::ROWS + row) * C::LD + d);
                sum += fw * sL[i4 * C::ROWS + row];
                x[0] += fw * y.x, x[1] += fw * y.y, x[2] += fw * y.z, x[3] += fw * y.w;
            }
            if (whole) out.store(row, d, x, top, sum);
            else put_part<D>(my_part, row, d, x, top, sum);
        }
        if (!whole) {
            const PagedPieces p = paged_pieces(plan, cuts[0].at + (int64_t)w.pos, w.steps + kPaItemCost);
            const int first = p.first, n = p.n, mine = (int)blockIdx.x - first;
            // counts this CTA in; true for the last of n
            auto arrive = [&](int32_t* ticket, int of) {
                __syncthreads();
                if (tid == 0) {
                    __threadfence();                         // of the whole CTA's results: they came before the barrier
                    last_flag = atomicAdd(ticket, 1) == of - 1;
                    if (last_flag) *ticket = 0;
                    __threadfence();
                }
                __syncthreads();
                return last_flag != 0;
            };
            // counters: of the item; of its first group; of a later group, by the group's first CTA (which may also begin an item)
            int32_t* tickets = a.tickets + first;
            if (n <= kPaJoin) {
                if (arrive(tickets, n)) join_pieces<D, F16Q>(a.part, first, 0, 1, n, rows, &out);
            } else {
                // levels: groups of kPaJoin pieces, then their results
                const int group = mine / kPaJoin, groups = (n + kPaJoin - 1) / kPaJoin, p0 = group * kPaJoin;
                const int count = min(kPaJoin, n - p0);
                if (arrive(tickets + kPaTicketRow * (group == 0 ? 1 : 2) + p0, count)) {
                    join_pieces<D, F16Q>(a.part, first, p0, 1, count, rows, nullptr);
                    if (arrive(tickets, groups)) {
                        // beyond kPaJoin^2 pieces one more level, by this CTA alone
                        for (int q0 = 0; groups > kPaJoin && q0 < groups; q0 += kPaJoin)
                            join_pieces<D, F16Q>(a.part, first, q0 * kPaJoin, kPaJoin, min(kPaJoin, groups - q0), rows, nullptr);
                        const int by = groups > kPaJoin ? kPaJoin * kPaJoin : kPaJoin;
                        __syncthreads();
                        join_pieces<D, F16Q>(a.part, first, 0, by, (n + by - 1) / by, rows, &out);
                    }
                }
            }
        }
        if (!another) break;
        if (!whole) request();
        w = x;
        __syncthreads();                    // shared memory is free for the next item
    }
}

template <int D, bool F16Q, bool E4M3, int HG>
__global__ void __launch_bounds__(kPaThreads, (Tile<D, F16Q, E4M3, HG>::CTAS)) paged_attn_kernel(const PagedAttnArgs a) {
    using C = Tile<D, F16Q, E4M3, HG>;
    extern __shared__ __align__(16) float sm[];
    __shared__ uint64_t plan_sum[kPaWarps];
    __shared__ uint32_t plan_longest[kPaWarps];
    __shared__ Cut cuts[2];
    __shared__ int32_t last_flag;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int H = a.n_kv * a.parts;                   // items a request

    grid_dep_wait();

    // ---- this CTA's share of all steps
    auto kept_at = [&](int r) { return kept_of(a, ld_index(a.lens + r)); };
    auto steps_of = [](const Kept& k) { return max((k.n + C::STEP - 1) / C::STEP, 1); };
    auto tiles_of = [](const Kept& k) { return (k.n + C::KT - 1) / C::KT; };
    PagedCuts plan;
    bool solo;
    {
        const int per = (a.n_requests + kPaThreads - 1) / kPaThreads;
        const int r0 = min(tid * per, a.n_requests), r1 = min(r0 + per, a.n_requests);
        uint64_t mine = 0;
        uint32_t longest = 0;
        for (int r = r0; r < r1; r += 4) {
            int32_t T[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) T[i] = r + i < r1 ? ld_index(a.lens + r + i) : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (r + i < r1) {
                    const Kept k = kept_of(a, T[i]);
                    mine += steps_of(k) + kPaItemCost;
                    longest = max(longest, (uint32_t)tiles_of(k));
                }
        }
        uint64_t inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 31) {
            plan_sum[warp] = inc;
            plan_longest[warp] = longest;
        }
        __syncthreads();
        uint64_t all = 0, before = inc - mine;
#pragma unroll
        for (int w = 0; w < kPaWarps; ++w) {
            if (w < warp) before += plan_sum[w];
            all += plan_sum[w];
            longest = max(longest, plan_longest[w]);
        }
        before *= H;
        solo = longest <= 2 && a.n_requests * H > (int)gridDim.x;       // (the same for every CTA)
        plan = paged_cuts(all * H, gridDim.x);
        if (!solo && blockIdx.x >= plan.n) return;
        const uint64_t b0 = paged_cut(plan, blockIdx.x), b1 = paged_cut(plan, blockIdx.x + 1);
#pragma unroll 1
        for (int i = 0; i < 2 && !solo; ++i) {
            const uint64_t b = i ? b1 : b0;
            if (b >= plan.all) {
                if (tid == 0) cuts[i] = Cut{plan.all, plan.all, a.n_requests, 0};
            } else if (b >= before && b < before + mine * H) {
                uint64_t at = before;
                int r = r0, cost = 0;
                for (; r < r1; ++r) {
                    cost = steps_of(kept_at(r)) + kPaItemCost;
                    if (b < at + (uint64_t)H * cost) break;
                    at += (uint64_t)H * cost;
                }
                Cut c;
                c.r = r;
                c.item = (int)div_u64(b - at, cost);
                c.item_at = at + (uint64_t)c.item * cost;
                const int moves = paged_cut_moves(plan, (int)(b - c.item_at), cost);
                c.at = moves < 0 ? c.item_at : b;
                if (moves > 0) {                                 // on to the next item
                    c.item_at += cost;
                    c.at = c.item_at;
                    if (++c.item == H) c.item = 0, ++c.r;
                }
                cuts[i] = c;
            }
        }
        __syncthreads();
    }
    if (solo) attend<D, F16Q, E4M3, HG, true>(a, plan, cuts, sm, last_flag);
    else attend<D, F16Q, E4M3, HG, false>(a, plan, cuts, sm, last_flag);
}

template <int D, bool F16Q, bool E4M3, int HG>
bool set_attributes() {
    using C = Tile<D, F16Q, E4M3, HG>;
    return cudaFuncSetAttribute(paged_attn_kernel<D, F16Q, E4M3, HG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM) == cudaSuccess;
}

template <int D, bool F16Q, bool E4M3, int HG>
pafu_status launch(const PagedAttnArgs& a, cudaStream_t stream) {
    using C = Tile<D, F16Q, E4M3, HG>;
    static bool done[kMaxDevices] = {};
    static int ctas[kMaxDevices] = {};
    const int dev = current_device();
    if (dev < 0 || !once_per_device(done, [] { return set_attributes<D, F16Q, E4M3, HG>(); })) return PAFU_ERR_CUDA;
    if (ctas[dev] == 0) {
        int n = 0;
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, paged_attn_kernel<D, F16Q, E4M3, HG>, kPaThreads, C::SMEM) != cudaSuccess || n < 1)
            return PAFU_ERR_CUDA;
        ctas[dev] = n < kPagedCtasPerSm ? n : kPagedCtasPerSm;
    }
    return cuda_ok(launch_dependent(paged_attn_kernel<D, F16Q, E4M3, HG>, dim3(ctas[dev] * device_sm_count()), dim3(kPaThreads), C::SMEM,
                                    stream, 1, a));
}

template <int D, bool F16Q, bool E4M3>
pafu_status launch_rows(const PagedAttnArgs& a, cudaStream_t stream) {
    return a.group <= 8 ? launch<D, F16Q, E4M3, 1>(a, stream) : launch<D, F16Q, E4M3, 2>(a, stream);
}
template <int D>
pafu_status launch_type(const PagedAttnArgs& a, bool f16q, bool e4m3, cudaStream_t stream) {
    if (e4m3) return f16q ? launch_rows<D, true, true>(a, stream) : launch_rows<D, false, true>(a, stream);
    return f16q ? launch_rows<D, true, false>(a, stream) : launch_rows<D, false, false>(a, stream);
}

}  // namespace

pafu_status launch_paged_attn(const pafu_paged_cache& c, const void* Q, int64_t q_token, int64_t q_head, const int32_t* lens,
                              int64_t n_sink, int64_t n_recent, float scale, void* O, float* LSE, void* ws, cudaStream_t stream) {
    PagedAttnArgs a;
    a.pool = pool_of(c);
    a.Q = static_cast<const char*>(Q);
    a.q_token = q_token * 2;
    a.q_head = q_head * 2;
    a.lens = lens;
    a.n_requests = c.n_requests;
    a.n_heads = c.n_heads;
    a.n_kv = c.n_kv_heads;
    a.group = c.n_heads / c.n_kv_heads;
    a.parts = (a.group + kPagedRows - 1) / kPagedRows;
    a.sink = (int32_t)(n_sink < 0x7fffffff ? n_sink : 0x7fffffff);
    a.recent = n_recent < 0 ? -1 : (int32_t)(n_recent < 0x7fffffff ? n_recent : 0x7fffffff);
    a.scale = scale * 1.4426950408889634f;
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.O = static_cast<char*>(O);
    a.LSE = LSE;
    a.status = static_cast<int32_t*>(ws) + kStatusWordPaged;
    a.tickets = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + kWsHeaderBytes);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + kPagedPartOffset);
    const bool f16q = c.type == PAFU_TYPE_F16, e4m3 = c.cache_type == PAFU_TYPE_E4M3;
    return c.d_head == 128 ? launch_type<128>(a, f16q, e4m3, stream) : launch_type<64>(a, f16q, e4m3, stream);
}

}  // namespace pafu
