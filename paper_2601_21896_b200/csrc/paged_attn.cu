// Attention of one new token a request over a paged cache: for request r and query head n
//   o = sum_j softmax_j(scale * q . k_j) v_j,   j over the kept positions [0, n_sink) U [T - n_recent, T).
//
// Every key is used by the n_heads / n_kv_heads query heads of its group, 2 flop a byte and head: the cache's bytes bound
// the call, and what a kernel has to do is keep enough of them on their way.  So nothing is staged: a warp's lanes load
// 16-byte pieces of the rows straight into the registers in which mma.sync wants them.  The order of the contraction
// index is free as long as both operands follow it, so a lane's 16 contiguous bytes of a key row serve as two (8 bits: four)
// B fragments of Q K^T, and the queries are loaded in the same order; the columns of P V are free too, so eight
// neighbouring lanes read a 128-byte line of a value row and a byte permute pairs the rows of two keys.  The rows' addresses
// come from the page table one tile ahead, so pages of any length, order and stride cost the same and may end inside a tile.
// Up to eight query heads fill half of the 16 rows of a product's tile; the other half then carries what rounding the
// probabilities to 16 bits leaves over, which makes P V nearly exact at no cost.  With 9 to 16 heads a second product does
// that for bf16; fp16 probabilities (2^-12) need none.
// 8-bit caches are widened to fp16, which holds every e4m3 value; bf16 queries are scaled by a power of two a row so that
// their largest component lies in [2^14, 2^15) and fp16 holds them to 2^-39 of it.
//
// Split over the length: every (request, group of heads) is an item of ceil(kept / step) steps (a step is one tile for each of
// the four warps) and a fixed cost.  All items laid end to end are cut into equal shares, one a CTA, by arithmetic that every
// CTA does for itself from the lengths on the device: the grid does not depend on the lengths, and a captured launch follows
// them.  A share's first and last item may continue in other CTAs: their fp32 partial results go to the workspace,
// and the CTA that arrives last (a counter; nothing waits) joins them in a fixed order, so results do not depend on timing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "paged.cuh"

namespace pafu {

namespace {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = kPaWarps * 32;
constexpr int kPaItemCost = 1;        // what an item costs beside its steps, in steps
constexpr int kPaMinShare = 4;        // steps and item costs that a CTA takes at least

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

// 16 bytes (8) of a row, or zeros
__device__ __forceinline__ void ld_row(uint32_t (&w)[4], const char* p, bool ok) {
    w[0] = w[1] = w[2] = w[3] = 0u;
    asm volatile(
        "{\n\t.reg .pred P;\n\tsetp.ne.b32 P, %5, 0;\n\t"
        "@P ld.global.nc.L1::no_allocate.L2::128B.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]) : "l"(p), "r"((int)ok) : "memory");
}
__device__ __forceinline__ void ld_row(uint32_t (&w)[2], const char* p, bool ok) {
    w[0] = w[1] = 0u;
    asm volatile(
        "{\n\t.reg .pred P;\n\tsetp.ne.b32 P, %3, 0;\n\t"
        "@P ld.global.nc.L1::no_allocate.L2::128B.v2.u32 {%0, %1}, [%2];\n\t}"
        : "+r"(w[0]), "+r"(w[1]) : "l"(p), "r"((int)ok) : "memory");
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

// two e4m3 values (a 16-bit pair) as two fp16 ones
__device__ __forceinline__ uint32_t widen2(uint32_t pair) {
    uint32_t r;
    asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(pair));
    return r;
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
    static constexpr int KT = D * ES >= 256 ? 16 : 32;            // keys of a warp's tile: 4 to 8 KB of K and V in flight a warp
    static constexpr int KR = KT / 8;                             // key rows that a lane has a part of
    static constexpr int KW = D * ES / 16;                        // words of each
    static constexpr int VR = KT / 4;                             // value rows
    static constexpr int VB = D * ES / 8 < 16 ? 8 : 16;           // bytes of a value load
    static constexpr int VC = D * ES / 8 / VB;                    // loads a value row
    static constexpr int VE = VB / ES;                            // elements of a value load
    static constexpr int NT = D / 8;                              // column tiles of O
    static constexpr int STEP = KT * kPaWarps;
    static constexpr bool F16 = F16Q || E4M3;                     // type of the products
    static constexpr int ROWS = HG * 8;
    static constexpr int LD = D + 4;
    static constexpr size_t SMEM = sizeof(float) * (kPaWarps * ROWS * LD + 2 * kPaWarps * ROWS);
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

template <int D, bool F16Q, bool E4M3, int HG>
__global__ void __launch_bounds__(kPaThreads, HG == 1 ? 3 : 2) paged_attn_kernel(const PagedAttnArgs a) {
    using C = Tile<D, F16Q, E4M3, HG>;
    extern __shared__ __align__(16) float sm[];
    float* sO = sm;                                   // [warp][row][LD]
    float* sM = sm + kPaWarps * C::ROWS * C::LD;      // [warp][row]
    float* sL = sM + kPaWarps * C::ROWS;
    __shared__ int64_t plan_sum[kPaWarps], plan_at;
    __shared__ int32_t plan_r, last_flag;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int H = a.n_kv * a.parts;                   // items a request

    grid_dep_wait();

    // ---- this CTA's share of all steps
    int64_t share, begin;
    {
        const int per = (a.n_requests + kPaThreads - 1) / kPaThreads;
        const int r0 = min(tid * per, a.n_requests), r1 = min(r0 + per, a.n_requests);
        int64_t mine = 0;
        for (int r = r0; r < r1; ++r) mine += max((kept_of(a, ld_index(a.lens + r)).n + C::STEP - 1) / C::STEP, 1) + kPaItemCost;
        int64_t inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) plan_sum[warp] = inc;
        __syncthreads();
        int64_t all = 0, before = inc - mine;
        for (int w = 0; w < kPaWarps; ++w) {
            if (w < warp) before += plan_sum[w];
            all += plan_sum[w];
        }
        all *= H;
        before *= H;
        share = (all + gridDim.x - 1) / gridDim.x;
        if (share < kPaMinShare) share = kPaMinShare;
        begin = share * blockIdx.x;
        if (begin >= all) return;
        if (begin >= before && begin < before + mine * H) {
            int64_t at = before;
            int r = r0;
            for (; r < r1; ++r) {
                const int64_t c = (int64_t)H * (max((kept_of(a, ld_index(a.lens + r)).n + C::STEP - 1) / C::STEP, 1) + kPaItemCost);
                if (begin < at + c) break;
                at += c;
            }
            plan_r = r;
            plan_at = at;
        }
        __syncthreads();
    }
    const int64_t end = begin + share;
    int r = plan_r;
    Kept kept = kept_of(a, ld_index(a.lens + r));
    int steps = max((kept.n + C::STEP - 1) / C::STEP, 1);
    int item = (int)((begin - plan_at) / (steps + kPaItemCost));
    int64_t at = plan_at + (int64_t)item * (steps + kPaItemCost);     // where the item starts

    while (true) {
        const int lo = (int)min((int64_t)steps, max(begin - at, (int64_t)0));
        const int hi = (int)min((int64_t)steps, end - at);
        const bool whole = lo == 0 && hi == steps;
        if (lo < hi) {
            const int kv = item / a.parts, head0 = kv * a.group + (item - kv * a.parts) * kPagedRows;
            const int rows = min(kPagedRows, (kv + 1) * a.group - head0);       // query heads of the item
            const int32_t* table = a.pool.table + (int64_t)r * a.pool.max_pages;
            const uint32_t head_u = (uint32_t)kv * a.pool.head_u;

            uint32_t K[C::KR][C::KW / 4][4], V[C::VR][C::VC][C::VB / 4];
            auto load_K = [&](uint32_t off) {
#pragma unroll
                for (int i = 0; i < C::KR; ++i) {
                    const uint32_t o = __shfl_sync(0xffffffffu, off, i * 8 + g);
                    const char* p = a.pool.K + (uint64_t)o * 16 + t * 16;
#pragma unroll
                    for (int c = 0; c < C::KW / 4; ++c) ld_row(K[i][c], p + c * 64, o != ~0u);
                }
            };
            auto load_V = [&](uint32_t off) {
#pragma unroll
                for (int i = 0; i < C::VR; ++i) {
                    const uint32_t o = __shfl_sync(0xffffffffu, off, (i >> 2) * 16 + ((i >> 1) & 1) * 8 + 2 * t + (i & 1));
                    const char* p = a.pool.V + (uint64_t)o * 16 + g * C::VB;
#pragma unroll
                    for (int c = 0; c < C::VC; ++c) ld_row(V[i][c], p + c * 8 * C::VB, o != ~0u);
                }
            };

            // the first tile's rows are requested before the queries
            int32_t j = (lo * kPaWarps + warp) * C::KT + (lane & (C::KT - 1));
            const int32_t j_end = hi * C::STEP;           // exclusive; keys past kept.n do not exist
            auto ask = [&](int32_t jj) { return key_at(a, kept, table, jj < j_end ? jj : 0x7fffffff, head_u); };
            uint32_t off = key_offset(a, ask(j));
            KeyAt next = ask(j + C::STEP);
            load_K(off);
            load_V(off);

            // queries: rows g (and g + 8), in the order in which the lane's key words come
            uint32_t qf[HG][D / 16][2];
            float c_row[HG];
#pragma unroll
            for (int hg = 0; hg < HG; ++hg) {
                const bool have = hg * 8 + g < rows;
                const char* qp = a.Q + r * a.q_token + (int64_t)(head0 + hg * 8 + g) * a.q_head;
#pragma unroll
                for (int c = 0; c < C::KW / 4; ++c) {
                    // elements of 16 bytes of a key row: 8 or 16
                    constexpr int PER = 16 / C::ES;
                    const char* p = qp + (c * 4 * PER + t * PER) * 2;
#pragma unroll
                    for (int h = 0; h < PER / 8; ++h) {
                        uint4 w = make_uint4(0, 0, 0, 0);
                        if (have) w = *reinterpret_cast<const uint4*>(p + h * 16);
                        const int ks = c * (PER / 4) + h * 2;
                        qf[hg][ks][0] = w.x;
                        qf[hg][ks][1] = w.y;
                        qf[hg][ks + 1][0] = w.z;
                        qf[hg][ks + 1][1] = w.w;
                    }
                }
                c_row[hg] = a.scale;
                if (E4M3 && a.k_scale != nullptr) c_row[hg] *= a.k_scale[kv];
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
                    c_row[hg] *= __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 v = unpack2<false>(qf[hg][ks][i]);
                            qf[hg][ks][i] = pack2<true>(v.x * f, v.y * f);
                        }
                }
            }

            float o[C::NT][4];
            float m[HG], l[HG];
#pragma unroll
            for (int n = 0; n < C::NT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
            for (int hg = 0; hg < HG; ++hg) m[hg] = -INFINITY, l[hg] = 0.f;

            for (int s = lo; s < hi; ++s) {
                const uint32_t valid = __ballot_sync(0xffffffffu, off != ~0u) & (C::KT == 32 ? ~0u : (1u << C::KT % 32) - 1u);
                const uint32_t off_next = key_offset(a, next);
                j += C::STEP;
                next = ask(j + C::STEP);
                // S = Q K^T: rows are heads, columns keys
                float S[C::KR][4];
#pragma unroll
                for (int i = 0; i < C::KR; ++i) {
                    S[i][0] = S[i][1] = S[i][2] = S[i][3] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        uint32_t b0, b1;
                        if (E4M3) {
                            const uint32_t w = K[i][ks / 4][ks % 4];
                            b0 = widen2(w & 0xffffu);
                            b1 = widen2(w >> 16);
                        } else {
                            b0 = K[i][ks / 2][ks % 2 * 2];
                            b1 = K[i][ks / 2][ks % 2 * 2 + 1];
                        }
                        mma<C::F16>(S[i], qf[0][ks][0], HG == 2 ? qf[HG - 1][ks][0] : 0u, qf[0][ks][1], HG == 2 ? qf[HG - 1][ks][1] : 0u, b0, b1);
                    }
                }
                if (s + 1 < hi) load_K(off_next);

                // running maximum and sum, one or two rows a lane, shared by the four lanes of a row
                uint32_t ph[C::KR][HG], pl[C::KR][HG];
                float f[HG];
                bool moved = false;
#pragma unroll
                for (int hg = 0; hg < HG; ++hg) {
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < C::KR; ++i)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float x = S[i][hg * 2 + k] * c_row[hg];
                            if (!(valid >> (i * 8 + 2 * t + k) & 1u)) x = -INFINITY;
                            S[i][hg * 2 + k] = x;
                            top = fmaxf(top, x);
                        }
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const float now = fmaxf(m[hg], top);
                    const float base = now == -INFINITY ? 0.f : now;
                    f[hg] = ex2(m[hg] - base);
                    moved |= now != m[hg];
                    m[hg] = now;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < C::KR; ++i) {
                        const float x = ex2(S[i][hg * 2] - base), y = ex2(S[i][hg * 2 + 1] - base);
                        sum += x + y;
                        ph[i][hg] = pack2<C::F16>(x, y);
                        const float2 back = unpack2<C::F16>(ph[i][hg]);
                        pl[i][hg] = pack2<C::F16>(x - back.x, y - back.y);
                    }
                    l[hg] = l[hg] * f[hg] + sum;
                }
                if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                    for (int n = 0; n < C::NT; ++n) {
                        o[n][0] *= f[0];
                        o[n][1] *= f[0];
                        o[n][2] *= f[HG - 1];
                        o[n][3] *= f[HG - 1];
                    }
                }
                // O += P V
#pragma unroll
                for (int v = 0; v < C::KT / 16; ++v)
#pragma unroll
                    for (int c = 0; c < C::VC; ++c)
#pragma unroll
                        for (int e = 0; e < C::VE; ++e) {
                            uint32_t b0, b1;
                            if (E4M3) {
                                const uint32_t sel = 0x40u + 0x11u * (e % 4);
                                b0 = widen2(__byte_perm(V[v * 4][c][e / 4], V[v * 4 + 1][c][e / 4], sel));
                                b1 = widen2(__byte_perm(V[v * 4 + 2][c][e / 4], V[v * 4 + 3][c][e / 4], sel));
                            } else {
                                const uint32_t sel = e % 2 ? 0x7632u : 0x5410u;
                                b0 = __byte_perm(V[v * 4][c][e / 2], V[v * 4 + 1][c][e / 2], sel);
                                b1 = __byte_perm(V[v * 4 + 2][c][e / 2], V[v * 4 + 3][c][e / 2], sel);
                            }
                            float (&acc)[4] = o[c * C::VE + e];
                            if (HG == 1) {
                                mma<C::F16>(acc, ph[2 * v][0], pl[2 * v][0], ph[2 * v + 1][0], pl[2 * v + 1][0], b0, b1);
                            } else {
                                mma<C::F16>(acc, ph[2 * v][0], ph[2 * v][HG - 1], ph[2 * v + 1][0], ph[2 * v + 1][HG - 1], b0, b1);
                                if (!C::F16) mma<C::F16>(acc, pl[2 * v][0], pl[2 * v][HG - 1], pl[2 * v + 1][0], pl[2 * v + 1][HG - 1], b0, b1);
                            }
                        }
                if (s + 1 < hi) load_V(off_next);
                off = off_next;
            }

            // ---- the four warps' results, joined through shared memory
#pragma unroll
            for (int hg = 0; hg < HG; ++hg) {
                l[hg] += __shfl_xor_sync(0xffffffffu, l[hg], 1);
                l[hg] += __shfl_xor_sync(0xffffffffu, l[hg], 2);
                if (t == 0) {
                    sM[warp * C::ROWS + hg * 8 + g] = m[hg];
                    sL[warp * C::ROWS + hg * 8 + g] = l[hg];
                }
                if (hg * 8 + g < rows) {
                    float* row = sO + (warp * C::ROWS + hg * 8 + g) * C::LD;
#pragma unroll
                    for (int c = 0; c < C::VC; ++c)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int e = 0; e < C::VE; e += 4) {
                                float4 x;
                                float* xs = &x.x;
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float (&acc)[4] = o[c * C::VE + e + i];
                                    xs[i] = HG == 1 ? acc[half] + acc[2 + half] : acc[hg * 2 + half];
                                }
                                *reinterpret_cast<float4*>(row + c * 8 * C::VE + (2 * t + half) * C::VE + e) = x;
                            }
                }
            }
            __syncthreads();

            const int64_t first = at / share, last = (at + steps - 1) / share;      // CTAs that have a piece of the item
            float* my_part = a.part + (size_t)(2 * blockIdx.x + (lo == 0)) * kPagedRows * (D + 2);
            constexpr int PER = 4;                             // neighbouring columns a thread
            const float v_scale = E4M3 && a.v_scale != nullptr ? a.v_scale[kv] : 1.f;
            auto store = [&](int row, int d, const float (&x)[PER], float top, float sum) {
                const float inv = sum == 0.f ? 0.f : v_scale / sum;
                uint2 w;
                w.x = pack2<F16Q>(x[0] * inv, x[1] * inv);
                w.y = pack2<F16Q>(x[2] * inv, x[3] * inv);
                *reinterpret_cast<uint2*>(a.O + (((int64_t)r * a.n_heads + head0 + row) * D + d) * 2) = w;
                if (a.LSE != nullptr && d == 0) a.LSE[(int64_t)(head0 + row) * a.n_requests + r] = top * 0.6931471805599453f + logf(sum);
            };
            for (int i = tid; i < rows * (D / PER); i += kPaThreads) {
                const int row = i / (D / PER), d = i % (D / PER) * PER;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kPaWarps; ++w) top = fmaxf(top, sM[w * C::ROWS + row]);
                const float base = top == -INFINITY ? 0.f : top;
                float x[PER] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
                for (int w = 0; w < kPaWarps; ++w) {
                    const float f = ex2(sM[w * C::ROWS + row] - base);
                    const float4 y = *reinterpret_cast<const float4*>(sO + (w * C::ROWS + row) * C::LD + d);
                    sum += f * sL[w * C::ROWS + row];
                    x[0] += f * y.x, x[1] += f * y.y, x[2] += f * y.z, x[3] += f * y.w;
                }
                if (whole) {
                    store(row, d, x, top, sum);
                } else {
                    *reinterpret_cast<float4*>(my_part + row * D + d) = make_float4(x[0], x[1], x[2], x[3]);
                    if (d == 0) {
                        my_part[kPagedRows * D + row] = top;
                        my_part[kPagedRows * D + kPagedRows + row] = sum;
                    }
                }
            }
            if (!whole) {
                // the pieces' CTAs count themselves in; the last one joins them, first piece first
                __threadfence();
                __syncthreads();
                if (tid == 0) last_flag = atomicAdd(a.tickets + first, 1) == (int)(last - first);
                __syncthreads();
                if (last_flag) {
                    __threadfence();
                    if (tid == 0) a.tickets[first] = 0;
                    const int n = (int)(last - first) + 1;
                    auto piece = [&](int p) { return a.part + (size_t)(2 * (first + p) + (p == 0)) * kPagedRows * (D + 2); };
                    for (int i = tid; i < rows * (D / PER); i += kPaThreads) {
                        const int row = i / (D / PER), d = i % (D / PER) * PER;
                        float top = -INFINITY;
                        for (int p = 0; p < n; ++p) top = fmaxf(top, __ldcg(piece(p) + kPagedRows * D + row));
                        const float base = top == -INFINITY ? 0.f : top;
                        float x[PER] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll 4
                        for (int p = 0; p < n; ++p) {
                            const float* q = piece(p);
                            const float f = ex2(__ldcg(q + kPagedRows * D + row) - base);
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(q + row * D + d));
                            sum += f * __ldcg(q + kPagedRows * D + kPagedRows + row);
                            x[0] += f * y.x, x[1] += f * y.y, x[2] += f * y.z, x[3] += f * y.w;
                        }
                        store(row, d, x, top, sum);
                    }
                }
            }
            __syncthreads();                    // shared memory is free for the next item
        }
        at += steps + kPaItemCost;
        if (at >= end) break;
        if (++item == H) {
            item = 0;
            if (++r == a.n_requests) break;
            kept = kept_of(a, ld_index(a.lens + r));
            steps = max((kept.n + C::STEP - 1) / C::STEP, 1);
        }
    }
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
    a.recent = (int32_t)(n_recent < 0x7fffffff ? n_recent : 0x7fffffff);
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
