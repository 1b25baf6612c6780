// Attention of few query rows per KV head (a decoded token, a few speculated ones) over a long cache.
//
// o_r = sum_j p_rj v_j / sum_j p_rj with p_rj = 2^(c s_rj - m_r), one pass over the keys with a running maximum m_r.  With 8 or 16
// rows in a tile every cache byte is used for that many multiply-adds, so the kernel is bound by HBM and is built to keep
// loads in flight:
//   - A unit of work is 64 keys (16-bit cache) or 128 keys (8-bit) of one (problem, KV head, row tile).  The units of the whole
//     call, in that order, are cut into runs of equal cost, one per CTA, from the lengths on the device, so that ragged batches
//     balance; an item costs its units plus kDecItemCost (the merge of its warps and the drained pipeline).  A run that starts
//     or ends inside an item leaves a partial (o, m, l) that combine_kernel merges.
//   - Within a unit each of the four warps owns a slice of 16 (32) keys and a private ring of three slices in shared memory, filled
//     by its own 16-byte cp.async: no barrier between warps until an item ends.  Two CTAs per SM hold 128 KB of loads in
//     flight and cover each other's item ends.  cp.async takes any page size and any 16-byte-aligned stride and
//     zero-fills rows past the prefix, so their contents never enter the sums.
//   - Products run on mma.sync with the keys as the M dimension: S^T = K Q^T (16 keys x 8 rows), O^T += V^T P^T (16 elements x 8
//     rows), so a tile of eight rows, which is what one token of most models gives, wastes nothing; a 128-row tcgen05 tile would
//     be 15/16 padding.  The fragments come straight out of registers, which the 8-bit cache needs anyway.  (With the rows as M, 16 at
//     a time, the 8-bit kernel took an eighth longer on a ragged batch: twice the products and exponentials, half of them padding.)
// 8-bit keys are multiplied as they are (m16n8k32, e4m3): the query is split into hi + lo e4m3 codes under a power-of-two
// scale of its row.  A bf16 number has eight significant bits, hi takes the upper four, lo the rest exactly, down to elements
// 2^-10 of the row's largest; below that the error is at most 2^-17 of the largest, far under the bf16 rounding of q itself.
// 8-bit values are f16 numbers exactly; their scales multiply P, taken over a running power of two so that f16 holds the product.  In a
// slice with a scale below 2^-21 of it f16 would take bits from that key: there P and the values (bf16 numbers, too) are bf16.
#pragma once
#include <type_traits>

#include "chunk.cuh"

namespace mage {
namespace chunk {

constexpr int kDecWarps = 4;
constexpr int kDecStages = 3;
// Fixed cost of an item in units' worth of time.  (2, 4, 7 units.  8 bits, 32 sequences of 1 to 131072 tokens, 28 + 4 heads: 128, 102, 104 us; other
// lengths 82, 70, 74; 32 + 8 heads 216, 171, 176; 64 sequences of up to 3000: 18.8, 20.2, 24.  16 bits, 16 sequences: 328, 327, 328.)
constexpr int kDecItemCost = 4;
// floats of a partial result of a tile of n rows: o[n][128], m[n], l[n]
__host__ __device__ constexpr int slot_floats(int n) { return n * kD + 2 * n; }
template <bool KV8, int NQ = 1>                       // NQ: groups of eight rows in a tile
struct Dec {
    static constexpr int kRows = 8 * NQ;
    static constexpr int kSlice = KV8 ? 32 : 16;      // keys of a warp's slice
    static constexpr int kUnit = kSlice * kDecWarps;  // keys of a unit
    static constexpr int kMinCost = KV8 ? 1 : 2;      // least cost of a run (16 bits, one token over 8000 keys, 8 + 2 heads: 1 unit 12.2 us, 2 units 10.6, 4 units 10.9)
    static constexpr int kHalf = KV8 ? 32 * 128 : 16 * 256;        // bytes of the K (or V) part of a slice
    static constexpr int kStage = 2 * kHalf + (KV8 ? 256 : 0);     // + scales of the keys, then of the values
    static constexpr size_t kSmem = (size_t)kDecWarps * kDecStages * kStage;
};

// An item whose keys are cut over the runs c0 .. c1, as combine_kernel needs it: in the record of run c0, and for prompts in those of
// the runs between, which lie inside the item (at most one such item per run); count 0: there is none.
struct Split {
    int a, h, pos0, N;        // first packed token, KV head, position of that token, length
    int first, count;         // decode: first row (token * G + head) and rows of the tile; prefill: first token and tokens
    int c1, c0;               // the last run and the first with a part of it
};
static_assert(sizeof(Split) == 32, "");

struct AttnArgs {
    Strided q;
    int mask_block;
    float scale_log2;
    __nv_bfloat16 *out;
    float *lse;
};

// A row (or a part of its keys) that took no key, all of them behind the mask or on bad pages, has reference -inf: its result is zeros.
// Where the keys that it took have no logit above -inf (infinite keys, NaN) the reference is the lowest finite number: 0 / 0, as by the
// definition.
constexpr float kLowest = -3.4028234663852886e38f;
// Keys that the row at position t sees.
__device__ __forceinline__ int visible(int t, int N, int mask_block) {
    if (t < 0) return 0;
    if (mask_block == 0) return N;
    const long long end = ((long long)(t / mask_block) + 1) * mask_block;
    return end < N ? (int)end : N;
}

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 8 x 8 sixteen-bit values, a row in four lanes: transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void cp_async_16z(uint32_t dst, const void *src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_4z(uint32_t dst, const void *src, bool take) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(take ? 4 : 0) : "memory");
}
// Query rows as hi + lo e4m3 codes under a power-of-two factor f of the row (the row over f has its largest magnitude in (224, 448]; NaN
// for a row with a NaN or an infinity).  amax: the row's largest bf16 bit pattern without sign.  Everything is exact in f16
// arithmetic: bf16 numbers have eight significant bits, f16 eleven, and what lies below f16's range is far below lo's smallest step.
__device__ __forceinline__ float row_factor(uint32_t amax, float &inv) {
    inv = 1.f;
    if (amax >= 0x7f80u) return __uint_as_float(0x7fc00000u);
    if (amax == 0u) return 1.f;
    int e = (int)(amax >> 7) - 127;
    e = (amax & 0x7fu) <= 0x60u ? e - 8 : e - 7;      // mantissa <= 1.75: 2^8 * 1.75 = 448
    e = max(e, -120);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}
__device__ __forceinline__ uint32_t amax_bits(uint32_t m, uint32_t two) { return __vmaxu2(m, two & 0x7fff7fffu); }     // per 16-bit half
__device__ __forceinline__ uint32_t amax_of_halves(uint32_t m) { return max(m & 0xffffu, m >> 16); }
// two bf16 -> two codes of hi (low 16 bits of the result) and of lo (high 16 bits)
__device__ __forceinline__ uint32_t code_pair(uint32_t two, float inv) {
    uint32_t x, back, r;
    unsigned short hi, lo;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(x) : "f"(__uint_as_float(two & 0xffff0000u) * inv), "f"(__uint_as_float(two << 16) * inv));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(hi) : "r"(x));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(back) : "h"(hi));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(back));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(lo) : "r"(r));
    return (uint32_t)hi | ((uint32_t)lo << 16);
}

// The items of the call in order (problem, KV head, row tile): cost of a problem's, its row tiles, units of each.
struct UnitMap {
    __device__ static long long of_problem(const KvView &kv, const ChunkView &cv, int p, int unit, int rows, int &tiles, int &units, unsigned *status) {
        int a;
        const int n = chunk_len_of(cv, p, &a, status);
        tiles = (n * kv.G + rows - 1) / rows;
        units = max(1, (seq_len_of(kv, p) + unit - 1) / unit);
        return (long long)tiles * kv.H_kv * (units + kDecItemCost);
    }
};

template <bool KV8, int NQ>
__global__ void __launch_bounds__(kDecWarps * 32, 2)
decode_kernel(KvView kv, Kv8View c8, ChunkView cv, AttnArgs at, Split *__restrict__ split, float *__restrict__ part, unsigned *status) {
    using namespace ptx;
    using C = Dec<KV8, NQ>;
    constexpr int kRows = C::kRows;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    __shared__ long long s_scan[kDecWarps + 1];
    __shared__ long long s_start[2];
    __shared__ float s_m[kDecWarps][kRows], s_l[kDecWarps][kRows];
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // ---- this CTA's run of units
    const int per = (kv.P + blockDim.x - 1) / blockDim.x, p_lo = min(kv.P, tid * per), p_hi = min(kv.P, p_lo + per);
    long long mine = 0;
    for (int p = p_lo; p < p_hi; ++p) {
        int tiles, units;
        mine += UnitMap::of_problem(kv, cv, p, C::kUnit, C::kRows, tiles, units, blockIdx.x == 0 ? status : nullptr);
    }
    long long incl = mine;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, incl, w);
        if (lane >= w) incl += o;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
    }
    const long long excl = before + incl - mine;
    if (split && tid == 0) split[blockIdx.x].count = 0;
    const int n_runs = (int)min((long long)gridDim.x, (total + C::kMinCost - 1) / C::kMinCost);
    if ((int)blockIdx.x >= n_runs) return;
    const long long run0 = total * blockIdx.x / n_runs, run1 = total * (blockIdx.x + 1) / n_runs;
    if (excl <= run0 && run0 < excl + mine) {
        long long off = excl;
        for (int p = p_lo; p < p_hi; ++p) {
            int tiles, units;
            const long long n = UnitMap::of_problem(kv, cv, p, C::kUnit, C::kRows, tiles, units, nullptr);
            if (run0 < off + n) { s_start[0] = p; s_start[1] = off; break; }
            off += n;
        }
    }
    __syncthreads();
    int p = (int)s_start[0];
    long long p_off = s_start[1];

    const int g = lane >> 2, c = lane & 3;                // fragment coordinates: key (or element) g, pair of rows (or keys) c
    uint8_t *ring = smem_raw + warp * (kDecStages * C::kStage);
    const uint32_t ring_u = smem_u32(ring);

    for (long long u = run0; u < run1;) {
        int tiles, units;
        for (;;) {
            const long long n = UnitMap::of_problem(kv, cv, p, C::kUnit, C::kRows, tiles, units, nullptr);
            if (u < p_off + n) break;
            p_off += n;
            ++p;
        }
        // an item's units come first, its fixed cost last: a run that ends there has all of them
        const long long local = u - p_off;
        const int cost = units + kDecItemCost, u0 = (int)(local % cost), item = (int)(local / cost), h = item / tiles, rt = item % tiles;
        const int taken = (int)min((long long)(cost - u0), run1 - u), u1 = min(units, u0 + taken);
        const long long x0 = u - u0;
        u += taken;
        if (u0 >= units) continue;
        int a;
        const int n_new = chunk_len_of(cv, p, &a, nullptr), N = seq_len_of(kv, p), rows = min(kRows, n_new * kv.G - rt * kRows);
        if (tid == 0 && u0 == 0 && u1 < units) split[blockIdx.x] = {a, h, N - n_new, N, rt * kRows, rows, (int)(((x0 + units) * n_runs - 1) / total), (int)blockIdx.x};

        // ---- rows of this tile: a thread holds rows 8 nq + 2 c + e of S^T and O^T, and row 8 nq + g of Q as B fragments
        int lim[NQ][2], lim_lo = 0x7fffffff, lim_hi = 0;
        float cs[NQ][2];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nq * 8 + 2 * c + e;
                lim[nq][e] = r < rows ? visible(N - n_new + (rt * kRows + r) / kv.G, N, at.mask_block) : 0;
                if (r < rows) lim_lo = min(lim_lo, lim[nq][e]);
                lim_hi = max(lim_hi, lim[nq][e]);
                cs[nq][e] = at.scale_log2;
            }
#pragma unroll
        for (int w = 1; w < 4; w <<= 1) {
            lim_lo = min(lim_lo, __shfl_xor_sync(0xffffffffu, lim_lo, w));
            lim_hi = max(lim_hi, __shfl_xor_sync(0xffffffffu, lim_hi, w));
        }
        // 16-bit: qb[nq][ks] = k-step ks (16 elements).  8-bit: qb[nq][ks], qb[nq][4 + ks] = hi and lo codes of k-step ks (32 elements).
        uint32_t qb[NQ][8][2];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int r = nq * 8 + g, R = rt * kRows + r;
            const bool ok = r < rows;
            const __nv_bfloat16 *qp = at.q.p + (long long)(a + R / kv.G) * at.q.st + (long long)(h * kv.G + R % kv.G) * at.q.sh;
            if (!KV8) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
#pragma unroll
                    for (int x = 0; x < 2; ++x) qb[nq][ks][x] = ok ? *reinterpret_cast<const uint32_t *>(qp + ks * 16 + x * 8 + 2 * c) : 0u;
            } else {
                uint2 raw[8];                             // elements 16 x + 4 c .. + 3 of the row, x = 0..7
                uint32_t m = 0;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    raw[x] = ok ? *reinterpret_cast<const uint2 *>(qp + x * 16 + 4 * c) : make_uint2(0u, 0u);
                    m = amax_bits(amax_bits(m, raw[x].x), raw[x].y);
                }
                m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
                float inv;
                const float f = row_factor(amax_of_halves(m), inv);
#pragma unroll
                for (int e = 0; e < 2; ++e) cs[nq][e] *= __shfl_sync(0xffffffffu, f, (2 * c + e) * 4);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t a01 = code_pair(raw[x].x, inv), a23 = code_pair(raw[x].y, inv);
                    qb[nq][x >> 1][x & 1] = __byte_perm(a01, a23, 0x5410);
                    qb[nq][4 + (x >> 1)][x & 1] = __byte_perm(a01, a23, 0x7632);
                }
            }
        }

        // ---- this warp's slices of units u0 .. u1-1 that hold a visible key
        const int j_first = u0 * C::kUnit + warp * C::kSlice;
        const int n_sl = lim_hi <= j_first ? 0 : min(u1 - u0, (lim_hi - j_first + C::kUnit - 1) / C::kUnit);
        const long long row_step = kv.page_size ? kD : kv.stride_n;
        long long base = 0, sbase = 0;                    // contiguous: row 0 of the head
        const int *table = nullptr;
        if (kv.page_size) table = kv.block_table + (long long)p * kv.max_pages;
        else { base = (long long)p * kv.stride_p + (long long)h * kv.stride_h; sbase = ((long long)p * kv.H_kv + h) * kv.N_max; }
        constexpr int kGroups = C::kSlice / 16;           // 16-key groups: a group lies inside one page
        int ent[kGroups];                                 // lane l: page entries of slice (s & ~31) + l
        uint32_t bad_bits = 0;                            // 2 bits per slice in flight, the oldest at the bottom
        auto lookup = [&](int s) {
#pragma unroll
            for (int q = 0; q < kGroups; ++q) {
                const int j = j_first + (s + lane) * C::kUnit + q * 16;
                ent[q] = s + lane < n_sl && j < N ? table[j / kv.page_size] : -2;
            }
        };
        // A lane's copies of a slice: row lane / kLanes + it * kRowsPer, 16-byte piece lane % kLanes.  Whole slices go by pointers that
        // advance by constants; slices that end the prefix or touch a bad page are copied row by row with zero fill.
        constexpr int kLanes = KV8 ? 8 : 16, kRowsPer = 32 / kLanes, kEb = KV8 ? 1 : 2, kRowB = 128 * kEb;
        const int my_r = lane / kLanes, my_ch = lane % kLanes;
        const uint8_t *k_src = KV8 ? c8.k8 : reinterpret_cast<const uint8_t *>(kv.k), *v_src = KV8 ? c8.v8 : reinterpret_cast<const uint8_t *>(kv.v);
        const long long my_off = (my_r * row_step + (KV8 ? my_ch * 16 : my_ch * 8)) * kEb, it_step = row_step * kRowsPer * kEb;
        const uint32_t my_dst = my_r * kRowB + ((my_ch ^ my_r) << 4);                     // r & 7 = my_r ^ (it * kRowsPer & 7)
        int st_in = 0;                                    // stage of the next slice issued
        auto issue = [&](int s) {
            if (s < n_sl) {
                if (kv.page_size && (s & 31) == 0) lookup(s);
                const int j0 = j_first + s * C::kUnit;
                const uint32_t dst = ring_u + st_in * C::kStage;
                uint32_t bad = 0;
                long long soff[kGroups], off[kGroups];    // first row of a group: its scale, its bytes
#pragma unroll
                for (int q = 0; q < kGroups; ++q) {
                    if (kv.page_size) {
                        const int page = __shfl_sync(0xffffffffu, ent[q], s & 31), j = j0 + q * 16;
                        if (j < N && (page < 0 || page >= kv.num_pages)) bad |= 1u << q;
                        soff[q] = ((long long)page * kv.H_kv + h) * kv.page_size + (j & (kv.page_size - 1));
                        off[q] = soff[q] * kRowB;
                    } else {
                        soff[q] = sbase + j0 + q * 16;
                        off[q] = (base + (long long)(j0 + q * 16) * kv.stride_n) * kEb;
                    }
                }
                if (j0 + C::kSlice <= N && bad == 0) {
#pragma unroll
                    for (int q = 0; q < kGroups; ++q) {
                        const uint8_t *kp = k_src + off[q] + my_off, *vp = v_src + off[q] + my_off;
#pragma unroll
                        for (int i = 0; i < 16 / kRowsPer; ++i) {
                            const uint32_t d = dst + ((my_dst + (q * 16 + i * kRowsPer) * kRowB) ^ (((i * kRowsPer) & 7) << 4));
                            cp_async_16(d, kp);
                            cp_async_16(d + C::kHalf, vp);
                            kp += it_step;
                            vp += it_step;
                        }
                    }
                    if (KV8) {
                        const long long so = (lane < 16 ? soff[0] : soff[kGroups - 1]) + (lane & 15);
                        cp_async_4z(dst + 2 * C::kHalf + lane * 4, c8.k_scale + so, true);
                        cp_async_4z(dst + 2 * C::kHalf + 128 + lane * 4, c8.v_scale + so, true);
                    }
                } else {
                    if (bad && status && lane == 0) atomicOr(status, MAGE_DEV_BAD_PAGE);
#pragma unroll 1
                    for (int r = my_r; r < C::kSlice; r += kRowsPer) {
                        const int q = r >> 4;
                        const bool take = !((bad >> q) & 1u) && j0 + r < N;
                        const long long o = take ? (q ? off[kGroups - 1] : off[0]) + ((r & 15) * row_step + (KV8 ? my_ch * 16 : my_ch * 8)) * kEb : 0;
                        const uint32_t d = dst + r * kRowB + ((my_ch ^ (r & 7)) << 4);
                        cp_async_16z(d, k_src + o, take);
                        cp_async_16z(d + C::kHalf, v_src + o, take);
                    }
                    if (KV8) {
                        const bool take = !((bad >> (lane >> 4)) & 1u) && j0 + lane < N;
                        const long long o = take ? (lane < 16 ? soff[0] : soff[kGroups - 1]) + (lane & 15) : 0;
                        cp_async_4z(dst + 2 * C::kHalf + lane * 4, c8.k_scale + o, take);
                        cp_async_4z(dst + 2 * C::kHalf + 128 + lane * 4, c8.v_scale + o, take);
                    }
                }
                bad_bits |= bad << (2 * st_in);
                if (++st_in == kDecStages) st_in = 0;
            }
            cp_async_commit();
        };

        float o[NQ][8][4];
        float m[NQ][2], l[NQ][2];
        uint32_t v_ref = 22u << 23;                       // (a power of two: its bits)
        int first_key = 0x7fffffff;                       // of this warp that is not left out: rows that see it took a key
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            m[nq][0] = m[nq][1] = -INFINITY;
            l[nq][0] = l[nq][1] = 0.f;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[nq][t][0] = o[nq][t][1] = o[nq][t][2] = o[nq][t][3] = 0.f;
        }

#pragma unroll 1
        for (int s = 0; s < kDecStages - 1; ++s) issue(s);
#pragma unroll 1
        for (int s = 0, st = 0; s < n_sl; ++s, st = st + 1 == kDecStages ? 0 : st + 1) {
            issue(s + kDecStages - 1);
            cp_async_wait<kDecStages - 1>();
            __syncwarp();
            const int j0 = j_first + s * C::kUnit, mi = lane >> 3, lr8 = lane & 7;
            const uint32_t k_u = ring_u + st * C::kStage, v_u = k_u + C::kHalf;
            const float *ksc = reinterpret_cast<const float *>(ring + st * C::kStage + 2 * C::kHalf), *vsc = ksc + 32;
            const uint32_t bad = (bad_bits >> (2 * st)) & 3u;
            bad_bits &= ~(3u << (2 * st));
            constexpr int KT = C::kSlice / 16;            // tiles of 16 keys
            first_key = min(first_key, bad == 0 ? j0 : (KT > 1 && bad == 1u ? j0 + 16 : 0x7fffffff));
            // S^T: keys 16 t + g, + 8 and rows 2 c, 2 c + 1; two sums each, so that the products do not wait for one another
            float x[KT][NQ][4];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                float y[NQ][4];
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][nq][e] = y[nq][e] = 0.f;
                const uint32_t row = k_u + (t * 16 + (mi & 1) * 8 + lr8) * kRowB;
                if (!KV8) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        uint32_t a[4];
                        ldsm4(row + (((2 * ks + (mi >> 1)) ^ lr8) << 4), a);
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) mma_bf16(ks & 1 ? y[nq] : x[t][nq], a, qb[nq][ks][0], qb[nq][ks][1]);
                    }
                } else {
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) {
                        uint32_t a[4];
                        ldsm4(row + (((2 * ks + (mi >> 1)) ^ lr8) << 4), a);
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) {
                            mma_e4m3(x[t][nq], a, qb[nq][ks][0], qb[nq][ks][1]);
                            mma_e4m3(y[nq], a, qb[nq][4 + ks][0], qb[nq][4 + ks][1]);
                        }
                    }
                }
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][nq][e] += y[nq][e];
            }
            // Logits up to the row's factor cs > 0 (8-bit: times the keys' scales); what a row does not see becomes -inf whatever it was
            const bool masked = j0 + C::kSlice > lim_lo || bad != 0;
            float mx[NQ][2];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mx[nq][0] = mx[nq][1] = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const float k0 = KV8 ? ksc[t * 16 + g] : 1.f, k1 = KV8 ? ksc[t * 16 + 8 + g] : 1.f;
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) {
                    if (KV8) { x[t][nq][0] *= k0; x[t][nq][1] *= k0; x[t][nq][2] *= k1; x[t][nq][3] *= k1; }
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (j0 + t * 16 + g + (e >> 1) * 8 >= lim[nq][e & 1] || ((bad >> t) & 1u)) x[t][nq][e] = -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) mx[nq][e] = max3(mx[nq][e], x[t][nq][e], x[t][nq][2 + e]);
                }
            }
            // 8-bit: the running power of two v_ref >= every value scale so far, of keys that some row of the tile sees; o is kept over v_ref / 2^14
            uint32_t ref_new = v_ref;
            bool wide = false;                            // some scale is below 2^-21 of it
            if (KV8) {
                uint32_t vb = __float_as_uint(vsc[lane]);
                if (vb >= __float_as_uint(kScaleEnd) || j0 + lane >= lim_hi) vb = 0;      // (NaN, or no scale, takes no part)
                ref_new = max(v_ref, (__reduce_max_sync(0xffffffffu, vb) + 0x7fffffu) & 0x7f800000u);
                wide = __any_sync(0xffffffffu, vb - 1u < ref_new - (21u << 23) - 1u);       // (as bits; 0 is no scale)
            }
            bool moved = ref_new != v_ref;
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) mx[nq][e] = fmaxf(mx[nq][e], __shfl_xor_sync(0xffffffffu, mx[nq][e], w));
                    mx[nq][e] = __fmul_rn(mx[nq][e], cs[nq][e]);
                    moved |= mx[nq][e] > m[nq][e];
                }
            if (__any_sync(0xffffffffu, moved)) {
                const float g_ref = KV8 ? __uint_as_float(v_ref) / __uint_as_float(ref_new) : 1.f;
                v_ref = ref_new;
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float m_new = fmaxf(m[nq][e], mx[nq][e]);
                        f[e] = m_new == -INFINITY ? 1.f : ex2(m[nq][e] - m_new);
                        m[nq][e] = m_new;
                        l[nq][e] *= f[e];
                        f[e] *= g_ref;
                    }
#pragma unroll
                    for (int t = 0; t < 8; ++t) { o[nq][t][0] *= f[0]; o[nq][t][1] *= f[1]; o[nq][t][2] *= f[0]; o[nq][t][3] *= f[1]; }
                }
            }
            const float v_mul = KV8 ? __uint_as_float((268u << 23) - v_ref) : 1.f;          // 2^14 / v_ref
            uint32_t pb[KT][NQ][2];                       // P^T as B fragments: keys 16 t + 2 c, + 1 (and + 8) of row g
            auto weigh = [&](auto in_bf16) {              // P, and with an 8-bit cache times the value scales
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    const float v0 = KV8 ? vsc[t * 16 + g] * v_mul : 1.f, v1 = KV8 ? vsc[t * 16 + 8 + g] * v_mul : 1.f;
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) {
                        float pr[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float ref = m[nq][e & 1] == -INFINITY ? 0.f : m[nq][e & 1];
                            // the logit is rounded before the reference, the largest rounded one, is taken off: no exponent is above 0, and the
                            // largest key's is 0 (the remainder of an fma would be up to half a step of the reference, however large that is)
                            pr[e] = ex2(__fsub_rn(__fmul_rn(x[t][nq][e], cs[nq][e & 1]), ref));
                            l[nq][e & 1] += pr[e];
                        }
                        uint32_t u0, u1;
                        if (KV8) {
                            // P times the value scales in f16: at most 2^14, eleven bits down to 2^-28 of the largest, nothing lost above 2^-38
                            pr[0] *= v0; pr[1] *= v0; pr[2] *= v1; pr[3] *= v1;
                            if (masked) {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (x[t][nq][e] == -INFINITY) pr[e] = 0.f;    // (a NaN scale behind the mask)
                            }
                            u0 = in_bf16.value ? pack_bf16x2(pr[0], pr[1]) : pack_f16x2(pr[0], pr[1]);
                            u1 = in_bf16.value ? pack_bf16x2(pr[2], pr[3]) : pack_f16x2(pr[2], pr[3]);
                        } else {
                            u0 = pack_bf16x2(pr[0], pr[1]);   // rounding of P: 2^-8 relative, like the output's own
                            u1 = pack_bf16x2(pr[2], pr[3]);
                        }
                        pb[t][nq][0] = transpose8(u0);
                        pb[t][nq][1] = transpose8(u1);
                    }
                }
            };
            if (!KV8) {
                weigh(std::true_type{});
                bool plain = true;
                if (j0 + C::kSlice > lim_lo) {
                    // Some row does not see some key of this slice.  0 * v is 0 only for a finite v: look for others.
                    bool odd = false;
#pragma unroll
                    for (int it = 0; it < 8; ++it) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(ring + st * C::kStage + C::kHalf + (it * 32 + lane) * 16);
                        const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) odd |= (w4[q] & 0x7f80u) == 0x7f80u || (w4[q] & 0x7f800000u) == 0x7f800000u;
                    }
                    plain = !__any_sync(0xffffffffu, odd);
                }
                const uint32_t row = v_u + ((mi >> 1) * 8 + lr8) * kRowB;                 // V^T: elements 16 t + g, + 8; keys 2 c, + 1 and + 8
                if (plain) {
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        uint32_t a[4];
                        ldsm4t(row + (((2 * t + (mi & 1)) ^ lr8) << 4), a);
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) mma_bf16(o[nq][t], a, pb[0][nq][0], pb[0][nq][1]);
                    }
                } else {
                    // the slice row by row, every key taken out of the product for the rows that do not see it (error path of
                    // tokens whose values are NaN or infinite: earlier rows must not notice them)
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll 1
                        for (int r = 0; r < 8; ++r) {
                            const int l0 = __shfl_sync(0xffffffffu, lim[nq][0], r >> 1), l1 = __shfl_sync(0xffffffffu, lim[nq][1], r >> 1), lr = r & 1 ? l1 : l0;
#pragma unroll
                            for (int t = 0; t < 8; ++t) {
                                uint32_t a[4];
                                ldsm4t(row + (((2 * t + (mi & 1)) ^ lr8) << 4), a);
#pragma unroll
                                for (int q = 0; q < 4; ++q) {                 // keys (q >> 1) * 8 + 2 c, + 1
                                    const int j = j0 + (q >> 1) * 8 + 2 * c;
                                    if (j >= lr) a[q] &= 0xffff0000u;
                                    if (j + 1 >= lr) a[q] &= 0x0000ffffu;
                                }
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_bf16(d, a, pb[0][nq][0], pb[0][nq][1]);
                                if (c == r >> 1) {
                                    if (r & 1) { o[nq][t][1] += d[1]; o[nq][t][3] += d[3]; }
                                    else { o[nq][t][0] += d[0]; o[nq][t][2] += d[2]; }
                                }
                            }
                        }
                }
            } else {
                auto product = [&](auto in_bf16) {
#pragma unroll
                    for (int t = 0; t < 8; ++t) {             // V^T: elements 16 t + 2 g (A rows g) and 16 t + 2 g + 1 (A rows g + 8)
                        uint32_t b[4];                        // both elements of keys 8 q + 2 c, + 1
                        ldsm4t(v_u + lane * 128 + ((t ^ lr8) << 4), b);
                        uint32_t ev[4], od[4];                // codes of a key pair side by side, then exactly to f16
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t w = __byte_perm(b[q], 0, 0x3120);
                            asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(ev[q]), "=r"(od[q]) : "r"(w));
                        }
                        if (in_bf16.value) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const float2 x0 = __half22float2(*reinterpret_cast<const __half2 *>(&ev[q])), x1 = __half22float2(*reinterpret_cast<const __half2 *>(&od[q]));
                                ev[q] = pack_bf16x2(x0.x, x0.y);
                                od[q] = pack_bf16x2(x1.x, x1.y);
                            }
                        }
                        const uint32_t a0[4] = {ev[0], od[0], ev[1], od[1]}, a1[4] = {ev[2], od[2], ev[3], od[3]};
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) {
                            if (in_bf16.value) {
                                mma_bf16(o[nq][t], a0, pb[0][nq][0], pb[0][nq][1]);
                                mma_bf16(o[nq][t], a1, pb[KT - 1][nq][0], pb[KT - 1][nq][1]);
                                continue;
                            }
                            mma_f16(o[nq][t], a0, pb[0][nq][0], pb[0][nq][1]);
                            mma_f16(o[nq][t], a1, pb[KT - 1][nq][0], pb[KT - 1][nq][1]);
                        }
                    }
                };
                if (__builtin_expect(wide, 0)) {          // (code of its own: 32 sequences of 1 to 131072 tokens 109.6 us, within the common code 114, without it 107.8)
                    weigh(std::true_type{});
                    product(std::true_type{});
                } else {
                    weigh(std::false_type{});
                    product(std::false_type{});
                }
            }
            __syncwarp();
        }
        cp_async_wait<0>();
        __syncwarp();

        // ---- merge of the four warps: each stages its o in its own ring (16-byte pieces permuted by row against bank conflicts)
        const float back = KV8 ? __uint_as_float(v_ref - (14u << 23)) : 1.f;
        float *stg = reinterpret_cast<float *>(ring);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = nq * 8 + 2 * c + e, sw = (r & 7) << 2;
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[nq][e] += __shfl_xor_sync(0xffffffffu, l[nq][e], w);
                if (m[nq][e] == -INFINITY && lim[nq][e] > first_key) m[nq][e] = kLowest;
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    if (KV8) {
                        *reinterpret_cast<float2 *>(stg + r * kD + ((t * 16 + 2 * g) ^ sw)) = make_float2(o[nq][t][e] * back, o[nq][t][2 + e] * back);
                    } else {
                        stg[r * kD + ((t * 16 + g) ^ sw)] = o[nq][t][e];
                        stg[r * kD + ((t * 16 + 8 + g) ^ sw)] = o[nq][t][2 + e];
                    }
                }
                if (g == 0) { s_m[warp][r] = m[nq][e]; s_l[warp][r] = l[nq][e]; }
            }
        __syncthreads();
        {
            constexpr int kPerRow = kDecWarps * 32 / kRows;                               // threads of a row
            const int r = tid / kPerRow, sw = (r & 7) << 2, R = rt * kRows + r;
            float m_all = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kDecWarps; ++w) m_all = fmaxf(m_all, s_m[w][r]);
            float wt[kDecWarps], l_all = 0.f;
#pragma unroll
            for (int w = 0; w < kDecWarps; ++w) {
                wt[w] = s_m[w][r] == -INFINITY ? 0.f : ex2(s_m[w][r] - m_all);
                l_all += s_l[w][r] * wt[w];
            }
            const bool whole = u0 == 0 && u1 == units;
            const int i = R / kv.G, hq = h * kv.G + R % kv.G;
            const bool sees = visible(N - n_new + i, N, at.mask_block) > 0 && m_all != -INFINITY;     // (the second: some key that it sees was not left out)
            float *slot = whole ? nullptr : part + ((size_t)blockIdx.x * 2 + (u0 > 0 ? 0 : 1)) * slot_floats(kRows);
            const float inv = sees ? 1.f / l_all : 0.f;
            if (r < rows) {
#pragma unroll
                for (int col = (tid % kPerRow) * 4; col < kD; col += kPerRow * 4) {
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < kDecWarps; ++w) {
                        const float4 v = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem_raw + w * (kDecStages * C::kStage)) + r * kD + (col ^ sw));
                        acc.x = fmaf(v.x, wt[w], acc.x); acc.y = fmaf(v.y, wt[w], acc.y); acc.z = fmaf(v.z, wt[w], acc.z); acc.w = fmaf(v.w, wt[w], acc.w);
                    }
                    if (whole) {
                        const uint2 b = sees ? make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv)) : make_uint2(0u, 0u);
                        *reinterpret_cast<uint2 *>(at.out + ((long long)(a + i) * kv.H_q + hq) * kD + col) = b;
                    } else {
                        *reinterpret_cast<float4 *>(slot + r * kD + col) = acc;
                    }
                }
                if (tid % kPerRow == 0) {
                    if (whole) {
                        if (at.lse) at.lse[(long long)(a + i) * kv.H_q + hq] = sees ? (m_all + log2f(l_all)) * 0.6931471805599453f : -INFINITY;
                    } else {
                        slot[kRows * kD + r] = m_all;
                        slot[kRows * kD + kRows + r] = l_all;
                    }
                }
            }
        }
        __syncthreads();
    }
}

// Merge of one row's partial results, of runs c0 .. c1 in ascending order, so that the result does not depend on timing.
// slot(c): o[n_rows][128], m[n_rows], l[n_rows] of run c.
__device__ __forceinline__ void store_merged(int lane, const float4 &acc, float m_all, float l_all, bool sees, const AttnArgs &at, long long row) {
    sees = sees && m_all != -INFINITY;
    const float inv = 1.f / l_all;
    const uint2 b = sees ? make_uint2(ptx::pack_bf16x2(acc.x * inv, acc.y * inv), ptx::pack_bf16x2(acc.z * inv, acc.w * inv)) : make_uint2(0u, 0u);
    *reinterpret_cast<uint2 *>(at.out + row * kD + lane * 4) = b;
    if (at.lse && lane == 0) at.lse[row] = sees ? (m_all + log2f(l_all)) * 0.6931471805599453f : -INFINITY;
}
__device__ __forceinline__ void add_scaled(float4 &acc, const float4 &v, float f) {
    acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y); acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
}
__device__ __forceinline__ float part_weight(float m_c, float m_all) { return m_c == -INFINITY ? 0.f : ptx::ex2(m_c - m_all); }

// Few parts (at most eight): one warp.
template <typename SlotOf>
__device__ __forceinline__ void merge_row_warp(int lane, int c0, int c1, int r, int n_rows, SlotOf slot, bool sees, const AttnArgs &at, long long row) {
    const int n = c1 - c0 + 1;
    float4 v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < n) v[q] = *reinterpret_cast<const float4 *>(slot(c0 + q) + r * kD + lane * 4);
    const float m_c = lane < n ? slot(c0 + lane)[n_rows * kD + r] : -INFINITY;
    float m_all = m_c;
#pragma unroll
    for (int s = 4; s; s >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, s));
    m_all = __shfl_sync(0xffffffffu, m_all, 0);
    const float wt = part_weight(m_c, m_all);
    const float l_c = lane < n ? slot(c0 + lane)[n_rows * kD + n_rows + r] * wt : 0.f;
    float l_all = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        l_all += __shfl_sync(0xffffffffu, l_c, q);
        const float f = __shfl_sync(0xffffffffu, wt, q);
        if (q < n) add_scaled(acc, v[q], f);
    }
    store_merged(lane, acc, m_all, l_all, sees, at, row);
}
// Many parts (a long cache and little else in the call): the four warps of a CTA take every fourth part, eight in flight each.
constexpr int kMostParts = 2 * 148;
constexpr int kMergeY = 16;                                // CTAs per run of the merge of prompts
template <typename SlotOf>
__device__ __forceinline__ void merge_row_block(int c0, int c1, int r, int n_rows, SlotOf slot, bool sees, const AttnArgs &at, long long row) {
    __shared__ float wts[kMostParts], red[8];
    __shared__ float4 accs[4][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = c1 - c0 + 1;
    float m_all = -INFINITY;
    for (int c = tid; c < n; c += 128) m_all = fmaxf(m_all, wts[c] = slot(c0 + c)[n_rows * kD + r]);
#pragma unroll
    for (int s = 16; s; s >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, s));
    if (lane == 0) red[warp] = m_all;
    __syncthreads();
    m_all = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float l = 0.f;
    for (int c = tid; c < n; c += 128) {
        const float w = part_weight(wts[c], m_all);
        wts[c] = w;
        l += slot(c0 + c)[n_rows * kD + n_rows + r] * w;
    }
#pragma unroll
    for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
    if (lane == 0) red[4 + warp] = l;
    __syncthreads();
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int cb = warp; cb < n; cb += 32) {
        float4 v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (cb + 4 * q < n) v[q] = *reinterpret_cast<const float4 *>(slot(c0 + cb + 4 * q) + r * kD + lane * 4);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (cb + 4 * q < n) add_scaled(acc, v[q], wts[cb + 4 * q]);
    }
    accs[warp][lane] = acc;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) add_scaled(acc, accs[w][lane], 1.f);
        store_merged(lane, acc, m_all, (red[4] + red[5]) + (red[6] + red[7]), sees, at, row);
    }
    __syncthreads();
}

// Two parts, the common case of a prompt: a warp takes four rows at once, so that 128 bytes a lane are in flight.
// Row q of the four is r0 + q * step of the tile; row_of(q): its output row, -1 if there is none; sees(q): whether it sees a key.
template <typename SlotOf, typename RowOf, typename Sees>
__device__ __forceinline__ void merge_rows_pair(int lane, int c0, int r0, int step, int n_rows, SlotOf slot, RowOf row_of, Sees sees, const AttnArgs &at) {
    const float *s0 = slot(c0), *s1 = slot(c0 + 1);
    float4 v[4][2];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (row_of(q) >= 0) {
            v[q][0] = *reinterpret_cast<const float4 *>(s0 + (r0 + q * step) * kD + lane * 4);
            v[q][1] = *reinterpret_cast<const float4 *>(s1 + (r0 + q * step) * kD + lane * 4);
        }
    // (every row of a slot has room for its numbers; those of rows that are none are read and not used)
    const float *ml = (lane & 1 ? s1 : s0) + n_rows * kD + r0 + ((lane >> 1) & 3) * step;
    const float m_c = ml[0], l_c = ml[n_rows];
    const float m_all = fmaxf(m_c, __shfl_xor_sync(0xffffffffu, m_c, 1)), wt = part_weight(m_c, m_all), lw = l_c * wt, l_all = lw + __shfl_xor_sync(0xffffffffu, lw, 1);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float w0 = __shfl_sync(0xffffffffu, wt, 2 * q), w1 = __shfl_sync(0xffffffffu, wt, 2 * q + 1);
        const float ma = __shfl_sync(0xffffffffu, m_all, 2 * q), la = __shfl_sync(0xffffffffu, l_all, 2 * q);
        if (row_of(q) < 0) continue;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        add_scaled(acc, v[q][0], w0);
        add_scaled(acc, v[q][1], w1);
        store_merged(lane, acc, ma, la, sees(q), at, row_of(q));
    }
}

// Items whose keys were cut over several runs.  The first run's part is in its second slot (its last segment), the others' in their first.
// Decode: blockIdx.x = the first run, blockIdx.y = the row.  Prompts: blockIdx.y = y takes the rows y + kMergeY q of the tile, sixteen
// of them: with two parts four per warp at once (with four rows a CTA and one at a time per warp, 24 mixed chunks of 1 to 700 tokens took
// 6 % longer in all); with more the runs inside the item help, each with its share of the q, since an item of
// many parts comes with few others (4 tokens of 28 + 4 heads over 5000 keys: 45 us without, 18 with).
template <int kRows>                                  // rows of a tile; 256: prefill
__global__ void __launch_bounds__(128) combine_kernel(AttnArgs at, const Split *__restrict__ split, const float *__restrict__ part, int H_q, int G, int mt_toks) {
    constexpr bool PREFILL = kRows == 256;
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    const Split sp = split[blockIdx.x];
    if (sp.count == 0) return;
    const int c0 = sp.c0, n = sp.c1 - c0 + 1, col = blockIdx.x - c0, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto slot = [&](int c) { return part + ((size_t)c * 2 + (c > c0 ? 0 : 1)) * slot_floats(kRows); };
    // a row of the tile: its token (within the problem) and query head of the group; token -1: none
    auto token_of = [&](int r, int &g) -> int {
        if (PREFILL) {
            const int in = r & 127, t_in = in / G, i = (r >> 7) * mt_toks + t_in;
            g = in - t_in * G;
            return t_in < mt_toks && i < sp.count ? sp.first + i : -1;
        }
        g = (sp.first + r) % G;
        return r < sp.count ? (sp.first + r) / G : -1;
    };
    auto sees_of = [&](int tok) { return visible(sp.pos0 + tok, sp.N, at.mask_block) > 0; };
    constexpr int kStep = PREFILL ? kMergeY : 1, kPer = PREFILL ? kRows / kMergeY : 1;
    const int r0 = blockIdx.y;
    if (PREFILL && n == 2) {
        const int rw = r0 + warp * 4 * kStep;
        int row[4];                                        // (below 2^31 by the host's check)
        bool sees[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            int g;
            const int tok = token_of(rw + q * kStep, g);
            row[q] = tok < 0 ? -1 : (sp.a + tok) * H_q + sp.h * G + g;
            sees[q] = tok >= 0 && sees_of(tok);
        }
        merge_rows_pair(lane, c0, rw, kStep, kRows, slot, [&](int q) { return row[q]; }, [&](int q) { return sees[q]; }, at);
        return;
    }
    const bool few = n <= 8;
    const int cols = PREFILL ? max(1, n - 1) : 1;          // runs that share the work
#pragma unroll 1
    for (int q = few ? col + cols * warp : col; q < kPer; q += few ? cols * 4 : cols) {
        int g;
        const int tok = token_of(r0 + q * kStep, g);
        if (tok < 0) continue;
        const long long row = (long long)(sp.a + tok) * H_q + sp.h * G + g;
        if (few) merge_row_warp(lane, c0, sp.c1, r0 + q * kStep, kRows, slot, sees_of(tok), at, row);
        else merge_row_block(c0, sp.c1, r0 + q * kStep, kRows, slot, sees_of(tok), at, row);
    }
}

}  // namespace chunk
}  // namespace mage
