// Attention of many query rows per KV head (prompts and chunks of them) over the cache: the tensor-core kernel.
//
// A 128-row M-tile holds the G query heads of floor(128 / G) tokens, row = token * G + head, so that one TMA box per d-half fetches its
// queries straight out of a packed projection; a row tile is two M-tiles.  An item is (row tile, KV head), its units are the 128-key
// tiles that its last row sees.  The units of the whole call, in the order (problem, row tile, head, key tile), are cut into
// runs of equal cost, one per CTA (one CTA per SM), from the lengths on the device: causal masks, ragged batches and a number of
// items that is no multiple of 148 all balance.  A unit of an item with one M-tile costs less, and every item a fixed share.  A run that
// starts or ends inside an item leaves a partial (o, m, l) that combine_kernel merges.
//
// Per item the CTA runs the online softmax on tcgen05: two 128-row M-tiles, S = Q K^T into tensor memory, one warpgroup per M-tile
// (thread = row) turns S into P = 2^(c s - m) in place, O += P V.  The two M-tiles alternate, so one's products run under the
// other's exponentials.  With at most 128 rows the two warpgroups take alternate key tiles of the same rows instead, each with a
// sum of its own, merged at the end.  A row's reference m moves only when it lags (Ref::kRescale), at the start of the next tile; a
// jump inside a part of a tile that P could not hold (Ref::kMost) redoes that part, once, with the new reference.
//
// Roles (all hand-offs by mbarriers with bounded waits; ring positions run on over the items, so the next item's keys are on their
// way while this one is finished):
//   16-bit cache:  warps 0-7 softmax, 8 K tiles by TMA, 9 MMA issue, 10 item list, Q tiles and the check of V tiles, 11 V tiles by TMA
//   8-bit cache:   warps 0-7 Q rows as e4m3 hi + lo codes and softmax, 8 item list, K and V tiles by TMA, scales, 9 MMA issue,
//                  10-11 V codes widened to f16
//
// 8-bit cache: S is the sum of two e4m3 products (hi and lo codes of the query, see chunk_decode.cuh) at twice the bf16 rate each, so
// it costs what the 16-bit product costs; the scale of a key multiplies its column of S.  Values are widened to f16 (exact) and
// multiplied by 2^7 times their scales over v_ref, a power of two that is at least every scale of the item's tiles so far (448 * 2^7
// fits f16, and a scale keeps eleven bits down to 2^-21 of the largest: a row of zeros has scale 1, others may be far below);
// O is kept over v_ref / 2^7 and P is f16 too, with the reference four binades below the maximum, so that nothing above 2^-28 of a row's largest P is lost.
// (Multiplying P's columns by the scales instead keeps the softmax warps, which set the pace, busy longer: a fifth more time for 2001
// tokens behind 16384 when it was tried.)
// Where a tile has a scale below 2^-21 of v_ref (a large row anywhere in front of it, or a row of zeros beside very small ones), f16 would
// take bits from it, or all of them: such a tile is in bf16, whose range needs no such care, the values times the scale's power of two (exact)
// and P times its mantissa, so that there is one rounding as elsewhere.
// A value row with a NaN scale enters as zeros, and rows that see it are made NaN at the end.
//
// 0 * v is 0 only for a finite v.  Rows of V at or behind the prefix's end are zeroed in shared memory; in a key tile that some row of
// the CTA does not see whole, warp 10 looks for NaN and infinite values.  If there are any, every row notes for which of the 128
// columns it sees one (added back to its result at the end), and they are zeroed before the product.
#pragma once
#include <type_traits>

#include "chunk_decode.cuh"

namespace mage {
namespace chunk {

constexpr int kPreRows = 256, kPreTile = 128;
constexpr int kPreSlot = slot_floats(kPreRows);
constexpr int kPreHalf = kPreTile * 128;                   // 128 rows of 128 bytes: one swizzled d-half (16 bits) or a whole tile of codes
constexpr int kPreTileBytes = 2 * kPreHalf;
constexpr int kSegRing = 8;
// Relative times of a key tile, of a key tile of an item with one M-tile, and of an item's begin and end, where the 8-bit cache has
// the queries to code.  (24 mixed chunks of 1 to 700 tokens: 16 bits 88.3 us with an item at 4, 87.1 at 6, 88.6 at 8, 92.1
// at 10; 8 bits 133 at 6, 122 at 8, 124 at 10; another mix 81.6, 81.4, 82.9, 86.1 and 126, 118, 119.)
constexpr int kUnitCost = 3, kUnitCost1 = 2, kItemCost16 = 6, kItemCost8 = 8;
// A row's reference moves at the next tile when the tile's sum of 2^(x - m) has passed kRescale (to where that sum would be
// 2^kUp); a half tile whose sum has passed kMost is redone.  The sum stands for the maximum, which the sweep then need not track:
// it is at most 128 times 2^(max - m).  kMost is what the sum O of P v has to bear on top of the values themselves: 2^30 leaves room for
// values of 2^70 in a cache of 2^20 rows.
// With P in f16 (8-bit cache) the reference sits kUp binades below the maximum and a half tile is redone before P leaves f16's range.
// The mantissa of a scale, 1 <= m < 2 (something finite for those that enter as zeros).
__device__ __forceinline__ float mantissa(float scale) { return __uint_as_float((__float_as_uint(scale) & 0x7fffffu) | 0x3f800000u); }
template <bool KV8>
struct Ref {
    static constexpr float kUp = KV8 ? 4.f : 0.f, kRescale = KV8 ? 16384.f : 1024.f, kMost = KV8 ? 32768.f : 1073741824.f, kMostLog = KV8 ? 15.f : 24.f;
};

// Straight-line code takes the reference off the unrounded product c s in one fma, which is exact enough while half a step of the
// reference is small (2^-9 here).  Beyond, and wherever a reference is chosen, the logit is rounded first: the row's largest one is then
// at most 2 kUp above a reference taken from it (0 where its step is larger than that), however large it is.
constexpr float kFar = 65536.f;

constexpr uint32_t kValueBits = 7;                         // 8-bit cache: binades between the largest value factor and 1

struct Seg {                                               // a run's part of one item, published by one warp for the others
    int p, h, a, n_new, N;                                 // problem, KV head, first packed token, new tokens, length
    int tok0, toks;                                        // first token of the row tile (within the problem's), tokens in it
    int t0, t1;                                            // key tiles
    int lim_first;                                         // keys that the tile's first row sees
    int slot;                                              // partial result: its slot; -1: whole item
    int lim_last;                                          // keys that the tile's last row sees (of the publishing warp)
    int pad[4];
};
static_assert(sizeof(Seg) == 64, "");

template <bool KV8>
struct Pre {
    static constexpr int kThreads = 384;           // twelve warps: 168 registers a thread
    static constexpr int kKSlots = 2, kVSlots = 2;
    static constexpr int kKBytes = KV8 ? kPreHalf : kPreTileBytes;
    static constexpr int kPubBytes = 2576;
    // Products of a tile as a loop of this many per turn.  Code that stays in the instruction cache counts for short items, no gap between
    // products for long ones: 24 mixed chunks and 4096 tokens behind 32768, 16 bits, 8 a turn 91.5 and 1984 us, 4: 87.3 and 1946, 2: 88.1
    // and 2050; 8 bits (and 2001 behind 16384), 8: 141 and 750, 2: 129 and 675, 1: 124 and 658.
    static constexpr int kMmaUnroll = KV8 ? 1 : 4;
    static constexpr int kItemCost = KV8 ? kItemCost8 : kItemCost16;
    static constexpr int offQ = 0, offK = 2 * kPreTileBytes, offV = offK + kKSlots * kKBytes, offV8 = offV + kVSlots * kPreTileBytes,
                         offPub = offV8 + (KV8 ? 2 * kPreHalf : 0), offSc = offPub + 4 * kPubBytes, offRowF = offSc + (KV8 ? 4 * 2 * kPreTile * 4 : 0),
                         offSeg = offRowF + (KV8 ? 2 * kPreRows * 4 : 0), offBar = offSeg + kSegRing * (int)sizeof(Seg);
    static constexpr size_t kSmem = 1024 + offBar + 512;
};

struct PreMaps {
    CUtensorMap q, k, v;
    int box_rows;                                          // rows of a TMA box: 128 (one box per tile and operand), or 16 .. 64
    int test_stall;
};

// Row tiles of `tt` tokens have fixed slots: problem p's are base(p) .. base(p) + tiles - 1 with base(p) = floor(q_start[p] / tt) + p, which
// ascend without overlap for any lengths.
__device__ __forceinline__ int slot_base(const ChunkView &cv, int p, int tt) { return cv.q_start[p] / tt + p; }
// Key tiles of row tile rt of a problem with n new tokens and length N (at least one, so that every row is written).
__device__ __forceinline__ int units_of(int n, int N, int tt, int rt, int mask_block) {
    return max(1, (visible(N - n + min((rt + 1) * tt, n) - 1, N, mask_block) + kPreTile - 1) / kPreTile);
}

// Walks row-tile slots in order, with the problem's numbers at hand.
// (kv.seq_lens and cv.q_start may point to copies in shared memory.)
struct SlotWalk {
    int p, a, n, N, tiles, base, next, tt, item;           // next: first slot of the problem behind; item: fixed cost of an item
    __device__ void load(const KvView &kv, const ChunkView &cv) {
        n = chunk_len_of(cv, p, &a, nullptr);
        N = seq_len_of(kv, p);
        base = slot_base(cv, p, tt);
        next = p + 1 < kv.P ? slot_base(cv, p + 1, tt) : 0x7fffffff;
        tiles = (n + tt - 1) / tt;
    }
    __device__ void seek(const KvView &kv, const ChunkView &cv, int slot) {            // the last p with base(p) <= slot
        int lo = 0, hi = kv.P - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (slot_base(cv, mid, tt) <= slot) lo = mid;
            else hi = mid - 1;
        }
        p = lo;
        load(kv, cv);
    }
    __device__ int units(const KvView &kv, const ChunkView &cv, int slot, int mask_block) {   // 0: no row tile in this slot
        while (next <= slot) {
            ++p;
            load(kv, cv);
        }
        const int rt = slot - base;
        return rt >= 0 && rt < tiles ? units_of(n, N, tt, rt, mask_block) : 0;
    }
    __device__ int unit_cost(int slot) { return n - (slot - base) * tt <= tt / 2 ? kUnitCost1 : kUnitCost; }       // (of a slot that units() has walked to)
    __device__ int cost(const KvView &kv, const ChunkView &cv, int slot, int mask_block) {
        const int u = units(kv, cv, slot, mask_block);
        return u ? u * unit_cost(slot) + item : 0;
    }
};

struct PreGrid {
    int slots;                                             // row-tile slots of the call
    int mt_toks;                                           // tokens of an M-tile: floor(128 / G)
    int min_cost;                                          // least cost of a run (at least kUnitCost: a run inside an item has a key tile)
    Split *split;                                          // [grid]
    float *part;
};
__device__ __forceinline__ long long runs_of(long long total, int grid, int min_cost) {
    const long long most = total / min_cost;
    return most < grid ? (most > 0 ? most : 1) : grid;
}

// Start of run b of n over a total cost.  (32-bit divisions where they do: a 64-bit one takes longer than the rest of a record.)
__device__ __forceinline__ long long run_start(long long total, int b, int n) {
    if (total < 0x7fffffff) {
        const unsigned t = (unsigned)total, q = t / (unsigned)n, r = t - q * (unsigned)n;
        return (long long)q * b + (r * (unsigned)b) / (unsigned)n;
    }
    return total * b / n;
}

// Bits of the 32 columns from c0 on that take part: inside the row's visible keys and not in a 16-key group with a bad page.
__device__ __forceinline__ uint32_t cols_ok(int c0, int valid, uint32_t bad) {
    uint32_t okm = valid - c0 >= 32 ? 0xffffffffu : (valid - c0 <= 0 ? 0u : (1u << (valid - c0)) - 1u);
    if (bad) {
        const uint32_t b = bad >> (c0 >> 4);
        if (b & 1u) okm &= 0xffff0000u;
        if (b & 2u) okm &= 0x0000ffffu;
    }
    return okm;
}

// Error path: which columns of d carry a non-finite value in a key that this row sees (first `valid` keys of the tile) and some other
// row does not (those from `seen` on).  tP: the row's P, since 0 * inf is NaN.  Called by whole warps.
__device__ __noinline__ void note_odd_values(const uint8_t *v_tile, int seen, int valid, uint32_t tP, uint32_t *pos, uint32_t *neg) {
    uint32_t zero[4];                                      // keys whose P is 0
#pragma unroll 1
    for (int c0 = 0; c0 < 4; ++c0) {
        uint32_t pr[16], z = 0;
        ptx::tmem_ld16(tP + c0 * 16, pr);
        ptx::tmem_wait_ld(pr);
#pragma unroll
        for (int e = 0; e < 16; ++e) z |= ((pr[e] & 0xffffu) == 0u ? 1u << (2 * e) : 0u) | ((pr[e] >> 16) == 0u ? 2u << (2 * e) : 0u);
        zero[c0] = z;
    }
    for (int r = seen; r < valid; ++r)
        for (int ch = 0; ch < 16; ++ch) {
            const uint4 v = *reinterpret_cast<const uint4 *>(v_tile + (ch >> 3) * kPreHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            for (int e = 0; e < 8; ++e) {
                const uint32_t x = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
                if ((x & 0x7f80u) != 0x7f80u) continue;
                const int d = ch * 8 + e;
                const bool nan = (x & 0x7fu) != 0 || ((zero[r >> 5] >> (r & 31)) & 1u);
                if (nan || !(x & 0x8000u)) pos[d >> 5] |= 1u << (d & 31);
                if (nan || (x & 0x8000u)) neg[d >> 5] |= 1u << (d & 31);
            }
        }
}

template <bool KV8>
__global__ void __launch_bounds__(Pre<KV8>::kThreads, 1)
prefill_kernel(const __grid_constant__ PreMaps maps, KvView kv, Kv8View c8, ChunkView cv, AttnArgs at, PreGrid pg, unsigned *status) {
    using namespace ptx;
    using C = Pre<KV8>;
    using R_ = Ref<KV8>;
    constexpr int kKSlots = C::kKSlots, kVSlots = C::kVSlots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *q_s = base + C::offQ, *k_s = base + C::offK, *v_s = base + C::offV;
    [[maybe_unused]] uint8_t *v8_s = base + C::offV8;
    [[maybe_unused]] float *sc_s = reinterpret_cast<float *>(base + C::offSc);         // [4][keys' scales 128, values' scales 128]
    [[maybe_unused]] float *rowf_s = reinterpret_cast<float *>(base + C::offRowF);     // [2][256] factors of the query rows
    Seg *seg_s = reinterpret_cast<Seg *>(base + C::offSeg);
    uint64_t *bars = reinterpret_cast<uint64_t *>(base + C::offBar);
    enum { SEG_FULL = 0, SEG_EMPTY = SEG_FULL + kSegRing, Q_FULL = SEG_EMPTY + kSegRing, Q_EMPTY, K_FULL, K_EMPTY = K_FULL + 2, V_FULL = K_EMPTY + 2, V_EMPTY = V_FULL + 2, V8_FULL = V_EMPTY + 2,
           V8_EMPTY = V8_FULL + 2, V_SCAN = V8_EMPTY + 2, V_READY = V_SCAN + 2, NOTED = V_READY + 2, S_FULL, P_FULL = S_FULL + 2, O_DONE = P_FULL + 2, PUB = O_DONE + 2,
           SEG_DONE = PUB + 2, N_BARS = SEG_DONE + 2 };
    static_assert(N_BARS * 8 + 80 <= 512, "");
    uint32_t *tmem_ptr_s = reinterpret_cast<uint32_t *>(bars + N_BARS);
    volatile int *abort_s = reinterpret_cast<volatile int *>(tmem_ptr_s + 1);
    volatile int *odd_s = reinterpret_cast<volatile int *>(tmem_ptr_s + 4);            // [2] per V slot: the tile holds non-finite values
    volatile uint32_t *bad_s = reinterpret_cast<volatile uint32_t *>(tmem_ptr_s + 6);  // [4] per key tile: 16-key groups with a bad page
    volatile int *vnan_s = reinterpret_cast<volatile int *>(tmem_ptr_s + 10);          // [4] per key tile (8-bit): some value row's scale is NaN
    volatile uint32_t *vref_s = reinterpret_cast<volatile uint32_t *>(tmem_ptr_s + 14);    // [4] per key tile (8-bit): v_ref as bits, + 1 for a tile in bf16
    long long *scan_s = reinterpret_cast<long long *>(seg_s);                          // prologue only
    auto bar = [&](int i) { return smem_u32(bars + i); };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        abort_s[0] = 0;
        abort_s[1] = maps.test_stall;
        for (int i = 0; i < kSegRing; ++i) {
            mbar_init(bar(SEG_FULL + i), 1);
            mbar_init(bar(SEG_EMPTY + i), C::kThreads / 32 - 1);     // every warp but the one that publishes reads every record
        }
        mbar_init(bar(Q_FULL), KV8 ? 8 : 1);
        mbar_init(bar(Q_EMPTY), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(K_FULL + i), 1);
            mbar_init(bar(K_EMPTY + i), 1);
            mbar_init(bar(V_FULL + i), KV8 ? 2 : 1);
            mbar_init(bar(V_EMPTY + i), 1);
            mbar_init(bar(V8_FULL + i), 1);
            mbar_init(bar(V8_EMPTY + i), 2);
            mbar_init(bar(V_SCAN + i), 1);
            mbar_init(bar(V_READY + i), 1);
            mbar_init(bar(S_FULL + i), 1);
            mbar_init(bar(P_FULL + i), 4);
            mbar_init(bar(PUB + i), 4);
            mbar_init(bar(O_DONE + i), 1);
            mbar_init(bar(SEG_DONE + i), 4);
        }
        mbar_init(bar(NOTED), 8);
        fence_mbar_init();
        fence_proxy_async();
        prefetch_tensormap(&maps.k);
        prefetch_tensormap(&maps.v);
    }
    if (warp == 9) { tmem_alloc(smem_u32(tmem_ptr_s), 512); tmem_relinquish(); }
    pdl_wait();
    pdl_launch_dependents();

    // ---- this CTA's run: prefix sums of the row tiles' costs, each thread over a contiguous share of the slots
    const int tt = 2 * pg.mt_toks;
    long long run0 = 0, run1 = 0, total = 0;
    int n_runs = 1;
    {
        // (lengths and ranges of up to 8000 problems are copied to the ring of value tiles first: the search below is a chain of loads)
        KvView kvp = kv;
        ChunkView cvp = cv;
        if (kv.P <= 8000) {
            int *qs = reinterpret_cast<int *>(v_s), *sl = qs + kv.P + 1;
            for (int p = tid; p <= kv.P; p += blockDim.x) {
                qs[p] = cv.q_start[p];
                if (p < kv.P && kv.seq_lens) sl[p] = kv.seq_lens[p];
            }
            cvp.q_start = qs;
            if (kv.seq_lens) kvp.seq_lens = sl;
            __syncthreads();
        }
        SlotWalk w;
        w.tt = tt;
        w.item = C::kItemCost;
        const int per = (pg.slots + (int)blockDim.x - 1) / (int)blockDim.x, s_lo = min(pg.slots, tid * per), s_hi = min(pg.slots, s_lo + per);
        long long mine = 0;
        if (s_lo < s_hi) {
            w.seek(kvp, cvp, s_lo);
            for (int s = s_lo; s < s_hi; ++s) mine += w.cost(kvp, cvp, s, at.mask_block);
        }
        if (blockIdx.x == 0 && status)                      // ranges that are none are reported once
            for (int p = tid; p < kv.P; p += blockDim.x) { int a; chunk_len_of(cvp, p, &a, status); }
        long long incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
        if (lane == 31) scan_s[warp] = incl;
        __syncthreads();
        long long before = 0;
        for (int i = 0; i < (int)(blockDim.x >> 5); ++i) {
            if (i < warp) before += scan_s[i];
            total += scan_s[i];
        }
        const long long first = before + incl - mine;
        total *= kv.H_kv;
        n_runs = (int)runs_of(total, gridDim.x, pg.min_cost);
        if ((int)blockIdx.x < n_runs) {
            run0 = run_start(total, (int)blockIdx.x, n_runs);
            run1 = run_start(total, (int)blockIdx.x + 1, n_runs);
        }
        // where the run starts: its slot, and the costs of one head in front of it
        const bool starts = run0 < run1 && run0 >= first * kv.H_kv && run0 < (first + mine) * kv.H_kv;
        if (starts) {
            if (per > 1 && s_lo < s_hi) w.seek(kvp, cvp, s_lo);
            long long off = first;
            for (int s = s_lo; s < s_hi; ++s) {
                const int n = w.cost(kvp, cvp, s, at.mask_block);
                if (run0 < (off + n) * kv.H_kv) {
                    scan_s[32] = off;
                    int *at_s = reinterpret_cast<int *>(scan_s + 33);
                    at_s[0] = s; at_s[1] = w.p; at_s[2] = w.a; at_s[3] = w.n; at_s[4] = w.N; at_s[5] = w.tiles; at_s[6] = w.base; at_s[7] = w.next;
                    break;
                }
                off += n;
            }
        }
        if (tid == 0) pg.split[blockIdx.x].count = 0;
    }
    fence_proxy_async();                                   // (the copies above lie where TMA will write)
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_ptr_s;
    // ---- the list of items, kept by one warp, from where the run starts
    SlotWalk walk;
    walk.tt = tt;
    walk.item = C::kItemCost;
    const int *at_s = reinterpret_cast<const int *>(scan_s + 33);
    int slot_at = at_s[0];
    walk.p = at_s[1]; walk.a = at_s[2]; walk.n = at_s[3]; walk.N = at_s[4]; walk.tiles = at_s[5]; walk.base = at_s[6]; walk.next = at_s[7];
    long long off_at = scan_s[32], u_at = run0;
    bool lists_ok = true;
    __syncthreads();                                       // scan_s shares the item ring

    // the next item's record; false at the end of the list
    auto next_seg = [&](int s, Seg &g) -> bool {
        if (!__all_sync(0xffffffffu, mbar_wait(bar(SEG_FULL + (s & (kSegRing - 1))), (s / kSegRing) & 1, abort_s, status))) return false;
        const volatile int *src = reinterpret_cast<const volatile int *>(seg_s + (s & (kSegRing - 1)));
        int *dst = reinterpret_cast<int *>(&g);
#pragma unroll
        for (int i = 0; i < 11; ++i) dst[i] = src[i];
        mbar_arrive_warp(bar(SEG_EMPTY + (s & (kSegRing - 1))));
        return g.t1 > g.t0;
    };

    auto publish = [&](int s) -> Seg {                 // record s, t1 = t0 = 0 behind the last item
        Seg g = {};
        if (!__all_sync(0xffffffffu, mbar_wait(bar(SEG_EMPTY + (s & (kSegRing - 1))), ((s / kSegRing) & 1) ^ 1, abort_s, status))) {
            lists_ok = false;
            return g;
        }
        long long x_item = 0, x_last = 0;                  // where the item's first and last tiles start
        bool cut = false;
        while (u_at < run1 && slot_at < pg.slots) {          // (the second condition holds unless q_start does not ascend)
            const int n = walk.units(kv, cv, slot_at, at.mask_block), uc = n ? walk.unit_cost(slot_at) : 1, cost = n ? n * uc + walk.item : 0;
            const long long local = u_at - off_at * kv.H_kv;
            if (local >= (long long)cost * kv.H_kv) {
                off_at += cost;
                ++slot_at;
                continue;
            }
            // an item's key tiles come first, its fixed cost last: a run that ends there has all of them; a tile is the run's in which it starts
            const int h = local < 0x7fffffff ? (int)((unsigned)local / (unsigned)cost) : (int)(local / cost), x0 = (int)(local - (long long)h * cost), x1 = (int)min((long long)cost, x0 + (run1 - u_at));
            const int t0 = (x0 + uc - 1) / uc, t1 = (x1 + uc - 1) / uc;
            u_at += x1 - x0;
            if (t0 >= min(t1, n)) continue;
            g.p = walk.p; g.h = h; g.a = walk.a; g.n_new = walk.n; g.N = walk.N;
            g.t0 = t0;
            g.t1 = min(t1, n);
            g.tok0 = (slot_at - walk.base) * tt;
            g.toks = min(tt, walk.n - g.tok0);
            g.lim_first = visible(walk.N - walk.n + g.tok0, walk.N, at.mask_block);
            g.lim_last = visible(walk.N - walk.n + g.tok0 + g.toks - 1, walk.N, at.mask_block);
            g.slot = g.t0 == 0 && g.t1 == n ? -1 : (int)blockIdx.x * 2 + (g.t0 > 0 ? 0 : 1);
            x_item = off_at * kv.H_kv + (long long)h * cost;
            x_last = x_item + (long long)(n - 1) * uc;
            cut = g.t1 < n;
            break;
        }
        if (lane == 0) seg_s[s & (kSegRing - 1)] = g;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(SEG_FULL + (s & (kSegRing - 1))));
        if (lane == 0 && cut) {                            // its parts lie in the runs in which its first and last tiles start
            auto run_at = [&](long long x) { return (int)min((long long)n_runs - 1, ((x + 1) * n_runs - 1) / total); };     // (the bound holds by itself unless q_start does not ascend)
            pg.split[blockIdx.x] = {g.a, g.h, g.N - g.n_new, g.N, g.tok0, g.toks, run_at(x_last), g.t0 == 0 ? (int)blockIdx.x : run_at(x_item)};
        }
        return g;
    };
    // ---- K and V tiles: lane b < n_box fetches box b of every tile; page entries are looked up a tile ahead
    const int n_box = kPreTile / maps.box_rows;
    constexpr uint32_t kLoadBytes = KV8 ? kPreHalf : kPreTileBytes;
    auto entry_at = [&](const Seg &g, int t) {
        const int j = t * kPreTile + lane * maps.box_rows;
        return kv.page_size && lane < n_box && t < g.t1 && j < g.N ? kv.block_table[(long long)g.p * kv.max_pages + j / kv.page_size] : -2;
    };
    // tile t of the item (the tc-th of the run) into its slot; ent: this lane's page entry
    auto fetch = [&](bool is_v, const Seg &g, int t, int tc, int ent) -> bool {
        const int slot = tc & 1, par = (tc >> 1) & 1, FULL = is_v ? (KV8 ? V8_FULL : V_FULL) : K_FULL, EMPTY = is_v ? (KV8 ? V8_EMPTY : V_EMPTY) : K_EMPTY;
        if (!__all_sync(0xffffffffu, mbar_wait(bar(EMPTY + slot), par ^ 1, abort_s, status)) || maps.test_stall) return false;
        const int j = t * kPreTile + lane * maps.box_rows;
        int c1 = 0, c3 = 0;
        bool bad = false;
        if (kv.page_size) {
            c1 = j & (kv.page_size - 1);
            c3 = kv.num_pages;                             // out of range: zero fill
            if (ent >= 0 && ent < kv.num_pages) c3 = ent;
            else bad = ent != -2;
        } else {
            c1 = j < g.N ? j : kv.N_max + 64;              // behind the prefix: zero fill
            c3 = g.p;
        }
        const uint32_t bad_boxes = __ballot_sync(0xffffffffu, bad);
        if (!is_v && lane == 0) {
            uint32_t groups = 0;
            if (bad_boxes) {
                for (int q = 0; q < 8; ++q)
                    if ((bad_boxes >> (q * 16 / maps.box_rows)) & 1u) groups |= 1u << q;
                if (status) atomicOr(status, MAGE_DEV_BAD_PAGE);
            }
            bad_s[tc & 3] = groups;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_expect_tx(bar(FULL + slot), kLoadBytes);
        __syncwarp();
        if (lane < n_box) {
            uint8_t *ring = is_v ? (KV8 ? v8_s : v_s) : k_s;
            const CUtensorMap *map = is_v ? &maps.v : &maps.k;
            const uint32_t dst = smem_u32(ring + slot * (int)kLoadBytes + lane * maps.box_rows * 128);
            tma_load_4d(dst, map, bar(FULL + slot), 0, c1, g.h, c3);
            if (!KV8) tma_load_4d(dst + kPreHalf, map, bar(FULL + slot), 64, c1, g.h, c3);
        }
        return true;
    };
    auto drain = [&](int FULL, int tc) {                   // after a wait that gave up: copies in flight land before the CTA leaves
        if (*abort_s)
            for (int x = max(0, tc - 2); x < tc; ++x) {
                const long long c0 = clock64();
                while (!mbar_try_wait(bar(FULL + (x & 1)), (x >> 1) & 1) && clock64() - c0 < 2000000) {}
            }
    };

    if (run0 >= run1) {
        // more CTAs than work
    } else if (!KV8 && (warp == 8 || warp == 11)) {
        // ------------------------------------------------------------------ 16-bit cache: K (warp 8) or V (warp 11) tiles
        const bool is_v = warp == 11;
        int tc = 0;                                        // tiles so far, over all items
        Seg g;
        bool ok = true;
        for (int s = 0; ok && next_seg(s, g); ++s) {
            int ent = entry_at(g, g.t0);
            for (int t = g.t0; ok && t < g.t1; ++t) {
                const int ent_next = entry_at(g, t + 1);
                ok = fetch(is_v, g, t, tc, ent);
                if (ok) ++tc;
                ent = ent_next;
            }
        }
        drain(is_v ? V_FULL : K_FULL, tc);
    } else if (KV8 && warp == 8) {
        // ------------------------------------------------------------------ 8-bit cache: item list, K and V tiles, scales
        Seg g = publish(0);
        int tc = 0, vc = 0;
        bool ok = lists_ok;
        for (int s = 0; ok && g.t1 > g.t0; ++s) {
            const Seg nxt = publish(s + 1);
            ok = lists_ok;
            int ent = entry_at(g, g.t0);
            uint32_t v_ref = 20u << 23;                    // (bits of a power of two)
            for (int t = g.t0; ok && t < g.t1; ++t) {
                const int ent_next = entry_at(g, t + 1);
                // scales of the tile's rows: in shared memory before the tile's barrier; 0 for keys that none of the queries sees, so that
                // they have no part in v_ref and their values enter as zeros
                float sk[4], sv[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = q * 32 + lane, j = t * kPreTile + r;
                    const int page = __shfl_sync(0xffffffffu, ent, r / maps.box_rows);
                    sk[q] = sv[q] = 0.f;
                    if (j < g.lim_last && (kv.page_size == 0 || (page >= 0 && page < kv.num_pages))) {
                        const long long so = kv.page_size ? ((long long)page * kv.H_kv + g.h) * kv.page_size + (j & (kv.page_size - 1))
                                                          : ((long long)g.p * kv.H_kv + g.h) * kv.N_max + j;
                        sk[q] = c8.k_scale[so];
                        sv[q] = c8.v_scale[so];
                    }
                }
                // (the slot of scales was last read four tiles ago, whose product P V is behind the K slot's last use)
                if (!__all_sync(0xffffffffu, mbar_wait(bar(K_EMPTY + (tc & 1)), ((tc >> 1) & 1) ^ 1, abort_s, status))) { ok = false; break; }
                float *sc = sc_s + (tc & 3) * 2 * kPreTile;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (!(sv[q] < kScaleEnd)) sv[q] = __uint_as_float(0x7fc00000u);       // (no scale: like NaN)
                    sc[q * 32 + lane] = sk[q];
                    sc[kPreTile + q * 32 + lane] = sv[q];
                }
                const bool nan = __any_sync(0xffffffffu, sv[0] != sv[0] || sv[1] != sv[1] || sv[2] != sv[2] || sv[3] != sv[3]);
                uint32_t vb = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) vb = max(vb, sv[q] == sv[q] ? __float_as_uint(sv[q]) : 0u);
                v_ref = max(v_ref, (__reduce_max_sync(0xffffffffu, vb) + 0x7fffffu) & 0x7f800000u);
                bool small = false;
#pragma unroll
                for (int q = 0; q < 4; ++q) small |= sv[q] > 0.f && sv[q] * 2097152.f < __uint_as_float(v_ref);
                small = __any_sync(0xffffffffu, small);
                if (lane == 0) {
                    vnan_s[tc & 3] = nan;
                    vref_s[tc & 3] = v_ref + small;
                }
                ok = fetch(false, g, t, tc, ent);
                if (!ok) break;
                ++tc;
                ok = fetch(true, g, t, vc, ent);
                if (ok) ++vc;
                ent = ent_next;
            }
            g = nxt;
        }
        drain(K_FULL, tc);
        drain(V8_FULL, vc);
    } else if (!KV8 && warp == 10) {
        // ------------------------------------------------------------------ 16-bit cache: item list, Q tiles, check of V tiles
        Seg g = publish(0);
        int vc = 0, odd_count = 0;
        bool ok = lists_ok;
        for (int s = 0; ok && g.t1 > g.t0; ++s) {
            if (s > 0 && !__all_sync(0xffffffffu, mbar_wait(bar(Q_EMPTY), (s - 1) & 1, abort_s, status))) { ok = false; break; }
            {
                if (lane == 0) {
                    // (boxes reach past the problem's last token: other tokens' rows, or zeros behind the tensor; nobody reads the results)
                    const int n_mt = g.toks > pg.mt_toks ? 2 : 1;
                    const uint32_t box = (uint32_t)(pg.mt_toks * kv.G) * 128;
                    mbar_arrive_expect_tx(bar(Q_FULL), n_mt * 2 * box);
                    for (int mt = 0; mt < n_mt; ++mt)
                        for (int dh = 0; dh < 2; ++dh)
                            tma_load_4d(smem_u32(q_s + mt * kPreTileBytes + dh * kPreHalf), &maps.q, bar(Q_FULL), dh * 64, 0, g.h, g.a + g.tok0 + mt * pg.mt_toks);
                }
                __syncwarp();
            }
            const Seg nxt = publish(s + 1);
            ok = lists_ok;
            {
                for (int t = g.t0; ok && t < g.t1; ++t, ++vc) {
                    const int vs = vc % kVSlots, par = (vc / kVSlots) & 1;
                    if (!__all_sync(0xffffffffu, mbar_wait(bar(V_FULL + vs), par, abort_s, status))) { ok = false; break; }
                    const int j0 = t * kPreTile;
                    if (j0 + kPreTile > g.lim_first) {     // some row does not see all of this tile
                        uint8_t *v_tile = v_s + vs * kPreTileBytes;
                        // 16-byte piece x of the tile: row x / 16, rows in front of `seen` are seen by every row
                        auto piece = [&](int x) { return reinterpret_cast<uint4 *>(v_tile + ((x >> 3) & 1) * kPreHalf + (x >> 4) * 128 + (((x & 7) ^ ((x >> 4) & 7)) << 4)); };
                        const int seen = max(0, g.lim_first - j0), end = min(kPreTile, max(0, g.N - j0));
                        bool odd = false;
#pragma unroll 2
                        for (int x = seen * 16 + lane; x < end * 16; x += 32) {
                            const uint4 v = *piece(x);
                            const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd |= (w4[e] & 0x7f80u) == 0x7f80u || (w4[e] & 0x7f800000u) == 0x7f800000u;
                        }
#pragma unroll 2
                        for (int x = end * 16 + lane; x < kPreTile * 16; x += 32) *piece(x) = make_uint4(0, 0, 0, 0);
                        odd = __any_sync(0xffffffffu, odd);
                        if (lane == 0) odd_s[vs] = odd;
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(V_SCAN + vs));
                        if (odd) {
                            if (!__all_sync(0xffffffffu, mbar_wait(bar(NOTED), odd_count & 1, abort_s, status))) { ok = false; break; }
                            ++odd_count;
                            for (int x = seen * 16 + lane; x < end * 16; x += 32) {
                                uint4 v = *piece(x);
                                uint32_t w4[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if ((w4[e] & 0x7f80u) == 0x7f80u) w4[e] &= 0xffff0000u;
                                    if ((w4[e] & 0x7f800000u) == 0x7f800000u) w4[e] &= 0x0000ffffu;
                                }
                                *piece(x) = make_uint4(w4[0], w4[1], w4[2], w4[3]);
                            }
                            fence_proxy_async();
                            __syncwarp();
                        }
                    } else {
                        if (lane == 0) mbar_arrive(bar(V_SCAN + vs));
                    }
                    if (lane == 0) mbar_arrive(bar(V_READY + vs));
                }
            }
            g = nxt;
        }
        if (*abort_s && lane == 0) {                       // (a Q load in flight lands before the CTA leaves)
            const long long c0 = clock64();
            while (clock64() - c0 < 100000) {}
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ MMA issue (one lane)
        // The issuing thread runs in step with the tensor pipe, so what it executes between two products is idle time of the pipe:
        // descriptors are a base plus constants, and the waits of a tile are taken in front of its products.
        constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
        constexpr uint32_t kTileU = kPreTileBytes >> 4, kHalfU = kPreHalf >> 4, kKU = C::kKBytes >> 4;
        auto desc = [](uint32_t lo) { return ((uint64_t)kDescHi << 32) | lo; };
        const uint32_t q_lo = ((smem_u32(q_s) >> 4) & 0x3FFFu) | (1u << 16), k_lo = ((smem_u32(k_s) >> 4) & 0x3FFFu) | (1u << 16);
        const uint32_t v_lo = ((smem_u32(v_s) >> 4) & 0x3FFFu) | (kHalfU << 16);
        constexpr uint32_t idesc_qk = KV8 ? idesc_e4m3_f32(kPreTile) : idesc_bf16_f32(kPreTile, false, false), idesc_pv = KV8 ? idesc_f16_f32(kD, false, true) : idesc_bf16_f32(kD, false, true),
                           idesc_pv_wide = idesc_bf16_f32(kD, false, true);
        int kc = 0, vc = 0, sc[2] = {0, 0};                // tiles taken from the K and V rings; products S of each region
        bool tp_before = false;
        Seg g;
        bool ok = true;
        for (int s = 0; ok && next_seg(s, g); ++s) {
            if (lane == 0) {
                const bool tp = g.toks <= pg.mt_toks;
                const int n = g.t1 - g.t0;
                auto qk = [&](int slot, int reg) {
                    const uint32_t a0 = q_lo + (tp ? 0u : (uint32_t)reg * kTileU), b0 = k_lo + (uint32_t)slot * kKU;
                    if (KV8) {
#pragma unroll C::kMmaUnroll
                        for (int ks = 0; ks < 8; ++ks)
                            umma_ss_f8(tmem_base + reg * 128, desc(a0 + (ks >> 2) * kHalfU + (ks & 3) * 2), desc(b0 + (ks & 3) * 2), idesc_qk, ks > 0);
                    } else {
#pragma unroll C::kMmaUnroll
                        for (int ks = 0; ks < 8; ++ks) {
                            const uint32_t off = (ks >> 2) * kHalfU + (ks & 3) * 2;
                            umma_ss(tmem_base + reg * 128, desc(a0 + off), desc(b0 + off), idesc_qk, ks > 0);
                        }
                    }
                };
                auto pv = [&](int slot, int reg, uint32_t acc, uint32_t idesc) {
                    const uint32_t b0 = v_lo + (uint32_t)slot * kTileU;
#pragma unroll C::kMmaUnroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_ts(tmem_base + 256 + reg * 128, tmem_base + reg * 128 + ks * 8, desc(b0 + ks * (2048 >> 4)), idesc, ks > 0 ? 1u : acc);
                };
                auto wait = [&](int b, int par) { return mbar_wait(bar(b), par & 1, abort_s, status); };
                auto wait_k = [&](int c) { return wait(K_FULL + c % kKSlots, c / kKSlots); };
                auto idesc_of = [&](int c) { return KV8 && (vref_s[c & 3] & 1u) ? idesc_pv_wide : idesc_pv; };     // of V tile c, which has come
                auto wait_v = [&](int c) {
                    const int sl = c % kVSlots, par = c / kVSlots;
                    return wait(V_FULL + sl, par) && (KV8 || wait(V_READY + sl, par));
                };
                ok = wait(Q_FULL, s);
                // first S of every region in use
                for (int i = 0; ok && i < (tp ? min(2, n) : 1); ++i) {
                    ok = wait_k(kc);
                    if (!ok) break;
                    tc_fence_after_sync();
                    qk(kc % kKSlots, i);
                    umma_commit(bar(S_FULL + i));
                    if (!tp) {
                        qk(kc % kKSlots, 1);
                        umma_commit(bar(S_FULL + 1));
                    }
                    umma_commit(bar(K_EMPTY + kc % kKSlots));
                    ++kc;
                }
                if (ok && n == (tp ? min(2, n) : 1)) umma_commit(bar(Q_EMPTY));
                // With two M-tiles a warpgroup's first P comes after its own results of the item before are out.  With one, the first
                // warpgroup reads both parts of O: then the item before has to be out of both.
                if (ok && s > 0 && (tp || tp_before)) ok = wait(SEG_DONE + 0, s - 1) && wait(SEG_DONE + 1, s - 1);
                tp_before = tp;
                if (tp) {
                    for (int i = 0; ok && i < n; ++i) {
                        const int reg = i & 1;
                        ok = wait_v(vc) && wait(P_FULL + reg, sc[reg]);
                        if (!ok) break;
                        ++sc[reg];
                        const uint32_t idesc = idesc_of(vc);
                        tc_fence_after_sync();
                        pv(vc % kVSlots, reg, i > 1 ? 1u : 0u, idesc);
                        umma_commit(bar(V_EMPTY + vc % kVSlots));
                        ++vc;
                        if (i + 2 < n) {
                            ok = wait_k(kc);
                            if (!ok) break;
                            tc_fence_after_sync();
                            qk(kc % kKSlots, reg);
                            umma_commit(bar(S_FULL + reg));
                            umma_commit(bar(K_EMPTY + kc % kKSlots));
                            ++kc;
                            if (i + 3 == n) umma_commit(bar(Q_EMPTY));
                        }
                    }
                } else {
                    for (int i = 0; ok && i < n; ++i) {
                        const bool more = i + 1 < n;
                        const uint32_t acc = i > 0 ? 1u : 0u;
                        ok = wait_v(vc) && (!more || wait_k(kc)) && wait(P_FULL + 0, sc[0]);
                        if (!ok) break;
                        ++sc[0];
                        const uint32_t idesc = idesc_of(vc);
                        tc_fence_after_sync();
                        pv(vc % kVSlots, 0, acc, idesc);
                        if (more) {
                            qk(kc % kKSlots, 0);
                            umma_commit(bar(S_FULL + 0));
                        } else {
                            umma_commit(bar(O_DONE + 0));
                        }
                        ok = wait(P_FULL + 1, sc[1]);
                        if (!ok) break;
                        ++sc[1];
                        tc_fence_after_sync();
                        pv(vc % kVSlots, 1, acc, idesc);
                        umma_commit(bar(V_EMPTY + vc % kVSlots));
                        ++vc;
                        if (more) {
                            qk(kc % kKSlots, 1);
                            umma_commit(bar(S_FULL + 1));
                            umma_commit(bar(K_EMPTY + kc % kKSlots));
                            ++kc;
                            if (i + 2 == n) umma_commit(bar(Q_EMPTY));
                        }
                    }
                }
                if (ok && tp) umma_commit(bar(O_DONE + 0));
                if (ok) umma_commit(bar(O_DONE + 1));
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        }
    } else if (KV8 && warp >= 10) {
        // ------------------------------------------------------------------ 8-bit cache: widened values
        const int w2 = warp - 10;
        int vc = 0;
        Seg g;
        bool ok = true;
        for (int s = 0; ok && next_seg(s, g); ++s) {
            // V: a thread takes two key rows of 128 codes: eight 16-byte pieces in, sixteen out, each
            for (int t = g.t0; t < g.t1; ++t, ++vc) {
                const int vs = vc % kVSlots, par = (vc / kVSlots) & 1;
                if (!__all_sync(0xffffffffu, mbar_wait(bar(V8_FULL + vs), par, abort_s, status)) ||
                    !__all_sync(0xffffffffu, mbar_wait(bar(V_EMPTY + vs), par ^ 1, abort_s, status))) { ok = false; break; }
                const uint8_t *src = v8_s + vs * kPreHalf;
                uint8_t *dst = v_s + vs * kPreTileBytes;
                const float *vsc = sc_s + (vc & 3) * 2 * kPreTile + kPreTile;
                // the rows' factors, 2^7 scale / v_ref <= 2^7; 0 for rows behind the prefix or on a bad page (whose codes may be NaN) and NaN scales
                const uint32_t v_raw = vref_s[vc & 3];
                const float inv = __uint_as_float(((254u + kValueBits) << 23) - (v_raw & 0x7f800000u));
                auto factor = [&](float sc) { return sc > 0.f ? sc * inv : 0.f; };
                float g0 = factor(vsc[w2 * 64 + lane]), g1 = factor(vsc[w2 * 64 + 32 + lane]);
                if (v_raw & 1u) {                          // (scales of very different size) bf16, the scales' mantissas are in P
                    g0 /= mantissa(vsc[w2 * 64 + lane]);
                    g1 /= mantissa(vsc[w2 * 64 + 32 + lane]);
#pragma unroll 1
                    for (int x = 0; x < 16; ++x) {
                        const int r = w2 * 64 + (x & 8) * 4 + lane, ch = x & 7;
                        const uint4 v = *reinterpret_cast<const uint4 *>(src + r * 128 + ((ch ^ (r & 7)) << 4));
                        const float f = (x & 8) ? g1 : g0;
                        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                        uint32_t o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            uint32_t h2;
                            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)(w[e >> 1] >> (16 * (e & 1)))));
                            const float2 c = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
                            o[e] = f > 0.f ? pack_bf16x2(c.x * f, c.y * f) : 0u;
                        }
                        const int c0 = 2 * ch, c1 = 2 * ch + 1;
                        *reinterpret_cast<uint4 *>(dst + (c0 >> 3) * kPreHalf + r * 128 + (((c0 & 7) ^ (r & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                        *reinterpret_cast<uint4 *>(dst + (c1 >> 3) * kPreHalf + r * 128 + (((c1 & 7) ^ (r & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
                    }
                    fence_proxy_async();
                    mbar_arrive_warp(bar(V_FULL + vs));
                    mbar_arrive_warp(bar(V8_EMPTY + vs));
                    continue;
                }
                const uint32_t f0 = pack_f16x2(g0, g0), f1 = pack_f16x2(g1, g1);
#pragma unroll 4
                for (int x = 0; x < 16; ++x) {
                    const int r = w2 * 64 + (x & 8) * 4 + lane, ch = x & 7;
                    const uint4 v = *reinterpret_cast<const uint4 *>(src + r * 128 + ((ch ^ (r & 7)) << 4));
                    const uint32_t f2 = (x & 8) ? f1 : f0;
                    const uint32_t w[4] = {f2 ? v.x : 0u, f2 ? v.y : 0u, f2 ? v.z : 0u, f2 ? v.w : 0u};
                    uint32_t o[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {          // four codes -> two f16 pairs, times the row's factor
                        uint32_t lo, hi;
                        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w[e]));
                        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * e]) : "r"(lo), "r"(f2));
                        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o[2 * e + 1]) : "r"(hi), "r"(f2));
                    }
                    const int c0 = 2 * ch, c1 = 2 * ch + 1;
                    *reinterpret_cast<uint4 *>(dst + (c0 >> 3) * kPreHalf + r * 128 + (((c0 & 7) ^ (r & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4 *>(dst + (c1 >> 3) * kPreHalf + r * 128 + (((c1 & 7) ^ (r & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
                }
                fence_proxy_async();
                mbar_arrive_warp(bar(V_FULL + vs));
                mbar_arrive_warp(bar(V8_EMPTY + vs));
            }
        }
    } else if (warp < 8) {
        // ------------------------------------------------------------------ softmax warpgroups
        const int mt = warp >> 2, w4 = warp & 3, row = w4 * 32 + lane;
        const uint32_t lane_off = (uint32_t)(w4 * 32) << 16;
        const uint32_t tS = tmem_base + mt * 128 + lane_off, tO = tmem_base + 256 + mt * 128 + lane_off;
        // what a warp of the second warpgroup publishes to its counterpart in the first (one M-tile), twice by turns: (reference, sum) of
        // its 32 rows, the columns that it noted, whether it noted any
        uint8_t *pubw = base + C::offPub + w4 * C::kPubBytes;
        const int my_tok = row / kv.G, my_g = row % kv.G;
        int cnt = 0, tile0 = 0, merges = 0;                // products S of this region, key tiles and merged items so far
        // 8-bit cache: the query rows of an item as e4m3 hi and lo codes with a factor per row.  Each warp codes its share while it would
        // otherwise wait for the last product of the item before (two warps of their own took longer over 256 rows than a short
        // item's tiles do: 24 mixed chunks of 1 to 700 tokens took half as long again).  Sixteen lanes a row, eight elements a lane, two rows of a
        // lane's column in flight ahead of the two being coded (short code: with eight at once they took a tenth longer).
        auto code_queries = [&](const Seg &g, int s) -> bool {
            const int n_mt = g.toks > pg.mt_toks ? 2 : 1, qt = warp * n_mt >> 3, n_rows = min(pg.mt_toks, g.toks - qt * pg.mt_toks) * kv.G, l16 = lane & 15;
            const __nv_bfloat16 *src0 = at.q.p + (long long)(g.a + g.tok0 + qt * pg.mt_toks) * at.q.st + (long long)(g.h * kv.G) * at.q.sh + l16 * 8;
            int r_at = (warp * n_mt * 16 & 127) + (lane >> 4), ti = r_at / kv.G, gi = r_at % kv.G, r_ld = r_at;
            uint4 next[2];
            auto load = [&]() {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    next[q] = r_ld < n_rows ? *reinterpret_cast<const uint4 *>(src0 + (long long)ti * at.q.st + (long long)gi * at.q.sh) : make_uint4(0, 0, 0, 0);
                    r_ld += 2;
                    gi += 2;
                    while (gi >= kv.G) { gi -= kv.G; ++ti; }
                }
            };
            load();
            if (s > 0 && !__all_sync(0xffffffffu, mbar_wait(bar(Q_EMPTY), (s - 1) & 1, abort_s, status))) return false;
#pragma unroll 1
            for (int b = 0; b < 4 * n_mt; ++b, r_at += 4) {
                uint4 raw[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) raw[q] = next[q];
                if (b + 1 < 4 * n_mt) load();
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int r = r_at + 2 * q;
                    const uint32_t w[4] = {raw[q].x, raw[q].y, raw[q].z, raw[q].w};
                    uint32_t m = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) m = amax_bits(m, w[e]);
#pragma unroll
                    for (int d = 8; d; d >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, d));
                    float inv;
                    const float f = row_factor(amax_of_halves(m), inv);
                    uint32_t hi[2], lo[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t a01 = code_pair(w[2 * e], inv), a23 = code_pair(w[2 * e + 1], inv);
                        hi[e] = __byte_perm(a01, a23, 0x5410);
                        lo[e] = __byte_perm(a01, a23, 0x7632);
                    }
                    uint8_t *dst = q_s + qt * kPreTileBytes + r * 128 + (((l16 >> 1) ^ (r & 7)) << 4) + (l16 & 1) * 8;
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(hi[0], hi[1]);
                    *reinterpret_cast<uint2 *>(dst + kPreHalf) = make_uint2(lo[0], lo[1]);
                    if (l16 == 0) rowf_s[(s & 1) * kPreRows + qt * kPreTile + r] = f;
                }
            }
            fence_proxy_async();
            mbar_arrive_warp(bar(Q_FULL));
            return true;
        };
        Seg g, g_next;
        bool have = next_seg(0, g);
        if (KV8 && have) have = code_queries(g, 0);
        for (int s = 0; have; ++s) {
            const bool tp = g.toks <= pg.mt_toks;
            const int n = g.t1 - g.t0, first = tp ? mt : 0, stride = tp ? 2 : 1;
            const int r_tile = (tp ? 0 : mt * kPreTile) + row;
            const int tok = g.tok0 + (tp ? 0 : mt * pg.mt_toks) + my_tok;                   // this row's token within the problem
            const int rows = min(pg.mt_toks, g.toks - (tp ? 0 : mt * pg.mt_toks)) * kv.G;   // rows of this M-tile
            const bool row_ok = row < rows, warp_has_rows = w4 * 32 < rows;
            const int lim = row_ok ? visible(g.N - g.n_new + tok, g.N, at.mask_block) : g.N;
            float m_used = 0.f, l = 0.f, pend_m = 0.f;
            bool pending = false, ok = true, odd_seen = false, unset = true;       // unset: no key taken yet, the reference stands for nothing
            bool far = false;                              // (of the warp) some row's reference is beyond kFar
            auto any_far = [&]() { return __any_sync(0xffffffffu, row_ok && !(fabsf(m_used) <= kFar)) != 0; };
            uint32_t odd_pos[4], odd_neg[4], v_ref = 0;    // v_ref: what O is kept over (8-bit), as bits
            float scale = at.scale_log2;
            for (int i = first; i < n; i += stride, ++cnt) {
                if (!__all_sync(0xffffffffu, mbar_wait(bar(S_FULL + mt), cnt & 1, abort_s, status))) { ok = false; break; }
                tc_fence_after_sync();
                if (KV8 && i == first) scale = at.scale_log2 * rowf_s[(s & 1) * kPreRows + r_tile];
                const uint64_t c2 = pack2(scale, scale);
                const int j0 = (g.t0 + i) * kPreTile, tcur = tile0 + i;
                const uint32_t bad = bad_s[tcur & 3];
                [[maybe_unused]] const float *ksc = sc_s + (tcur & 3) * 2 * kPreTile, *vsc = ksc + kPreTile;                 // 8-bit: the tile's scales
                const bool diag = j0 + kPreTile > g.lim_first;
                auto rescale_o = [&](float f) {
#pragma unroll 1
                    for (int c0 = 0; c0 < kD; c0 += 32) {
                        uint32_t r[32];
                        tmem_ld32(tO + c0, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                        tmem_st32(tO + c0, r);
                    }
                    tmem_wait_st();
                };
                const int valid = min(kPreTile, max(0, lim - j0));               // keys of the tile that this row sees
                const bool masked = diag || bad != 0;
                if (warp_has_rows) {
                    // One sweep with the reference carried over from earlier tiles.  Tiles that every row sees whole run straight-line
                    // code; masked ones, and halves that have to be redone, a loop of 32 columns a turn (rarely run code is kept
                    // small: fetching it costs more than running it).
                    // (rows of M-tile padding and of tokens behind the problem's last hold anything: they have no say in the warp's
                    // decisions, so that a result depends on its own problem alone)
                    uint32_t ra[32], rb[32], pa[16], pb[16];
                    tmem_ld32(tS, ra);
                    const uint32_t v_raw = KV8 ? vref_s[tcur & 3] : 0u, v_new = v_raw & 0x7f800000u;
                    const bool wide = KV8 && (v_raw & 1u);
                    if (KV8 && i == first) v_ref = v_new;
                    if (__any_sync(0xffffffffu, pending) || v_new != v_ref) {
                        const float f = pending ? ex2(m_used - pend_m) : 1.f;
                        rescale_o(KV8 ? f * (__uint_as_float(v_ref) / __uint_as_float(v_new)) : f);
                        v_ref = v_new;
                        l *= f;
                        if (pending) m_used = pend_m;
                        pending = false;
                        far = any_far();
                    }
                    tmem_wait_ld(ra);
                    if (i == first) {
                        // the reference starts at the maximum of the row's first 32 logits, with masked columns at that of the first 32 columns
                        // that have one; the sweep moves it on like any later rise
                        float m0 = -INFINITY;
                        if (!masked) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                float x[4] = {__uint_as_float(ra[e]), __uint_as_float(ra[e + 1]), __uint_as_float(ra[e + 2]), __uint_as_float(ra[e + 3])};
                                if (KV8) {
                                    const float4 ks = lds128(smem_u32(ksc + e));
                                    x[0] *= ks.x; x[1] *= ks.y; x[2] *= ks.z; x[3] *= ks.w;
                                }
                                m0 = max3(max3(m0, x[0], x[1]), x[2], x[3]);
                            }
                        }
                        unset = m0 == -INFINITY;
                        m_used = unset ? 0.f : __fsub_rn(__fmul_rn(m0, scale), R_::kUp);
                        far = any_far();
                    }
                    uint64_t neg_m2 = pack2(-m_used, -m_used), l2a, l2b;
                    float mx = -INFINITY, sum_all = 0.f;
                    // 32 columns of S -> 16 packed bf16 pairs of P and their sum; may_mask: logits rounded first, and the largest of them
                    auto chunk32 = [&](auto may_mask, auto in_bf16, uint32_t (&r)[32], uint32_t (&pk)[16], int c0) {
                        if (KV8) {                         // (scales are read well before they are used: 2 % for 2001 tokens behind 16384)
                            float4 ksv[8];
#pragma unroll
                            for (int e = 0; e < 4; ++e) ksv[e] = lds128(smem_u32(ksc + c0 + 4 * e));
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                if (e == 8) {
#pragma unroll
                                    for (int x = 4; x < 8; ++x) ksv[x] = lds128(smem_u32(ksc + c0 + 4 * x));
                                }
                                const float4 ks = ksv[e >> 2];
                                float a0, a1;
                                unpack2(mul2(pack2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), pack2(ks.x, ks.y)), a0, a1);
                                r[e] = __float_as_uint(a0); r[e + 1] = __float_as_uint(a1);
                                unpack2(mul2(pack2(__uint_as_float(r[e + 2]), __uint_as_float(r[e + 3])), pack2(ks.z, ks.w)), a0, a1);
                                r[e + 2] = __float_as_uint(a0); r[e + 3] = __float_as_uint(a1);
                            }
                        }
                        if (may_mask.value && (bad != 0 || __any_sync(0xffffffffu, valid < c0 + 32))) {      // what a row does not see becomes -inf whatever it was
                            const uint32_t okm = cols_ok(c0, valid, bad);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((okm >> e) & 1u)) r[e] = 0xff800000u;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const uint64_t s2 = pack2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]));
                            float x0, x1;
                            if (may_mask.value) {
                                const uint64_t t2 = mul2(s2, c2);
                                unpack2(t2, x0, x1);
                                mx = max3(mx, x0, x1);
                                unpack2(add2(t2, neg_m2), x0, x1);
                            } else {
                                unpack2(fma2(s2, c2, neg_m2), x0, x1);
                            }
                            const float p0 = ex2(x0), p1 = ex2(x1);
                            if (e & 1) l2b = add2(l2b, pack2(p0, p1));
                            else l2a = add2(l2a, pack2(p0, p1));
                            if (KV8 && may_mask.value && in_bf16.value) {
                                const float2 sv = *reinterpret_cast<const float2 *>(vsc + c0 + 2 * e);
                                pk[e] = pack_bf16x2(p0 * mantissa(sv.x), p1 * mantissa(sv.y));
                                continue;
                            }
                            pk[e] = KV8 ? pack_f16x2(p0, p1) : pack_bf16x2(p0, p1);       // rounding of P to bf16: 2^-8 relative, like the output's own
                        }
                    };
                    auto half_sum = [&]() {
                        float a0, a1, b0, b1;
                        unpack2(l2a, a0, a1);
                        unpack2(l2b, b0, b1);
                        return (a0 + a1) + (b0 + b1);
                    };
                    auto keep_half = [&](int half, float sum) {
                        tmem_st16(tS + half * 32, pa);
                        tmem_st16(tS + half * 32 + 16, pb);
                        l += sum;
                        sum_all += sum;
                    };
                    int done = 0;                          // quarters of the tile whose P is stored
                    if (!masked && !far && !wide) {
                        const std::false_type no = {};
                        tmem_ld32(tS + 32, rb);
                        l2a = l2b = pack2(0.f, 0.f);
                        chunk32(no, no, ra, pa, 0);
                        tmem_wait_ld(rb);
                        tmem_ld32(tS + 64, ra);
                        chunk32(no, no, rb, pb, 32);
                        tmem_wait_ld(ra);
                        const float sum0 = half_sum();
                        if (!__any_sync(0xffffffffu, row_ok && (sum0 > R_::kMost || unset))) {
                            keep_half(0, sum0);
                            done = 2;
                            tmem_ld32(tS + 96, rb);
                            l2a = l2b = pack2(0.f, 0.f);
                            chunk32(no, no, ra, pa, 64);
                            tmem_wait_ld(rb);
                            chunk32(no, no, rb, pb, 96);
                            const float sum1 = half_sum();
                            if (!__any_sync(0xffffffffu, row_ok && sum1 > R_::kMost)) {
                                keep_half(1, sum1);
                                done = 4;
                            }
                        }
                    }
                    bool redo = false;                     // this turn does its quarter a second time
#pragma unroll 1
                    for (; done < 4; ++done) {
                        const std::true_type yes = {};
                        const int c0 = done * 32;
                        if (!__any_sync(0xffffffffu, row_ok && valid > c0)) {          // behind what any row of the warp sees
#pragma unroll
                            for (int e = 0; e < 16; ++e) pa[e] = 0u;
                            tmem_st16(tS + done * 16, pa);
                            continue;
                        }
                        tmem_ld32(tS + c0, ra);
                        tmem_wait_ld(ra);
                        mx = (bad == 0 ? valid > c0 : cols_ok(c0, valid, bad) != 0u) ? kLowest : -INFINITY;      // -inf: no key taken here
                        l2a = l2b = pack2(0.f, 0.f);
                        if (KV8 && wide) chunk32(yes, yes, ra, pa, c0);
                        else chunk32(yes, std::false_type{}, ra, pa, c0);
                        // A rise past kMostLog (exponentials out of range), or the first key that the row sees: move the reference,
                        // scale what is there -- O, the sum, the P of the quarters before -- and redo this quarter, whose S is still
                        // whole.  The new reference is kUp below the quarter's largest rounded logit (or, where its step is larger, that
                        // logit or a step below it, at most 8), so the second time no row needs another; a quarter is never
                        // redone twice, whatever it holds.
                        const bool need = row_ok && (mx - m_used > R_::kMostLog || (unset && mx > -INFINITY));
                        if (!redo && __any_sync(0xffffffffu, need)) {
                            const float m_new = need ? __fsub_rn(mx, R_::kUp) : m_used, f = need && !unset ? ex2(m_used - m_new) : 1.f;
                            if (i != first) rescale_o(f);
                            l *= f;
                            tmem_wait_st();
#pragma unroll 1
                            for (int x = 0; x < done * 16; x += 16) {
                                uint32_t pr[16];
                                tmem_ld16(tS + x, pr);
                                tmem_wait_ld(pr);
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    if (KV8 && !wide) {
                                        const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&pr[e]));
                                        pr[e] = pack_f16x2(h.x * f, h.y * f);
                                    } else {
                                        pr[e] = pack_bf16x2(__uint_as_float(pr[e] << 16) * f, __uint_as_float(pr[e] & 0xffff0000u) * f);
                                    }
                                }
                                tmem_st16(tS + x, pr);
                            }
                            if (need) unset = false;
                            m_used = m_new;
                            neg_m2 = pack2(-m_used, -m_used);
                            sum_all = 0.f;
                            far = any_far();
                            redo = true;
                            --done;
                            continue;
                        }
                        redo = false;
                        tmem_st16(tS + done * 16, pa);
                        const float sum = half_sum();
                        l += sum;
                        sum_all += sum;
                    }
                    if (sum_all > R_::kRescale && !far) { pending = true; pend_m = m_used + __log2f(sum_all) - R_::kUp; }
                }
                if (KV8 && vnan_s[tcur & 3]) {             // (error path)
#pragma unroll 1
                    for (int j = 0; j < valid; ++j) odd_seen |= vsc[j] != vsc[j];
                }
                if (!KV8 && diag) {
                    const int vs = tcur % kVSlots;
                    if (!__all_sync(0xffffffffu, mbar_wait(bar(V_SCAN + vs), (tcur / kVSlots) & 1, abort_s, status))) { ok = false; break; }
                    if (odd_s[vs]) {
                        if (!odd_seen) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) odd_pos[q] = odd_neg[q] = 0u;
                        }
                        odd_seen = true;
                        tmem_wait_st();
                        note_odd_values(v_s + vs * kPreTileBytes, max(0, g.lim_first - j0), valid, tS, odd_pos, odd_neg);
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(bar(NOTED));
                            if (tp) mbar_arrive(bar(NOTED));       // four warps of one warpgroup stand for eight
                        }
                    }
                }
                tmem_wait_st();
                tc_fence_before_sync();
                mbar_arrive_warp(bar(P_FULL + mt));
            }
            tile0 += n;
            if (!ok) break;
            have = next_seg(s + 1, g_next);
            if (KV8 && have && !code_queries(g_next, s + 1)) break;
            if (unset) m_used = -INFINITY;
            // ---- the item's result.  One M-tile: the second warpgroup publishes its (reference, sum), the first adds its part of O.
            const bool merge = tp && n > 1;
            float2 *pub = reinterpret_cast<float2 *>(pubw) + (merges & 1) * 32;
            float w0 = 1.f, w1 = 0.f;
            // (and, on the error path, the columns with non-finite values that it noted)
            uint32_t *pub_odd = reinterpret_cast<uint32_t *>(pubw + 512) + (merges & 1) * (KV8 ? 32 : 256), *pub_flag = reinterpret_cast<uint32_t *>(pubw + 2560) + (merges & 1);
            if (tp && mt == 1) {
                if (merge) {
                    pub[lane] = make_float2(m_used, l);
                    if (KV8) {
                        pub_odd[lane] = odd_seen;
                        pub_odd[64 + lane] = v_ref;
                    } else {
                        if (odd_seen) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) { pub_odd[q * 32 + lane] = odd_pos[q]; pub_odd[(4 + q) * 32 + lane] = odd_neg[q]; }
                        }
                        if (lane == 0) *pub_flag = odd_seen;
                    }
                    mbar_arrive_warp(bar(PUB + (merges & 1)));
                }
            }
            // (the second warpgroup waits also where only the first needs O, so that neither runs ahead through items without tiles for it)
            if (!__all_sync(0xffffffffu, mbar_wait(bar(O_DONE + mt), s & 1, abort_s, status))) break;
            if (!(tp && mt == 1)) {
                if (merge && !__all_sync(0xffffffffu, mbar_wait(bar(PUB + (merges & 1)), (merges >> 1) & 1, abort_s, status))) break;
                tc_fence_after_sync();
                if (KV8 && !merge) w0 = __uint_as_float(v_ref - (kValueBits << 23));
                if (merge) {
                    const float2 o = pub[lane];
                    const float m_all = fmaxf(m_used, o.x);
                    w0 = unset ? 0.f : ex2(m_used - m_all);
                    w1 = o.x == -INFINITY ? 0.f : ex2(o.x - m_all);
                    l = l * w0 + o.y * w1;
                    if (KV8) {
                        w0 *= __uint_as_float(v_ref - (kValueBits << 23));
                        w1 *= __uint_as_float(pub_odd[64 + lane] - (kValueBits << 23));
                    }
                    m_used = m_all;
                    if (KV8) {
                        odd_seen |= pub_odd[lane] != 0;
                    } else if (*pub_flag) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            odd_pos[q] = (odd_seen ? odd_pos[q] : 0u) | pub_odd[q * 32 + lane];
                            odd_neg[q] = (odd_seen ? odd_neg[q] : 0u) | pub_odd[(4 + q) * 32 + lane];
                        }
                        odd_seen = true;
                    }
                }
                const bool whole = g.slot < 0;
                float *slot = whole ? nullptr : pg.part + (size_t)g.slot * kPreSlot;
                const bool sees = m_used != -INFINITY;                      // (or it took no key)
                const float inv = whole ? (sees ? 1.f / l : 0.f) : 1.f;
                const int my_row = (g.a + tok) * kv.H_q + g.h * kv.G + my_g;               // (below 2^31 by the host's check)
                // A thread holds a row of O and stores it in pieces of 32 bytes, whole sectors.
                uint8_t *dst = whole ? reinterpret_cast<uint8_t *>(at.out) + (long long)my_row * (kD * 2) : reinterpret_cast<uint8_t *>(slot + r_tile * kD);
                const bool wide = (reinterpret_cast<uintptr_t>(at.out) & 16) == 0;     // (partial results always are)
                if (warp_has_rows) {
#pragma unroll 1
                    for (int c0 = 0; c0 < kD; c0 += 32) {
                        uint32_t r[32];
                        tmem_ld32(tO + c0, r);
                        if (merge) {
                            uint32_t q[32];
                            tmem_ld32(tO + 128 + c0, q);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(fmaf(__uint_as_float(q[e]), w1, __uint_as_float(r[e]) * w0));
                        } else {
                            tmem_wait_ld(r);
                            if (KV8) {
#pragma unroll
                                for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * w0);
                            }
                        }
                        if (whole) {
                            uint32_t v[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] = sees ? pack_bf16x2(__uint_as_float(r[2 * e]) * inv, __uint_as_float(r[2 * e + 1]) * inv) : 0u;
                            if (row_ok) {
                                st_global32(dst + c0 * 2, v, wide);
                                st_global32(dst + c0 * 2 + 32, v + 8, wide);
                            }
                        } else if (row_ok) {
#pragma unroll
                            for (int e = 0; e < 32; e += 8) st_global32(dst + (c0 + e) * 4, r + e, true);
                        }
                    }
                    if (odd_seen && row_ok) {              // (error path) the columns in which this row saw infinities or NaN
#pragma unroll 1
                        for (int d = 0; d < kD; ++d) {
                            const bool up = KV8 || ((odd_pos[d >> 5] >> (d & 31)) & 1u), down = KV8 || ((odd_neg[d >> 5] >> (d & 31)) & 1u);
                            if (!up && !down) continue;
                            const float v = up && down ? __uint_as_float(0x7fc00000u) : (up ? INFINITY : -INFINITY);
                            if (whole) at.out[(long long)my_row * kD + d] = __float2bfloat16(l == l ? v : l);
                            else slot[r_tile * kD + d] = v;
                        }
                    }
                    if (row_ok) {
                        if (!whole) {
                            slot[kPreRows * kD + r_tile] = m_used;
                            slot[kPreRows * kD + kPreRows + r_tile] = l;
                        } else if (at.lse) {
                            at.lse[my_row] = sees ? (m_used + log2f(l)) * 0.6931471805599453f : -INFINITY;
                        }
                    }
                }
            }
            if (merge) ++merges;
            tc_fence_before_sync();
            mbar_arrive_warp(bar(SEG_DONE + mt));
            g = g_next;
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 9) { tc_fence_after_sync(); tmem_dealloc(tmem_base, 512); }
}

}  // namespace chunk
}  // namespace mage
