// Packed chunks of new tokens: which problem a token belongs to, where its rows sit in the cache, and the kernels that write
// the rows (16 bits, or quantised to e4m3 on the way) and read an 8-bit cache back.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mage {
namespace chunk {

struct ChunkView {
    const int *q_start;
    int n_tokens, max_len;
};
struct Kv8View {
    uint8_t *k8, *v8;
    float *k_scale, *v_scale;
};
struct Strided {                              // element (t, h, c) of a packed token tensor at t*st + h*sh + c
    const __nv_bfloat16 *p;
    long long st, sh;
};

constexpr float kE4m3Max = 448.f;
constexpr float kScaleEnd = 1.329227995784916e36f;    // 2^120: scales are below it (the largest bf16 number over 448), or NaN

// New tokens of problem p: first packed row and count; 0 and a status bit when the entries are no valid range.
__device__ __forceinline__ int chunk_len_of(const ChunkView &cv, int p, int *first, unsigned *status) {
    const int a = cv.q_start[p], b = cv.q_start[p + 1];
    *first = a;
    if (a < 0 || b < a || b > cv.n_tokens || b - a > cv.max_len) {
        if (status) atomicOr(status, MAGE_DEV_BAD_CHUNK);
        return 0;
    }
    return b - a;
}

// The problem that owns packed row t: the last p with q_start[p] <= t, -1 if there is none.  Called by whole warps: 32 entries
// are compared per step, so up to 32 problems cost one load and 1024 cost two dependent ones.
__device__ __forceinline__ int find_problem(const int *q_start, int P, int t, int lane) {
    int lo = 0, n = P;
    bool first = true;
    while (n > 1 || first) {
        first = false;
        const int step = (n + 31) >> 5, e = lane * step;
        const unsigned le = __ballot_sync(0xffffffffu, e < n && q_start[lo + e] <= t);
        if (le == 0) return -1;
        const int at = (31 - __clz(le)) * step;
        lo += at;
        n = min(step, n - at);
    }
    return lo;
}

// Offset of cache row (p, h, j) in elements, and of its scale; false (and a status bit) when the page id is bad.  (Page sizes are
// powers of two: shifts, because a division costs as much as the rest of the row.)
__device__ __forceinline__ bool row_at(const KvView &kv, int p, int h, int j, long long &off, long long &soff, unsigned *status) {
    if (kv.page_size == 0) {
        off = (long long)p * kv.stride_p + (long long)h * kv.stride_h + (long long)j * kv.stride_n;
        soff = ((long long)p * kv.H_kv + h) * kv.N_max + j;
        return true;
    }
    const int page = kv.block_table[(long long)p * kv.max_pages + (j >> (31 - __clz(kv.page_size)))];
    if (page < 0 || page >= kv.num_pages) {
        if (status) atomicOr(status, MAGE_DEV_BAD_PAGE);
        return false;
    }
    soff = ((long long)page * kv.H_kv + h) * kv.page_size + (j & (kv.page_size - 1));
    off = soff * kD;
    return true;
}

// ---- e4m3 codes of a row
__device__ __forceinline__ unsigned e4m3x2(float lo, float hi) {              // low byte = code of lo
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// A row's scale s from the largest bit pattern m of its magnitudes, and y = RN(1/s).
__device__ __forceinline__ float row_scale(uint32_t m, float &y) {
    y = 0.f;
    if (m >= 0x7f80u) return __uint_as_float(0x7fc00000u);                    // NaN or infinity in the row
    const float s = m ? __fdiv_rn(__uint_as_float(m << 16), kE4m3Max) : 1.f;
    y = __frcp_rn(s);
    return s;
}
__device__ __forceinline__ uint32_t pair_max(const uint4 &raw) {              // of magnitudes as bit patterns, which order like them, NaN above infinity
    return __vmaxu2(__vmaxu2(raw.x & 0x7fff7fffu, raw.y & 0x7fff7fffu), __vmaxu2(raw.z & 0x7fff7fffu, raw.w & 0x7fff7fffu));
}
// This lane's eight codes.  x / s is rounded to nearest with one reciprocal for the row: y = RN(1/s), q = RN(x y), r = x - q s
// (exact in an fma), RN(q + r y) is the correctly rounded quotient (Markstein's correction) while nothing over- or underflows;
// scales outside 2^-100 .. 2^100 take the division itself.  Elements below 2^-20 s need no exactness: their code is 0 either way.
__device__ __forceinline__ uint2 row_codes(const uint4 &raw, float s, float y) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    unsigned c[4];
    if (s > 7.9e-31f && s < 1.2e30f) {
        const uint64_t y2 = ptx::pack2(y, y), neg_s2 = ptx::pack2(-s, -s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t x = ptx::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), q = ptx::mul2(x, y2);
            float lo, hi;
            ptx::unpack2(ptx::fma2(ptx::fma2(q, neg_s2, x), y2, q), lo, hi);
            c[i] = e4m3x2(lo, hi);
        }
    } else if (s == s) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
            const unsigned v = e4m3x2(__fdiv_rn(__uint_as_float(w[i] << 16), s), __fdiv_rn(__uint_as_float(w[i] & 0xffff0000u), s));
            if (i == 0) c[0] = v;
            if (i == 1) c[1] = v;
            if (i == 2) c[2] = v;
            if (i == 3) c[3] = v;
        }
    } else {
        return make_uint2(0u, 0u);
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
// Scales of kRows rows whose pieces lie in sixteen lanes each (eight elements a lane), the same in all sixteen.  The kernel that calls this
// is bound by instructions as much as by bytes: four rows are reduced together, each lane ending with one of them, so that the
// division and the reciprocal run once for four (16 prompts of 300 to 2048 tokens, 8 heads: 19.4 us, one row at a time 23.0).
template <int kRows>
__device__ __forceinline__ void row_scales(const uint4 (&raw)[kRows], int lane, float (&s)[kRows], float (&y)[kRows]) {
    if (kRows == 4) {
        const uint32_t v0 = pair_max(raw[0]), v1 = pair_max(raw[1 % kRows]), v2 = pair_max(raw[2 % kRows]), v3 = pair_max(raw[3 % kRows]);
        const bool b8 = lane & 8, b4 = lane & 4;
        const uint32_t a0 = __vmaxu2(b8 ? v2 : v0, __shfl_xor_sync(0xffffffffu, b8 ? v0 : v2, 8)), a1 = __vmaxu2(b8 ? v3 : v1, __shfl_xor_sync(0xffffffffu, b8 ? v1 : v3, 8));
        uint32_t m = __vmaxu2(b4 ? a1 : a0, __shfl_xor_sync(0xffffffffu, b4 ? a0 : a1, 4));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        float my_y;
        const float my_s = row_scale(max(m & 0xffffu, m >> 16), my_y);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            s[r] = __shfl_sync(0xffffffffu, my_s, (lane & 16) | (r >> 1) * 8 | (r & 1) * 4);
            y[r] = __shfl_sync(0xffffffffu, my_y, (lane & 16) | (r >> 1) * 8 | (r & 1) * 4);
        }
    } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            uint32_t m = pair_max(raw[r]);
#pragma unroll
            for (int d = 8; d; d >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, d));
            s[r] = row_scale(max(m & 0xffffu, m >> 16), y[r]);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------
// Cache write.  A warp takes kRows consecutive KV heads of one token: lanes 0-15 the K row, 16-31 the V row, one 16-byte load
// each, all kRows loads in flight before the first is used.  Bound by HBM bytes for long chunks and by the chain
// q_start -> (range, length) -> page table -> store for single tokens; the data loads do not wait for that chain.
// ------------------------------------------------------------------------------------------------------------
template <bool KV8, int kRows>
__global__ void __launch_bounds__(128) append_kernel(KvView kv, Kv8View c8, ChunkView cv, Strided kn, const __nv_bfloat16 *__restrict__ v_new, unsigned *status) {
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    const int lane = threadIdx.x & 31, t = blockIdx.x * 4 + (threadIdx.x >> 5), h0 = blockIdx.y * kRows;
    if (blockIdx.x == 0 && blockIdx.y == 0 && status)       // ranges that are none are reported, whether a token falls into them or not
        for (int p = threadIdx.x; p < kv.P; p += 128) { int a; chunk_len_of(cv, p, &a, status); }
    if (t >= cv.n_tokens) return;
    const int half = lane >> 4, l16 = lane & 15;
    const __nv_bfloat16 *src = (half ? v_new : kn.p) + (long long)t * kn.st + (long long)h0 * kn.sh + l16 * 8;
    uint4 raw[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        raw[r] = h0 + r < kv.H_kv ? *reinterpret_cast<const uint4 *>(src + r * kn.sh) : make_uint4(0, 0, 0, 0);
    const int p = find_problem(cv.q_start, kv.P, t, lane);
    if (p < 0) return;
    int a;
    const int n = chunk_len_of(cv, p, &a, nullptr);
    if (t - a >= n) return;
    const int N = kv.seq_lens ? kv.seq_lens[p] : kv.N_max;
    if (N > kv.N_max || n > N) {
        if (status && lane == 0) atomicOr(status, MAGE_DEV_CACHE_FULL);
        return;
    }
    const int j = N - n + (t - a);
    long long off, soff;
    if (!row_at(kv, p, h0, j, off, soff, lane == 0 ? status : nullptr)) return;
    // the next head's row: a page further by its rows, or the caller's head stride
    const long long step = kv.page_size ? (long long)kv.page_size * kD : kv.stride_h, sstep = kv.page_size ? kv.page_size : kv.N_max;
    [[maybe_unused]] float s[kRows], y[kRows];
    if (KV8) row_scales<kRows>(raw, lane, s, y);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (h0 + r >= kv.H_kv) break;
        if (KV8) {
            *reinterpret_cast<uint2 *>((half ? c8.v8 : c8.k8) + off + r * step + l16 * 8) = row_codes(raw[r], s[r], y[r]);
            if (l16 == 0) (half ? c8.v_scale : c8.k_scale)[soff + r * sstep] = s[r];
        } else {
            *reinterpret_cast<uint4 *>(const_cast<__nv_bfloat16 *>(half ? kv.v : kv.k) + off + r * step + l16 * 8) = raw[r];
        }
    }
}

// ------------------------------------------------------------------------------------------------------------
// Cache read: a warp takes kReadRows rows of one (problem, KV head), sixteen lanes the K row and sixteen the V row, eight codes
// (8 bytes) in and eight bf16 (16 bytes) out per lane; all loads of the warp's rows are in flight together.
// ------------------------------------------------------------------------------------------------------------
constexpr int kReadRows = 4;
__global__ void __launch_bounds__(256) read_kernel(KvView kv, Kv8View c8, const int *__restrict__ indices, const int *__restrict__ k_eff, int row_begin, int n_rows,
                                                   __nv_bfloat16 *__restrict__ k_out, __nv_bfloat16 *__restrict__ v_out, unsigned *status) {
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const int z = blockIdx.y, r0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * kReadRows, p = z / kv.H_kv, h = z % kv.H_kv, N = seq_len_of(kv, p);
    if (r0 >= n_rows) return;
    const int n_here = indices ? min(max(k_eff[p], 0), n_rows) : n_rows;
    int j[kReadRows];
#pragma unroll
    for (int r = 0; r < kReadRows; ++r) {
        j[r] = -1;
        if (r0 + r < n_here) {
            if (indices) {
                j[r] = indices[(long long)z * n_rows + r0 + r];
                if (j[r] < 0 || j[r] >= N) {
                    if (status && lane == 0) atomicOr(status, MAGE_DEV_BAD_INDEX);
                    j[r] = -1;
                }
            } else if (r0 + r < N - row_begin) {
                j[r] = row_begin + r0 + r;
            }
        }
    }
    uint2 code[kReadRows];
    float s[kReadRows];
#pragma unroll
    for (int r = 0; r < kReadRows; ++r) {
        long long off, soff;
        if (j[r] >= 0 && row_at(kv, p, h, j[r], off, soff, lane == 0 ? status : nullptr)) {
            code[r] = *reinterpret_cast<const uint2 *>((half ? c8.v8 : c8.k8) + off + l16 * 8);
            s[r] = (half ? c8.v_scale : c8.k_scale)[soff];
        } else {
            j[r] = -1;
        }
    }
#pragma unroll
    for (int r = 0; r < kReadRows; ++r) {
        if (j[r] < 0) continue;
        unsigned o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned short two = (unsigned short)((i < 2 ? code[r].x : code[r].y) >> (16 * (i & 1)));
            unsigned h2;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(two));             // exact
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
            o[i] = ptx::pack_bf16x2(f.x * s[r], f.y * s[r]);                      // two roundings: single precision, then bf16
        }
        *reinterpret_cast<uint4 *>((half ? v_out : k_out) + ((long long)z * n_rows + r0 + r) * kD + l16 * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

}  // namespace chunk
}  // namespace mage
