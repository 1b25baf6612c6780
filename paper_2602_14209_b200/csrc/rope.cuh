// Rotary positions with several axes on packed queries and keys, alone or on the way into the cache.
#pragma once
#include "chunk.cuh"
#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mage {
namespace rope {

struct Args {
    const __nv_bfloat16 *in[2];                  // queries, keys
    __nv_bfloat16 *out[2];
    long long st[2], sh[2], ost[2], osh[2];
    int heads[2];
    int n_tokens, rot, halves, n_axes;
    float mult;
    const int *positions;
    long long pos_stride;
    const float *inv_freq;
    uint8_t axis[64];
};

__device__ __forceinline__ uint4 pack8(const float *y) {
    return make_uint4(ptx::pack_bf16x2(y[0], y[1]), ptx::pack_bf16x2(y[2], y[3]), ptx::pack_bf16x2(y[4], y[5]), ptx::pack_bf16x2(y[6], y[7]));
}

// A pair, turned.  Which product is rounded is spelled out, since the kernels of this file promise one another's bits and would otherwise have them by the
// compiler's choice of what to contract.
__device__ __forceinline__ void turn_pair(float x1, float x2, float c, float s, float &y1, float &y2) {
    const float x2s = __fmul_rn(x2, s), x1s = __fmul_rn(x1, s);
    y1 = fmaf(x1, c, -x2s);
    y2 = fmaf(x2, c, x1s);
}
// Two of them, by (cos, sin) twice: the four products first (with pairs (i, i + rot/2) 15385 tokens take 54.4 us so, 54.9 pair by pair).
__device__ __forceinline__ void turn_two(float x1, float x2, float z1, float z2, const float4 &cs, float &y1, float &y2, float &w1, float &w2) {
    const float x2s = __fmul_rn(x2, cs.y), z2s = __fmul_rn(z2, cs.w), x1s = __fmul_rn(x1, cs.y), z1s = __fmul_rn(z1, cs.w);
    y1 = fmaf(x1, cs.x, -x2s);
    w1 = fmaf(z1, cs.z, -z2s);
    y2 = fmaf(x2, cs.x, x1s);
    w2 = fmaf(z2, cs.z, z1s);
}

// A CTA takes kTok tokens: it computes their rot/2 (cos, sin) pairs once -- the turn pos * inv_freq / 2 pi in double, reduced to
// its fraction exactly, then sincospif -- and applies them to all heads.  A thread's unit is 16 elements of one head (two
// 16-byte pieces that hold eight whole pairs), so every load and store is 16 bytes wide and a warp covers four heads.
// Bound by HBM bytes for prompts; for a few tokens by one dependent chain (position -> table in shared memory -> rotation),
// under which the data loads of the first units are already in flight.
template <int kTok, int kThreads, int kAhead>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Args a) {
    __shared__ __align__(16) float2 cs[kTok][64];
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    const int t0 = blockIdx.x * kTok, pairs = a.rot >> 1, heads = a.heads[0] + a.heads[1];
    const int n_tok = min(kTok, a.n_tokens - t0), units = n_tok * heads * 8, rot_units = a.rot >> 4;
    struct Unit {                                // token, head, eight pairs (or sixteen elements to copy)
        uint4 r0, r1;
        __nv_bfloat16 *dst;
        int d0, d1, u, tok;
    };
    auto fetch = [&](Unit &x, int i) {
        x.u = i & 7;
        const int th = i >> 3, hh = th % heads;
        x.tok = th / heads;
        const int k = hh >= a.heads[0], h = hh - (k ? a.heads[0] : 0);
        const __nv_bfloat16 *src = a.in[k] + (long long)(t0 + x.tok) * a.st[k] + (long long)h * a.sh[k];
        x.dst = a.out[k] + (long long)(t0 + x.tok) * a.ost[k] + (long long)h * a.osh[k];
        x.d0 = a.halves && x.u < rot_units ? x.u * 8 : x.u * 16;
        x.d1 = a.halves && x.u < rot_units ? pairs + x.u * 8 : x.u * 16 + 8;
        x.r0 = *reinterpret_cast<const uint4 *>(src + x.d0);
        x.r1 = *reinterpret_cast<const uint4 *>(src + x.d1);
    };
    auto finish = [&](Unit &v) {
        if (v.u < rot_units) {
            float x[16], y[16];
            bf16x8_to_float(v.r0, x);
            bf16x8_to_float(v.r1, x + 8);
            const float4 *w = reinterpret_cast<const float4 *>(cs[v.tok] + v.u * 8);      // (cos, sin) of two pairs each
            if (a.halves) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) turn_two(x[e], x[e + 8], x[e + 1], x[e + 9], w[e >> 1], y[e], y[e + 8], y[e + 1], y[e + 9]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float4 c = w[e >> 1];
                    turn_pair(x[2 * e], x[2 * e + 1], c.x, c.y, y[2 * e], y[2 * e + 1]);
                    turn_pair(x[2 * e + 2], x[2 * e + 3], c.z, c.w, y[2 * e + 2], y[2 * e + 3]);
                }
            }
            v.r0 = pack8(y);
            v.r1 = pack8(y + 8);
        }
        *reinterpret_cast<uint4 *>(v.dst + v.d0) = v.r0;
        *reinterpret_cast<uint4 *>(v.dst + v.d1) = v.r1;
    };
    Unit x[kAhead];                              // units in flight; the first ones under the table's computation
    int i = threadIdx.x;
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
        if (i + q * kThreads < units) fetch(x[q], i + q * kThreads);
    for (int e = threadIdx.x; e < n_tok * pairs; e += kThreads) {
        const int tk = e / pairs, pr = e % pairs;
        const double t = (double)a.positions[a.axis[pr] * a.pos_stride + t0 + tk] * (double)a.inv_freq[pr] * 0.15915494309189533577;
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        cs[tk][pr] = make_float2(c * a.mult, s * a.mult);
    }
    __syncthreads();
    for (; i < units; i += kAhead * kThreads) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (i + q * kThreads < units) finish(x[q]);
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            if (i + (kAhead + q) * kThreads < units) fetch(x[q], i + (kAhead + q) * kThreads);
    }
}

// ------------------------------------------------------------------------------------------------------------
// Rotation and cache write in one pass: queries rotated to q_out, keys rotated and written to the cache, values written, the new tokens read
// once and nothing of them written but the cache's own format.
//
// A CTA takes kTok tokens.  Their (cos, sin) are computed once into shared memory, and one warp per token looks up its place in the cache
// (problem, range, length, page: a chain of loads) beside that; the data loads of the first units are in flight meanwhile.  Queries go as in
// rope_kernel.  A key row is sixteen lanes of eight neighbouring elements, as the codes need it: with the pairs (i, i + rot/2) a lane
// loads its partner's piece too (from L1) instead of exchanging; the other sixteen lanes hold the value row of the same head.
// The key is rounded to bf16 before it is coded: the cache holds what a rotation and a write one after the other would leave.
// Bound by HBM bytes for prompts (15385 tokens, 32 + 8 + 8 heads: 65 us for 378 MB, rotation and write one after the other 76; scalar products 73, units placed by
// divisions 79) and by the chain for single tokens (48 tokens 3.5 us, 4.3).  Over 8 and 4 bits by issue slots (74 and 73 %: rows are coded one at a time here, where the
// write alone shares the work on their scales among four): 73.8 and 70.5 us, one after the other 75.9 and 75.8 (pairs of neighbours 73.0 and 69.7, 84.1 and 83.9).
// ------------------------------------------------------------------------------------------------------------
// Eight elements and their partners: x cos -+ partner sin as in turn_pair, on two elements at once.
struct Turn {
    float4 c[2], s[2];
    __device__ __forceinline__ Turn(const float *cos_p, const float *sin_p) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            c[i] = reinterpret_cast<const float4 *>(cos_p)[i];
            s[i] = reinterpret_cast<const float4 *>(sin_p)[i];
        }
    }
    static __device__ __forceinline__ uint64_t wide(uint32_t w) { return ptx::pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    __device__ __forceinline__ uint4 apply(const uint4 &own, const uint4 &far, float sign) const {
        const uint32_t x[4] = {own.x, own.y, own.z, own.w}, f[4] = {far.x, far.y, far.z, far.w};
        const uint64_t sign2 = ptx::pack2(sign, sign);
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 &ci = c[i >> 1], &si = s[i >> 1];
            const uint64_t c2 = i & 1 ? ptx::pack2(ci.z, ci.w) : ptx::pack2(ci.x, ci.y), s2 = i & 1 ? ptx::pack2(si.z, si.w) : ptx::pack2(si.x, si.y);
            float lo, hi;
            ptx::unpack2(ptx::fma2(wide(x[i]), c2, ptx::mul2(wide(f[i]), ptx::mul2(s2, sign2))), lo, hi);
            y[i] = ptx::pack_bf16x2(lo, hi);
        }
        return make_uint4(y[0], y[1], y[2], y[3]);
    }
};
// Four pairs of neighbours.
__device__ __forceinline__ uint4 turn_neighbours(const uint4 &own, const float *cos_p, const float *sin_p) {
    const float4 c4 = *reinterpret_cast<const float4 *>(cos_p), s4 = *reinterpret_cast<const float4 *>(sin_p);
    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
    const uint32_t x[4] = {own.x, own.y, own.z, own.w};
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __uint_as_float(x[i] << 16), hi = __uint_as_float(x[i] & 0xffff0000u);
        float y1, y2;
        turn_pair(lo, hi, c[i], s[i], y1, y2);
        y[i] = ptx::pack_bf16x2(y1, y2);
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

struct Place {
    int p, j, page;                              // problem, position (page's entry); p < 0: nobody's token; j < 0: nothing is written
};
template <int BITS, int kTok, int kThreads, int kRows, int kPerSm>
__global__ void __launch_bounds__(kThreads, kPerSm) rope_append_kernel(const __grid_constant__ Args a, KvView kv, chunk::CodeView<BITS> cc, chunk::ChunkView cv,
                                                               const __nv_bfloat16 *__restrict__ v_new, unsigned *status) {
    __shared__ __align__(16) float cos_s[kTok][64], sin_s[kTok][64];
    __shared__ Place place[kTok];
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
    const int t0 = blockIdx.x * kTok, pairs = a.rot >> 1, n_tok = min(kTok, a.n_tokens - t0), hkv = kv.H_kv, groups = (hkv + kRows - 1) / kRows;
    if (blockIdx.x == 0 && status)                          // ranges that are none are reported, whether a token falls into them or not
        for (int p = threadIdx.x; p < kv.P; p += kThreads) { int first; chunk::chunk_len_of(cv, p, &first, status); }

    // ---- keys and values: a job is kRows heads of one token; this lane's piece of eight elements and its partner's
    const int e0 = l16 * 8;
    const bool turns = !half && e0 < a.rot, upper = e0 >= pairs;
    const int e_far = upper ? e0 - pairs : e0 + pairs;
    struct Job {
        uint4 own[kRows], far[kRows];
    };
    auto fetch_job = [&](Job &x, int tk, int h0) {
        const __nv_bfloat16 *src = (half ? v_new : a.in[1]) + (long long)(t0 + tk) * a.st[1] + (long long)h0 * a.sh[1];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            x.own[r] = x.far[r] = make_uint4(0, 0, 0, 0);
            if (h0 + r < hkv) {
                x.own[r] = *reinterpret_cast<const uint4 *>(src + r * a.sh[1] + e0);
                if (turns && a.halves) x.far[r] = *reinterpret_cast<const uint4 *>(src + r * a.sh[1] + e_far);
            }
        }
    };
    // ---- queries: as in rope_kernel
    const int heads = a.heads[0], units = n_tok * heads * 8, rot_units = a.rot >> 4;
    // (a thread keeps its place in a head and goes on by kThreads / 8 heads: no divisions)
    struct Unit {
        uint4 r0, r1;
        int h, tok;
    };
    const int u = threadIdx.x & 7, d0 = a.halves && u < rot_units ? u * 8 : u * 16, d1 = a.halves && u < rot_units ? pairs + u * 8 : u * 16 + 8;
    int h_at = threadIdx.x >> 3, tok_at = 0;
    while (h_at >= heads) { h_at -= heads; ++tok_at; }
    auto fetch = [&](Unit &x) {
        x.h = h_at;
        x.tok = tok_at;
        const __nv_bfloat16 *src = a.in[0] + (long long)(t0 + tok_at) * a.st[0] + (long long)h_at * a.sh[0];
        x.r0 = *reinterpret_cast<const uint4 *>(src + d0);
        x.r1 = *reinterpret_cast<const uint4 *>(src + d1);
        h_at += kThreads / 8;
        while (h_at >= heads) { h_at -= heads; ++tok_at; }
    };
    auto finish = [&](Unit &v) {
        if (place[v.tok].p < 0) return;
        if (u < rot_units) {
            if (a.halves) {
                const Turn t(cos_s[v.tok] + u * 8, sin_s[v.tok] + u * 8);
                const uint4 lo = v.r0;
                v.r0 = t.apply(lo, v.r1, -1.f);
                v.r1 = t.apply(v.r1, lo, 1.f);
            } else {
                v.r0 = turn_neighbours(v.r0, cos_s[v.tok] + u * 8, sin_s[v.tok] + u * 8);
                v.r1 = turn_neighbours(v.r1, cos_s[v.tok] + u * 8 + 4, sin_s[v.tok] + u * 8 + 4);
            }
        }
        __nv_bfloat16 *dst = a.out[0] + (long long)(t0 + v.tok) * a.ost[0] + (long long)v.h * a.osh[0];
        *reinterpret_cast<uint4 *>(dst + d0) = v.r0;
        *reinterpret_cast<uint4 *>(dst + d1) = v.r1;
    };

    Job job;
    Unit unit;
    int jb = warp, i = threadIdx.x;
    const int jobs = n_tok * groups;
    int tk = 0, hg = warp;                       // the job's token and group of heads
    while (hg >= groups) { hg -= groups; ++tk; }
    if (jb < jobs) fetch_job(job, tk, hg * kRows);
    if (i < units) fetch(unit);

    // ---- places of the tokens, and the table
    if (warp < n_tok) {
        Place at = {-1, -1, 0};
        const int t = t0 + warp, p = chunk::find_problem(cv.q_start, kv.P, t, lane);
        int first = 0;
        const int n = p < 0 ? 0 : chunk::chunk_len_of(cv, p, &first, nullptr);
        if (t - first < n) {
            at.p = p;
            const int N = kv.seq_lens ? kv.seq_lens[p] : kv.N_max;
            if (N > kv.N_max || n > N) {
                if (status && lane == 0) atomicOr(status, MAGE_DEV_CACHE_FULL);
            } else {
                at.j = N - n + (t - first);
                if (kv.page_size) {
                    at.page = kv.block_table[(long long)p * kv.max_pages + (at.j >> (31 - __clz(kv.page_size)))];
                    if (at.page < 0 || at.page >= kv.num_pages) {
                        if (status && lane == 0) atomicOr(status, MAGE_DEV_BAD_PAGE);
                        at.j = -1;
                    }
                }
            }
        }
        if (lane == 0) place[warp] = at;
    }
    for (int e = threadIdx.x; e < n_tok * pairs; e += kThreads) {
        const int tk = e / pairs, pr = e % pairs;
        const double t = (double)a.positions[a.axis[pr] * a.pos_stride + t0 + tk] * (double)a.inv_freq[pr] * 0.15915494309189533577;
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        cos_s[tk][pr] = c * a.mult;
        sin_s[tk][pr] = s * a.mult;
    }
    __syncthreads();

#pragma unroll 1
    for (; jb < jobs; jb += kThreads / 32) {
        const int h0 = hg * kRows;
        const Place at = place[tk];
        uint4 raw[kRows];
        if (turns) {
            if (a.halves) {
                const Turn t(cos_s[tk] + (upper ? e_far : e0), sin_s[tk] + (upper ? e_far : e0));
#pragma unroll
                for (int r = 0; r < kRows; ++r) raw[r] = t.apply(job.own[r], job.far[r], upper ? 1.f : -1.f);
            } else {
#pragma unroll
                for (int r = 0; r < kRows; ++r) raw[r] = turn_neighbours(job.own[r], cos_s[tk] + (e0 >> 1), sin_s[tk] + (e0 >> 1));
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRows; ++r) raw[r] = job.own[r];
        }
        hg += kThreads / 32;
        while (hg >= groups) { hg -= groups; ++tk; }
        if (jb + kThreads / 32 < jobs) fetch_job(job, tk, hg * kRows);
        __syncwarp();
        if (at.j < 0) continue;
        long long off, soff, step, sstep;
        if (kv.page_size) {
            sstep = kv.page_size;
            soff = ((long long)at.page * hkv + h0) * kv.page_size + (at.j & (kv.page_size - 1));
            off = soff * kD;
            step = sstep * kD;
        } else {
            sstep = kv.N_max;
            soff = ((long long)at.p * hkv + h0) * kv.N_max + at.j;
            off = (long long)at.p * kv.stride_p + (long long)h0 * kv.stride_h + (long long)at.j * kv.stride_n;
            step = kv.stride_h;
        }
        chunk::put_rows<BITS, kRows>(kv, cc, raw, off, soff, step, sstep, hkv - h0, lane);
    }
#pragma unroll 1
    for (; i < units; i += kThreads) {
        Unit v = unit;
        if (i + kThreads < units) fetch(unit);
        finish(v);
    }
}

}  // namespace rope
}  // namespace mage
