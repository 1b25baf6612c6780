// Rotary positions with several axes on packed queries and keys.
#pragma once
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
                for (int e = 0; e < 8; e += 2) {
                    const float4 c = w[e >> 1];
                    y[e] = x[e] * c.x - x[e + 8] * c.y;
                    y[e + 8] = x[e + 8] * c.x + x[e] * c.y;
                    y[e + 1] = x[e + 1] * c.z - x[e + 9] * c.w;
                    y[e + 9] = x[e + 9] * c.z + x[e + 1] * c.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float4 c = w[e >> 1];
                    y[2 * e] = x[2 * e] * c.x - x[2 * e + 1] * c.y;
                    y[2 * e + 1] = x[2 * e + 1] * c.x + x[2 * e] * c.y;
                    y[2 * e + 2] = x[2 * e + 2] * c.z - x[2 * e + 3] * c.w;
                    y[2 * e + 3] = x[2 * e + 3] * c.z + x[2 * e + 2] * c.w;
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

}  // namespace rope
}  // namespace mage
