// Per-head RMSNorm of queries and keys and the rotation by position in one pass, with the new keys' and values' way into
// the cache:
//   y = x * gamma / sqrt(mean(x^2) + eps)                          over the head (no gamma: y = x)
//   (y1, y2) -> (y1 cos t - y2 sin t, y2 cos t + y1 sin t),  t = position * inv_freq[i]
// for the pairs (i, i + rot / 2), or (2 i, 2 i + 1) interleaved, i < rot / 2; the columns from rot on stay y.  All in single
// precision, rounded once to fp16; the angle in double (single would be off by 2^-24 of the angle: 0.008 at position 131072).
//
// A lane holds both members of four pairs, so that the rotation needs no exchange between lanes; the lanes of a head share
// its sum of squares.  A workgroup takes one token (or some of its heads): cosines and sines are computed once per token and
// pair and stay in the lanes' registers over the heads.  Bound by memory: 8192 tokens of 64 + 8 + 8 heads of 128, 336 MB, 78 us
// (4.3 TB/s; a plain copy 4.9).  Four tokens a workgroup with the loads a round ahead: 99 us; 512 lanes: 89; the heads of a token over
// several workgroups there too: 99.
#include "block_common.h"

namespace intscale {
namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ void widen4(uint2 v, float* f) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
    const float2 a = __half22float2(h[0]), b = __half22float2(h[1]);
    f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
}
__device__ __forceinline__ uint2 narrow4(const float* f) {
    uint2 v;
    __half2* h = reinterpret_cast<__half2*>(&v);
    h[0] = __floats2half2_rn(f[0], f[1]);
    h[1] = __floats2half2_rn(f[2], f[3]);
    return v;
}

// Read once and written for a later kernel: past the caches (82 us without the marks).
__device__ __forceinline__ uint2 load_past(const __half* p) {
    const unsigned long long v = __builtin_nontemporal_load(reinterpret_cast<const unsigned long long*>(p));
    return make_uint2((unsigned)v, (unsigned)(v >> 32));
}
__device__ __forceinline__ void store_past(__half* p, uint2 v) {
    __builtin_nontemporal_store(((unsigned long long)v.y << 32) | v.x, reinterpret_cast<unsigned long long*>(p));
}

// L lanes a head (a power of two, head_dim / 8 of them at work).
template <int L>
__global__ __launch_bounds__(kRopeThreads) void qk_norm_rope_kernel(RopeArgs a, int slots_per_wg) {
    __shared__ float2 turn[128];  // cos, sin
    const int m = blockIdx.x, tid = threadIdx.x, j = tid % L;
    const int pairs = a.rot_dim >> 1;
    if (tid < pairs) {
        // angle in turns, its whole part taken off in double
        const double t = (double)a.positions[m] * (double)a.inv_freq[tid] * 0.15915494309189533577;
        float sn, cs;
        sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
        turn[tid] = make_float2(cs, sn);
    }
    __syncthreads();
    const bool work = j * 8 < a.head_dim, rot = j * 8 < a.rot_dim;
    // columns of this lane: two runs of four
    const int first = rot && !a.interleaved ? 4 * j : 8 * j, second = rot && !a.interleaved ? pairs + 4 * j : 8 * j + 4;
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = rot ? turn[4 * j + i] : make_float2(1.0f, 0.0f);
        cs[i] = t.x, sn[i] = t.y;
    }
    const long long row = a.kv_rows ? a.kv_rows[m] : m;
    const bool row_in = row >= 0 && row < a.cache_rows;  // (a row outside the cache, a padding token's, goes nowhere)
    const int heads = a.heads_q + a.heads_k, slots = heads + (a.v ? a.heads_k : 0);
    const int to = min(slots, (int)(blockIdx.y + 1) * slots_per_wg);
    const float inv_dim = 1.0f / (float)a.head_dim;
    for (int s0 = blockIdx.y * slots_per_wg; s0 < to; s0 += kRopeThreads / L) {
        const int s = s0 + tid / L;
        const bool is_q = s < a.heads_q, is_v = s >= heads, on = s < to && work;
        const int h = is_q ? s : is_v ? s - heads : s - a.heads_q;
        const __half* src = is_q ? a.q + (size_t)m * a.ldq : is_v ? a.v + (size_t)m * a.ldv : a.k + (size_t)m * a.ldk;
        src += (size_t)h * a.head_dim;
        uint2 u1 = make_uint2(0u, 0u), u2 = u1;
        if (on) {
            u1 = load_past(src + first);
            u2 = load_past(src + second);
        }
        float x[8];
        widen4(u1, x);
        widen4(u2, x + 4);
        const __half* gamma = is_q ? a.gamma_q : a.gamma_k;
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int d = 1; d < L; d *= 2) ss += __shfl_xor(ss, d, kWave);
        if (!on) continue;
        if (!is_v) {
            if (gamma != nullptr) {
                const float r = 1.0f / sqrtf(fmaf(ss, inv_dim, a.eps));
                float g[8];
                widen4(*reinterpret_cast<const uint2*>(gamma + first), g);
                widen4(*reinterpret_cast<const uint2*>(gamma + second), g + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[i];
            }
            if (rot) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = a.interleaved ? 2 * i : i, q = a.interleaved ? 2 * i + 1 : i + 4;
                    const float y1 = x[p], y2 = x[q];
                    x[p] = y1 * cs[i] - y2 * sn[i];
                    x[q] = y2 * cs[i] + y1 * sn[i];
                }
            }
            u1 = narrow4(x);
            u2 = narrow4(x + 4);
        }
        if (!is_q && !row_in) continue;
        __half* dst = is_q ? a.q_out + (size_t)m * a.ldqo : is_v ? a.v_out + (size_t)row * a.ldvo : a.k_out + (size_t)row * a.ldko;
        dst += (size_t)h * a.head_dim;
        store_past(dst + first, u1);
        store_past(dst + second, u2);
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream) {
    int lanes = 1;
    while (lanes * 8 < a.head_dim) lanes *= 2;
    const int slots = a.heads_q + a.heads_k * (a.v ? 2 : 1), at_once = kRopeThreads / lanes;
    // few tokens: their heads over several workgroups
    const int rounds = (slots + at_once - 1) / at_once;
    const int parts = a.M < cu_count() ? rounds : 1;
    const int per_wg = (rounds + parts - 1) / parts * at_once;
    const dim3 grid(a.M, (slots + per_wg - 1) / per_wg);
#define ROPE_LAUNCH(L) \
    case L: hipLaunchKernelGGL((qk_norm_rope_kernel<L>), grid, dim3(kRopeThreads), 0, stream, a, per_wg); break
    switch (lanes) {
        ROPE_LAUNCH(1);
        ROPE_LAUNCH(2);
        ROPE_LAUNCH(4);
        ROPE_LAUNCH(8);
        ROPE_LAUNCH(16);
        ROPE_LAUNCH(32);
        default: return hipErrorInvalidValue;
    }
#undef ROPE_LAUNCH
    return hipGetLastError();
}

}  // namespace intscale
