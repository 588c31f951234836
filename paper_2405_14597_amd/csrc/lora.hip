// Low-rank adapters of many requests beside a shared projection:
//   out[m] = base[m] + scale_e (x[m] A_e^T) B_e^T,  e = the row's adapter; rows without one: out[m] = base[m]
// Two kernels a call: the inner products t = x A_e^T [M, R] in single precision to the workspace, then the outer product added to
// the base.  Two forms of them:
//   by rows   every row by itself with its own adapter, on the vector units: a decode step's rows have an adapter each, and
//             what such a step computes is little; bound by latency (64 rows of 32 adapters, rank 16, 4096 x 4096: 3.9 + 2.9 us, 7.2 in
//             all where the tiles take 40; one row 3.0 + 2.3 us);
//   by tiles  32 or 64 rows at a time on the matrix units, for prompts, whose rows share an adapter in long runs: bound by the reading
//             of x and base and the writing of out, of which too little is on its way at a time (4096 rows of nine requests, rank 64,
//             4096 x 6144: 28 + 40 us, 72 in all, 138 MB at 1.9 TB/s).  A tile walks the adapters that occur in it and keeps each row's own
//             result (selected, not masked by a factor, so that nothing of one adapter, an infinity for one, reaches another
//             request's rows).
#include <algorithm>

#include "block_common.h"

namespace intscale {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kLoraWaves = 4;

// The adapter of a row, -1 for none.
__device__ __forceinline__ int own_adapter(const LoraArgs& a, int row) {
    const int e = row < a.M ? a.row_adapter[row] : -1;
    return e >= 0 && e < a.adapters ? e : -1;
}
__device__ __forceinline__ int rank_of(const LoraArgs& a, int e) { return a.ranks ? min(max(a.ranks[e], 0), a.R) : a.R; }

__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d, kWave);
    return v;
}

// ---- by rows
// t[row][r]: a wave takes two r, its lanes eight k each of every 512.
__global__ __launch_bounds__(kLoraWaves* kWave) void lora_inner_rows_kernel(LoraArgs a) {
    const int lane = threadIdx.x & (kWave - 1), row = blockIdx.x;
    const int r = (blockIdx.y * kLoraWaves + threadIdx.x / kWave) * 2;
    const int e = own_adapter(a, row);
    if (e < 0 || r >= a.R) return;  // (R is even: r + 1 < R)
    const int rank = rank_of(a, e);
    const __half* x = a.x + (size_t)row * a.ldx;
    const __half* w0 = a.a + ((size_t)e * a.R + r) * a.K;
    const __half* w1 = w0 + a.K;
    float t0 = 0.0f, t1 = 0.0f;
    if (r < rank) {
        constexpr int kAtOnce = 4;
        for (int k0 = lane * 8; k0 < a.K; k0 += kAtOnce * kWave * 8) {
            h8 xv[kAtOnce], u[kAtOnce], v[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int k = k0 + i * kWave * 8;
                const bool in = k < a.K;
                xv[i] = in ? *reinterpret_cast<const h8*>(x + k) : h8{};
                u[i] = in ? *reinterpret_cast<const h8*>(w0 + k) : h8{};
                v[i] = in ? *reinterpret_cast<const h8*>(w1 + k) : h8{};
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    t0 = fmaf((float)xv[i][j], (float)u[i][j], t0);
                    t1 = fmaf((float)xv[i][j], (float)v[i][j], t1);
                }
        }
    }
    t0 = lanes_sum(t0);
    t1 = lanes_sum(t1);
    if (lane == 0) *reinterpret_cast<float2*>(a.inner + (size_t)row * a.R + r) = make_float2(r < rank ? t0 : 0.0f, r + 1 < rank ? t1 : 0.0f);
}

// One column of out a lane: the row of B behind it is R contiguous elements, t[row] the same for all lanes.
__global__ __launch_bounds__(kLoraWaves* kWave) void lora_outer_rows_kernel(LoraArgs a) {
    const int row = blockIdx.x, n = blockIdx.y * kLoraWaves * kWave + threadIdx.x;
    const int e = own_adapter(a, row);
    if (n >= a.N || (e < 0 && a.base == a.out)) return;  // (rows without an adapter stay as they are)
    const __half base = a.base ? a.base[(size_t)row * a.ldb + n] : __float2half(0.0f);
    float y = 0.0f;
    if (e >= 0) {
        const int rank = rank_of(a, e);
        const __half* w = a.b + ((size_t)e * a.N + n) * a.R;
        const float* t = a.inner + (size_t)row * a.R;
        int r = 0;
#pragma unroll 4
        for (; r + 8 <= rank; r += 8) {
            const h8 v = *reinterpret_cast<const h8*>(w + r);
#pragma unroll
            for (int j = 0; j < 8; ++j) y = fmaf((float)v[j], t[r + j], y);
        }
        for (; r < rank; ++r) y = fmaf(__half2float(w[r]), t[r], y);
        y *= a.scales ? a.scales[e] : 1.0f;
    }
    a.out[(size_t)row * a.ldo + n] = e >= 0 ? __float2half(__half2float(base) + y) : base;
}

// ---- by tiles
constexpr int kInnerBlocks = 2;                 // 16-row blocks of a tile of the inner products
constexpr int kOuterBlocks = 2;                 // a wave's of the outer product
constexpr int kOuterRows = 64, kOuterCols = 64; // a workgroup's tile of it: two waves down, two across

// The adapters in a tile's rows, one after the other: `todo[b]` holds the rows of block b whose adapter has not come yet.
template <int CB>
__device__ __forceinline__ int next_adapter(const int (&mine)[CB], unsigned long long (&todo)[CB]) {
    int e = -1;
#pragma unroll
    for (int b = 0; b < CB; ++b)
        if (e < 0 && todo[b]) e = __builtin_amdgcn_readlane(mine[b], __builtin_ctzll(todo[b]));
#pragma unroll
    for (int b = 0; b < CB; ++b) todo[b] &= ~__ballot(mine[b] == e);
    return e;
}

// t[row][r] of one slab of K.  First operand: 16 rows of A (r), second: 16 rows of x, 32 k an instruction; the four waves take
// turns of four (two) runs of 32 k and meet in LDS.  A result's lane holds row lane & 15 and r = 16 i + 4 (lane >> 4) + 0..3.
template <int RT>  // R in tiles of 16
__global__ __launch_bounds__(kLoraWaves* kWave) void lora_inner_kernel(LoraArgs a) {
    constexpr int CB = kInnerBlocks;
    __shared__ float4 part[kLoraWaves][RT][CB][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, col = lane & 15, quad = lane >> 4;
    const int runs = (a.K + 31) / 32, per = (runs + a.slabs - 1) / a.slabs;
    const int r0 = blockIdx.y * per, r1 = min(r0 + per, runs);
    int mine[CB];
    unsigned long long todo[CB], any = 0;
    const __half* x[CB];
    f4 t[CB][RT];
#pragma unroll
    for (int b = 0; b < CB; ++b) {
        const int row = (blockIdx.x * CB + b) * 16 + col;
        mine[b] = own_adapter(a, row);
        todo[b] = __ballot(mine[b] >= 0);
        any |= todo[b];
        x[b] = a.x + (size_t)min(row, a.M - 1) * a.ldx;
#pragma unroll
        for (int i = 0; i < RT; ++i) t[b][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    if (any == 0) return;
    for (int e = next_adapter(mine, todo); e >= 0; e = next_adapter(mine, todo)) {
        const int rank = rank_of(a, e);
        const __half* w = a.a + (size_t)e * a.R * a.K;
        f4 s[CB][RT];
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int i = 0; i < RT; ++i) s[b][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int kAtOnce = RT <= 4 ? 4 : 2;  // runs on their way
        for (int run = r0 + wave * kAtOnce; run < r1; run += kAtOnce * kLoraWaves) {  // (whole lines of a row to one wave)
            h8 xv[kAtOnce][CB], wv[kAtOnce][RT];
            // (a row's pieces one behind the other: together they are whole lines)
            auto inside = [&](int u) { return run + u < r1 && (run + u) * 32 + quad * 8 < a.K; };
#pragma unroll
            for (int b = 0; b < CB; ++b)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) xv[u][b] = inside(u) ? *reinterpret_cast<const h8*>(x[b] + (run + u) * 32 + quad * 8) : h8{};
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    wv[u][i] = inside(u) && i * 16 + col < rank ? *reinterpret_cast<const h8*>(w + (size_t)(i * 16 + col) * a.K + (run + u) * 32 + quad * 8) : h8{};
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int b = 0; b < CB; ++b)
#pragma unroll
                    for (int i = 0; i < RT; ++i) s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv[u][i], xv[u][b], s[b][i], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    // (past the rank by a choice, too: the zeros above times an infinity of x would be NaN)
                    t[b][i][j] = mine[b] != e ? t[b][i][j] : i * 16 + quad * 4 + j < rank ? s[b][i][j] : 0.0f;
    }
#pragma unroll
    for (int b = 0; b < CB; ++b)
#pragma unroll
        for (int i = 0; i < RT; ++i) part[wave][i][b][lane] = make_float4(t[b][i][0], t[b][i][1], t[b][i][2], t[b][i][3]);
    __syncthreads();
    for (int at = threadIdx.x; at < RT * CB * kWave; at += kLoraWaves * kWave) {
        const int l = at & (kWave - 1), b = at / kWave % CB, i = at / kWave / CB;
        float4 s = part[0][i][b][l];
#pragma unroll
        for (int w = 1; w < kLoraWaves; ++w) {
            const float4 p = part[w][i][b][l];
            s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
        }
        const int row = (blockIdx.x * CB + b) * 16 + (l & 15), r = i * 16 + (l >> 4) * 4;
        if (row < a.M && r < a.R) *reinterpret_cast<float4*>(a.inner + ((size_t)blockIdx.y * a.M + row) * a.R + r) = s;
    }
}

// One element of scale t B^T as it stands in the formula, for those that are not finite: of an infinity (of B's, of t's) a second term of
// zero or of the other sign makes NaN, and a row with an infinite t[r] has no power of two that keeps its others from overflowing.
__device__ __forceinline__ float plain_product(const LoraArgs& a, int row, int e, int n) {
    const int rank = rank_of(a, e);
    float y = 0.0f;
#pragma unroll 1
    for (int r = 0; r < rank; ++r) {
        float t = 0.0f;
#pragma unroll 1
        for (int slab = 0; slab < a.slabs; ++slab) t += a.inner[((size_t)slab * a.M + row) * a.R + r];
        y = fmaf(__half2float(a.b[((size_t)e * a.N + n) * a.R + r]), t, y);
    }
    return a.scales ? a.scales[e] * y : y;
}

// out = base + scale t B^T: 32 rows x 32 columns a wave, 64 x 64 a workgroup.  First operand: rows of B (columns of out),
// second: t.  Row i of operand tile j is column 16 (i / 4) + 4 j + i % 4, so that a lane's four results of the four tiles are 16
// columns in a row.  t goes in as two fp16 terms, the row's largest brought to [0.5, 1) by a power of two: rounded to one it would add an
// error of the size of the output's own rounding, and a large t would overflow.  The second term is what the first leaves, at most 2^-12,
// times 2^27, with an accumulator of its own: so it stays a normal number, and a t[r] far below the row's largest keeps its bits (to 2^-22
// of itself, 2^-11 at worst; without the factor all below 2^-25 of the largest was lost).  The terms are made once a workgroup, for `steps`
// tiles of 64 columns, and lie in LDS as the instructions take them.
constexpr float kLowUp = 0x1p27f;
template <int RS>  // R in steps of 32
__global__ __launch_bounds__(kLoraWaves* kWave) __attribute__((amdgpu_waves_per_eu(RS <= 2 ? 4 : 2))) void lora_outer_kernel(LoraArgs a, int wide, int steps) {
    constexpr int CB = kOuterBlocks, kBlocks = kOuterRows / 16;
    __shared__ h8 hi[kBlocks][RS][kWave], lo[kBlocks][RS][kWave];
    __shared__ int power[kOuterRows];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, col = lane & 15, quad = lane >> 4;
    const int b0 = wave / 2 * CB;  // this wave's first block of 16 rows in the tile
    int mine[CB];
    unsigned long long all[CB];
#pragma unroll
    for (int b = 0; b < CB; ++b) {
        mine[b] = own_adapter(a, blockIdx.y * kOuterRows + (b0 + b) * 16 + col);
        all[b] = __ballot(mine[b] >= 0);
    }
    // ---- block `wave` of t
    static_assert(kBlocks == kLoraWaves && CB == 2, "a wave makes the terms of one block and has the results of two");
    {
        const int row = blockIdx.y * kOuterRows + wave * 16 + col;
        const bool has = own_adapter(a, row) >= 0;
        float t[RS][8], most = 0.0f;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int r = s * 32 + quad * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) t[s][i] = 0.0f;
            if (has && r < a.R) {
#pragma unroll 4
                for (int slab = 0; slab < a.slabs; ++slab) {
                    const float4* src = reinterpret_cast<const float4*>(a.inner + ((size_t)slab * a.M + row) * a.R + r);
                    const float4 u = src[0], v = src[1];
                    t[s][0] += u.x, t[s][1] += u.y, t[s][2] += u.z, t[s][3] += u.w;
                    t[s][4] += v.x, t[s][5] += v.y, t[s][6] += v.z, t[s][7] += v.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(t[s][i]));
        }
        most = fmaxf(most, __shfl_xor(most, 16, kWave));
        most = fmaxf(most, __shfl_xor(most, 32, kWave));
        // the row's largest is at least 0.5 and below 1 after it; infinities and NaN go through as they are
        const int up = most > 0.0f && most < INFINITY ? -__builtin_amdgcn_frexp_expf(most) : 0;
        if (quad == 0) power[wave * 16 + col] = -up;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            h8 h, l;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = __builtin_amdgcn_ldexpf(t[s][i], up);
                h[i] = (_Float16)v;
                l[i] = fabsf(v) < INFINITY ? (_Float16)(kLowUp * (v - (float)h[i])) : (_Float16)0.0f;
            }
            hi[wave][s][lane] = h;
            lo[wave][s][lane] = l;
        }
    }
    __syncthreads();
    // the adapters in the wave's rows, with their ranks and scales: lane i has the i-th
    unsigned long long todo[CB];
#pragma unroll
    for (int b = 0; b < CB; ++b) todo[b] = all[b];
    int count = 0, listed = 0;
    for (int e = next_adapter(mine, todo); e >= 0; e = next_adapter(mine, todo), ++count) listed = lane == count ? e : listed;
    const int rank_listed = lane < count ? rank_of(a, listed) : 0;
    const float scale_listed = lane < count && a.scales ? a.scales[listed] : 1.0f;
    auto adapter_at = [&](int i) { return __builtin_amdgcn_readlane(listed, i); };
    auto rank_at = [&](int i) { return __builtin_amdgcn_readlane(rank_listed, i); };
    auto scale_at = [&](int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale_listed), i)); };
    auto first_column = [&](int step) { return (blockIdx.x * steps + step) * kOuterCols + wave % 2 * 32; };
    auto load_base = [&](h8 (&base)[CB], int step) {
        const int n = first_column(step) + 8 * quad;
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            const int row = blockIdx.y * kOuterRows + (b0 + b) * 16 + col;
            base[b] = wide && a.base && row < a.M && n < a.N ? *reinterpret_cast<const h8*>(a.base + (size_t)row * a.ldb + n) : h8{};
        }
    };
    auto load_b = [&](h8 (&wv)[2][RS], int e, int step) {
        const __half* w = a.b + (size_t)e * a.N * a.R;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = first_column(step) + 8 * (col >> 2) + 4 * j + (col & 3);
#pragma unroll
            for (int st = 0; st < RS; ++st) {
                const int r = st * 32 + quad * 8;
                wv[j][st] = n < a.N && r < a.R ? *reinterpret_cast<const h8*>(w + (size_t)n * a.R + r) : h8{};
            }
        }
    };
    f4 sum[CB][2];
    auto add = [&](h8 (&wv)[2][RS], int e, int rank, float scale) {
        if (rank < a.R) {  // (the columns of B past the adapter's rank are not its own)
#pragma unroll
            for (int st = 0; st < RS; ++st)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool own = st * 32 + quad * 8 + i < rank;
#pragma unroll
                    for (int j = 0; j < 2; ++j) wv[j][st][i] = own ? wv[j][st][i] : (_Float16)0.0f;
                }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int b = 0; b < CB; ++b) {
                f4 s = f4{0.0f, 0.0f, 0.0f, 0.0f}, low = s;
#pragma unroll
                for (int st = 0; st < RS; ++st) {
                    s = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv[j][st], hi[b0 + b][st][lane], s, 0, 0, 0);
                    low = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv[j][st], lo[b0 + b][st][lane], low, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = fmaf(low[i], 1.0f / kLowUp, s[i]);
                const int up = power[(b0 + b) * 16 + col];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[b][j][i] = mine[b] == e ? scale * __builtin_amdgcn_ldexpf(s[i], up) : sum[b][j][i];
            }
    };
    for (int step = 0; step < steps && first_column(step) < a.N; ++step) {
        const int n = first_column(step) + 8 * quad;
        h8 base[CB];
        load_base(base, step);
#pragma unroll
        for (int b = 0; b < CB; ++b) sum[b][0] = sum[b][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (int k = 0; k < count; ++k) {
            h8 wv[2][RS];
            load_b(wv, adapter_at(k), step);
            add(wv, adapter_at(k), rank_at(k), scale_at(k));
        }
        unsigned odd = 0;  // bit 8 b + i: result i of block b is not finite
#pragma unroll
        for (int i = 0; i < 8 * CB; ++i) odd |= fabsf(sum[i / 8][i % 8 / 4][i % 4]) < INFINITY ? 0u : 1u << i;
        if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll 1
            for (; odd != 0; odd &= odd - 1) {
                const int at = __builtin_ctz(odd), b = at / 8;
                const int e = b == 0 ? mine[0] : mine[1], column = n + at % 8;
                const float y = column < a.N ? plain_product(a, blockIdx.y * kOuterRows + (b0 + b) * 16 + col, e, column) : 0.0f;
#pragma unroll
                for (int i = 0; i < 8 * CB; ++i) sum[i / 8][i % 8 / 4][i % 4] = i == at ? y : sum[i / 8][i % 8 / 4][i % 4];
            }
        }
#pragma unroll
        for (int b = 0; b < CB; ++b) {
            const int row = blockIdx.y * kOuterRows + (b0 + b) * 16 + col;
            if (row >= a.M || (mine[b] < 0 && a.base == a.out)) continue;  // (rows without an adapter stay as they are)
            __half* out = a.out + (size_t)row * a.ldo + n;
            if (wide) {
                if (n >= a.N) continue;
                h8 v = base[b];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = mine[b] >= 0 ? (_Float16)((float)v[i] + sum[b][i / 4][i % 4]) : v[i];
                *reinterpret_cast<h8*>(out) = v;
            } else {
                const __half* src = a.base ? a.base + (size_t)row * a.ldb + n : nullptr;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (n + i >= a.N) continue;
                    const __half v = src ? src[i] : __float2half(0.0f);
                    out[i] = mine[b] >= 0 ? __float2half(__half2float(v) + sum[b][i / 4][i % 4]) : v;
                }
            }
        }
    }
}

// The form by rows reads an adapter once for every row of it (from L2, mostly), whatever the rows' mix; a tile walks every adapter in it.
// Which rows have which adapter is known on the device alone, so that the limit lies between what either mix would want.  On 4096 x 4096
// the 2^26 products are 1024 rows at rank 16, 256 at rank 64; us by rows / by tiles:
//              rows in runs of four adapters                an adapter of 32 a row
//   rank 16    512: 15 / 12   1024: 24 / 19   2048: 41 / 20   512: 18 / 47   1024: 27 / 63   2048: 44 / 115
//   rank 64    128: 17 / 18    256: 27 / 19    512: 47 / 28   128: 24 / 79    256: 36 / 78    512: 56 / 92
// and on 28672 x 8192 at rank 64 (36 rows) 16: 19 / 27, 64: 38 / 31 in runs, 19 / 57, 56 / 108 mixed.
bool by_rows(int M, int N, int K, int R) { return (long long)M * R * std::max(K, N) <= 1LL << 26; }

int lora_slabs(int M, int K) {
    const int tiles = (M + 16 * kInnerBlocks - 1) / (16 * kInnerBlocks);
    return std::max(1, std::min(std::min(2 * cu_count() / tiles, 16), K / 256));
}

}  // namespace

size_t lora_workspace_bytes(int M, int N, int K, int R) { return (size_t)(by_rows(M, N, K, R) ? 1 : lora_slabs(M, K)) * M * R * 4; }

hipError_t launch_lora_add(const LoraArgs& args, void* workspace, hipStream_t stream) {
    LoraArgs a = args;
    a.inner = static_cast<float*>(workspace);
    const int threads = kLoraWaves * kWave;
    if (by_rows(a.M, a.N, a.K, a.R)) {
        hipLaunchKernelGGL(lora_inner_rows_kernel, dim3(a.M, (a.R + 2 * kLoraWaves - 1) / (2 * kLoraWaves)), dim3(threads), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(lora_outer_rows_kernel, dim3(a.M, (a.N + threads - 1) / threads), dim3(threads), 0, stream, a);
        return hipGetLastError();
    }
    a.slabs = lora_slabs(a.M, a.K);
    const int wide = a.N % 8 == 0 && a.ldo % 8 == 0 && (a.base == nullptr || a.ldb % 8 == 0);
    const dim3 inner((a.M + 16 * kInnerBlocks - 1) / (16 * kInnerBlocks), a.slabs);
    // Four workgroups a unit, each over as many columns as that leaves: every one of them adds up the slabs of t, and with more the
    // sums take longer, with fewer too little of base is on its way (4096 x 6144, rank 64, three adapters in the worst tile: 72 us with the
    // inner products; with 2 and 6 a unit 83 and 77).
    const int row_tiles = (a.M + kOuterRows - 1) / kOuterRows, col_tiles = (a.N + kOuterCols - 1) / kOuterCols;
    const int steps = std::max(1, col_tiles * row_tiles / (4 * cu_count()));
    const dim3 outer((col_tiles + steps - 1) / steps, row_tiles);
    const int rt = (a.R + 15) / 16;
    if (rt <= 1) hipLaunchKernelGGL((lora_inner_kernel<1>), inner, dim3(threads), 0, stream, a);
    else if (rt <= 2) hipLaunchKernelGGL((lora_inner_kernel<2>), inner, dim3(threads), 0, stream, a);
    else if (rt <= 4) hipLaunchKernelGGL((lora_inner_kernel<4>), inner, dim3(threads), 0, stream, a);
    else hipLaunchKernelGGL((lora_inner_kernel<8>), inner, dim3(threads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.R <= 32) hipLaunchKernelGGL((lora_outer_kernel<1>), outer, dim3(threads), 0, stream, a, wide, steps);
    else if (a.R <= 64) hipLaunchKernelGGL((lora_outer_kernel<2>), outer, dim3(threads), 0, stream, a, wide, steps);
    else hipLaunchKernelGGL((lora_outer_kernel<4>), outer, dim3(threads), 0, stream, a, wide, steps);
    return hipGetLastError();
}

}  // namespace intscale
