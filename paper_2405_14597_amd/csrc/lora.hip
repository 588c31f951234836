// Low-rank adapters of many requests beside a shared projection:
//   out[m] = base[m] + scale_e (x[m] A_e^T) B_e^T,  e = the row's adapter; rows without one: out[m] = base[m]
// Two kernels: the inner products t = x A_e^T [M, R] in single precision, cut along K so that few rows fill the chip (each
// slab's sums to the workspace), then the outer product added to the base.  Rows are taken 16 at a time whatever their
// adapters; a tile walks the adapters that occur in it and keeps each row's own result (selected, not masked by a factor, so
// that nothing of one adapter, an infinity for one, reaches another request's rows).
#include "block_common.h"

namespace intscale {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kRows = 16;      // rows of a tile: the second operand's columns
constexpr int kLoraWaves = 4;

// The adapter of this lane's row (lane & 15), -1 for none.
__device__ __forceinline__ int own_adapter(const LoraArgs& a, int row) {
    const int e = row < a.M ? a.row_adapter[row] : -1;
    return e >= 0 && e < a.adapters ? e : -1;
}
__device__ __forceinline__ int rank_of(const LoraArgs& a, int e) { return a.ranks ? min(max(a.ranks[e], 0), a.R) : a.R; }

// t[row][r] of one slab.  First operand: 16 rows of A (r), second: 16 rows of x, 32 k an instruction; the four waves take
// every fourth run of 32 k and meet in LDS.  A result's lane holds row lane & 15 and r = 16 i + 4 (lane >> 4) + 0..3.
template <int RT>  // R in tiles of 16
__global__ __launch_bounds__(kLoraWaves* kWave) void lora_inner_kernel(LoraArgs a) {
    __shared__ float4 part[kLoraWaves][RT][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, col = lane & 15, quad = lane >> 4;
    const int row = blockIdx.x * kRows + col;
    const int mine = own_adapter(a, row);
    const int runs = (a.K + 31) / 32, per = (runs + a.slabs - 1) / a.slabs;
    const int r0 = blockIdx.y * per, r1 = min(r0 + per, runs);
    const __half* x = a.x + (size_t)min(row, a.M - 1) * a.ldx;
    f4 t[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) t[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    unsigned long long todo = __ballot(mine >= 0 && quad == 0);
    if (todo == 0) return;
    while (todo) {
        const int e = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
        todo &= ~__ballot(mine == e);
        const int rank = rank_of(a, e);
        const __half* w = a.a + (size_t)e * a.R * a.K;
        f4 s[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int run = r0 + wave; run < r1; run += kLoraWaves) {
            const int k = run * 32 + quad * 8;
            const h8 xv = k < a.K ? *reinterpret_cast<const h8*>(x + k) : h8{};
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int r = i * 16 + col;
                const h8 wv = k < a.K && r < rank ? *reinterpret_cast<const h8*>(w + (size_t)r * a.K + k) : h8{};
                s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv, xv, s[i], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) t[i][j] = mine == e ? s[i][j] : t[i][j];
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) part[wave][i][lane] = make_float4(t[i][0], t[i][1], t[i][2], t[i][3]);
    __syncthreads();
    for (int i = wave; i < RT; i += kLoraWaves) {
        float4 s = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < kLoraWaves; ++w) {
            const float4 p = part[w][i][lane];
            s.x += p.x, s.y += p.y, s.z += p.z, s.w += p.w;
        }
        const int r = i * 16 + quad * 4;
        if (mine >= 0 && r < a.R) *reinterpret_cast<float4*>(a.inner + ((size_t)blockIdx.y * a.M + row) * a.R + r) = s;
    }
}

// out = base + scale t B^T: 16 rows x 64 columns a wave.  First operand: rows of B (columns of out), second: t.  Row i of
// operand tile j is column 16 (i / 4) + 4 j + i % 4, so that a lane's four results of the four tiles are 16 columns in a row.
// t goes in as two fp16 terms (together 2^-22 of the row's largest) after a power of two of the row: rounded to one it would
// add an error of the size of the output's own rounding, and a large t would overflow.
template <int RS>  // R in steps of 32
__global__ __launch_bounds__(kLoraWaves* kWave) void lora_outer_kernel(LoraArgs a, int wide) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, col = lane & 15, quad = lane >> 4;
    const int row = blockIdx.x * kRows + col;
    const int mine = own_adapter(a, row);
    const int n0 = (blockIdx.y * kLoraWaves + wave) * 64;
    if (n0 >= a.N) return;
    f4 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    unsigned long long todo = __ballot(mine >= 0 && quad == 0);
    if (todo) {
        float t[RS][8];
        float most = 0.0f;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            const int r = s * 32 + quad * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) t[s][i] = 0.0f;
            if (mine >= 0 && r < a.R) {
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
        // 2^power is the row's largest rounded down to a power of two; NaN and infinities go through as they are
        const int power = most > 0.0f && most < INFINITY ? ilogbf(most) : 0;
        h8 hi[RS], lo[RS];
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = ldexpf(t[s][i], -power);
                hi[s][i] = (_Float16)v;
                lo[s][i] = fabsf(v) < INFINITY ? (_Float16)(v - (float)hi[s][i]) : (_Float16)0.0f;
            }
        while (todo) {
            const int e = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
            todo &= ~__ballot(mine == e);
            const int rank = rank_of(a, e);
            const float scale = a.scales ? a.scales[e] : 1.0f;
            const __half* w = a.b + (size_t)e * a.N * a.R;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + 16 * (col >> 2) + 4 * j + (col & 3);
                f4 s = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int st = 0; st < RS; ++st) {
                    const int r = st * 32 + quad * 8;
                    h8 wv = n < a.N && r < a.R ? *reinterpret_cast<const h8*>(w + (size_t)n * a.R + r) : h8{};
                    if (rank < a.R)  // (the columns of B past the adapter's rank are not its own)
#pragma unroll
                        for (int i = 0; i < 8; ++i) wv[i] = r + i < rank ? wv[i] : (_Float16)0.0f;
                    s = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv, hi[st], s, 0, 0, 0);
                    s = __builtin_amdgcn_mfma_f32_16x16x32_f16(wv, lo[st], s, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[j][i] = mine == e ? scale * ldexpf(s[i], power) : sum[j][i];
            }
        }
    }
    if (row >= a.M || (mine < 0 && a.base == a.out)) return;  // (rows without an adapter stay as they are)
    const int n = n0 + 16 * quad;
    const __half* base = a.base ? a.base + (size_t)row * a.ldb + n : nullptr;
    __half* out = a.out + (size_t)row * a.ldo + n;
    if (wide) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (n + 8 * c >= a.N) continue;
            h8 v = base ? *reinterpret_cast<const h8*>(base + 8 * c) : h8{};
            if (mine >= 0)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (_Float16)((float)v[i] + sum[2 * c + i / 4][i % 4]);
            *reinterpret_cast<h8*>(out + 8 * c) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (n + i >= a.N) continue;
            const __half v = base ? base[i] : __float2half(0.0f);
            out[i] = mine >= 0 ? __float2half(__half2float(v) + sum[i / 4][i % 4]) : v;
        }
    }
}

}  // namespace

int lora_slabs(int M, int K) {
    const int tiles = (M + kRows - 1) / kRows, most = (K + 127) / 128;
    const int want = 2 * cu_count() / tiles;
    return want < 1 ? 1 : want > 32 ? (most < 32 ? most : 32) : want > most ? most : want;
}

size_t lora_workspace_bytes(int M, int K, int R) { return (size_t)lora_slabs(M, K) * M * R * 4; }

hipError_t launch_lora_add(const LoraArgs& args, void* workspace, hipStream_t stream) {
    LoraArgs a = args;
    a.inner = static_cast<float*>(workspace);
    a.slabs = lora_slabs(a.M, a.K);
    const int tiles = (a.M + kRows - 1) / kRows, threads = kLoraWaves * kWave;
    const int wide = a.N % 8 == 0 && a.ldo % 8 == 0 && (a.base == nullptr || a.ldb % 8 == 0);
    const dim3 inner(tiles, a.slabs), outer(tiles, (a.N + 64 * kLoraWaves - 1) / (64 * kLoraWaves));
    const int rt = (a.R + 15) / 16;
    if (rt <= 1) hipLaunchKernelGGL((lora_inner_kernel<1>), inner, dim3(threads), 0, stream, a);
    else if (rt <= 2) hipLaunchKernelGGL((lora_inner_kernel<2>), inner, dim3(threads), 0, stream, a);
    else if (rt <= 4) hipLaunchKernelGGL((lora_inner_kernel<4>), inner, dim3(threads), 0, stream, a);
    else hipLaunchKernelGGL((lora_inner_kernel<8>), inner, dim3(threads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.R <= 32) hipLaunchKernelGGL((lora_outer_kernel<1>), outer, dim3(threads), 0, stream, a, wide);
    else if (a.R <= 64) hipLaunchKernelGGL((lora_outer_kernel<2>), outer, dim3(threads), 0, stream, a, wide);
    else hipLaunchKernelGGL((lora_outer_kernel<4>), outer, dim3(threads), 0, stream, a, wide);
    return hipGetLastError();
}

}  // namespace intscale
