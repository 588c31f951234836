// Attention over packed sequences of different lengths, grouped heads:
//   out[i, h] = sum_j softmax_j(scale * q[i, h] . k[j, h / group]) v[j, h / group],  j < lim(i)
// with lim(i) = i + kv_len - q_len + 1 (the last query row sees every key) or, both ways, kv_len.
//
// One pass over the keys with a running maximum and sum per query row.  The transposed product S^T = K Q^T comes first:
// in its result a lane holds one query row (lane & 31) and half of the keys of the tile, so that the maximum and the sum
// of a row are in-lane operations and one exchange between the wave's halves, and the fp16 probabilities already lie as
// the second operand of O^T = V^T P^T wants them: no trip through LDS between the two products.  V^T comes out of row-major
// V in LDS by the transposing read (a group of 16 lanes turns 4 keys x 16 columns).
//
// Query rows and the query heads of a key head are one axis ("packed rows": row * group + head), so that a tile of 32 packed
// rows a wave is full for single tokens of grouped heads too and the keys are read once for the whole group.
#include "block_common.h"
#include "tile_common.h"

namespace intscale {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) unsigned char* LdsPtr;

constexpr int kKeys = 64;        // keys of a tile
constexpr int kRowsPerWave = 32; // packed rows of a wave
// A row's running maximum is raised only when it would grow by more than this (in powers of two): until then the
// probabilities are larger than 1, at most 2^8, which fp16 holds as exactly as those below 1, and the accumulators need no
// rescaling.
constexpr float kLazyMax = 8.0f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum (sum) of a value and of the one in the other half of the wave (lane ^ 32).
__device__ __forceinline__ float halves_max(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// A sequence of the batch as the kernels see it: lengths and places clamped to the tensors, so that no offset leads outside.
struct Seq {
    int q0, qlen, kvlen;
    long long kv0;
};
__device__ __forceinline__ Seq seq_at(const AttnArgs& a, int s) {
    Seq r;
    r.q0 = min(max(a.q_offsets[s], 0), a.M);
    r.qlen = max(min(max(a.q_offsets[s + 1], 0), a.M) - r.q0, 0);
    const long long start = a.kv_starts ? a.kv_starts[s] : (long long)r.q0;
    const int len = a.kv_lens ? a.kv_lens[s] : r.qlen;
    const bool inside = start >= 0 && start <= a.kv_rows;
    r.kv0 = inside ? start : 0;
    const long long room = inside ? a.kv_rows - start : 0;
    r.kvlen = (int)min((long long)max(min(len, a.max_kv), 0), room);
    return r;
}

// Which sequence the row tile `target` of the batch belongs to (every sequence has whole tiles of `rows` packed rows) and
// which of its tiles it is; seq < 0 past the last one.  Each wave by itself, 64 sequences at a time.
struct RowTile {
    int seq, tile;
};
__device__ __forceinline__ RowTile row_tile(const AttnArgs& a, int target, int rows) {
    const int lane = threadIdx.x & (kWave - 1);
    int before = 0;
    for (int s0 = 0; s0 < a.seqs; s0 += kWave) {
        const int s = s0 + lane;
        int n = 0;
        if (s < a.seqs) {
            const int b = min(max(a.q_offsets[s], 0), a.M), e = min(max(a.q_offsets[s + 1], 0), a.M);
            n = (max(e - b, 0) * a.group + rows - 1) / rows;
        }
        const int upto = lanes_up_to(n, lane);
        const unsigned long long past = __ballot(before + upto > target);
        if (past) {
            const int first = __builtin_ctzll(past);
            const int skipped = before + __builtin_amdgcn_readlane(upto - n, first);
            return RowTile{s0 + first, target - skipped};
        }
        before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return RowTile{-1, 0};
}

// Where 16-byte chunk c of row r of a tile lies in LDS (in chunks from the row's start): rows are a power of two of bytes
// apart, so without it the rows that one read touches would meet in the same banks.
template <int D>
__device__ __forceinline__ int k_chunk(int r, int c) {  // 16 rows, one chunk each
    return D == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_chunk(int r, int c) {  // 4 rows, four chunks each
    return D == 128 ? c ^ ((r & 3) << 2) : c ^ (((r >> 1) & 1) << 2);
}

__device__ __forceinline__ h8 lds_h8(LdsPtr p) { return *(const __attribute__((address_space(3))) h8*)p; }
__device__ __forceinline__ h4 lds_h4_turned(LdsPtr p) {
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
    return __builtin_bit_cast(h4, v);
}

// One workgroup: NW waves of 32 packed rows of one sequence and key head, one chunk of its keys.  Grid: x = key head +
// heads_kv * row tile (the key heads of a row tile go to different XCDs, and with 8 of them one head's keys stay in one
// XCD's L2), y = chunk.  The last row tile of a sequence, which sees the most keys, comes first.
template <int D, int NW>
__global__ __launch_bounds__(NW* kWave) __attribute__((amdgpu_waves_per_eu(2, 2))) void attention_tile_kernel(AttnArgs a) {
    constexpr int kRowBytes = 2 * D, kTileBytes = kKeys * kRowBytes, kLoads = kTileBytes / 1024 / NW;
    constexpr int kSteps = D / 16, kBlocks = D / 32;
    static_assert(kLoads >= 1, "every wave loads a part of a tile");
    extern __shared__ __align__(1024) unsigned char lds[];  // [2][K tile | V tile], [2][NW] words
    const LdsPtr lds_p = (LdsPtr)lds;
    const unsigned lds_base = (unsigned)(uintptr_t)lds_p;
    int* found = reinterpret_cast<int*>(lds + 4 * kTileBytes);

    const int head = blockIdx.x % a.heads_kv;
    const RowTile at = row_tile(a, blockIdx.x / a.heads_kv, NW * kRowsPerWave);
    if (at.seq < 0) return;
    const Seq s = seq_at(a, at.seq);
    const int rows = s.qlen * a.group;  // packed rows of the sequence
    const int tiles = (rows + NW * kRowsPerWave - 1) / (NW * kRowsPerWave);
    const int first = (tiles - 1 - at.tile) * NW * kRowsPerWave;
    const int c0 = blockIdx.y * a.chunk;
    if (c0 > 0 && c0 >= s.kvlen) return;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1), half = lane >> 5;
    // keys seen by packed row p: lim(p); it does not fall with p
    auto limit = [&](int p) { return a.causal ? max(min(p / a.group + s.kvlen - s.qlen + 1, s.kvlen), 0) : s.kvlen; };
    const int wg_most = limit(min(first + NW * kRowsPerWave, rows) - 1), wg_least = limit(first);
    const int w_first = first + wave * kRowsPerWave;
    const int w_least = limit(min(w_first, rows - 1)), w_most = w_first < rows ? limit(min(w_first + kRowsPerWave, rows) - 1) : 0;
    const int p = w_first + (lane & 31);
    const bool mine = p < rows;
    const int lim = mine ? limit(p) : 0;
    const int qrow = s.q0 + (mine ? p / a.group : 0), qhead = head * a.group + (mine ? p % a.group : 0);

    h8 q[kSteps];
    {
        const __half* src = a.q + (size_t)qrow * a.ldq + (size_t)qhead * D + half * 8;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) q[kk] = mine ? *reinterpret_cast<const h8*>(src + kk * 16) : h8{};
    }

    // a tile's rows to LDS: kilobyte i of the tile is wave i / kLoads's, its rows' chunks permuted on the way
    int k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int byte = (wave * kLoads + j) * 1024 + lane * 16, r = byte / kRowBytes, c = byte % kRowBytes / 16;
        k_off[j] = r * (int)(a.ldk * 2) + k_chunk<D>(r, c) * 16;
        v_off[j] = r * (int)(a.ldv * 2) + v_chunk<D>(r, c) * 16;
    }
    const __half* k_head = a.k + (size_t)s.kv0 * a.ldk + (size_t)head * D;
    const __half* v_head = a.v + (size_t)s.kv0 * a.ldv + (size_t)head * D;
    auto fetch = [&](int t, int buf) {
        // rows past the sequence's last read as zero
        const int left = min(s.kvlen - t * kKeys, kKeys);
        const v4i kd = make_desc(k_head + (size_t)t * kKeys * a.ldk, left > 0 ? (size_t)(left - 1) * a.ldk * 2 + kRowBytes : 0);
        const v4i vd = make_desc(v_head + (size_t)t * kKeys * a.ldv, left > 0 ? (size_t)(left - 1) * a.ldv * 2 + kRowBytes : 0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const unsigned to = buf * 2 * kTileBytes + (wave * kLoads + j) * 1024;
            load_to_lds_b128(kd, lds_base, to, k_off[j], 0);
            load_to_lds_b128(vd, lds_base, to + kTileBytes, v_off[j], 0);
        }
    };

    f16v o[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    float top = -INFINITY, sum = 0.0f;  // running maximum of scale * q.k (powers of two), sum over this lane's half of the keys
    const float factor = a.scale * 1.44269504088896340736f;

    const int t0 = c0 / kKeys, t1 = (min(c0 + a.chunk, wg_most) + kKeys - 1) / kKeys;
    if (t0 < t1) fetch(t0, 0);
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1, buf ^ 1);
        const LdsPtr kt = lds_p + buf * 2 * kTileBytes, vt = kt + kTileBytes;
        // Keys that some rows see and others do not: a product with a probability of zero still turns an infinity or a NaN among
        // their values into a NaN, so such a tile is looked through first.
        bool odd_values = false;
        if (min((t + 1) * kKeys, s.kvlen) > wg_least) {
            bool odd = false;
#pragma unroll
            for (int i = threadIdx.x * 16; i < kTileBytes; i += NW * kWave * 16) {
                const v4i w = *(const __attribute__((address_space(3))) v4i*)(vt + i);
                auto is_odd = [](unsigned x) { return (x & 0x7C00u) == 0x7C00u || (x & 0x7C000000u) == 0x7C000000u; };
                odd = odd || is_odd(w[0]) || is_odd(w[1]) || is_odd(w[2]) || is_odd(w[3]);
            }
            const bool any_odd = __any(odd);
            if (lane == 0) found[buf * NW + wave] = any_odd;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) odd_values = odd_values || found[buf * NW + w];
        }
        if (t * kKeys >= w_most) continue;  // (wave-uniform: no row of this wave sees the tile)

        f16v sc[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[m][i] = 0.0f;
            const int r = m * 32 + (lane & 31);
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk)
                sc[m] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_h8(kt + r * kRowBytes + k_chunk<D>(r, 2 * kk + half) * 16), q[kk],
                                                               sc[m], 0, 0, 0);
        }
        const int seen = lim - t * kKeys - 4 * half;  // element i of block m: key m * 32 + 8 * (i / 4) + i % 4 of this half
        if ((t + 1) * kKeys > w_least) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[m][i] = m * 32 + 8 * (i / 4) + i % 4 < seen ? sc[m][i] : -INFINITY;
        }
        float most = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, sc[i / 16][i % 16]);
        most = halves_max(most) * factor;
        if (__any(most > top + kLazyMax)) {  // (the first tile too: top is -inf)
            const float now = fmaxf(top, most);
            const float shrink = now == -INFINITY ? 1.0f : exp2_fast(top - now);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= shrink;
            sum *= shrink;
            top = now;
        }
        const float less = top == -INFINITY ? 0.0f : top;
        h8 pr[4];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float p0 = exp2_fast(fmaf(sc[i / 16][i % 16], factor, -less)), p1 = exp2_fast(fmaf(sc[i / 16][i % 16 + 1], factor, -less));
            sum += p0 + p1;
            // (to the nearest, half a step of 2^-11 each: towards zero would leave every output too small)
            pr[i / 8][i % 8] = (_Float16)p0;
            pr[i / 8][i % 8 + 1] = (_Float16)p1;
        }
        // V^T's operand: lane's column 32 b + (lane & 31), keys 16 s + 4 half + 0..3 and those 8 further on, as the probabilities lie
        const int vr = 4 * half + (lane & 15) / 4, vc = (lane >> 4 & 1) * 32 + (lane & 3) * 8;  // row, byte column
        auto values = [&](int step, int b) {
            const int r = step * 16 + vr, c = b * 64 + vc;
            const h4 x = lds_h4_turned(vt + r * kRowBytes + v_chunk<D>(r, c >> 4) * 16 + (c & 15));
            const h4 y = lds_h4_turned(vt + (r + 8) * kRowBytes + v_chunk<D>(r + 8, c >> 4) * 16 + (c & 15));
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if (!odd_values) {
#pragma unroll
            for (int step = 0; step < 4; ++step)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values(step, b), pr[step], o[b], 0, 0, 0);
        } else {  // key by key, and only into the rows that see it
#pragma unroll 1
            for (int key = 0; key < kKeys; ++key) {
                const int step = key / 16, h = key / 4 & 1, e = (key / 8 & 1) * 4 + key % 4;
                h8 pk = step == 0 ? pr[0] : step == 1 ? pr[1] : step == 2 ? pr[2] : pr[3];
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    h8 v = values(step, b);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (j != e || h != half) v[j] = (_Float16)0.0f;
                        if (j != e || h != half) pk[j] = (_Float16)0.0f;
                    }
                    f16v one;
#pragma unroll
                    for (int i = 0; i < 16; ++i) one[i] = 0.0f;
                    one = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pk, one, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][i] = t * kKeys + key < lim ? o[b][i] + one[i] : o[b][i];
                }
            }
        }
    }

    sum = halves_sum(sum);
    if (s.kvlen <= a.chunk) {
        // a row that sees no key is zero; one whose scores are all -inf (or that saw a NaN) is NaN, as the formula's 0 / 0
        const float inv = 1.0f / sum;
        __half* dst = a.out + (size_t)qrow * a.ldo + (size_t)qhead * D;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                h4 x, y;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = lim > 0 ? (_Float16)(o[b][i + j] * inv) : (_Float16)0.0f;
                    y[j] = lim > 0 ? (_Float16)(o[b][i + 4 + j] * inv) : (_Float16)0.0f;
                }
                // columns 8 (i / 4) + 4 half + 0..3 and those 8 further on: after the exchange 8 columns in a row a lane
                const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
                const auto s0 = __builtin_amdgcn_permlane32_swap(xu.x, yu.x, false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(xu.y, yu.y, false, false);
                if (mine) *reinterpret_cast<uint4*>(dst + b * 32 + 2 * i + 8 * half) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
            }
    } else if (mine) {
        const size_t heads = (size_t)a.heads_kv * a.group, row = ((size_t)blockIdx.y * a.M + qrow) * heads + qhead;
        float* dst = a.part_o + row * D;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(dst + b * 32 + 2 * i + 4 * half) = make_float4(o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]);
        if (half == 0) a.part_ml[row] = make_float2(top, sum);
    }
}

// The chunks' partial results of a row and head, joined in the chunks' order: one wave each.
template <int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a) {
    const int lane = threadIdx.x & (kWave - 1);
    const int heads = a.heads_kv * a.group;
    const long long at = (long long)blockIdx.x * 4 + threadIdx.x / kWave;
    if (at >= (long long)a.M * heads) return;
    const int row = (int)(at / heads), head = (int)(at - (long long)row * heads);
    // the sequence of the row: the last one that starts at or before it and is not empty
    int seq = -1;
    for (int s0 = 0; s0 < a.seqs; s0 += kWave) {
        const int s = s0 + lane;
        const bool in = s < a.seqs && a.q_offsets[s] <= row && a.q_offsets[s + 1] > row;
        const unsigned long long found = __ballot(in);
        if (found) {
            seq = s0 + __builtin_ctzll(found);
            break;
        }
    }
    if (seq < 0) return;
    const Seq s = seq_at(a, seq);
    if (s.kvlen <= a.chunk) return;  // (written already)
    const int chunks = (s.kvlen + a.chunk - 1) / a.chunk;
    const size_t stride = (size_t)a.M * heads;
    float top = -INFINITY;
    for (int c = 0; c < chunks; ++c) top = fmaxf(top, a.part_ml[c * stride + at].x);
    const float less = top == -INFINITY ? 0.0f : top;
    constexpr int E = D / kWave;
    float acc[E] = {}, sum = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        const float2 ml = a.part_ml[c * stride + at];
        const float w = exp2_fast(ml.x - less);
        sum = fmaf(ml.y, w, sum);
        const float* src = a.part_o + (c * stride + at) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(src[e], w, acc[e]);
    }
    const int lim = a.causal ? row - s.q0 + s.kvlen - s.qlen + 1 : s.kvlen;
    __half* dst = a.out + (size_t)row * a.ldo + (size_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = __float2half(lim > 0 ? acc[e] / sum : 0.0f);
}

constexpr int kTileWaves = 8;

template <int D>
hipError_t launch_tiles(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
    constexpr int bytes = 4 * kKeys * 2 * D + 2 * kTileWaves * 4;
    static LdsLimit limit;
    const auto kernel = attention_tile_kernel<D, kTileWaves>;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    const long long tiles = (long long)a.M * a.group / (kTileWaves * kRowsPerWave) + a.seqs;  // no fewer than the sequences' whole tiles
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles * a.heads_kv), p.chunks), dim3(kTileWaves * kWave), bytes, stream, a);
    const hipError_t launched = hipGetLastError();
    if (launched != hipSuccess || p.chunks == 1) return launched;
    const long long waves = (long long)a.M * a.heads_kv * a.group;
    hipLaunchKernelGGL((attention_join_kernel<D>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

}  // namespace

// Keys are cut into chunks where the row tiles alone would leave most of the units idle.
AttnPlan attention_plan(int M, int seqs, int max_q, int max_kv, int heads_kv, int group, int head_dim) {
    const int whole = (int)ceil_div(max_kv, kKeys) * kKeys;
    AttnPlan p{whole > 0 ? whole : kKeys, 1};
    const long long rows = kTileWaves * kRowsPerWave;
    const long long tiles = ((long long)M * group / rows + seqs) * heads_kv;
    const long long want = 2LL * cu_count() / tiles;
    if (want > 1) {
        const long long chunk = ceil_div(ceil_div(max_kv, want), kKeys) * kKeys;
        p.chunk = (int)(chunk < 256 ? 256 : chunk);
        p.chunks = (int)ceil_div(max_kv, p.chunk);
        if (p.chunks < 1) p.chunks = 1;
    }
    return p;
}

size_t attention_workspace_bytes(const AttnPlan& p, int M, int heads_q, int head_dim) {
    return p.chunks == 1 ? 0 : (size_t)p.chunks * M * heads_q * (head_dim * 4 + 8);
}

hipError_t launch_attention(const AttnArgs& args, const AttnPlan& p, int head_dim, void* workspace, hipStream_t stream) {
    AttnArgs a = args;
    a.chunk = p.chunk;
    if (p.chunks > 1) {
        a.part_o = static_cast<float*>(workspace);
        a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)p.chunks * a.M * a.heads_kv * a.group * head_dim);
    }
    return head_dim == 128 ? launch_tiles<128>(a, p, stream) : launch_tiles<64>(a, p, stream);
}

}  // namespace intscale
