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
//
// Two kernels: row tiles (prompts and chunks of them), bound by the matrix instructions, the exponentials beside them and the clock that
// both leave (8192 rows, 64 heads of 128: 1090 to 1155 us from box to box, 0.95 to 1.01 PFLOP/s; counters of that call alone: matrix pipe
// busy 54 % of the cycles, vector instructions 50 %, LDS 27 %, no bank conflicts, the clock at 1.6 GHz on that box; of heads of 64, both
// ways, 27 %, 51 %, 14 %: vector instructions, twice the exponentials a product); few rows (single tokens), bound by memory (64 requests,
// 1.07 GB: 171 us, 6.2 TB/s; a plain streaming read 6.4; drafts of 5 tokens of 32 requests over 4000 keys 90 us at a group of 4, 5.8 TB/s,
// 115 at a group of 8, whose instance of 64 rows spills 90 registers).  Not kept for row tiles: the next tile's scores under this tile's
// probabilities (24 to 84 registers spilled at heads of 128, 1450 us and more; no gain at heads of 64), wave priorities (no change).
#include <math.h>

#include <algorithm>

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
// A row's running maximum is raised only when it would grow by more than kLazyMax (in powers of two): until then the accumulators need
// no rescaling.  The probabilities, fp16 for their product with V, are held times 2^kUp, the largest so far between 2^7 and 2^15: below
// fp16's normal numbers half a step is then 2^-32 of it.  In a long tail beside one dominant key each key may be 2^-20 of that and less
// (without the factor a tail of 131072 equal keys with 2 % of the weight came out 7 % off).  The factor is in the sum as well.
constexpr float kLazyMax = 8.0f, kUp = 7.0f;
// A maximum past this (in powers of two) is subtracted from the scores by itself, before anything is added: the fused multiply-add with
// the maximum, which is rounded, would leave what that rounding took (at 2^28 some powers of two, and the sum overflows or vanishes).
constexpr float kFarMax = 4096.0f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// x * y, rounded before anything else is done with it.
__device__ __forceinline__ float rounded_product(float x, float y) {
    float p = x * y;
    asm volatile("" : "+v"(p));
    return p;
}

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

// Which sequence the row tile `target` of the batch belongs to (every sequence of more than few_rows packed rows has whole tiles of
// `rows`) and which of its tiles it is; seq < 0 past the last one.  Each wave by itself.  Up to 64 sequences the longest come
// first, or the last workgroups to start would be the longest ones (twelve prompts of 17 to 2048 rows: 177 us in the batch's order,
// 172 so); one sequence after the other, since their keys and values stay in the caches that way.
struct RowTile {
    int seq, tile;
    Seq s;
};
__device__ __forceinline__ int row_tiles(const AttnArgs& a, const Seq& s, int rows) {
    const int packed = s.qlen * a.group;
    return packed > a.few_rows ? (packed + rows - 1) / rows : 0;
}
// The sequence that lane `at` has, to all lanes.
__device__ __forceinline__ Seq seq_of_lane(const Seq& mine, int at) {
    Seq s;
    s.q0 = __builtin_amdgcn_readlane(mine.q0, at);
    s.qlen = __builtin_amdgcn_readlane(mine.qlen, at);
    s.kvlen = __builtin_amdgcn_readlane(mine.kvlen, at);
    const unsigned lo = __builtin_amdgcn_readlane((int)mine.kv0, at), hi = __builtin_amdgcn_readlane((int)(mine.kv0 >> 32), at);
    s.kv0 = (long long)(((unsigned long long)hi << 32) | lo);
    return s;
}
__device__ __forceinline__ RowTile row_tile(const AttnArgs& a, int target, int rows) {
    const int lane = threadIdx.x & (kWave - 1);
    const Seq none{0, 0, 0, 0};
    if (a.seqs <= kWave) {
        const Seq mine = lane < a.seqs ? seq_at(a, lane) : none;
        const int n = row_tiles(a, mine, rows);
        int before = 0;
        for (int s = 0; s < a.seqs; ++s) {
            const int other = __builtin_amdgcn_readlane(n, s);
            before += other > n || (other == n && s < lane) ? other : 0;
        }
        const unsigned long long here = __ballot(target >= before && target < before + n);
        if (here == 0) return RowTile{-1, 0, none};
        const int at = __builtin_ctzll(here);
        return RowTile{at, target - __builtin_amdgcn_readlane(before, at), seq_of_lane(mine, at)};
    }
    // More of them: sequence s has the numbers from q_offsets[s] * group / rows + s on, as many as its rows can need and no more in all than
    // the grid has, so that a search finds it in as many steps as the number of sequences has bits (a walk over all of them in each of a
    // grid's workgroups would take their square).
    auto begin = [&](int s) { return (int)((long long)min(max(a.q_offsets[s], 0), a.M) * a.group / rows) + s; };
    int low = 0, past = a.seqs;
    while (past - low > 1) {
        const int mid = low + (past - low) / 2;
        (begin(mid) <= target ? low : past) = mid;
    }
    const Seq s = seq_at(a, low);
    const int tile = target - begin(low);
    if (tile >= 0 && tile < row_tiles(a, s, rows)) return RowTile{low, tile, s};
    return RowTile{-1, 0, none};
}

// Maximum (sum) of a value over the four lanes of equal lane & 15.
__device__ __forceinline__ float quads_max(float v) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return halves_max(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}
__device__ __forceinline__ float quads_sum(float v) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return halves_sum(__uint_as_float(s[0]) + __uint_as_float(s[1]));
}

// Sets the infinities and NaN among eight fp16 values in LDS to zero; whether there were any.
__device__ __forceinline__ bool take_out_odd_values(LdsPtr p) {
    v4i w = *(const __attribute__((address_space(3))) v4i*)p;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool low = (w[i] & 0x7C00) == 0x7C00, high = (w[i] & 0x7C000000) == 0x7C000000;
        w[i] &= (low ? 0 : 0xFFFF) | (high ? 0 : (int)0xFFFF0000);
        odd = odd || low || high;
    }
    if (odd) *(__attribute__((address_space(3))) v4i*)p = w;
    return odd;
}

// Infinities and NaN among the values: a row's column that sees one is the sum of those it sees, however small their probabilities are (a
// product with one that is rounded to zero, or a factor that vanishes later, would make NaN of an infinity).  The matrix instructions
// leave such columns not finite, or the values were taken out of a tile that not every row sees; either is found once at the end of a
// wave's keys, and the values are looked up then.
__device__ __forceinline__ bool is_odd(float x) { return !(fabsf(x) < INFINITY); }
// f * x, an infinity or a NaN as it is.
__device__ __forceinline__ float times_unless_odd(float f, float x) { return is_odd(x) ? x : f * x; }

// Keys `key` to `end` of a wave that looks such values up: each(key) for the keys of a tile that has one in the head's columns.
template <int D, class Each>
__device__ __forceinline__ void odd_tile(const __half* v_head, long long ldv, int key, int end, Each each) {
    bool odd = false;
#pragma unroll 1
    for (int i = threadIdx.x & (kWave - 1); i < (end - key) * (D / 8); i += kWave) {
        const v4i w = *reinterpret_cast<const v4i*>(v_head + (size_t)(key + i / (D / 8)) * ldv + i % (D / 8) * 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) odd = odd || (w[j] & 0x7C00) == 0x7C00 || (w[j] & 0x7C000000) == 0x7C000000;
    }
    if (!__any(odd)) return;
#pragma unroll 1
    for (; key < end; ++key) each(key);
}
// What such a value x of a key that the row sees comes to: itself, or the formula's 0 * x where the score is -inf.
template <int D>
__device__ __forceinline__ bool score_is_gone(const __half* q_row, const __half* k_row) {
    float score = 0.0f;
#pragma unroll 1
    for (int i = 0; i < D; ++i) score = fmaf(__half2float(q_row[i]), __half2float(k_row[i]), score);
    return !(score > -INFINITY);
}
__device__ __forceinline__ float odd_value(float x, bool gone) { return !is_odd(x) ? 0.0f : gone ? NAN : x; }

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
// XCD's L2), y = chunk.  The last row tile of a sequence, which sees the most keys, comes first.  (All sequences' last tiles before
// anybody's others: 84 us instead of 72 for five sequences both ways, 4 % more for a prompt of 8192.)  Four waves, two workgroups a unit
// (heads of 64: three): with eight waves, whose barrier holds all of a unit's, a prompt of 8192 rows takes 1 % less, five sequences both ways
// 74 us instead of 61, a chunk of 300 rows beside 24 requests 119 instead of 106.
template <int D, int NW>
__global__ __launch_bounds__(NW* kWave) __attribute__((amdgpu_waves_per_eu(2))) void attention_tile_kernel(AttnArgs a) {
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
    const Seq s = at.s;
    const int rows = s.qlen * a.group;  // packed rows of the sequence
    const int tiles = (rows + NW * kRowsPerWave - 1) / (NW * kRowsPerWave);
    const int first = (tiles - 1 - at.tile) * NW * kRowsPerWave;
    const int c0 = blockIdx.y * a.tile_chunk;
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
    float less = 0.0f;                  // what the exponents are brought down by
    bool far = false;                   // a row's maximum is past kFarMax
    bool taken_out = false;             // infinities or NaN were taken out of a tile
    const float factor = a.scale * 1.44269504088896340736f;

    const int t0 = c0 / kKeys, t1 = (min(c0 + a.tile_chunk, wg_most) + kKeys - 1) / kKeys;
    if (t0 < t1) fetch(t0, 0);
    h8 q[kSteps];
    {
        const __half* src = a.q + (size_t)qrow * a.ldq + (size_t)qhead * D + half * 8;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) q[kk] = mine ? *reinterpret_cast<const h8*>(src + kk * 16) : h8{};
        // Used here, so that they are waited for here: waited for at their first use in the loop, every tile would wait for the
        // next one's loads as well.
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(q[kk]));
    }
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1, buf ^ 1);
        const LdsPtr kt = lds_p + buf * 2 * kTileBytes, vt = kt + kTileBytes;
        // Keys that some rows see and others do not: a product with a probability of zero still turns an infinity or a NaN among
        // their values into a NaN.  Such a tile is looked through first, and those values are taken out; the rows that see them get
        // them at the end.
        if (min((t + 1) * kKeys, s.kvlen) > wg_least) {
            bool odd = false;
#pragma unroll
            for (int i = threadIdx.x * 16; i < kTileBytes; i += NW * kWave * 16) odd = take_out_odd_values(vt + i) || odd;
            const bool any_odd = __any(odd);
            if (lane == 0) found[(t & 1) * NW + wave] = any_odd;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) taken_out = taken_out || found[(t & 1) * NW + w];
        }
        if (t * kKeys >= w_most) continue;  // (wave-uniform: no row of this wave sees the tile)

        f16v sc[2];
#pragma unroll
        for (int i = 0; i < 32; ++i) sc[i / 16][i % 16] = 0.0f;
        // (the two blocks of 32 keys in turn: two products in a row into the same accumulators would wait for each other)
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const int r = m * 32 + (lane & 31);
                sc[m] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds_h8(kt + r * kRowBytes + k_chunk<D>(r, 2 * kk + half) * 16), q[kk], sc[m], 0, 0, 0);
            }
        // six (four) reads ahead of the products: two at a time would leave each pair of products waiting for LDS
        constexpr int kAhead = D == 128 ? 6 : 4;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < (2 * kSteps - kAhead) / 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        const int seen = lim - t * kKeys - 4 * half;  // element i of block m: key m * 32 + 8 * (i / 4) + i % 4 of this half
        if ((t + 1) * kKeys > w_least) {
            asm volatile("");  // (a branch: as selects in every tile these would be a sixth of its instructions)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[m][i] = m * 32 + 8 * (i / 4) + i % 4 < seen ? sc[m][i] : -INFINITY;
        }
        float most = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, sc[i / 16][i % 16]);
        most = rounded_product(halves_max(most), factor);
        if (__any(most > top + kLazyMax)) {  // (the first tile too: top is -inf)
            const float now = fmaxf(top, most);
            const float shrink = now == -INFINITY ? 1.0f : exp2_fast(top - now);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= shrink;
            sum *= shrink;
            top = now;
            far = __any(fabsf(top) > kFarMax && top != -INFINITY);
            less = top == -INFINITY ? 0.0f : far ? -kUp : top - kUp;
        }
        float times = factor;
        if (far) {
#pragma unroll
            for (int i = 0; i < 32; ++i) sc[i / 16][i % 16] = rounded_product(sc[i / 16][i % 16], factor) - (top == -INFINITY ? 0.0f : top);
            times = 1.0f;
        }
        h8 pr[4];
        float part = 0.0f;  // (a sum of the tile's own: next to the running one the terms of a long tail would lose their bits one by one)
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float p0 = exp2_fast(fmaf(sc[i / 16][i % 16], times, -less)), p1 = exp2_fast(fmaf(sc[i / 16][i % 16 + 1], times, -less));
            part += p0 + p1;
            // (to the nearest, half a step of 2^-11 each: towards zero would leave every output too small)
            pr[i / 8][i % 8] = (_Float16)p0;
            pr[i / 8][i % 8 + 1] = (_Float16)p1;
        }
        sum += part;
        // V^T's operand: lane's column 32 b + (lane & 31), keys 16 s + 4 half + 0..3 and those 8 further on, as the probabilities lie
        const int vr = 4 * half + (lane & 15) / 4, vc = (lane >> 4 & 1) * 32 + (lane & 3) * 8;  // row, byte column
        auto values = [&](int step, int b) {
            const int r = step * 16 + vr, c = b * 64 + vc;
            const h4 x = lds_h4_turned(vt + r * kRowBytes + v_chunk<D>(r, c >> 4) * 16 + (c & 15));
            const h4 y = lds_h4_turned(vt + (r + 8) * kRowBytes + v_chunk<D>(r + 8, c >> 4) * 16 + (c & 15));
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int step = 0; step < 4; ++step)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values(step, b), pr[step], o[b], 0, 0, 0);
    }

    sum = halves_sum(sum);
    float none = 0.0f;  // 0, or NaN
#pragma unroll
    for (int i = 0; i < 16 * kBlocks; ++i) none = fmaf(0.0f, o[i / 16][i % 16], none);
    if (__builtin_expect(__any((taken_out || is_odd(none)) && mine && !is_odd(sum)), 0)) {
        const __half* q_row = a.q + (size_t)qrow * a.ldq + (size_t)qhead * D;
#pragma unroll
        for (int i = 0; i < 16 * kBlocks; ++i) o[i / 16][i % 16] = is_odd(o[i / 16][i % 16]) ? 0.0f : o[i / 16][i % 16];
#pragma unroll 1
        for (int t = t0; t < t1 && t * kKeys < w_most; ++t)
            odd_tile<D>(v_head, a.ldv, t * kKeys, min((t + 1) * kKeys, w_most), [&](int key) {
                if (key >= lim) return;
                const bool gone = score_is_gone<D>(q_row, k_head + (size_t)key * a.ldk);
                const __half* src = v_head + (size_t)key * a.ldv + 4 * half;
#pragma unroll
                for (int i = 0; i < 16 * kBlocks; i += 4) {  // columns as below
                    const h4 v = *reinterpret_cast<const h4*>(src + 2 * i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i / 16][i % 16 + j] += odd_value((float)v[j], gone);
                }
            });
    }
    if (s.kvlen <= a.tile_chunk) {
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

// ---- few rows
// Sequences of at most kFewRows packed rows (single tokens; the drafts and short chunks of a step): bound by the reading of the
// keys and values.  Each of a workgroup's waves walks tiles of 32 keys of its own (every NW-th of the chunk's) with a stage of LDS
// of its own, so that no wave waits for another before the end, where their partial results meet in LDS.  A stage holds one tile
// of K and one of V: the next K is on its way while the probabilities and the product with V are computed, the next V during the
// next scores.  The 16-row forms of the matrix instructions, RB times: a group of 4 or 8 heads wastes less of them than of the
// 32-row ones.
// As load_to_lds_b128, for bytes that are read once: marked non-temporal they do not push each other through the caches (a decode
// step of 64 requests, 1.07 GB of keys and values: 198 us without the mark, 176 us with it when it came in; 171 now, 6.2 TB/s).
__device__ __forceinline__ void stream_to_lds_b128(v4i desc, unsigned lds_base, unsigned lds_offset, int voffset) {
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen nt lds"
                 :
                 : "s"(lds_base), "s"(lds_offset), "v"(voffset), "s"(desc)
                 : "memory", "scc");
}
constexpr int kFewKeys = 32;
constexpr int kFewRows = 64;
constexpr int few_waves(int rb) { return rb <= 2 ? 8 : 4; }  // (the partial results of 64 rows and eight waves would not fit LDS)

template <int D>
__device__ __forceinline__ int few_v_chunk(int r, int c) {  // 8 rows, two chunks each
    return D == 128 ? c ^ ((r & 7) << 1) : c ^ (((r >> 1) & 3) << 1);
}

// How the tiles of all these sequences are dealt out: numbered from sequence to sequence, every workgroup (and key head) takes the
// next `per` of them, so that ragged lengths leave nobody idle.  A workgroup's run may end one sequence, hold several whole and begin
// another; a sequence that lies in one run is finished there, the pieces of the others go to the workspace.
// Beginning and ending a sequence costs a workgroup about as much as kPiece of its tiles; every sequence counts so many more, in front
// of its own, so that a run of short ones is no longer than a piece of a long one.
constexpr int kPiece = 6;
struct Deal {
    int per;               // numbers of a workgroup
    int seq, tiles, begin; // the sequence (seqs: there is none), its tiles, the first number of it
    Seq s;
};
__device__ __forceinline__ int few_tiles(const AttnArgs& a, const Seq& s) {
    const int rows = s.qlen * a.group;
    return rows == 0 || rows > a.few_rows ? 0 : max((s.kvlen + kFewKeys - 1) / kFewKeys, 1);  // (rows without keys are written, too)
}
// By a wave: the sequence that holds the first number of `slot`.
__device__ __forceinline__ Deal few_deal(const AttnArgs& a, int slot) {
    const int lane = threadIdx.x & (kWave - 1);
    const Seq none{0, 0, 0, 0};
    const Seq mine0 = lane < a.seqs ? seq_at(a, lane) : none;
    auto numbers = [&](const Seq& s) {
        const int n = few_tiles(a, s);
        return n > 0 ? n + kPiece : 0;
    };
    int total = __builtin_amdgcn_readlane(lanes_up_to(numbers(mine0), lane), kWave - 1);
    for (int s0 = kWave; s0 < a.seqs; s0 += kWave)
        total += __builtin_amdgcn_readlane(lanes_up_to(s0 + lane < a.seqs ? numbers(seq_at(a, s0 + lane)) : 0, lane), kWave - 1);
    Deal d;
    d.per = max((total + a.slots - 1) / a.slots, a.least_tiles);
    const long long want = (long long)slot * d.per;
    int before = 0;
    for (int s0 = 0; s0 < a.seqs; s0 += kWave) {
        const Seq mine = s0 == 0 ? mine0 : s0 + lane < a.seqs ? seq_at(a, s0 + lane) : none;
        const int n = numbers(mine), upto = lanes_up_to(n, lane);
        const unsigned long long hit = __ballot(before + upto > want);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            d.seq = s0 + at;
            d.tiles = max(__builtin_amdgcn_readlane(n, at) - kPiece, 0);
            d.begin = before + __builtin_amdgcn_readlane(upto - n, at);
            d.s = seq_of_lane(mine, at);
            return d;
        }
        before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    d.seq = a.seqs, d.tiles = 0, d.begin = before, d.s = none;
    return d;
}
// By a wave: the next sequence from `seq` on that this kernel has (seqs: there is none), with its tiles.
__device__ __forceinline__ int few_next(const AttnArgs& a, int seq, Seq* s, int* tiles) {
    const int lane = threadIdx.x & (kWave - 1);
    for (; seq < a.seqs; seq += kWave) {
        const Seq mine = seq + lane < a.seqs ? seq_at(a, seq + lane) : Seq{0, 0, 0, 0};
        const int n = few_tiles(a, mine);
        const unsigned long long some = __ballot(n > 0);
        if (some) {
            const int at = __builtin_ctzll(some);
            *s = seq_of_lane(mine, at);
            *tiles = __builtin_amdgcn_readlane(n, at);
            return seq + at;
        }
    }
    return a.seqs;
}
// Where the piece of a sequence that begins in a run's middle (first: at the sequence's beginning) lies in the workspace, in rows.
__device__ __forceinline__ size_t piece_at(const AttnArgs& a, int slot, bool first, int head) {
    return (((size_t)slot * 2 + first) * a.heads_kv + head) * a.few_rows;
}

template <int D, int RB, int NW>
__global__ __launch_bounds__(NW* kWave) __attribute__((amdgpu_waves_per_eu(RB * D > 256 ? 1 : 2, 2))) void attention_few_kernel(AttnArgs a) {
    constexpr int kRowBytes = 2 * D, kTileBytes = kFewKeys * kRowBytes, kLoads = kTileBytes / 1024;
    constexpr int kSteps = D / 32, kBlocks = D / 16;
    extern __shared__ __align__(1024) unsigned char lds[];  // [NW][K tile | V tile]; at a piece's end [NW][RB * 16][D] partial results
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4;
    const LdsPtr kt = (LdsPtr)lds + wave * 2 * kTileBytes, vt = kt + kTileBytes;
    const unsigned kt_base = (unsigned)(uintptr_t)(LdsPtr)lds + wave * 2 * kTileBytes;
    float* part = reinterpret_cast<float*>(lds);                          // [NW][RB * 16][D], columns rotated by the row
    float2* ml = reinterpret_cast<float2*>(lds + NW * RB * 16 * D * 4);   // [NW][RB * 16]

    // (heads side by side: with 8 or 32 of them the workgroups i, i + 8, ... of an XCD read the same heads' columns; the heads of a run
    // on one XCD instead take 183 us where this takes 176, 1.07 GB)
    const int slot = blockIdx.x / a.heads_kv, head = blockIdx.x % a.heads_kv;
    const Deal deal = few_deal(a, slot);
    int seq = deal.seq, tiles = deal.tiles, begin = deal.begin, at = slot * deal.per;
    const int end = at + deal.per;
    Seq s = deal.s;

    int k_off[kLoads], v_off[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int byte = j * 1024 + lane * 16, r = byte / kRowBytes, c = byte % kRowBytes / 16;
        k_off[j] = r * (int)(a.ldk * 2) + k_chunk<D>(r, c) * 16;
        v_off[j] = r * (int)(a.ldv * 2) + few_v_chunk<D>(r, c) * 16;
    }
    const float factor = a.scale * 1.44269504088896340736f;

    while (seq < a.seqs && at < end) {
    const int rows = s.qlen * a.group;
    const int t0 = max(at - begin - kPiece, 0), t1 = min(end - begin - kPiece, tiles);
    if (t1 <= t0) break;  // (the run ends in front of the sequence's first tile)
    const bool whole = t0 == 0 && t1 == tiles;

    int lim[RB];
    h8 q[RB][kSteps];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int p = b * 16 + col, row = p / a.group;
        const bool mine = p < rows;
        lim[b] = !mine ? 0 : a.causal ? max(min(row + s.kvlen - s.qlen + 1, s.kvlen), 0) : s.kvlen;
        const __half* src = a.q + (size_t)(s.q0 + (mine ? row : 0)) * a.ldq + (size_t)(head * a.group + (mine ? p - row * a.group : 0)) * D + quad * 8;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) q[b][kk] = mine ? *reinterpret_cast<const h8*>(src + kk * 32) : h8{};
    }
    const int least = a.causal ? max(s.kvlen - s.qlen + 1, 0) : s.kvlen;  // keys that every row sees
    const __half* k_head = a.k + (size_t)s.kv0 * a.ldk + (size_t)head * D;
    const __half* v_head = a.v + (size_t)s.kv0 * a.ldv + (size_t)head * D;
    auto fetch = [&](const __half* base, long long ld, int t, const int (&off)[kLoads], unsigned to) {
        const int left = min(s.kvlen - t * kFewKeys, kFewKeys);  // (rows past the sequence's last read as zero)
        const v4i d = make_desc(base + (size_t)t * kFewKeys * ld, left > 0 ? (size_t)(left - 1) * ld * 2 + kRowBytes : 0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) stream_to_lds_b128(d, to, j * 1024, off[j]);
    };

    v4f o[RB][kBlocks];
    float top[RB], sum[RB];
    bool far[RB], taken_out = false;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        top[b] = -INFINITY, sum[b] = 0.0f, far[b] = false;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) o[b][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    int t = t0 + wave;
    if (t < t1) {
        fetch(k_head, a.ldk, t, k_off, kt_base);
        fetch(v_head, a.ldv, t, v_off, kt_base + kTileBytes);
    }
    // (used here to be waited for here: at their first use in the loop, K would wait for V as well)
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) asm volatile("" : "+v"(q[b][kk]));
    for (; t < t1; t += NW) {
        const bool more = t + NW < t1;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");  // K is here, V may be on its way
        v4f sc[RB][2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int b = 0; b < RB; ++b) sc[b][m] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            const int r = m * 16 + col;
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
                const h8 kv = lds_h8(kt + r * kRowBytes + k_chunk<D>(r, 4 * kk + quad) * 16);
#pragma unroll
                for (int b = 0; b < RB; ++b) sc[b][m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, q[b][kk], sc[b][m], 0, 0, 0);
            }
        }
        // (the next tile's loads write where this one was read: the reads have to be over)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) fetch(k_head, a.ldk, t + NW, k_off, kt_base);
        h8 pr[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int seen = lim[b] - t * kFewKeys - 4 * quad;  // element i of block m: key 16 m + 4 quad + i
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = sc[b][i / 4][i % 4];
            if ((t + 1) * kFewKeys > least) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 16 * (i / 4) + i % 4 < seen ? x[i] : -INFINITY;
            }
            float most = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            most = rounded_product(quads_max(most), factor);
            if (__any(most > top[b] + kLazyMax)) {
                const float now = fmaxf(top[b], most);
                const float shrink = now == -INFINITY ? 1.0f : exp2_fast(top[b] - now);
#pragma unroll
                for (int i = 0; i < kBlocks; ++i) o[b][i] *= shrink;
                sum[b] *= shrink;
                top[b] = now;
                far[b] = __any(fabsf(now) > kFarMax && now != -INFINITY);
            }
            float times = factor, less = top[b] == -INFINITY ? 0.0f : top[b] - kUp, part = 0.0f;
            if (far[b]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = rounded_product(x[i], factor) - top[b];
                times = 1.0f, less = -kUp;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = exp2_fast(fmaf(x[i], times, -less));
                part += p;
                pr[b][i] = (_Float16)p;
            }
            sum[b] += part;
        }
        if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (min((t + 1) * kFewKeys, s.kvlen) > least) {  // (keys that only some rows see, as in the kernel above)
            bool odd = false;
#pragma unroll
            for (int i = 0; i < kTileBytes; i += 1024) odd = take_out_odd_values(vt + i + lane * 16) || odd;
            taken_out = taken_out || __any(odd);
        }
        auto values = [&](int i) {  // V^T: column 16 i + (lane & 15), keys 4 quad + 0..3 and those 16 further on
            const int r = 4 * quad + (col >> 2), c = 2 * i + (col >> 1 & 1);
            const h4 x = lds_h4_turned(vt + r * kRowBytes + few_v_chunk<D>(r, c) * 16 + (col & 1) * 8);
            const h4 y = lds_h4_turned(vt + (r + 16) * kRowBytes + few_v_chunk<D>(r + 16, c) * 16 + (col & 1) * 8);
            return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        };
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const h8 v = values(i);
#pragma unroll
            for (int b = 0; b < RB; ++b) o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pr[b], o[b][i], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) fetch(v_head, a.ldv, t + NW, v_off, kt_base + kTileBytes);
    }

    bool odd = false;  // infinities and NaN among the values, as in the kernel above
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        sum[b] = quads_sum(sum[b]);
        float none = 0.0f;  // 0, or NaN
#pragma unroll
        for (int i = 0; i < 4 * kBlocks; ++i) none = fmaf(0.0f, o[b][i / 4][i % 4], none);
        odd = odd || ((taken_out || is_odd(none)) && lim[b] > 0 && !is_odd(sum[b]));
    }
    if (__builtin_expect(__any(odd), 0)) {
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = 0; i < 4 * kBlocks; ++i) o[b][i / 4][i % 4] = is_odd(o[b][i / 4][i % 4]) ? 0.0f : o[b][i / 4][i % 4];
#pragma unroll 1
        for (t = t0 + wave; t < t1; t += NW)
            odd_tile<D>(v_head, a.ldv, t * kFewKeys, min((t + 1) * kFewKeys, s.kvlen), [&](int key) {
                const __half* src = v_head + (size_t)key * a.ldv + 4 * quad;
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const int p = b * 16 + col, row = p / a.group;
                    if (key >= lim[b]) continue;
                    const bool gone = score_is_gone<D>(a.q + (size_t)(s.q0 + row) * a.ldq + (size_t)(head * a.group + p - row * a.group) * D,
                                                       k_head + (size_t)key * a.ldk);
#pragma unroll
                    for (int i = 0; i < kBlocks; ++i) {
                        const h4 v = *reinterpret_cast<const h4*>(src + 16 * i);
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[b][i][j] += odd_value((float)v[j], gone);
                    }
                }
            });
    }

    // ---- the waves' results: lane's row 16 b + col, columns 16 i + 4 quad + 0..3
    __syncthreads();
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = b * 16 + col;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
            *reinterpret_cast<v4f*>(part + (size_t)(wave * RB * 16 + r) * D + ((16 * i + 4 * quad + 4 * col) & (D - 1))) = o[b][i];
        if (quad == 0) ml[wave * RB * 16 + r] = make_float2(top[b], sum[b]);
    }
    __syncthreads();
    constexpr int kFours = RB * 16 * D / 4;
#pragma unroll
    for (int at = threadIdx.x; at < kFours; at += NW * kWave) {
        const int r = at / (D / 4), c = at % (D / 4) * 4;
        if (r >= rows) continue;
        float most = ml[r].x;
#pragma unroll
        for (int w = 1; w < NW; ++w) most = fmaxf(most, ml[w * RB * 16 + r].x);
        const float less = most == -INFINITY ? 0.0f : most;
        v4f acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 m = ml[w * RB * 16 + r];
            const float f = exp2_fast(m.x - less);
            total = fmaf(m.y, f, total);
            acc += f * *reinterpret_cast<const v4f*>(part + (size_t)(w * RB * 16 + r) * D + ((c + 4 * (r & 15)) & (D - 1)));
        }
        if (__builtin_expect(is_odd(acc[0] + acc[1] + acc[2] + acc[3]), 0)) {  // (a factor may have vanished)
            acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int w = 0; w < NW; ++w) {
                const float f = exp2_fast(ml[w * RB * 16 + r].x - less);
                const v4f v = *reinterpret_cast<const v4f*>(part + (size_t)(w * RB * 16 + r) * D + ((c + 4 * (r & 15)) & (D - 1)));
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += times_unless_odd(f, v[j]);
            }
        }
        if (whole) {
            const int row = r / a.group, seen = a.causal ? row + s.kvlen - s.qlen + 1 : s.kvlen;
            h4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = seen > 0 ? (_Float16)(acc[j] / total) : (_Float16)0.0f;
            *reinterpret_cast<h4*>(a.out + (size_t)(s.q0 + row) * a.ldo + (size_t)(head * a.group + (r - row * a.group)) * D + c) = y;
        } else {
            const size_t to = piece_at(a, slot, t0 == 0, head) + r;
            *reinterpret_cast<v4f*>(a.few_o + to * D + c) = acc;
            if (c == 0) a.few_ml[to] = make_float2(most, total);
        }
    }
    __syncthreads();  // (the next piece's tiles go where the partial results were)
    begin += kPiece + tiles;
    at = begin;
    if (at < end) seq = few_next(a, seq + 1, &s, &tiles);
    }
}

// The pieces of a sequence that several workgroups had, joined in their order: a workgroup for each slot but the first and key head,
// which has the sequence whose last piece is that slot's.
template <int D>
__global__ __launch_bounds__(256) void attention_few_join_kernel(AttnArgs a) {
    const int slot = 1 + blockIdx.x / a.heads_kv, head = blockIdx.x % a.heads_kv;
    const Deal d = few_deal(a, slot);
    if (d.tiles == 0) return;
    const int first = (d.begin + kPiece) / d.per, last = (d.begin + kPiece + d.tiles - 1) / d.per;
    if (first == last || last != slot) return;  // (written already, or another workgroup's)
    const Seq s = d.s;
    const int rows = s.qlen * a.group;
    for (int i = threadIdx.x; i < rows * (D / 4); i += 256) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float top = -INFINITY, sum = 0.0f;
        v4f acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int kAtOnce = 8;
        for (int p0 = first; p0 <= last; p0 += kAtOnce) {
            float2 m[kAtOnce];
            v4f v[kAtOnce];
            float now = top;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int p = min(p0 + j, last);
                const size_t from = piece_at(a, p, p == first, head) + r;
                m[j] = a.few_ml[from];
                v[j] = *reinterpret_cast<const v4f*>(a.few_o + from * D + c);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) now = fmaxf(now, m[j].x);
            const float less = now == -INFINITY ? 0.0f : now, shrink = exp2_fast(top - less);
            sum *= shrink;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = times_unless_odd(shrink, acc[e]);
            top = now;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (p0 + j <= last) {
                    const float f = exp2_fast(m[j].x - less);
                    sum = fmaf(m[j].y, f, sum);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] += times_unless_odd(f, v[j][e]);
                }
        }
        const int row = r / a.group, seen = a.causal ? row + s.kvlen - s.qlen + 1 : s.kvlen;
        h4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = seen > 0 ? (_Float16)(acc[j] / sum) : (_Float16)0.0f;
        *reinterpret_cast<h4*>(a.out + (size_t)(s.q0 + row) * a.ldo + (size_t)(head * a.group + (r - row * a.group)) * D + c) = y;
    }
}

// The chunks' partial results of a row and head, joined in the chunks' order: one wave each.
template <int D>
__global__ __launch_bounds__(256) void attention_tile_join_kernel(AttnArgs a) {
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
    const int chunk = a.tile_chunk;
    if (s.qlen * a.group <= a.few_rows || s.kvlen <= chunk) return;  // (not this kernel's, or written already)
    const int chunks = (s.kvlen + chunk - 1) / chunk;
    // the chunks' maxima and sums lie in the lanes, the partial rows come eight at a time
    const size_t stride = (size_t)a.M * heads;
    constexpr int E = D / kWave, kAtOnce = 8;
    float acc[E] = {}, sum = 0.0f, top = -INFINITY;
    for (int c0 = 0; c0 < chunks; c0 += kWave) {
        const int n = min(chunks - c0, kWave);
        const float2 ml = lane < n ? a.part_ml[(size_t)(c0 + lane) * stride + at] : make_float2(-INFINITY, 0.0f);
        float now = ml.x;
#pragma unroll
        for (int d = 1; d < 16; d *= 2) now = fmaxf(now, __shfl_xor(now, d, kWave));
        now = fmaxf(quads_max(now), top);
        const float less = now == -INFINITY ? 0.0f : now, shrink = exp2_fast(top - less), w = exp2_fast(ml.x - less);
        top = now;
        float part = ml.y * w;
#pragma unroll
        for (int d = 1; d < 16; d *= 2) part += __shfl_xor(part, d, kWave);
        sum = fmaf(sum, shrink, quads_sum(part));
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = times_unless_odd(shrink, acc[e]);
        const float* src = a.part_o + ((size_t)c0 * stride + at) * D + lane * E;
        for (int c = 0; c < n; c += kAtOnce) {
            float v[kAtOnce][E];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) v[i][e] = src[(size_t)min(c + i, n - 1) * stride * D + e];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), min(c + i, n - 1)));
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = c + i < n ? acc[e] + times_unless_odd(f, v[i][e]) : acc[e];
            }
        }
    }
    const int lim = a.causal ? row - s.q0 + s.kvlen - s.qlen + 1 : s.kvlen;
    __half* dst = a.out + (size_t)row * a.ldo + (size_t)head * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) dst[e] = __float2half(lim > 0 ? acc[e] / sum : 0.0f);
}

constexpr int kTileWaves = 4;

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

template <int D, int RB>
hipError_t launch_few(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
    constexpr int NW = few_waves(RB), stages = NW * 2 * kFewKeys * 2 * D, parts = NW * RB * 16 * (4 * D + 8), bytes = stages > parts ? stages : parts;
    static LdsLimit limit;
    const auto kernel = attention_few_kernel<D, RB, NW>;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.slots * a.heads_kv)), dim3(NW * kWave), bytes, stream, a);
    const hipError_t launched = hipGetLastError();
    if (launched != hipSuccess || !p.few_cut) return launched;
    hipLaunchKernelGGL((attention_few_join_kernel<D>), dim3((unsigned)((a.slots - 1) * a.heads_kv)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_tiles(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
    constexpr int bytes = 4 * kKeys * 2 * D + 2 * kTileWaves * 4;
    static LdsLimit limit;
    const auto kernel = attention_tile_kernel<D, kTileWaves>;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    const long long tiles = (long long)a.M * a.group / (kTileWaves * kRowsPerWave) + a.seqs;  // no fewer than the sequences' whole tiles
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles * a.heads_kv), p.tile_chunks), dim3(kTileWaves * kWave), bytes, stream, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_all(const AttnArgs& a, const AttnPlan& p, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (p.tiles) e = launch_tiles<D>(a, p, stream);
    if (e != hipSuccess) return e;
    if (p.few_rows > 0) e = p.few_rows <= 16 ? launch_few<D, 1>(a, p, stream) : p.few_rows <= 32 ? launch_few<D, 2>(a, p, stream) : launch_few<D, 4>(a, p, stream);
    if (e != hipSuccess || p.tile_chunks == 1) return e;
    const long long waves = (long long)a.M * a.heads_kv * a.group;
    hipLaunchKernelGGL((attention_tile_join_kernel<D>), dim3((unsigned)ceil_div(waves, 4)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// Pieces of the keys for the row tiles, by a fitted time: a unit takes 1.1 us for a tile of keys and one workgroup's rows, 0.9 of it
// when it has several workgroups (which then take turns, an uneven last turn half filled); two more tiles' time for a workgroup's
// beginning and end; pieces cost 7 us for a launch and the writing and reading of their partial rows.  Fitted to all numbers of pieces of
// 129 calls (70 to 4096 rows of 8 to 64 heads over as many keys and up to 60000): 3 % behind the best of each on average, 25 % at most; three
// workgroups a unit instead, whatever the rows: 17 %, 2.6 times at most.  900 rows over 900 keys, 32 + 8 heads of 128: 24.5 us whole, 42 in
// two pieces; 300 over 16000: 289 whole, 101 in six, 139 in 32; 128 over 60000: 1085 whole, 147 in sixteen.
int key_pieces(int M, int max_q, int max_kv, int heads_kv, int group, int head_dim) {
    const double workgroups = (double)(((long long)M * group / (kTileWaves * kRowsPerWave) + 1) * heads_kv), units = cu_count();
    const double seen = 1.0 - 0.5 * std::min(max_q, max_kv) / std::max(max_kv, 1);  // (of whole prompts a row sees half)
    const long long tiles = ceil_div(std::max(max_kv, 1), kKeys), most = std::min(tiles, (long long)(3.0 * units / workgroups) + 1);
    const double join = (double)M * heads_kv * group * (4 * head_dim + 8) / 4e6;
    long long best = 1;
    double least = 0.0;
    for (long long pieces = 1; pieces <= most; pieces += 1 + pieces / 16) {
        const long long each = ceil_div(tiles, pieces), n = ceil_div(tiles, each);
        const double turns = workgroups * n / units;
        double us = 1.1 * (each + 2);
        if (turns > 1.0) us = std::max(us, 1.1 * 0.9 * 0.5 * (turns + ceil(turns)) * (each * seen + 2));
        if (n > 1) us += 7.0 + n * join;
        if (pieces == 1 || us < least) best = n, least = us;
    }
    return (int)best;
}

}  // namespace

AttnPlan attention_plan(int M, int seqs, int max_q, int max_kv, int heads_kv, int group, int head_dim, bool own_lens) {
    AttnPlan p;
    max_q = std::min(max_q, M);
    const long long most = (long long)max_q * group;
    const int singles = group <= 16 ? 16 : group <= 32 ? 32 : group <= kFewRows ? kFewRows : 0;
    p.tiles = most > kFewRows;
    // beside longer sequences the kernel for few rows takes single tokens; there are none where all are equally long, and without
    // lengths of their own their keys are as few as their rows
    if (!p.tiles) p.few_rows = most <= 16 ? 16 : most <= 32 ? 32 : kFewRows;
    else p.few_rows = own_lens && M < (long long)seqs * max_q ? singles : 0;
    if (p.few_rows > 0) {
        // One workgroup a unit, none with less than 18 tiles (576 keys) of a sequence.
        constexpr int kLeast = 18 + kPiece;
        const long long most = ceil_div(max_kv < 1 ? 1 : max_kv, kFewKeys) + kPiece;  // numbers of a sequence
        p.least_tiles = kLeast;
        p.slots = (int)std::min(ceil_div(cu_count(), heads_kv), ceil_div(seqs * most, kLeast));
        p.few_cut = p.slots > 1 && (seqs > 1 || most > kLeast);
    }
    if (p.tiles) {
        const long long tiles = ceil_div(std::max(max_kv, 1), kKeys), each = ceil_div(tiles, key_pieces(M, max_q, max_kv, heads_kv, group, head_dim));
        p.tile_chunk = (int)(each * kKeys);
        p.tile_chunks = (int)ceil_div(tiles, each);
    }
    return p;
}

static size_t few_part_rows(const AttnPlan& p, int heads_kv) { return p.few_cut ? (size_t)p.slots * 2 * heads_kv * p.few_rows : 0; }
static size_t tile_part_rows(const AttnPlan& p, int M, int heads_q) { return p.tile_chunks == 1 ? 0 : (size_t)p.tile_chunks * M * heads_q; }

size_t attention_workspace_bytes(const AttnPlan& p, int M, int heads_kv, int group, int head_dim) {
    return (few_part_rows(p, heads_kv) + tile_part_rows(p, M, heads_kv * group)) * (head_dim * 4 + 8);
}

hipError_t launch_attention(const AttnArgs& args, const AttnPlan& p, int head_dim, void* workspace, hipStream_t stream) {
    AttnArgs a = args;
    a.few_rows = p.few_rows;
    a.slots = p.slots;
    a.least_tiles = p.least_tiles;
    a.tile_chunk = p.tile_chunk;
    const size_t few = few_part_rows(p, a.heads_kv), tile = tile_part_rows(p, a.M, a.heads_kv * a.group);
    a.few_o = static_cast<float*>(workspace);
    a.part_o = a.few_o + few * head_dim;
    a.few_ml = reinterpret_cast<float2*>(a.part_o + tile * head_dim);
    a.part_ml = a.few_ml + few;
    return head_dim == 128 ? launch_all<128>(a, p, stream) : launch_all<64>(a, p, stream);
}

}  // namespace intscale
