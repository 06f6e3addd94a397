// Causal attention with grouped heads over packed sequences (poseidon_layers.h), forward and backward:
//   s = scale q k^T for keys up to the query of the same sequence, lse = log sum exp s, p = exp(s - lse), out = p v;
//   delta = <dout, out>, dp = dout v^T, ds = p (dp - delta), dq = scale ds k, dk = scale ds^T q, dv = p^T dout.
//
// Scores are never in memory: a wave holds 32 queries (backward for dk and dv: 32 keys) in registers and goes through tiles of
// the others in LDS.  Products are laid out so that a lane holds one query (key) and its scores of 32 keys (queries)
// lie in the lane's registers as the next product's operand wants them, up to the order of what is summed over, which the
// other operand follows: nothing is exchanged between lanes but a row's largest score, and at the end its sum.
#include "layers_mfma.h"

#include <type_traits>

namespace pl {

constexpr uint32_t kTile = 64;               // keys (backward for dk and dv: queries) in LDS at a time
constexpr uint32_t kClearBlocks = 64;        // blocks that look for rows outside of all sequences
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Rows [tokens][heads][dim] of a 16-bit type: where a token's and a head's values begin.
struct Heads {
    const void *at;
    uint64_t token, head;
};

struct Attention {
    Heads q, k, v, dout, out, dq, dk, dv;    // written: out forward, dq, dk, dv backward
    float *lse, *delta;                      // [heads][tokens]
    const int32_t *offsets;                  // null: one sequence of all tokens
    uint32_t tokens, sequences, heads, kv_heads, dim, tiles;
    float scale;
};

template <class T>
__device__ __forceinline__ const typename T::raw *row_of(const Heads &x, uint64_t token, uint32_t head) {
    return (const typename T::raw *)x.at + token * x.token + head * x.head;
}

// Rows of D values lie in LDS in pieces of 16 bytes; piece p of row r at p ^ mixed(r).  Eight rows' pieces p and four rows'
// pieces [p, p + 4) are so in banks of their own.
template <int D>
__device__ __forceinline__ uint32_t mixed(uint32_t r) {
    if constexpr (D == 128)
        return (r >> 2 & 1) | (r & 2) | (r & 1) << 2 | (r & 2) << 2;
    else
        return (r >> 2 & 1) | (r & 1) << 1 | (r & 2) << 1;
}

// A tile of rows on its way to LDS, by `threads` threads; rows from `rows` on and values from `dim` on come as zeros.
template <int D, uint32_t THREADS>
struct Loader {
    static constexpr uint32_t kPieces = kTile * D / 8 / THREADS;
    uint32_t row[kPieces], piece[kPieces];
    __device__ __forceinline__ void aim(uint32_t dim) {
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i) {
            const uint32_t p = i * THREADS + threadIdx.x;
            row[i] = p / (D / 8);
            const uint32_t c = (p % (D / 8)) ^ mixed<D>(row[i]);
            piece[i] = c * 8 < dim ? c * 16 : kNowhere;
        }
    }
    template <class T>
    __device__ __forceinline__ void load(const typename T::raw *from, uint64_t pitch, uint32_t rows, uint16_t *to) const {
        const uint64_t bytes = rows * pitch * 2;
        const Rsrc r = buffer(from, (uint32_t)min(bytes, (uint64_t)kBufferBytes));
#pragma unroll
        for (uint32_t i = 0; i < kPieces; ++i)
            copy_to_lds(r, row[i] * ((uint32_t)pitch * 2) + piece[i], to + (i * THREADS + threadIdx.x / 64 * 64) * 8);
    }
};

// Operands from LDS: 16 values from 16 s on of rows 32 t + lane % 32, and the turned rows (lane: value 32 d + lane % 32) that
// go with the scores of rows [16 s, 16 s + 16) in a lane's registers: 4 half + {0..3}, then 8 + 4 half + {0..3}.
template <int D>
__device__ __forceinline__ Words4 rows_at(const uint16_t *lds, int t, int s, uint32_t lane) {
    const uint32_t r = lane % 32;
    return *(const Words4 *)(lds + (32 * t + r) * D + ((2 * s + lane / 32) ^ mixed<D>(r)) * 8);
}
template <int D>
__device__ __forceinline__ Words4 turned_at(const uint16_t *lds, int s, int d, uint32_t lane) {
    const uint32_t r = 4 * (lane / 32) + lane % 16 / 4;
    const uint32_t piece = (4 * d + 2 * (lane / 16 % 2) + lane % 4 / 2) ^ mixed<D>(r);
    const uint16_t *from = lds + (16 * s + r) * D + piece * 8 + lane % 2 * 4;
    const uint2 lo = read_turned(from), hi = read_turned(from + 8 * D);
    return Words4{lo.x, lo.y, hi.x, hi.y};
}

// Eight values [16 s + 8 (lane / 32), ...) of a row in memory, zeros from `dim` on.
template <class T>
__device__ __forceinline__ Words4 piece_of(const typename T::raw *row, int s, uint32_t lane, uint32_t dim) {
    const uint32_t c = 16 * s + 8 * (lane / 32);
    return c < dim ? *(const Words4 *)(row + c) : Words4{};
}

template <class T>
__device__ __forceinline__ Words4 packed(const float (&v)[16], int s) {
    return Words4{pair<T>(v[8 * s], v[8 * s + 1]), pair<T>(v[8 * s + 2], v[8 * s + 3]), pair<T>(v[8 * s + 4], v[8 * s + 5]),
                  pair<T>(v[8 * s + 6], v[8 * s + 7])};
}

// Values of the same lane of the other half of the wave.
__device__ __forceinline__ float larger_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_half(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Sums whose column is the lane's row, times f, to that row in memory.
template <class T, int D>
__device__ __forceinline__ void store_turned(const Acc (&sum)[D / 32], float f, typename T::raw *row, uint32_t dim, uint32_t lane) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[d][8 * h + i] * f),
                                                                __float_as_uint(sum[d][8 * h + 4 + i] * f), false, false);
                v[i] = __uint_as_float(r[0]);
                v[4 + i] = __uint_as_float(r[1]);
            }
            const uint32_t c = 32 * d + 16 * h + 8 * (lane / 32);
            if (row && c < dim) store_slice<T>(row, c, dim, v);
        }
}

// The tile and head of a block.  Blocks go round the eight XCDs in turn, so the heads that share keys are a multiple of
// kv_heads apart: an XCD sees few heads of keys.
struct Work {
    uint32_t tile, head, kv;
};
__device__ __forceinline__ Work work_of(uint32_t id, uint32_t heads, uint32_t kv_heads) {
    const uint32_t h = id % heads, kv = h % kv_heads;
    return {id / heads, kv * (heads / kv_heads) + h / kv_heads, kv};
}

__device__ __forceinline__ Place sequence_of(const Attention &a, uint32_t tile, uint32_t size, uint32_t &begin) {
    Place p = {0, tile * size, a.tokens, tile * size < a.tokens};
    begin = 0;
    if (a.offsets) {
        p = place_of(a.offsets, a.sequences, a.tokens, tile, size);
        begin = bound_of(a.offsets, p.range, a.tokens);
    }
    return p;
}

// f(token) for the tokens outside of all sequences that fall to block `block` of `blocks`.
template <class F>
__device__ __forceinline__ void outside(const Attention &a, uint32_t block, uint32_t blocks, F f) {
    const uint32_t begin = bound_of(a.offsets, 0, a.tokens), end = max(begin, bound_of(a.offsets, a.sequences, a.tokens));
    for (uint32_t i = block; i < begin + a.tokens - end; i += blocks) f((uint64_t)(i < begin ? i : end + (i - begin)));
}
template <class T>
__device__ __forceinline__ void clear_token(const Heads &x, uint64_t token, uint32_t heads, uint32_t dim) {
    const float zero[8] = {};
    for (uint32_t i = threadIdx.x; i < heads * (dim / 8); i += blockDim.x)
        store_slice<T>((typename T::raw *)row_of<T>(x, token, i / (dim / 8)), i % (dim / 8) * 8, dim, zero);
}

// WAVES waves of 32 queries each.  The running largest score m follows a row's scores only when one outgrows it by 2^8:
// the sums then stay below 2^8 times the number of keys, and most tiles leave what was summed alone.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_forward_kernel(Attention a) {
    constexpr uint32_t kQueries = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * kStage];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.heads;
    if (blockIdx.x >= blocks) {
        outside(a, blockIdx.x - blocks, gridDim.x - blocks, [&](uint64_t t) {
            clear_token<T>(a.out, t, a.heads, a.dim);
            for (uint32_t h = threadIdx.x; h < a.heads; h += blockDim.x) a.lse[(uint64_t)h * a.tokens + t] = -__builtin_inff();
        });
        return;
    }
    const Work w = work_of(blockIdx.x, a.heads, a.kv_heads);
    uint32_t begin;    // the longest rows of a sequence first
    const Place at = sequence_of(a, a.tiles - 1 - w.tile, kQueries, begin);
    if (!at.there) return;
    const uint32_t q0 = at.begin + 32 * wave, q = q0 + lane % 32;    // the wave's first query, the lane's
    const uint32_t last = min(at.begin + kQueries, at.end);
    const uint32_t tiles = (last - begin + kTile - 1) / kTile;

    using raw = typename T::raw;
    Words4 query[D / 16];
    {
        const raw *row = row_of<T>(a.q, min(q, at.end - 1), w.head);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) query[s] = piece_of<T>(row, s, lane, a.dim);
    }
    Loader<D, 64 * WAVES> loader;
    loader.aim(a.dim);
    const auto fetch = [&](uint32_t i) {
        const uint32_t t = begin + i * kTile, rows = at.end - t;
        uint16_t *to = lds + (i & 1) * kStage;
        loader.template load<T>(row_of<T>(a.k, t, w.kv), a.k.token, rows, to);
        loader.template load<T>(row_of<T>(a.v, t, w.kv), a.v.token, rows, to + kTile * D);
    };

    const float c = a.scale * kLog2e;
    float m = -__builtin_inff(), total = 0.0f;
    Acc sum[D / 32] = {};
    fetch(0);
    for (uint32_t i = 0; i < tiles; ++i) {
        __builtin_amdgcn_s_waitcnt(0x0f70);    // vmcnt(0): this wave's part of the tile is in LDS
        __syncthreads();
        if (i + 1 < tiles) fetch(i + 1);
        const uint32_t t0 = begin + i * kTile;
        if (t0 > q0 + 31) continue;            // all of it after the wave's queries
        const uint16_t *keys = lds + (i & 1) * kStage, *vals = keys + kTile * D;
        Acc s[2] = {};
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mfma<T>(rows_at<D>(keys, t, j, lane), query[j], s[t]);
        float p[2][16];
        float most = -__builtin_inff();
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) p[t][r] = s[t][r];
        if (t0 + kTile - 1 > q0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (t0 + 32 * t + (r & 3) + 8 * (r >> 2) + 4 * (lane / 32) > q) p[t][r] = -__builtin_inff();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, p[t][r]);
        most = larger_half(most);
        if (__any((most - m) * c > 8.0f)) {
            const float to = fmaxf(m, most), f = __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            total *= f;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) sum[d] *= f;
        }
        const float mc = m * c;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[t][r] = __builtin_amdgcn_exp2f(fmaf(p[t][r], c, -mc));
                total += p[t][r];
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Words4 w = packed<T>(p[j / 2], j % 2);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) sum[d] = mfma<T>(turned_at<D>(vals, j, d, lane), w, sum[d]);
        }
    }
    total = sum_half(total);
    const bool there = q < at.end;
    store_turned<T, D>(sum, 1.0f / total, there ? (raw *)row_of<T>(a.out, q, w.head) : nullptr, a.dim, lane);
    if (there && lane < 32) a.lse[(uint64_t)w.head * a.tokens + q] = m * a.scale + __logf(total);
}

// dq, as the forward pass goes, with delta = <dout, out> for the other kernel.  p and ds are rounded to the operands' type.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_queries_kernel(Attention a) {
    constexpr uint32_t kQueries = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * kStage];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.heads;
    if (blockIdx.x >= blocks) {
        outside(a, blockIdx.x - blocks, gridDim.x - blocks, [&](uint64_t t) { clear_token<T>(a.dq, t, a.heads, a.dim); });
        return;
    }
    const Work w = work_of(blockIdx.x, a.heads, a.kv_heads);
    uint32_t begin;
    const Place at = sequence_of(a, a.tiles - 1 - w.tile, kQueries, begin);
    if (!at.there) return;
    const uint32_t q0 = at.begin + 32 * wave, q = q0 + lane % 32;
    const uint32_t last = min(at.begin + kQueries, at.end);
    const uint32_t tiles = (last - begin + kTile - 1) / kTile;
    const bool there = q < at.end;

    using raw = typename T::raw;
    Words4 query[D / 16], dout[D / 16];
    float delta = 0.0f;
    const uint32_t mine = min(q, at.end - 1);
    {
        const raw *qr = row_of<T>(a.q, mine, w.head), *dr = row_of<T>(a.dout, mine, w.head), *outr = row_of<T>(a.out, mine, w.head);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            query[s] = piece_of<T>(qr, s, lane, a.dim);
            dout[s] = piece_of<T>(dr, s, lane, a.dim);
            const Words4 o = piece_of<T>(outr, s, lane, a.dim);
            raw x[8], y[8];
            __builtin_memcpy(x, &dout[s], 16);
            __builtin_memcpy(y, &o, 16);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(T::up(x[i]), T::up(y[i]), delta);
        }
        delta = sum_half(delta);
        if (there && lane < 32) a.delta[(uint64_t)w.head * a.tokens + q] = delta;
    }
    Loader<D, 64 * WAVES> loader;
    loader.aim(a.dim);
    const auto fetch = [&](uint32_t i) {
        const uint32_t t = begin + i * kTile, rows = at.end - t;
        uint16_t *to = lds + (i & 1) * kStage;
        loader.template load<T>(row_of<T>(a.k, t, w.kv), a.k.token, rows, to);
        loader.template load<T>(row_of<T>(a.v, t, w.kv), a.v.token, rows, to + kTile * D);
    };

    const float c = a.scale * kLog2e, lse = a.lse[(uint64_t)w.head * a.tokens + mine] * kLog2e;
    Acc sum[D / 32] = {};
    fetch(0);
    for (uint32_t i = 0; i < tiles; ++i) {
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        if (i + 1 < tiles) fetch(i + 1);
        const uint16_t *keys = lds + (i & 1) * kStage, *vals = keys + kTile * D;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t t0 = begin + i * kTile + 32 * t;
            if (t0 > q0 + 31) continue;
            Acc s = {}, dp = {};
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                s = mfma<T>(rows_at<D>(keys, t, j, lane), query[j], s);
                dp = mfma<T>(rows_at<D>(vals, t, j, lane), dout[j], dp);
            }
            float ds[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse)) * (dp[r] - delta);
            if (t0 + 31 > q0) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (t0 + (r & 3) + 8 * (r >> 2) + 4 * (lane / 32) > q) ds[r] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Words4 w = packed<T>(ds, j);
#pragma unroll
                for (int d = 0; d < D / 32; ++d) sum[d] = mfma<T>(turned_at<D>(keys, 2 * t + j, d, lane), w, sum[d]);
            }
        }
    }
    store_turned<T, D>(sum, a.scale, there ? (raw *)row_of<T>(a.dq, q, w.head) : nullptr, a.dim, lane);
}

// dk and dv: WAVES waves of 32 keys each go through the queries of every head that shares them, in one order.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_keys_kernel(Attention a) {
    constexpr uint32_t kKeys = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * kStage];
    __shared__ __attribute__((aligned(16))) float rows[2][2][kTile];    // lse and delta
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.kv_heads;
    if (blockIdx.x >= blocks) {
        outside(a, blockIdx.x - blocks, gridDim.x - blocks, [&](uint64_t t) {
            clear_token<T>(a.dk, t, a.kv_heads, a.dim);
            clear_token<T>(a.dv, t, a.kv_heads, a.dim);
        });
        return;
    }
    const uint32_t kv = blockIdx.x % a.kv_heads, group = a.heads / a.kv_heads;
    uint32_t begin;    // keys early in a sequence have the most queries: these first
    const Place at = sequence_of(a, blockIdx.x / a.kv_heads, kKeys, begin);
    if (!at.there) return;
    const uint32_t k0 = at.begin + 32 * wave, key = k0 + lane % 32;
    const bool there = key < at.end;
    const uint32_t tiles = (at.end - at.begin + kTile - 1) / kTile;    // of queries, from the block's first key on

    using raw = typename T::raw;
    Words4 keys[D / 16], vals[D / 16];
    {
        const uint32_t mine = min(key, at.end - 1);
        const raw *kr = row_of<T>(a.k, mine, kv), *vr = row_of<T>(a.v, mine, kv);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            keys[s] = piece_of<T>(kr, s, lane, a.dim);
            vals[s] = piece_of<T>(vr, s, lane, a.dim);
        }
    }
    Loader<D, 64 * WAVES> loader;
    loader.aim(a.dim);
    const auto fetch = [&](uint32_t set, uint32_t head, uint32_t i) {
        const uint32_t t = at.begin + i * kTile, n = at.end - t;
        uint16_t *to = lds + set * kStage;
        loader.template load<T>(row_of<T>(a.q, t, head), a.q.token, n, to);
        loader.template load<T>(row_of<T>(a.dout, t, head), a.dout.token, n, to + kTile * D);
        if (wave < 2) {    // rows past the end: zeros, as q and dout have there
            const float *from = (wave ? a.delta : a.lse) + (uint64_t)head * a.tokens + t;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(from, min(n, kTile) * 4),
                                                     (__attribute__((address_space(3))) void *)rows[set][wave], 4, lane * 4, 0, 0, 0);
        }
    };

    const float c = a.scale * kLog2e;
    Acc dk[D / 32] = {}, dv[D / 32] = {};
    uint32_t set = 0;
    fetch(0, kv * group, 0);
    for (uint32_t g = 0; g < group; ++g)
        for (uint32_t i = 0; i < tiles; ++i, set ^= 1) {
            __builtin_amdgcn_s_waitcnt(0x0f70);
            __syncthreads();
            if (i + 1 < tiles)
                fetch(set ^ 1, kv * group + g, i + 1);
            else if (g + 1 < group)
                fetch(set ^ 1, kv * group + g + 1, 0);
            const uint16_t *queries = lds + set * kStage, *douts = queries + kTile * D;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t t0 = at.begin + i * kTile + 32 * t;
                if (t0 + 31 < k0) continue;    // all of them before the wave's keys
                Acc s = {}, dp = {};
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    s = mfma<T>(rows_at<D>(queries, t, j, lane), keys[j], s);
                    dp = mfma<T>(rows_at<D>(douts, t, j, lane), vals[j], dp);
                }
                float p[16], ds[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t r0 = 32 * t + 8 * q + 4 * (lane / 32);
                    const float4 lse = *(const float4 *)&rows[set][0][r0], delta = *(const float4 *)&rows[set][1][r0];
                    const float l[4] = {lse.x, lse.y, lse.z, lse.w}, d[4] = {delta.x, delta.y, delta.z, delta.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 4 * q + e;
                        p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -l[e] * kLog2e));
                        ds[r] = p[r] * (dp[r] - d[e]);
                    }
                }
                if (t0 < k0 + 31) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (t0 + (r & 3) + 8 * (r >> 2) + 4 * (lane / 32) < key) p[r] = ds[r] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const Words4 pw = packed<T>(p, j), dw = packed<T>(ds, j);
#pragma unroll
                    for (int d = 0; d < D / 32; ++d) {
                        dv[d] = mfma<T>(turned_at<D>(douts, 2 * t + j, d, lane), pw, dv[d]);
                        dk[d] = mfma<T>(turned_at<D>(queries, 2 * t + j, d, lane), dw, dk[d]);
                    }
                }
            }
        }
    store_turned<T, D>(dk, a.scale, there ? (raw *)row_of<T>(a.dk, key, kv) : nullptr, a.dim, lane);
    store_turned<T, D>(dv, 1.0f, there ? (raw *)row_of<T>(a.dv, key, kv) : nullptr, a.dim, lane);
}

inline int check_heads(const void *p, uint64_t token, uint64_t head, uint64_t tokens, uint64_t heads, uint64_t dim) {
    if (token < dim || (heads > 1 && head < dim) || token % 8 || head % 8) return POSEIDON_E_INVAL;
    if (token > POSEIDON_PITCH_MAX || (heads > 1 && head > (1ull << 40))) return POSEIDON_E_RANGE;
    return tokens && (!p || !aligned(p, 16)) ? POSEIDON_E_INVAL : POSEIDON_OK;
}

inline int check_attention(uint64_t tokens, uint64_t heads, uint64_t kv_heads, uint64_t dim, float scale,
                           const int32_t *offsets, uint32_t sequences) {
    if (!heads || !kv_heads || heads % kv_heads || !dim || dim % 8 || !sequences || (!offsets && sequences != 1) ||
        !aligned(offsets, 4) || !(scale > -__builtin_inff() && scale < __builtin_inff()))
        return POSEIDON_E_INVAL;
    if (tokens > POSEIDON_ROWS_MAX || heads > POSEIDON_HEADS_MAX || dim > POSEIDON_HEAD_MAX || sequences > POSEIDON_ROWS_MAX)
        return POSEIDON_E_RANGE;
    return POSEIDON_OK;
}

// Runs f(type, padded dim) for a head's width.
template <class F>
inline int for_heads(uint32_t type, uint64_t dim, F f) {
    using Small = std::integral_constant<int, 64>;
    using Large = std::integral_constant<int, 128>;
    if (type == POSEIDON_F16) return dim <= 64 ? f(F16{}, Small{}) : f(F16{}, Large{});
    return dim <= 64 ? f(BF16{}, Small{}) : f(BF16{}, Large{});
}

template <class K>
inline int run_attention(K kernel, Attention &a, uint32_t heads, uint32_t waves, void *hip_stream) {
    const uint64_t size = 32 * waves;
    const uint64_t tiles = a.offsets ? tiles_for(a.tokens, a.sequences, (uint32_t)size) : (a.tokens + size - 1) / size;
    if (tiles * heads > 0x7fffff00ull) return POSEIDON_E_RANGE;
    a.tiles = (uint32_t)tiles;
    kernel<<<(uint32_t)(tiles * heads) + (a.offsets ? kClearBlocks : 0), 64 * waves, 0, (hipStream_t)hip_stream>>>(a);
    return launched();
}

}  // namespace pl

using namespace pl;

extern "C" {

int poseidon_attention_forward(const void *q, uint64_t q_token, uint64_t q_head, const void *k, uint64_t k_token,
                               uint64_t k_head, const void *v, uint64_t v_token, uint64_t v_head, uint32_t type,
                               uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dim, float scale,
                               const int32_t *offsets, uint32_t sequences, void *out, uint64_t out_token,
                               uint64_t out_head, float *lse, void *hip_stream) {
    PL_TRY(check_attention(tokens, heads, kv_heads, dim, scale, offsets, sequences));
    if (type != POSEIDON_F16 && type != POSEIDON_BF16) return POSEIDON_E_INVAL;
    PL_TRY(check_heads(q, q_token, q_head, tokens, heads, dim));
    PL_TRY(check_heads(k, k_token, k_head, tokens, kv_heads, dim));
    PL_TRY(check_heads(v, v_token, v_head, tokens, kv_heads, dim));
    PL_TRY(check_heads(out, out_token, out_head, tokens, heads, dim));
    if (tokens && (!lse || !aligned(lse, 4))) return POSEIDON_E_INVAL;
    if (!tokens) return POSEIDON_OK;
    Attention a = {};
    a.q = {q, q_token, q_head};
    a.k = {k, k_token, k_head};
    a.v = {v, v_token, v_head};
    a.out = {out, out_token, out_head};
    a.lse = lse;
    a.offsets = offsets;
    a.tokens = (uint32_t)tokens;
    a.sequences = sequences;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.dim = dim;
    a.scale = scale;
    return for_heads(type, dim, [&](auto t, auto d) {
        return run_attention(attention_forward_kernel<decltype(t), d.value, 4>, a, heads, 4, hip_stream);
    });
}

uint64_t poseidon_attention_backward_workspace(uint64_t tokens, uint32_t heads) {
    return tokens > POSEIDON_ROWS_MAX || !heads || heads > POSEIDON_HEADS_MAX ? UINT64_MAX : tokens * heads * 4;
}

int poseidon_attention_backward(const void *dout, uint64_t dout_token, uint64_t dout_head, const void *q,
                                uint64_t q_token, uint64_t q_head, const void *k, uint64_t k_token, uint64_t k_head,
                                const void *v, uint64_t v_token, uint64_t v_head, const void *out, uint64_t out_token,
                                uint64_t out_head, const float *lse, uint32_t type, uint64_t tokens, uint32_t heads,
                                uint32_t kv_heads, uint32_t dim, float scale, const int32_t *offsets,
                                uint32_t sequences, void *dq, uint64_t dq_token, uint64_t dq_head, void *dk,
                                uint64_t dk_token, uint64_t dk_head, void *dv, uint64_t dv_token, uint64_t dv_head,
                                void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    PL_TRY(check_attention(tokens, heads, kv_heads, dim, scale, offsets, sequences));
    if (type != POSEIDON_F16 && type != POSEIDON_BF16) return POSEIDON_E_INVAL;
    PL_TRY(check_heads(dout, dout_token, dout_head, tokens, heads, dim));
    PL_TRY(check_heads(q, q_token, q_head, tokens, heads, dim));
    PL_TRY(check_heads(k, k_token, k_head, tokens, kv_heads, dim));
    PL_TRY(check_heads(v, v_token, v_head, tokens, kv_heads, dim));
    PL_TRY(check_heads(out, out_token, out_head, tokens, heads, dim));
    PL_TRY(check_heads(dq, dq_token, dq_head, tokens, heads, dim));
    PL_TRY(check_heads(dk, dk_token, dk_head, tokens, kv_heads, dim));
    PL_TRY(check_heads(dv, dv_token, dv_head, tokens, kv_heads, dim));
    if (tokens && (!lse || !aligned(lse, 4))) return POSEIDON_E_INVAL;
    PL_TRY(check_workspace(workspace, workspace_bytes, poseidon_attention_backward_workspace(tokens, heads)));
    if (!tokens) return POSEIDON_OK;
    Attention a = {};
    a.q = {q, q_token, q_head};
    a.k = {k, k_token, k_head};
    a.v = {v, v_token, v_head};
    a.dout = {dout, dout_token, dout_head};
    a.out = {out, out_token, out_head};
    a.dq = {dq, dq_token, dq_head};
    a.dk = {dk, dk_token, dk_head};
    a.dv = {dv, dv_token, dv_head};
    a.lse = const_cast<float *>(lse);
    a.delta = (float *)workspace;
    a.offsets = offsets;
    a.tokens = (uint32_t)tokens;
    a.sequences = sequences;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.dim = dim;
    a.scale = scale;
    return for_heads(type, dim, [&](auto t, auto d) -> int {
        PL_TRY(run_attention(attention_queries_kernel<decltype(t), d.value, 4>, a, heads, 4, hip_stream));
        return run_attention(attention_keys_kernel<decltype(t), d.value, 4>, a, kv_heads, 4, hip_stream);
    });
}

}  // extern "C"
