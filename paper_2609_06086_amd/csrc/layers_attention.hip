// Causal attention with grouped heads over packed sequences (poseidon_layers.h), forward and backward:
//   s = scale q k^T for keys up to the query of the same sequence, lse = log sum exp s, p = exp(s - lse), out = p v;
//   delta = <dout, out>, dp = dout v^T, ds = p (dp - delta), dq = scale ds k, dk = scale ds^T q, dv = p^T dout.
//
// Scores are never in memory: a wave holds 32 queries (backward for dk and dv: 32 keys) in registers and goes through tiles of
// the others in LDS.  Products are laid out so that a lane holds one query (key) and its scores of 32 keys (queries)
// lie in the lane's registers as the next product's operand wants them, up to the order of what is summed over, which the
// other operand follows: nothing is exchanged between lanes but a row's largest score, and at the end its sum.
//
// p and ds go to their products in 16 bits, as the matrix instructions take operands; the sums of p, and all other
// statistics, are made of what they were before.  In bf16 outputs are off by 0.0018 to 0.0022 of their norm and dq and dk by 0.0027 where
// the rounding of results alone gives 0.0016.  What the rounding drops could go through products of its own: three in place of two
// forward, ten in place of seven backward.
#include "layers_mfma.h"

#include <type_traits>

namespace pl {

constexpr uint32_t kTile = 64;               // keys (backward for dk and dv: queries) in LDS at a time
constexpr int kWaves = 4;                    // of a block
constexpr uint32_t kClearBlocks = 64;        // blocks that look for rows outside of all sequences
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Rows [tokens][heads][dim] of a 16-bit type: where a token's and a head's values begin.
struct Heads {
    const void *at;
    uint64_t token, head;
};

struct Attention {
    Heads q, k, v, dout, out, dq, dk, dv;    // written: out forward, dq, dk, dv backward
    float *lse, *delta, *base;               // [heads][tokens]; base: -lse / ln 2 + kRaised
    const int32_t *offsets;                  // null: one sequence of all tokens
    float *parts;                            // [split][dk, dv][tokens][kv heads][dim] sums, where split > 1
    uint32_t tokens, sequences, heads, kv_heads, dim, tiles, split, first;    // first: block of this launch
    float scale;
};

template <class T>
__device__ __forceinline__ const typename T::raw *row_of(const Heads &x, uint64_t token, uint32_t head) {
    return (const typename T::raw *)x.at + token * x.token + head * x.head;
}

// Rows of D values lie in LDS in pieces of 16 bytes; piece p of row r at p ^ mixed(r).  The pieces p of sixteen rows, which
// LDS reads at a time, and the pieces [4 p, 4 p + 4) of four rows, which a turned read takes, are so in banks of their own.
template <int D>
__device__ __forceinline__ uint32_t mixed(uint32_t r) {
    const uint32_t high = (r >> 2 & 1) | (r >> 2 & 2);
    if constexpr (D == 128)
        return (r & 3) << 2 | high;
    else
        return (r & 2) << 1 | high;    // two rows to all banks
}

// A tile of rows on its way to LDS, by THREADS threads, some rows in each of a few copies; rows from `rows` on and values from
// `dim` on come as zeros.  A copy's rows are a multiple of 16, so a lane's piece lies at the same place in all of them.
template <int D, uint32_t THREADS>
struct Loader {
    static constexpr uint32_t kRows = THREADS / (D / 8);
    static_assert(kRows % 16 == 0 && kTile % kRows == 0);
    uint32_t row, piece;
    __device__ __forceinline__ explicit Loader(uint32_t dim) {
        row = threadIdx.x / (D / 8);
        const uint32_t c = (threadIdx.x % (D / 8)) ^ mixed<D>(row);
        piece = c * 8 < dim ? c * 16 : kNowhere;
    }
    __device__ __forceinline__ uint32_t place(uint64_t pitch) const { return row * ((uint32_t)pitch * 2) + piece; }
    template <class T>
    __device__ __forceinline__ void load(const typename T::raw *from, uint64_t pitch, uint32_t place, uint32_t rows, uint16_t *to) const {
#pragma unroll
        for (uint32_t i = 0; i < kTile / kRows; ++i) {
            const uint32_t left = rows > i * kRows ? min(rows - i * kRows, kRows) : 0;
            copy_to_lds<false>(buffer(from + i * kRows * pitch, __builtin_amdgcn_readfirstlane(left * ((uint32_t)pitch * 2))), place,
                        to + (i * THREADS + __builtin_amdgcn_readfirstlane(threadIdx.x & ~63u)) * 8);
        }
    }
};

// Two stages of two tiles in LDS.  The boundary is SmallReader's.
template <int D>
struct alignas(2 * D) Stages {
    uint16_t at[4 * kTile * D];
};

// Operands from a tile in LDS that begins OFFSET values into it: 16 values from 16 s on of rows 32 t + lane % 32, and the
// turned rows (lane: value 32 d + lane % 32) that go with the scores of rows [16 s, 16 s + 16) in a lane's registers:
// 4 half + {0..3}, then 8 + 4 half + {0..3}.  A lane's places are found once; tiles and rows are offsets in the instructions.
template <int D>
struct Reader {
    using Bytes = __attribute__((address_space(3))) const char *;
    uint32_t rows[D / 16], lo[D / 32], hi[D / 32];
    __device__ __forceinline__ Reader(const Stages<D> &lds, uint32_t lane) {
        const uint32_t base = (uint32_t)(uintptr_t)(Bytes)(const char *)lds.at;
        const uint32_t r = lane % 32, u = 4 * (lane / 32) + lane % 16 / 4, c = 2 * (lane / 16 % 2) + lane % 4 / 2;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) rows[s] = base + r * (2 * D) + ((2 * s + lane / 32) ^ mixed<D>(r)) * 16;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
            lo[d] = base + u * (2 * D) + ((4 * d + c) ^ mixed<D>(u)) * 16 + lane % 2 * 8;
            hi[d] = base + (u + 8) * (2 * D) + ((4 * d + c) ^ mixed<D>(u + 8)) * 16 + lane % 2 * 8;
        }
    }
    template <uint32_t OFFSET>
    __device__ __forceinline__ Words4 row(int t, int s) const {
        return *(__attribute__((address_space(3))) const Words4 *)((Bytes)(uintptr_t)rows[s] + 2 * OFFSET + 64 * D * t);
    }
    template <uint32_t OFFSET>
    __device__ __forceinline__ Words4 turn(int s, int d) const {
        const uint2 a = read_turned((Bytes)(uintptr_t)lo[d] + 2 * OFFSET + 32 * D * s);
        const uint2 b = read_turned((Bytes)(uintptr_t)hi[d] + 2 * OFFSET + 32 * D * s);
        return Words4{a.x, a.y, b.x, b.y};
    }
};

// The same with three places, from which the others are an exclusive or away: for a kernel that needs its registers.  An exclusive
// or takes the place of an addition within a row of 2 D bytes, so rows begin at a multiple of that.
template <int D>
struct SmallReader {
    using Bytes = __attribute__((address_space(3))) const char *;
    uint32_t rows, lo, hi;
    static_assert(alignof(Stages<D>) % (2 * D) == 0 && 32 * (D / 16 - 1) < 2 * D && 64 * (D / 32 - 1) < 2 * D);
    __device__ __forceinline__ SmallReader(const Stages<D> &lds, uint32_t lane) {
        const Reader<D> all(lds, lane);
        rows = all.rows[0];
        lo = all.lo[0];
        hi = all.hi[0];
    }
    template <uint32_t OFFSET>
    __device__ __forceinline__ Words4 row(int t, int s) const {
        return *(__attribute__((address_space(3))) const Words4 *)((Bytes)(uintptr_t)(rows ^ 32 * s) + 2 * OFFSET + 64 * D * t);
    }
    template <uint32_t OFFSET>
    __device__ __forceinline__ Words4 turn(int s, int d) const {
        const uint2 a = read_turned((Bytes)(uintptr_t)(lo ^ 64 * d) + 2 * OFFSET + 32 * D * s);
        const uint2 b = read_turned((Bytes)(uintptr_t)(hi ^ 64 * d) + 2 * OFFSET + 32 * D * s);
        return Words4{a.x, a.y, b.x, b.y};
    }
};

template <uint32_t N>
using At = std::integral_constant<uint32_t, N>;

// Eight values [16 s + 8 (lane / 32), ...) of a row in memory, zeros from `dim` on.
template <class T>
__device__ __forceinline__ Words4 piece_of(const typename T::raw *row, int s, uint32_t lane, uint32_t dim) {
    const uint32_t c = 16 * s + 8 * (lane / 32);
    return c < dim ? *(const Words4 *)(row + c) : Words4{};
}

// Of the scores' operand in registers: scores are kept as their products, which `scale` only stretches, so a scale below zero
// turns this operand's signs round, and one of zero makes it zero.
__device__ __forceinline__ Words4 directed(Words4 w, float scale) {
    const uint32_t flip = scale < 0.0f ? 0x80008000u : 0u, keep = scale == 0.0f ? 0u : ~0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (w[i] ^ flip) & keep;
    return w;
}
// Of base-2 exponents: finite up to POSEIDON_SCALE_MAX.
__device__ __forceinline__ float stretch(float scale) { return scale == 0.0f ? kLog2e : fabsf(scale) * kLog2e; }

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

// f16 holds eleven bits from 2^-14 to 2^16 alone.  Backward, p lies below that for most keys of a long row, and ds at the small
// gradients (or above it at the large ones) of a loss that nobody scaled.  So p goes to the products as p 2^14, and ds times a
// power of two of the lane's own, taken back from the sums: it falls, and the sums with it, where a ds passes 2^15, to where the
// largest lies at 2^10.  What then lies below 2^-14 is 2^-24 of the largest or less.  bf16 has the range of 32 bits.
// 8192 tokens, 8 heads on 2 of 128, dout of 0.001: dq off by 2.2e-3 of its norm without, 4.6e-4 with this, its rounding alone
// 4.0e-4.  32 heads on 8: 1853 us, without 1779.
template <class T>
constexpr bool kNarrow = std::is_same_v<T, F16>;
template <class T>
constexpr int kRaised = kNarrow<T> ? 14 : 0;
template <class T>
constexpr int kUnseen = kNarrow<T> ? 50 : 0;    // the power's exponent until a ds is too large for it
// `ds`: times 2^up already, as long as it fits; true where it had to fall.
template <class T, int D>
__device__ __forceinline__ bool fit(float (&ds)[16], Acc (&sum)[D / 32], int &up) {
    if constexpr (kNarrow<T>) {
        float most = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(ds[r]));
        most = larger_half(most);
        if (__any(most > 0x1p15f)) {
            const int down = most > 0x1p15f ? 11 - __builtin_amdgcn_frexp_expf(most) : 0;
            const float f = __builtin_amdgcn_ldexpf(1.0f, down);
#pragma unroll
            for (int d = 0; d < D / 32; ++d) sum[d] *= f;
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] *= f;
            up += down;
            return true;
        }
    }
    return false;
}

// Sums whose column is the lane's row, times f, to that row in memory.
template <class O, int D>
__device__ __forceinline__ void store_turned(const Acc (&sum)[D / 32], float f, typename O::raw *row, uint32_t dim, uint32_t lane) {
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
            if (row && c < dim) store_slice<O>(row, c, dim, v);
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

// f(token) for the tokens outside of all sequences that fall to block `block` of kClearBlocks.
template <class F>
__device__ __forceinline__ void outside(const Attention &a, uint32_t block, F f) {
    const uint32_t begin = bound_of(a.offsets, 0, a.tokens), end = max(begin, bound_of(a.offsets, a.sequences, a.tokens));
    for (uint32_t i = block; i < begin + a.tokens - end; i += kClearBlocks) f((uint64_t)(i < begin ? i : end + (i - begin)));
}
template <class T>
__device__ __forceinline__ void clear_token(const Heads &x, uint64_t token, uint32_t heads, uint32_t dim) {
    const float zero[8] = {};
    for (uint32_t i = threadIdx.x; i < heads * (dim / 8); i += blockDim.x)
        store_slice<T>((typename T::raw *)row_of<T>(x, token, i / (dim / 8)), i % (dim / 8) * 8, dim, zero);
}

// WAVES waves of 32 queries each.  The running largest score m follows a row's scores only when one outgrows it by 2^8:
// the sums then stay below 2^8 times the number of keys, and most tiles leave what was summed alone.
//
// Here and in the two kernels below two waves a SIMD, one in its products while the other is in its scores, share it: of 8192 tokens
// and 32 heads of 128 values on 8 the matrix units take 57 % of the time and vector instructions' issue 48 % (dq: 60 and 38, dk and dv:
// 61 and 36), so neither alone bounds a long sequence.  16384 tokens, 16 heads on 4: 990 us, 1110 TFLOP/s of the 1386 to 1596 that
// large products reach, at 1.65 GHz, no bank conflicts.  Eight waves a block: 1321 us where four took 1234.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_forward_kernel(Attention a) {
    constexpr uint32_t kQueries = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ Stages<D> lds;
    static_assert(sizeof lds == 2 * 2 * kStage);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.heads, id = a.first + blockIdx.x;
    if (id >= blocks) {
        outside(a, id - blocks, [&](uint64_t t) {
            clear_token<T>(a.out, t, a.heads, a.dim);
            for (uint32_t h = threadIdx.x; h < a.heads; h += blockDim.x) a.lse[(uint64_t)h * a.tokens + t] = -__builtin_inff();
        });
        return;
    }
    const Work w = work_of(id, a.heads, a.kv_heads);
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
        for (int s = 0; s < D / 16; ++s) query[s] = directed(piece_of<T>(row, s, lane, a.dim), a.scale);
    }
    const Loader<D, 64 * WAVES> loader(a.dim);
    const Reader<D> reader(lds, lane);
    const uint32_t k_place = loader.place(a.k.token), v_place = loader.place(a.v.token);
    const auto fetch = [&](uint32_t i) {
        const uint32_t t = begin + i * kTile, rows = at.end - t;
        uint16_t *to = lds.at + (i & 1) * kStage;
        loader.template load<T>(row_of<T>(a.k, t, w.kv), a.k.token, k_place, rows, to);
        loader.template load<T>(row_of<T>(a.v, t, w.kv), a.v.token, v_place, rows, to + kTile * D);
    };

    const float c = stretch(a.scale);
    float m = -__builtin_inff(), total = 0.0f;
    Acc sum[D / 32] = {};
    fetch(0);
    const auto step = [&](auto stage, uint32_t i) {
        constexpr uint32_t kKeys = decltype(stage)::value, kValues = kKeys + kTile * D;
        __builtin_amdgcn_s_waitcnt(0x0f70);    // vmcnt(0): this wave's part of the tile is in LDS
        __syncthreads();
        if (i + 1 < tiles) fetch(i + 1);
        const uint32_t t0 = begin + i * kTile;
        if (t0 > q0 + 31) return;            // all of it after the wave's queries
        Acc s[2] = {};
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) s[t] = mfma<T>(reader.template row<kKeys>(t, j), query[j], s[t]);
        then<kReadLds, 6>();
#pragma unroll
        for (int j = 0; j < D / 8 - 6; ++j) {
            then<kMatrix, 1>();
            then<kReadLds, 1>();
        }
        then<kMatrix, 6>();
        float p[2][16];
        float most = -__builtin_inff();
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) p[t][r] = s[t][r];
        if (t0 + kTile - 1 > q0) {
            const int last_key = (int)(q - t0) - (int)(4 * (lane / 32));
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + (r & 3) + 8 * (r >> 2) > last_key) p[t][r] = -__builtin_inff();
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
            for (int d = 0; d < D / 32; ++d) sum[d] = mfma<T>(reader.template turn<kValues>(j, d), w, sum[d]);
        }
    };
    for (uint32_t i = 0; i < tiles; i += 2) {
        step(At<0>{}, i);
        if (i + 1 < tiles) step(At<kStage>{}, i + 1);
    }
    total = sum_half(total);
    const bool there = q < at.end;
    store_turned<T, D>(sum, 1.0f / total, there ? (raw *)row_of<T>(a.out, q, w.head) : nullptr, a.dim, lane);
    if (there && lane < 32) a.lse[(uint64_t)w.head * a.tokens + q] = (m * c + __builtin_amdgcn_logf(total)) * kLn2;
}

// dq, as the forward pass goes, with delta = <dout, out> for the other kernel.  p and ds are rounded to the operands' type.
// 8192 tokens, 32 heads of 128 values on 8: 745 us, 1107 TFLOP/s, at 1.65 GHz.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_queries_kernel(Attention a) {
    constexpr uint32_t kQueries = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ Stages<D> lds;
    static_assert(sizeof lds == 2 * 2 * kStage);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.heads, id = a.first + blockIdx.x;
    if (id >= blocks) {
        outside(a, id - blocks, [&](uint64_t t) { clear_token<T>(a.dq, t, a.heads, a.dim); });
        return;
    }
    const Work w = work_of(id, a.heads, a.kv_heads);
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
            query[s] = directed(piece_of<T>(qr, s, lane, a.dim), a.scale);
            dout[s] = piece_of<T>(dr, s, lane, a.dim);
            const Words4 o = piece_of<T>(outr, s, lane, a.dim);
            raw x[8], y[8];
            __builtin_memcpy(x, &dout[s], 16);
            __builtin_memcpy(y, &o, 16);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf(T::up(x[i]), T::up(y[i]), delta);
        }
        delta = sum_half(delta);
    }
    const Loader<D, 64 * WAVES> loader(a.dim);
    const Reader<D> reader(lds, lane);
    const uint32_t k_place = loader.place(a.k.token), v_place = loader.place(a.v.token);
    const auto fetch = [&](uint32_t i) {
        const uint32_t t = begin + i * kTile, rows = at.end - t;
        uint16_t *to = lds.at + (i & 1) * kStage;
        loader.template load<T>(row_of<T>(a.k, t, w.kv), a.k.token, k_place, rows, to);
        loader.template load<T>(row_of<T>(a.v, t, w.kv), a.v.token, v_place, rows, to + kTile * D);
    };

    const float c = stretch(a.scale), lse = a.lse[(uint64_t)w.head * a.tokens + mine] * kLog2e;
    if (there && lane < 32) {
        a.delta[(uint64_t)w.head * a.tokens + q] = delta;
        a.base[(uint64_t)w.head * a.tokens + q] = kRaised<T> - lse;
    }
    Acc sum[D / 32] = {};
    int up = kUnseen<T>;
    float base = kUnseen<T> - lse;
    fetch(0);
    const auto step = [&](auto stage, uint32_t i) {
        constexpr uint32_t kKeys = decltype(stage)::value, kValues = kKeys + kTile * D;
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        if (i + 1 < tiles) fetch(i + 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t t0 = begin + i * kTile + 32 * t;
            if (t0 > q0 + 31) continue;
            Acc s = {}, dp = {};
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                s = mfma<T>(reader.template row<kKeys>(t, j), query[j], s);
                dp = mfma<T>(reader.template row<kValues>(t, j), dout[j], dp);
            }
            then<kReadLds, 6>();
#pragma unroll
            for (int j = 0; j < D / 8 - 6; ++j) {
                then<kMatrix, 1>();
                then<kReadLds, 1>();
            }
            then<kMatrix, 6>();
            float ds[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, base)) * (dp[r] - delta);
            if (t0 + 31 > q0) {
                const int last_key = (int)(q - t0) - (int)(4 * (lane / 32));
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((r & 3) + 8 * (r >> 2) > last_key) ds[r] = 0.0f;
            }
            if (fit<T, D>(ds, sum, up)) base = up - lse;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Words4 w = packed<T>(ds, j);
#pragma unroll
                for (int d = 0; d < D / 32; ++d) sum[d] = mfma<T>(reader.template turn<kKeys>(2 * t + j, d), w, sum[d]);
            }
        }
    };
    for (uint32_t i = 0; i < tiles; i += 2) {
        step(At<0>{}, i);
        if (i + 1 < tiles) step(At<kStage>{}, i + 1);
    }
    store_turned<T, D>(sum, __builtin_amdgcn_ldexpf(a.scale, -up), there ? (raw *)row_of<T>(a.dq, q, w.head) : nullptr, a.dim, lane);
}

// dk and dv: WAVES waves of 32 keys each go through the queries of every head that shares them, in one order.  With 128
// values a head the keys, the values and both sums would leave no registers for what is read ahead, so some of the
// values lie in LDS.  The same 8192 tokens: 965 us, 1139 TFLOP/s, at 1.65 GHz.  Eight waves a block: 1905 us
// where four took 1678; one wave a SIMD with the next scores beside its products: 1772.
template <class T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_keys_kernel(Attention a) {
    constexpr uint32_t kKeys = 32 * WAVES, kStage = 2 * kTile * D;
    __shared__ Stages<D> lds;
    static_assert(sizeof lds == 2 * 2 * kStage);
    __shared__ __attribute__((aligned(16))) float rows[2][2][kTile];    // base and delta
    constexpr int kHeld = D == 128 ? 5 : D / 16, kSpare = D / 16 - kHeld;
    __shared__ Words4 spare[kSpare ? WAVES * kSpare * 64 : 1];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = a.tiles * a.split * a.kv_heads, id = a.first + blockIdx.x;
    if (id >= blocks) {
        outside(a, id - blocks, [&](uint64_t t) {
            clear_token<T>(a.dk, t, a.kv_heads, a.dim);
            clear_token<T>(a.dv, t, a.kv_heads, a.dim);
        });
        return;
    }
    const uint32_t kv = id % a.kv_heads, group = a.heads / a.kv_heads / a.split;
    const uint32_t tile = id / a.kv_heads / a.split, part = id / a.kv_heads % a.split;
    const uint32_t head0 = (kv * a.split + part) * group;    // the first of the block's query heads
    uint32_t begin;    // keys early in a sequence have the most queries: these first
    const Place at = sequence_of(a, tile, kKeys, begin);
    if (!at.there) return;
    const uint32_t k0 = at.begin + 32 * wave, key = k0 + lane % 32;
    const bool there = key < at.end;
    const uint32_t tiles = (at.end - at.begin + kTile - 1) / kTile;    // of queries, from the block's first key on

    using raw = typename T::raw;
    Words4 keys[D / 16], vals[kHeld];
    Words4 *const rest = spare + wave * (kSpare * 64) + lane;
    {
        const uint32_t mine = min(key, at.end - 1);
        const raw *kr = row_of<T>(a.k, mine, kv), *vr = row_of<T>(a.v, mine, kv);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            keys[s] = directed(piece_of<T>(kr, s, lane, a.dim), a.scale);
            const Words4 v = piece_of<T>(vr, s, lane, a.dim);
            if (s < kHeld)
                vals[s] = v;
            else
                rest[(s - kHeld) * 64] = v;
        }
    }
    const Loader<D, 64 * WAVES> loader(a.dim);
    const SmallReader<D> all(lds, lane);
    const uint32_t q_place = loader.place(a.q.token), dout_place = loader.place(a.dout.token);
    // From the last queries down, all heads at each: blocks that run together then ask for the same rows.
    uint32_t asked = tiles - 1, g = 0;
    bool more = true;
    const auto fetch = [&](uint32_t set) {    // the next tile
        if (!more) return;
        const uint32_t t = at.begin + asked * kTile, n = at.end - t, head = head0 + g;
        uint16_t *to = lds.at + set * kStage;
        loader.template load<T>(row_of<T>(a.q, t, head), a.q.token, q_place, n, to);
        loader.template load<T>(row_of<T>(a.dout, t, head), a.dout.token, dout_place, n, to + kTile * D);
        if (wave < 2) {    // rows past the end: zeros, as q and dout have there
            const float *from = (wave ? a.delta : a.base) + (uint64_t)head * a.tokens + t;
            const auto to = (__attribute__((address_space(3))) void *)rows[set][wave];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer(from, __builtin_amdgcn_readfirstlane(min(n, kTile) * 4)), to, 4, lane * 4, 0, 0, 0);
        }
        if (++g == group) {
            g = 0;
            more = asked-- != 0;
        }
    };

    const float c = stretch(a.scale);
    Acc dk[D / 32] = {}, dv[D / 32] = {};
    int up = kUnseen<T>;
    const auto use = [&](auto stage, int t, uint32_t t0) {    // 32 queries
        constexpr uint32_t kSet = decltype(stage)::value, kQueries = kSet * kStage, kDout = kQueries + kTile * D;
        if (t0 + 31 < k0) return;    // all of them before the wave's keys
        SmallReader<D> reader = all;
        uint32_t half = lane / 32;
        asm("" : "+v"(reader.rows), "+v"(reader.lo), "+v"(reader.hi), "+v"(half));    // places are found where they are used, not kept
        // What LDS gives is asked for two products of a kind before its use, and no earlier: there are no registers for more.
        Words4 x[2], y[2], z[2];
        const auto ask_x = [&](int j) { x[j & 1] = reader.template row<kQueries>(t, j); };
        const auto ask_y = [&](int j) {
            y[j & 1] = reader.template row<kDout>(t, j);
            if (j >= kHeld) z[j & 1] = rest[(j - kHeld) * 64];
        };
        Acc s = {}, dp = {};
        ask_x(0);
        ask_y(0);
        ask_x(1);
        ask_y(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            s = mfma<T>(x[j & 1], keys[j], s);
            if (j + 2 < D / 16) ask_x(j + 2);
            __builtin_amdgcn_sched_barrier(0);
            dp = mfma<T>(y[j & 1], j < kHeld ? vals[j] : z[j & 1], dp);
            if (j + 2 < D / 16) ask_y(j + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        float p[16], ds[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t r0 = 32 * t + 8 * q + 4 * half;
            const float4 base = *(const float4 *)&rows[kSet][0][r0], delta = *(const float4 *)&rows[kSet][1][r0];
            const float l[4] = {base.x, base.y, base.z, base.w}, d[4] = {delta.x, delta.y, delta.z, delta.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * q + e;
                p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, l[e]));
                ds[r] = p[r] * (dp[r] - d[e]);
                if constexpr (kNarrow<T>) ds[r] = __builtin_amdgcn_ldexpf(ds[r], up);
            }
        }
        if (t0 < k0 + 31) {
            const int before = (int)(key - t0) - (int)(4 * half);    // the first of these queries come before the key
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if ((r & 3) + 8 * (r >> 2) < before) p[r] = ds[r] = 0.0f;
        }
        fit<T, D>(ds, dk, up);
        const Words4 pw[2] = {packed<T>(p, 0), packed<T>(p, 1)}, dw[2] = {packed<T>(ds, 0), packed<T>(ds, 1)};
        Words4 u[3], v[3];
        const auto ask_turned = [&](int j) {
            u[j % 3] = reader.template turn<kDout>(2 * t + j / (D / 32), j % (D / 32));
            v[j % 3] = reader.template turn<kQueries>(2 * t + j / (D / 32), j % (D / 32));
        };
        ask_turned(0);
        ask_turned(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            if (j + 2 < D / 16) ask_turned(j + 2);
            constexpr int kTurns = D / 32;
            dv[j % kTurns] = mfma<T>(u[j % 3], pw[j / kTurns], dv[j % kTurns]);
            dk[j % kTurns] = mfma<T>(v[j % 3], dw[j / kTurns], dk[j % kTurns]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    uint32_t first = at.begin + (tiles - 1) * kTile, heads = 0;
    const uint64_t turns = (uint64_t)tiles * group;
    fetch(0);
    const auto step = [&](auto stage) {
        constexpr uint32_t kSet = decltype(stage)::value;
        __builtin_amdgcn_s_waitcnt(0x0f70);    // vmcnt(0): this wave's part of the tile is in LDS
        __syncthreads();
        fetch(kSet ^ 1);
        use(stage, 0, first);
        use(stage, 1, first + 32);
        if (++heads == group) {
            heads = 0;
            first -= kTile;
        }
    };
    for (uint64_t turn = 0; turn < turns; turn += 2) {
        step(At<0>{});
        if (turn + 1 < turns) step(At<1>{});
    }
    constexpr float kDown = kNarrow<T> ? 0x1p-14f : 1.0f;
    const float dk_down = __builtin_amdgcn_ldexpf(a.scale, -kRaised<T> - up);
    if (a.split == 1) {
        store_turned<T, D>(dk, dk_down, there ? (raw *)row_of<T>(a.dk, key, kv) : nullptr, a.dim, lane);
        store_turned<T, D>(dv, kDown, there ? (raw *)row_of<T>(a.dv, key, kv) : nullptr, a.dim, lane);
    } else {
        const uint64_t whole = (uint64_t)a.tokens * a.kv_heads * a.dim;
        float *to = a.parts + 2 * part * whole + ((uint64_t)key * a.kv_heads + kv) * a.dim;
        store_turned<F32, D>(dk, dk_down, there ? to : nullptr, a.dim, lane);
        store_turned<F32, D>(dv, kDown, there ? to + whole : nullptr, a.dim, lane);
    }
}

// dk and dv of the blocks that share a key's query heads, in order: eight values a lane.  Memory bounds it (the 8192
// tokens in two parts: 26 us for 168 MB, 6.4 TB/s).
template <class T>
__global__ __launch_bounds__(kBlock) void attention_join_kernel(Attention a) {
    const uint32_t per_token = a.kv_heads * (a.dim / 8);
    const uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const uint32_t token = (uint32_t)(i / per_token), at = (uint32_t)(i % per_token);
    if (i >= (uint64_t)a.tokens * per_token) return;
    if (a.offsets && (token < bound_of(a.offsets, 0, a.tokens) || token >= bound_of(a.offsets, a.sequences, a.tokens))) return;
    const uint64_t whole = (uint64_t)a.tokens * a.kv_heads * a.dim;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float sum[8] = {};
        for (uint32_t s = 0; s < a.split; ++s) {
            float v[8];
            load_slice<F32>(a.parts + (2 * s + w) * whole + i * 8, 0, 8, v);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] += v[c];
        }
        const Heads &to = w ? a.dv : a.dk;
        store_slice<T>((typename T::raw *)row_of<T>(to, token, at / (a.dim / 8)) + at % (a.dim / 8) * 8, 0, 8, sum);
    }
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
    if (fabsf(scale) > POSEIDON_SCALE_MAX || tokens > POSEIDON_ROWS_MAX || heads > POSEIDON_HEADS_MAX || dim > POSEIDON_HEAD_MAX || sequences > POSEIDON_ROWS_MAX)
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

inline uint64_t attention_tiles(uint64_t tokens, uint64_t sequences) {
    const uint32_t size = 32 * kWaves;
    return sequences ? tiles_for(tokens, sequences, size) : (tokens + size - 1) / size;
}

// Blocks that share a key's query heads, each with some of them: the keys with the most queries take longest and would go on
// alone.  1024 blocks, two for each that the chip has at a time, are enough for one sequence (8192 tokens, 32 heads on 8: 1444 us
// in 512 blocks, 1100 in 1024, 1111 in 2048, the sum of parts counted), 2048 for several, whose longest may
// come late (16384 tokens in 24 sequences, 16 heads on 8: 446 us in 1216 blocks, 413 in 2432).  The sums of parts take 1 GB at most.
inline uint32_t split_of(uint64_t tokens, uint64_t sequences, uint64_t heads, uint64_t kv_heads, uint64_t dim) {
    const uint64_t group = heads / kv_heads, blocks = attention_tiles(tokens, sequences) * kv_heads;
    const uint64_t least = sequences > 1 ? 2048 : 1024;
    uint64_t n = 1;
    while (n < group && (blocks * n < least || group % n)) ++n;
    while (n > 1 && (group % n || n * tokens * kv_heads * dim * 8 > 1ull << 30)) --n;
    return (uint32_t)n;
}

template <class K>
inline int run_attention(K kernel, Attention &a, uint64_t heads, void *hip_stream) {
    constexpr uint32_t waves = kWaves;
    const uint64_t tiles = attention_tiles(a.tokens, a.offsets ? a.sequences : 0);
    if (tiles * heads > kBlocksMost) return POSEIDON_E_RANGE;
    a.tiles = (uint32_t)tiles;
    return launch_blocks(kernel, a, tiles * heads + (a.offsets ? kClearBlocks : 0), 64 * waves, hip_stream);
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
        return run_attention(attention_forward_kernel<decltype(t), d.value, kWaves>, a, heads, hip_stream);
    });
}

uint64_t poseidon_attention_backward_workspace(uint64_t tokens, uint32_t heads, uint32_t kv_heads, uint32_t dim, uint32_t sequences) {
    if (check_attention(tokens, heads, kv_heads, dim, 1.0f, nullptr, 1) != POSEIDON_OK) return UINT64_MAX;
    uint64_t parts = 0;
    for (const uint64_t n : {(uint64_t)sequences, (uint64_t)0}) {    // the call may come without offsets
        const uint64_t split = split_of(tokens, n, heads, kv_heads, dim);
        if (split > parts) parts = split;
    }
    return tokens * heads * 8 + (parts > 1 ? parts * tokens * kv_heads * dim * 8 : 0);
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
    PL_TRY(check_workspace(workspace, workspace_bytes, poseidon_attention_backward_workspace(tokens, heads, kv_heads, dim, sequences)));
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
    a.base = a.delta + tokens * heads;
    a.parts = a.base + tokens * heads;
    a.split = split_of(tokens, offsets ? sequences : 0, heads, kv_heads, dim);
    a.offsets = offsets;
    a.tokens = (uint32_t)tokens;
    a.sequences = sequences;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.dim = dim;
    a.scale = scale;
    return for_heads(type, dim, [&](auto t, auto d) -> int {
        PL_TRY(run_attention(attention_queries_kernel<decltype(t), d.value, kWaves>, a, heads, hip_stream));
        PL_TRY(run_attention(attention_keys_kernel<decltype(t), d.value, kWaves>, a, (uint64_t)kv_heads * a.split, hip_stream));
        if (a.split == 1) return POSEIDON_OK;
        const uint64_t slices = tokens * kv_heads * (dim / 8);
        attention_join_kernel<decltype(t)><<<(uint32_t)((slices + kBlock - 1) / kBlock), kBlock, 0, (hipStream_t)hip_stream>>>(a);
        return launched();
    });
}

}  // extern "C"
