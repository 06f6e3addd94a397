// Products of rows with the weights of their range (poseidon_layers.h), for experts over ragged ranges and for one
// matrix: y[t] = W[r] x[t] forward, dx[t] = W[r]^T dy[t] backward, r the range of row t.
#include "layers_mfma.h"

#include <type_traits>

namespace pl {

constexpr uint32_t kDeep = 64;           // values along the sum in a step
constexpr uint32_t kClearing = 64;       // blocks that look for rows outside of all ranges

struct Product {
    const void *x, *weights;
    uint64_t pitch, out_pitch;
    uint32_t rows, ranges, deep, wide;    // deep: values that are summed, wide: values of an output row
    const int32_t *offsets;               // null: one range of all rows
    uint32_t tiles_r, tiles_c;            // tiles of rows (an upper bound), and of columns
    void *out;
    uint32_t out_type;
};

// Blocks go round the eight XCDs in turn, each with an L2 of its own, so an XCD takes a run of neighbouring tiles, which goes
// through them eight rows of tiles high: the 32 blocks on its CUs share 8 tiles of rows and 4 of weights.
struct Tile {
    uint32_t r, c;
};
__device__ __forceinline__ Tile tile_of(uint32_t id, uint32_t all, uint32_t tiles_r, uint32_t tiles_c) {
    constexpr uint32_t kHigh = 8;
    const uint32_t xcd = id & 7;
    id = xcd * (all / 8) + min(xcd, all & 7) + id / 8;
    const uint32_t band = id / (kHigh * tiles_c), high = min(kHigh, tiles_r - kHigh * band);
    id -= band * kHigh * tiles_c;
    return {kHigh * band + id % high, id / high};
}

template <class T>
__device__ __forceinline__ void clear_outside(const Product &g, uint32_t block, uint32_t blocks, uint32_t threads) {
    const uint32_t begin = bound_of(g.offsets, 0, g.rows), end = max(begin, bound_of(g.offsets, g.ranges, g.rows));
    const uint32_t gone = begin + g.rows - end, per_row = (g.wide + kSlice - 1) / kSlice;
    const float zero[8] = {};
    for (uint32_t i = block; i < gone; i += blocks) {
        const uint64_t row = i < begin ? i : end + (i - begin);
        for (uint32_t s = threadIdx.x; s < per_row; s += threads) {
            if (g.out_type == POSEIDON_F32)
                store_slice<F32>((float *)g.out + row * g.out_pitch, s * kSlice, g.wide, zero);
            else
                store_slice<T>((typename T::raw *)g.out + row * g.out_pitch, s * kSlice, g.wide, zero);
        }
    }
}

// R x C waves on a tile of 32 R M rows by 32 C N columns, 32 M x 32 N a wave.
// TURNED: W^T, whose values along the sum are a row apart.
template <class T, bool TURNED, bool ALIGNED, int R, int C, int M, int N>
__global__ __launch_bounds__(64 * R * C, 2) void product_kernel(Product g) {
    constexpr uint32_t kRows = 32 * R * M, kCols = 32 * C * N, kThreads = 64 * R * C;
    constexpr uint32_t kX = kRows * kDeep, kW = kCols * kDeep;    // values of a step
    constexpr uint32_t kLoadsX = kX / 8 / kThreads, kLoadsW = kW / 8 / kThreads;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * (kX + kW)];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const uint32_t tiles = g.tiles_r * g.tiles_c;
    if (blockIdx.x >= tiles) {
        clear_outside<T>(g, blockIdx.x - tiles, gridDim.x - tiles, kThreads);
        return;
    }
    const Tile tile = tile_of(blockIdx.x, tiles, g.tiles_r, g.tiles_c);
    Place at = {0, tile.r * kRows, g.rows, tile.r * kRows < g.rows};
    if (g.offsets) at = place_of(g.offsets, g.ranges, g.rows, tile.r, kRows);
    if (!at.there) return;
    const uint32_t row0 = at.begin, here = min(at.end - row0, kRows), col0 = tile.c * kCols;
    using raw = typename T::raw;
    const raw *x = (const raw *)g.x + row0 * g.pitch;
    const raw *w = (const raw *)g.weights + (uint64_t)at.range * g.deep * g.wide + (TURNED ? col0 : (uint64_t)col0 * g.deep);
    const uint32_t steps = (g.deep + kDeep - 1) / kDeep;

    // Rows of LDS hold 64 values along the sum in eight pieces of 16 bytes; piece p lies at p ^ (row & 7), so that
    // neighbouring lanes' rows, 128 bytes apart, are read from all banks.  TURNED: rows of kCols values of W, piece p
    // at p ^ 4 (row & 3), so that four rows are read from all banks.
    uint32_t x_at[kLoadsX], x_col[kLoadsX], w_at[kLoadsW], w_col[kLoadsW];
    uint64_t x_row[kLoadsX], w_row[kLoadsW];
#pragma unroll
    for (uint32_t i = 0; i < kLoadsX; ++i) {
        const uint32_t piece = i * kThreads + tid, row = piece / 8;
        x_col[i] = ((piece ^ row) & 7) * 8;
        x_row[i] = (uint64_t)min(row, here - 1) * g.pitch;
        x_at[i] = (uint32_t)(x_row[i] + x_col[i]) * 2;
    }
#pragma unroll
    for (uint32_t i = 0; i < kLoadsW; ++i) {
        const uint32_t piece = i * kThreads + tid;
        if constexpr (TURNED) {
            const uint32_t k = piece / (kCols / 8);
            w_col[i] = (piece % (kCols / 8) ^ 4 * (k & 3)) * 8;
            w_row[i] = k;
            w_at[i] = col0 + w_col[i] < g.wide ? (k * g.wide + w_col[i]) * 2 : kNowhere;
        } else {
            const uint32_t row = piece / 8;
            w_col[i] = ((piece ^ row) & 7) * 8;
            w_row[i] = (uint64_t)min(row, g.wide - 1 - col0) * g.deep;
            w_at[i] = (uint32_t)(w_row[i] + w_col[i]) * 2;
        }
    }
    Words4 held_x[ALIGNED ? 1 : kLoadsX], held_w[ALIGNED ? 1 : kLoadsW];
    const auto fetch = [&](uint32_t step) {    // asks for a step's values; ALIGNED: right into LDS
        const uint32_t k0 = step * kDeep;
        if constexpr (ALIGNED) {
            uint16_t *to = lds + (step & 1) * (kX + kW) + wave * 512;
            const Rsrc from_x = buffer(x + k0, kBufferBytes);
            const Rsrc from_w = buffer(TURNED ? w + (uint64_t)k0 * g.wide : w + k0, kBufferBytes);
#pragma unroll
            for (uint32_t i = 0; i < kLoadsX; ++i)
                copy_to_lds(from_x, k0 + x_col[i] < g.deep ? x_at[i] : kNowhere, to + i * kThreads * 8);
#pragma unroll
            for (uint32_t i = 0; i < kLoadsW; ++i)
                copy_to_lds(from_w, k0 + (TURNED ? (uint32_t)w_row[i] : w_col[i]) < g.deep ? w_at[i] : kNowhere,
                            to + kX + i * kThreads * 8);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kLoadsX; ++i) {
                const Slice<T> s = load_words<T>(x + x_row[i], k0 + x_col[i], g.deep);
                held_x[i] = Words4{s.w[0], s.w[1], s.w[2], s.w[3]};
            }
#pragma unroll
            for (uint32_t i = 0; i < kLoadsW; ++i) {
                Slice<T> s;
                if constexpr (TURNED) {
                    const uint32_t k = k0 + (uint32_t)w_row[i];
                    s = load_words<T>(w - col0 + (uint64_t)min(k, g.deep - 1) * g.wide, col0 + w_col[i], g.wide);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s.w[j] = k < g.deep ? s.w[j] : 0u;
                } else {
                    s = load_words<T>(w + w_row[i], k0 + w_col[i], g.deep);
                }
                held_w[i] = Words4{s.w[0], s.w[1], s.w[2], s.w[3]};
            }
        }
    };
    const auto deposit = [&](uint32_t step) {
        if constexpr (!ALIGNED) {
            Words4 *to = (Words4 *)(lds + (step & 1) * (kX + kW)) + tid;
#pragma unroll
            for (uint32_t i = 0; i < kLoadsX; ++i) to[i * kThreads] = held_x[i];
#pragma unroll
            for (uint32_t i = 0; i < kLoadsW; ++i) to[kX / 8 + i * kThreads] = held_w[i];
        }
    };

    const uint32_t r0 = wave / C * 32 * M, c0 = wave % C * 32 * N, l32 = lane % 32, half = lane / 32;
    const auto read_x = [&](uint32_t step, int s, int m) {
        return *(const Words4 *)(lds + (step & 1) * (kX + kW) + (r0 + 32 * m + l32) * kDeep + ((2 * s + half) ^ (l32 & 7)) * 8);
    };
    const auto read_w = [&](uint32_t step, int s, int n) {
        const uint16_t *from = lds + (step & 1) * (kX + kW) + kX;
        if constexpr (TURNED) {
            const uint32_t k = 8 * half + lane % 16 / 4, piece = (c0 / 8 + 4 * n) ^ 4 * (k & 3);
            from += (16 * s + k) * kCols + (piece + 2 * (lane / 16 % 2) + lane % 4 / 2) * 8 + lane % 2 * 4;
            const uint2 lo = read_turned(from), hi = read_turned(from + 4 * kCols);
            return Words4{lo.x, lo.y, hi.x, hi.y};
        } else {
            return *(const Words4 *)(from + (c0 + 32 * n + l32) * kDeep + ((2 * s + half) ^ (l32 & 7)) * 8);
        }
    };

    Acc acc[M][N] = {};
    fetch(0);
    deposit(0);
    for (uint32_t step = 0; step < steps; ++step) {
        if constexpr (ALIGNED) __builtin_amdgcn_s_waitcnt(0x0f70);    // vmcnt(0): this wave's part of the step is in LDS
        __syncthreads();
        if (step + 1 < steps) fetch(step + 1);
        Words4 a[2][M], b[2][N];
#pragma unroll
        for (int m = 0; m < M; ++m) a[0][m] = read_x(step, 0, m);
#pragma unroll
        for (int n = 0; n < N; ++n) b[0][n] = read_w(step, 0, n);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) {
#pragma unroll
                for (int m = 0; m < M; ++m) a[(s + 1) & 1][m] = read_x(step, s + 1, m);
#pragma unroll
                for (int n = 0; n < N; ++n) b[(s + 1) & 1][n] = read_w(step, s + 1, n);
            }
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int n = 0; n < N; ++n) acc[m][n] = mfma<T>(b[s & 1][n], a[s & 1][m], acc[m][n]);
        }
        if (step + 1 < steps) deposit(step + 1);
    }

    // A lane has a row, and of each 32 columns 4 of every 8: the two halves of the wave trade theirs, so that a lane
    // writes eight neighbouring ones.
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const uint32_t r = r0 + 32 * m + l32;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float lo = acc[m][n][8 * q + i], hi = acc[m][n][8 * q + 4 + i];
                    const float other = __shfl_xor(half ? lo : hi, 32, 64);
                    v[i] = half ? other : lo;
                    v[4 + i] = half ? hi : other;
                }
                const uint32_t col = col0 + c0 + 32 * n + 16 * q + 8 * half;
                if (r >= here || col >= g.wide) continue;
                const uint64_t row = row0 + r;
                if (g.out_type == POSEIDON_F32)
                    store_slice<F32>((float *)g.out + row * g.out_pitch, col, g.wide, v);
                else
                    store_slice<T>((raw *)g.out + row * g.out_pitch, col, g.wide, v);
            }
    }
}

}  // namespace pl

using namespace pl;

extern "C" {

int poseidon_expert_product(const void *x, uint64_t pitch, uint32_t type, uint64_t rows, const void *weights,
                            uint64_t out_width, uint64_t in_width, uint32_t transposed, const int32_t *offsets,
                            uint32_t n_ranges, void *out, uint64_t out_pitch, uint32_t out_type, void *hip_stream) {
    PL_TRY(check_sizes(rows, out_width));
    PL_TRY(check_sizes(rows, in_width));
    if (!n_ranges || (!offsets && n_ranges != 1) || transposed > 1) return POSEIDON_E_INVAL;
    if (n_ranges > POSEIDON_EXPERTS_MAX) return POSEIDON_E_RANGE;
    if (type != POSEIDON_F16 && type != POSEIDON_BF16) return POSEIDON_E_INVAL;
    if (out_type != type && out_type != POSEIDON_F32) return POSEIDON_E_INVAL;
    const uint64_t deep = transposed ? out_width : in_width, wide = transposed ? in_width : out_width;
    PL_TRY(check_matrix(x, pitch, type, rows, deep));
    PL_TRY(check_matrix(weights, wide, type, rows, wide));
    PL_TRY(check_matrix(out, out_pitch, out_type, rows, wide));
    if (rows && !aligned(offsets, 4)) return POSEIDON_E_INVAL;
    if (!rows) return POSEIDON_OK;
    Product g = {x, weights, pitch, out_pitch, (uint32_t)rows, n_ranges, (uint32_t)deep, (uint32_t)wide, offsets, 0, 0, out, out_type};
    // 16-byte pieces that lie on 16 bytes and end with the row, at offsets of less than 2^31 bytes within a tile
    const bool whole = deep % 8 == 0 && in_width % 8 == 0 && pitch % 8 == 0 && aligned(x, 16) && aligned(weights, 16) &&
                       pitch < (1u << 21) ;
    const auto run = [&](auto kernel, uint32_t tile_r, uint32_t tile_c, uint32_t threads) -> int {
        const uint64_t r = offsets ? tiles_for(rows, n_ranges, tile_r) : (rows + tile_r - 1) / tile_r, c = (wide + tile_c - 1) / tile_c;
        if (r * c > 0x7fffff00ull) return POSEIDON_E_RANGE;
        g.tiles_r = (uint32_t)r;
        g.tiles_c = (uint32_t)c;
        kernel<<<(uint32_t)(r * c) + (offsets ? kClearing : 0), threads, 0, (hipStream_t)hip_stream>>>(g);
        return launched();
    };
    const uint64_t large = tiles_for(rows, n_ranges, 256) * ((wide + 255) / 256);
    const auto pick = [&](auto t, auto turned, auto whole_) -> int {
        using T = decltype(t);
        constexpr bool kTurned = decltype(turned)::value, kWhole = decltype(whole_)::value;
        return large >= 256 ? run(product_kernel<T, kTurned, kWhole, 2, 4, 4, 2>, 256, 256, 512)
                            : run(product_kernel<T, kTurned, kWhole, 2, 2, 2, 2>, 128, 128, 256);
    };
    const auto of = [&](auto t) -> int {
        using Yes = std::true_type;
        using No = std::false_type;
        if (transposed) return whole ? pick(t, Yes{}, Yes{}) : pick(t, Yes{}, No{});
        return whole ? pick(t, No{}, Yes{}) : pick(t, No{}, No{});
    };
    return type == POSEIDON_F16 ? of(F16{}) : of(BF16{});
}

}  // extern "C"
