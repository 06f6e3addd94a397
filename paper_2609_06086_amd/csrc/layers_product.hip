// Products of rows with the weights of their range (poseidon_layers.h), for experts over ragged ranges and for one
// matrix: y[t] = W[r] x[t] forward, dx[t] = W[r]^T dy[t] backward, r the range of row t.
#include "layers_mfma.h"

namespace pl {

constexpr uint32_t kDeep = 64;           // values along the sum in a stage
constexpr uint32_t kClearing = 64;       // blocks that look for rows outside of all ranges

struct Product {
    const void *x, *weights;
    uint64_t pitch, out_pitch;
    uint32_t rows, ranges, deep, wide;    // deep: values that are summed, wide: values of an output row
    const int32_t *offsets;               // null: one range of all rows
    uint32_t tiles_r, tiles_c, first;     // tiles of rows (an upper bound), and of columns; block of this launch
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
__device__ __forceinline__ void clear_outside(const Product &g, uint32_t block, uint32_t threads) {
    const uint32_t begin = bound_of(g.offsets, 0, g.rows), end = max(begin, bound_of(g.offsets, g.ranges, g.rows));
    const uint32_t gone = begin + g.rows - end, per_row = (g.wide + kSlice - 1) / kSlice;
    const float zero[8] = {};
    for (uint32_t i = block; i < gone; i += kClearing) {
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
// TURNED: W^T, whose values along the sum are a row apart.  ALIGNED: rows begin on 16 bytes and are whole pieces of 16 bytes, which
// go to LDS without a register between; else they are read with plain loads, which take any address, and masked.
//
// LDS holds X stages (two or three) of 64 values along the sum, 128 bytes of a row, of x and three of the weights, which come
// from further away: other rows of them for every stage of W^T.  The last of a stage's operands are in registers when
// a quarter of its products is still to come: there the waves meet, the stage's place is given to the one after the
// next, and the next one's first operands are read beside the last products, so that no wave waits for LDS at a stage's start.
//
// 16384 rows of 8192 values by 4096 x 8192 take 862 us (1275 TFLOP/s; the library's product 844 to 881), W^T of 8192 x 4096 1030 us
// (1068; the library's 966 to 1000), 64 ragged ranges of 65536 rows by 4096 x 2048 1150 us (956).  In the last two the matrix units
// are busy for 51 % of the time at 1.67 GHz, and waves wait for memory, barriers and LDS for 32 % of theirs: a block has its CU
// alone, so its first loads and its stores have nothing beside them.  No bank conflicts.  Stages of 32 values with four places: the ragged ranges
// 1530 us where those of 64 took 1347.
template <class T, bool TURNED, bool ALIGNED, int R, int C, int M, int N, int X>
__global__ __launch_bounds__(64 * R * C, 2) void product_kernel(Product g) {
    constexpr uint32_t kRows = 32 * R * M, kCols = 32 * C * N, kThreads = 64 * R * C;
    constexpr uint32_t kX = kRows * kDeep, kW = kCols * kDeep, kStageW = X * kX;    // values of a stage; where the weights begin
    constexpr uint32_t kLoadsX = kX / 8 / kThreads, kLoadsW = kW / 8 / kThreads;
    constexpr uint32_t kPieces = kDeep / 8;                                         // of a row
    __shared__ __attribute__((aligned(16))) uint16_t lds[X * kX + 3 * kW];    // stages of x, then those of the weights
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const uint32_t tiles = g.tiles_r * g.tiles_c, id = g.first + blockIdx.x;
    if (id >= tiles) {
        clear_outside<T>(g, id - tiles, kThreads);
        return;
    }
    const Tile tile = tile_of(id, tiles, g.tiles_r, g.tiles_c);
    Place at = {0, tile.r * kRows, g.rows, tile.r * kRows < g.rows};
    if (g.offsets) at = place_of(g.offsets, g.ranges, g.rows, tile.r, kRows);
    if (!at.there) return;
    const uint32_t row0 = at.begin, here = min(at.end - row0, kRows), col0 = tile.c * kCols;
    using raw = typename T::raw;
    const raw *x = (const raw *)g.x + row0 * g.pitch;
    const raw *w = (const raw *)g.weights + (uint64_t)at.range * g.deep * g.wide + (TURNED ? col0 : (uint64_t)col0 * g.deep);
    const uint32_t stages = (g.deep + kDeep - 1) / kDeep;

    // Rows of LDS are eight pieces of 16 bytes; piece p lies at p ^ (row / 2 & 7), so that sixteen rows' are read from banks
    // of their own.  TURNED: rows of kCols values of W, piece p at p ^ 4 (row & 3), for four rows' next four pieces.
    // A lane's pieces of a stage lie at the same place of rows a multiple of 16 (4) apart.
    const uint32_t x_row = tid / kPieces, x_col = ((tid ^ x_row / 2) & 7) * 8;
    const uint32_t w_row = TURNED ? tid / (kCols / 8) : x_row, w_col = TURNED ? (tid % (kCols / 8) ^ 4 * (w_row & 3)) * 8 : x_col;
    constexpr uint32_t kStepX = kThreads / kPieces, kStepW = TURNED ? kThreads / (kCols / 8) : kStepX;    // rows from piece to piece
    static_assert(kStepX % 16 == 0 && kStepW % 4 == 0);
    const uint32_t x_at = (x_row * (uint32_t)g.pitch + x_col) * 2;
    const uint32_t w_at = TURNED ? (col0 + w_col < g.wide ? (w_row * g.wide + w_col) * 2 : kNowhere) : (w_row * g.deep + w_col) * 2;
    const uint32_t w_here = min(g.wide - col0, kCols), w_safe = col0 + w_col < g.wide ? w_col : 0;
    Words4 held_x[ALIGNED ? 1 : kLoadsX], held_w[ALIGNED ? 1 : kLoadsW];
    // A lane's pieces as buffers of their own, which end with the tile's rows and, TURNED, with the sum: only an offset
    // changes from stage to stage.
    Rsrc from_x[kLoadsX], from_w[kLoadsW];
    if constexpr (ALIGNED) {
#pragma unroll
        for (uint32_t i = 0; i < kLoadsX; ++i) {
            const uint32_t left = here > i * kStepX ? min(here - i * kStepX, kStepX) : 0;
            from_x[i] = buffer(x + i * kStepX * g.pitch, __builtin_amdgcn_readfirstlane(left * (uint32_t)g.pitch * 2));
        }
#pragma unroll
        for (uint32_t i = 0; i < kLoadsW; ++i) {
            const uint32_t row = i * kStepW, left = TURNED ? (g.deep > row ? g.deep - row : 0) : w_here > row ? min(w_here - row, kStepW) : 0;
            from_w[i] = buffer(w + (uint64_t)row * (TURNED ? g.wide : g.deep), __builtin_amdgcn_readfirstlane(left * (TURNED ? g.wide : g.deep) * 2));
        }
    }
    // Ask for a stage's values; ALIGNED: right into LDS.  Past the rows, the columns and the sum come zeros.
    const auto fetch_x = [&](uint32_t stage, auto place) __attribute__((always_inline)) {
        const uint32_t k0 = stage * kDeep;
        if constexpr (ALIGNED) {
            uint16_t *to = lds + decltype(place)::value * kX + wave * 512;
            const uint32_t offset = k0 + x_col < g.deep ? x_at + 2 * k0 : kNowhere;
#pragma unroll
            for (uint32_t i = 0; i < kLoadsX; ++i) copy_to_lds<TURNED>(from_x[i], offset, to + i * kThreads * 8);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kLoadsX; ++i) {
                const raw *row = x + min(x_row + i * kStepX, here - 1) * g.pitch;
                Slice<T> s;
                if (k0 + kDeep <= g.deep)
                    get<false>(s.w, row + k0 + x_col);
                else
                    s = load_words<T>(row, k0 + x_col, g.deep);
                held_x[i] = Words4{s.w[0], s.w[1], s.w[2], s.w[3]};
            }
        }
    };
    const auto fetch_w = [&](uint32_t stage, auto place) __attribute__((always_inline)) {
        const uint32_t k0 = stage * kDeep;
        if constexpr (ALIGNED) {
            uint16_t *to = lds + kStageW + decltype(place)::value * kW + wave * 512;
            const uint32_t offset = TURNED ? w_at + 2 * k0 * g.wide : k0 + w_col < g.deep ? w_at + 2 * k0 : kNowhere;
#pragma unroll
            for (uint32_t i = 0; i < kLoadsW; ++i) copy_to_lds<TURNED>(from_w[i], offset, to + i * kThreads * 8);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kLoadsW; ++i) {
                Slice<T> s;
                if constexpr (TURNED) {
                    const uint32_t k = k0 + w_row + i * kStepW;
                    const raw *row = w + (uint64_t)min(k, g.deep - 1) * g.wide;
                    if (k0 + kDeep < g.deep && g.wide >= kSlice) {    // past a row's end lies the next row: columns that nobody keeps
                        get<false>(s.w, row + w_safe);
                    } else {
                        s = load_words<T>(row - col0, col0 + w_col, g.wide);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s.w[j] = k < g.deep ? s.w[j] : 0u;
                    }
                } else {
                    const raw *row = w + (uint64_t)min(w_row + i * kStepW, w_here - 1) * g.deep;
                    if (k0 + kDeep <= g.deep)
                        get<false>(s.w, row + k0 + w_col);
                    else
                        s = load_words<T>(row, k0 + w_col, g.deep);
                }
                held_w[i] = Words4{s.w[0], s.w[1], s.w[2], s.w[3]};
            }
        }
    };
    const auto deposit = [&](auto place_x, auto place_w) __attribute__((always_inline)) {
        Words4 *to_x = (Words4 *)(lds + decltype(place_x)::value * kX) + tid;
        Words4 *to_w = (Words4 *)(lds + kStageW + decltype(place_w)::value * kW) + tid;
#pragma unroll
        for (uint32_t i = 0; i < kLoadsX; ++i) to_x[i * kThreads] = held_x[i];
#pragma unroll
        for (uint32_t i = 0; i < kLoadsW; ++i) to_w[i * kThreads] = held_w[i];
    };

    // A wave's operands: values [16 s + 8 (lane / 32), ...) of its rows and columns.
    const uint32_t r0 = wave / C * 32 * M, c0 = wave % C * 32 * N, l32 = lane % 32, half = lane / 32;
    const bool busy = r0 < here;    // a range's last tile may end before a wave's rows
    using Bytes = __attribute__((address_space(3))) const char *;
    const uint32_t base = (uint32_t)(uintptr_t)(Bytes)(const char *)lds;
    uint32_t x_from[4], w_from[TURNED ? N : 4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uint32_t piece = ((2 * s + half) ^ l32 / 2) & 7;
        x_from[s] = base + ((r0 + l32) * kDeep + piece * 8) * 2;
        if constexpr (!TURNED) w_from[s] = base + (kStageW + (c0 + l32) * kDeep + piece * 8) * 2;
    }
    if constexpr (TURNED) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t k = 8 * half + lane % 16 / 4, piece = ((c0 / 8 + 4 * n) ^ 4 * (k & 3)) + 2 * (lane / 16 % 2) + lane % 4 / 2;
            w_from[n] = base + (kStageW + k * kCols + piece * 8 + lane % 2 * 4) * 2;
        }
    }
    Words4 a[2][M], b[2][N];
    const auto read = [&](auto place_x, auto place_w, int s) {    // of the stage that lies there
        constexpr uint32_t kAtX = decltype(place_x)::value * kX * 2, kAt = decltype(place_w)::value * kW * 2;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (TURNED) {
                const uint2 lo = read_turned((Bytes)(uintptr_t)w_from[n] + kAt + 32 * s * kCols);
                const uint2 hi = read_turned((Bytes)(uintptr_t)w_from[n] + kAt + (32 * s + 8) * kCols);
                b[s & 1][n] = Words4{lo.x, lo.y, hi.x, hi.y};
            } else {
                b[s & 1][n] = *(__attribute__((address_space(3))) const Words4 *)((Bytes)(uintptr_t)w_from[s] + kAt + 64 * n * kDeep);
            }
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
            a[s & 1][m] = *(__attribute__((address_space(3))) const Words4 *)((Bytes)(uintptr_t)x_from[s] + kAtX + 64 * m * kDeep);
    };
    constexpr int kReads = M + (TURNED ? 2 * N : N), kProducts = M * N;
    Acc acc[M][N] = {};
    const auto multiply = [&](int s) {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int n = 0; n < N; ++n) acc[m][n] = mfma<T>(b[s & 1][n], a[s & 1][m], acc[m][n]);
        // one or two reads after a product
        constexpr int kTwo = kReads > kProducts ? kReads - kProducts : 0, kOne = (kReads < kProducts ? kReads : kProducts) - kTwo;
#pragma unroll
        for (int i = 0; i < kTwo; ++i) {
            then<kMatrix, 1>();
            then<kReadLds, 2>();
        }
#pragma unroll
        for (int i = 0; i < kOne; ++i) {
            then<kMatrix, 1>();
            then<kReadLds, 1>();
        }
        if constexpr (kProducts > kTwo + kOne) then<kMatrix, kProducts - kTwo - kOne>();
    };
    // Until every wave of the block has what it read, and what it asked for is in LDS but for the latest `left` loads.
    const auto meet = [&](auto left) {
        constexpr int n = decltype(left)::value;
        static_assert(n < 16);
        __builtin_amdgcn_s_waitcnt(ALIGNED ? 0x0070 | n : 0xc07f);    // vmcnt(n) lgkmcnt(0); not ALIGNED: lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    using N0 = std::integral_constant<int, 0>;
    using N1 = std::integral_constant<int, 1>;
    using N2 = std::integral_constant<int, 2>;
    // Loads that may be on their way when the stage before theirs has to be there.
    using Ahead = std::integral_constant<int, (int)(X == 3 ? kLoadsX + kLoadsW : kLoadsW)>;
    static_assert(X == 2 || (X == 3 && ALIGNED));
    fetch_x(0, N0{});
    fetch_w(0, N0{});
    if constexpr (!ALIGNED) deposit(N0{}, N0{});
    if (ALIGNED && stages > 1) {
        if constexpr (X == 3) fetch_x(1, N1{});
        fetch_w(1, N1{});
        meet(Ahead{});
    } else {
        meet(N0{});
    }
    if (stages > 1) {
        if constexpr (X == 2) fetch_x(1, N1{});
        if constexpr (!ALIGNED) {
            fetch_w(1, N1{});
            deposit(N1{}, N1{});
        }
    }
    if (ALIGNED && stages > 2) {
        if constexpr (X == 3) fetch_x(2, N2{});
        fetch_w(2, N2{});
    }
    read(N0{}, N0{}, 0);
    const auto step = [&](auto turn, uint32_t i) __attribute__((always_inline)) {
        constexpr int n = decltype(turn)::value;
        using AtX = std::integral_constant<int, n % X>;
        using AtW = std::integral_constant<int, n % 3>;
        using NextX = std::integral_constant<int, (n + 1) % X>;
        using NextW = std::integral_constant<int, (n + 1) % 3>;
        using AfterX = std::integral_constant<int, (n + 2) % X>;
        using AfterW = std::integral_constant<int, (n + 2) % 3>;
        if constexpr (!ALIGNED) {
            if (i + 2 < stages) {
                fetch_x(i + 2, AfterX{});
                fetch_w(i + 2, AfterW{});
            }
        }
        if (busy) {
            read(AtX{}, AtW{}, 1);
            multiply(0);
            read(AtX{}, AtW{}, 2);
            multiply(1);
            read(AtX{}, AtW{}, 3);
            multiply(2);
        }
        if (i + 2 < stages)    // what was asked for of the stage after the next may be on its way
            meet(Ahead{});
        else
            meet(N0{});
        if constexpr (ALIGNED) {
            if (i + X < stages) fetch_x(i + X, AtX{});
            if (i + 3 < stages) fetch_w(i + 3, AtW{});
        } else {
            if (i + 2 < stages) deposit(AfterX{}, AfterW{});
        }
        if (busy) {
            read(NextX{}, NextW{}, 0);    // after the last stage: of what lies there, to no use
            multiply(3);
        }
    };
    for (uint32_t i = 0; i < stages; i += X == 3 ? 3 : 6) {    // then the places are the same again
        step(N0{}, i);
        if (i + 1 < stages) step(N1{}, i + 1);
        if (i + 2 < stages) step(N2{}, i + 2);
        if constexpr (X == 2) {
            if (i + 3 < stages) step(std::integral_constant<int, 3>{}, i + 3);
            if (i + 4 < stages) step(std::integral_constant<int, 4>{}, i + 4);
            if (i + 5 < stages) step(std::integral_constant<int, 5>{}, i + 5);
        }
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
                    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[m][n][8 * q + i]),
                                                                    __float_as_uint(acc[m][n][8 * q + 4 + i]), false, false);
                    v[i] = __uint_as_float(w[0]);
                    v[4 + i] = __uint_as_float(w[1]);
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

// ---- few rows ----

constexpr uint32_t kFew = 32;        // rows of a block
constexpr uint32_t kFewCols = 16;    // columns of a block

// The tile-th piece of at most kFew rows of a range, empty ranges left out.  A lane looks at eight neighbouring ranges.
__device__ __forceinline__ Place few_of(const Product &g, uint32_t tile) {
    constexpr uint32_t kEach = (POSEIDON_EXPERTS_MAX + 64) / 64;
    const uint32_t lane = threadIdx.x & 63, first = lane * kEach;
    uint32_t bounds[kEach + 1], tiles = 0;
#pragma unroll
    for (uint32_t i = 0; i <= kEach; ++i) bounds[i] = bound_of(g.offsets, min(first + i, g.ranges), g.rows);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) tiles += (max(bounds[i], bounds[i + 1]) - bounds[i] + kFew - 1) / kFew;
    uint32_t sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(sum, d, 64);
        if ((int)lane >= d) sum += up;
    }
    const uint64_t after = __ballot(sum > tile);
    Place p = {0, 0, 0, after != 0};
    if (!p.there) return p;
    uint32_t at = tile - (sum - tiles), range = 0, begin = 0, end = 0;
    bool found = false;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t n = (max(bounds[i], bounds[i + 1]) - bounds[i] + kFew - 1) / kFew;
        const bool here = !found && at < n;
        range = here ? first + i : range;
        begin = here ? bounds[i] + at * kFew : begin;
        end = here ? bounds[i + 1] : end;
        found |= here;
        at -= found ? 0 : n;
    }
    const int owner = __ffsll((unsigned long long)after) - 1;
    p.range = __builtin_amdgcn_readfirstlane(__shfl(range, owner, 64));
    p.begin = __builtin_amdgcn_readfirstlane(__shfl(begin, owner, 64));
    p.end = __builtin_amdgcn_readfirstlane(__shfl(end, owner, 64));
    return p;
}

// out[t] = W x[t].  The weights' bytes bound it: they go from memory into operands, once, and a block has 16 columns alone,
// whose sum its four waves share, so that even one token's products are blocks for every CU.  A lane takes 16
// neighbouring values, so that one wave asks for whole lines (16 rows by 8192 x 8192: 33 us, with 8 neighbouring ones 39).
// One token's 8 ranges of 4096 x 2048, 134 MB of weights: 29 us, 4.6 TB/s; 512
// rows of 64 such ranges 218 us, 4.9 TB/s.  With one, three and four turns asked for ahead in place of two these are 30, 32 and 26 us, and
// 219, 252 and 222.
template <class T>
__global__ __launch_bounds__(kBlock) void few_rows_kernel(Product g) {
    constexpr uint32_t kEach = 64, kTurn = 4 * kEach;    // values that a wave and the block take in a turn
    constexpr uint32_t kAhead = 2;                           // turns that are asked for at a time
    __shared__ float sums[4][2][kFewCols][17];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t blocks = g.tiles_r * g.tiles_c, id = g.first + blockIdx.x;
    if (id >= blocks) {
        clear_outside<T>(g, id - blocks, kBlock);
        return;
    }
    const uint32_t tile = id / g.tiles_c, col0 = id % g.tiles_c * kFewCols;
    Place at = {0, tile * kFew, g.rows, tile * kFew < g.rows};
    if (g.offsets) at = few_of(g, tile);
    if (!at.there) return;
    const uint32_t here = min(at.end - at.begin, kFew), l16 = lane % 16, mine = 16 * (lane / 16);
    using raw = typename T::raw;
    // lanes of rows past the last read that one again
    const raw *x0 = (const raw *)g.x + (at.begin + min(l16, here - 1)) * g.pitch;
    const raw *x1 = (const raw *)g.x + (at.begin + min(16 + l16, here - 1)) * g.pitch;
    const raw *w = (const raw *)g.weights + ((uint64_t)at.range * g.wide + min(col0 + l16, g.wide - 1)) * g.deep;
    const auto words = [](const raw *p) {
        uint32_t u[4];
        get<false>(u, p);
        return Words4{u[0], u[1], u[2], u[3]};
    };
    const auto masked = [&](const raw *row, uint32_t k) {
        const Slice<T> u = load_words<T>(row, k, g.deep);
        return Words4{u.w[0], u.w[1], u.w[2], u.w[3]};
    };
    Acc4 sum[2] = {};
    uint32_t k = wave * kEach;
    const auto go = [&](auto two) __attribute__((always_inline)) {
        constexpr bool kTwo = decltype(two)::value;
        for (; k + (kAhead - 1) * kTurn + kEach <= g.deep; k += kAhead * kTurn) {
            Words4 a[kAhead][2], b[kAhead][2], c[kAhead][2];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) a[i][j] = words(w + k + i * kTurn + mine + 8 * j);
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    b[i][j] = words(x0 + k + i * kTurn + mine + 8 * j);
                    if constexpr (kTwo) c[i][j] = words(x1 + k + i * kTurn + mine + 8 * j);
                }
            __builtin_amdgcn_sched_barrier(0);    // all of them asked for before the first is used
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) {
                    sum[0] = mfma16<T>(a[i][j], b[i][j], sum[0]);
                    if constexpr (kTwo) sum[1] = mfma16<T>(a[i][j], c[i][j], sum[1]);
                }
        }
        for (; k < g.deep; k += kTurn)
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {
                const Words4 a = masked(w, k + mine + 8 * j);
                sum[0] = mfma16<T>(a, masked(x0, k + mine + 8 * j), sum[0]);
                if constexpr (kTwo) sum[1] = mfma16<T>(a, masked(x1, k + mine + 8 * j), sum[1]);
            }
    };
    if (here > 16)
        go(std::true_type{});
    else
        go(std::false_type{});
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][h][mine / 4 + r][l16] = sum[h][r];    // [column][row]
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < here * kFewCols; i += kBlock) {
        const uint32_t t = i / kFewCols, c = i % kFewCols;
        if (col0 + c >= g.wide) continue;
        float v = sums[0][t / 16][c][t % 16];
#pragma unroll
        for (int s = 1; s < 4; ++s) v += sums[s][t / 16][c][t % 16];
        const uint64_t to = (at.begin + t) * g.out_pitch + col0 + c;
        if (g.out_type == POSEIDON_F32)
            ((float *)g.out)[to] = v;
        else
            ((raw *)g.out)[to] = T::down(v);
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
    Product g = {x, weights, pitch, out_pitch, (uint32_t)rows, n_ranges, (uint32_t)deep, (uint32_t)wide, offsets, 0, 0, 0, out, out_type};
    // 16-byte pieces that lie on 16 bytes and end with the row, at offsets of less than 2^31 bytes within a tile's rows and, for
    // W^T, within W
    const bool whole = deep % 8 == 0 && in_width % 8 == 0 && pitch % 8 == 0 && aligned(x, 16) && aligned(weights, 16) &&
                       pitch < (1u << 21) && (!transposed || out_width * in_width < (1u << 30));
    const auto run = [&](auto kernel, uint32_t tile_r, uint32_t tile_c, uint32_t threads) -> int {
        const uint64_t r = offsets ? tiles_for(rows, n_ranges, tile_r) : (rows + tile_r - 1) / tile_r, c = (wide + tile_c - 1) / tile_c;
        if (r * c > kBlocksMost) return POSEIDON_E_RANGE;
        g.tiles_r = (uint32_t)r;
        g.tiles_c = (uint32_t)c;
        return launch_blocks(kernel, g, r * c + (offsets ? kClearing : 0), threads, hip_stream);
    };
    // A few rows a range on average, or in all, whose weights a tile would read no faster and whose columns would be too few
    // tiles (64 ranges of 4096 x 2048: 8 rows 29 us and in tiles 74 to 138, 384 rows 211 and 227, 512 rows 218 and 229, 768 rows 245 and
    // 235; one of 8192 x 8192: 1 row 33 and 57, 32 rows 47 and 59, 64 rows 88 and 62; of 2048 x 8192: 64 rows 24 and 43, of 4096 x 4096 24
    // either way).
    if (!transposed && (rows <= 32 || (rows <= 64 && wide <= 4096) || rows <= 8ull * n_ranges)) {
        const uint64_t r = rows < rows / kFew + n_ranges ? rows : rows / kFew + n_ranges, c = (wide + kFewCols - 1) / kFewCols;
        g.tiles_r = (uint32_t)r;
        g.tiles_c = (uint32_t)c;
        const uint64_t blocks = r * c + (offsets ? kClearing : 0);
        return type == POSEIDON_F16 ? launch_blocks(few_rows_kernel<F16>, g, blocks, kBlock, hip_stream)
                                    : launch_blocks(few_rows_kernel<BF16>, g, blocks, kBlock, hip_stream);
    }
    const uint64_t large = tiles_for(rows, n_ranges, 256) * ((wide + 255) / 256);
    const auto pick = [&](auto t, auto turned, auto whole_) -> int {
        using T = decltype(t);
        constexpr bool kTurned = decltype(turned)::value, kWhole = decltype(whole_)::value;
        // 256 x 256 tiles, one a CU, where most CUs get one (one range of 3000 x 3000, 4096 rows, 204 tiles: 89 us, in 128 x 128 120;
        // 6000 rows of 2048 x 2048, 192: 57 and 60; 5120 rows, 168: 59 and 56).
        if (large >= 180) return run(product_kernel<T, kTurned, kWhole, 2, 4, 4, 2, 2>, 256, 256, 512);
        // 128 x 128 where every CU gets one (4096 rows in 16 ranges of 1024 x 1024, 384 tiles: 18 us, in 64 x 128 21; 512 rows of 4096 x
        // 4096, 160: 35 and 26; 256 rows of them 33 and 24).
        if (tiles_for(rows, n_ranges, 128) * ((wide + 127) / 128) >= 256) return run(product_kernel<T, kTurned, kWhole, 2, 2, 2, 2, 2>, 128, 128, 256);
        // with a third stage of x, as nothing else on a CU hides its way from memory (256 rows of 4096 x 4096: 24 us, with two 28)
        return run(product_kernel<T, kTurned, kWhole, 2, 2, 1, 2, kWhole ? 3 : 2>, 64, 128, 256);
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
