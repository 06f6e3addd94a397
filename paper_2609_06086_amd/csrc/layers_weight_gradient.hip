// Weight gradients from activations kept in 8 bits (poseidon_layers.h):
//   grad[r][o][i] = sum over rows t of range r of dy[t][o] * x[t][i].
//
// A kept value is q 2^e with |q| <= 127: exact in bf16 (8 significant bits) and, kept
// from f16, in f16.  So the codes become operands of the 16-bit matrix instructions without a
// rounding, and the only error of the product is that of its 32-bit sums.
//
// Both operands are summed over their slow axis, the rows.  A matrix
// instruction wants eight neighbouring rows of one column in a lane, so a
// thread loads an 8 x 8 block (eight rows of eight columns: coalesced), turns
// it in registers with byte permutes, and writes each column's eight rows as 16
// bytes to LDS, where a column's 64 rows of a step lie together.  Every thread
// brings a block of dy and one of the codes, which it also unpacks and scales.
#include "layers_device.h"

namespace pl {

using Acc = float __attribute__((ext_vector_type(16)));
using HalfVec = _Float16 __attribute__((ext_vector_type(8)));
using BrainVec = __bf16 __attribute__((ext_vector_type(8)));
using Words4 = uint32_t __attribute__((ext_vector_type(4)));

constexpr uint32_t kStep = 64;    // rows of a step

template <class T>
__device__ __forceinline__ Acc mfma(Words4 a, Words4 b, Acc c);
template <>
__device__ __forceinline__ Acc mfma<BF16>(Words4 a, Words4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(BrainVec, a), __builtin_bit_cast(BrainVec, b), c,
                                                   0, 0, 0);
}
template <>
__device__ __forceinline__ Acc mfma<F16>(Words4 a, Words4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(HalfVec, a), __builtin_bit_cast(HalfVec, b), c, 0,
                                                  0, 0);
}

// Two values as a pair.  BF16 holds every kept value exactly, and F16 those that were kept from it.  Of the others, this
// conversion toward zero holds large ones to the type's last finite value in the same instruction, which rounding to nearest
// would make infinite, and cuts what lies below 2^-24 off small ones: at most 2^-24, where nearest is 2^-25.
template <class T>
__device__ __forceinline__ uint32_t pack(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack<BF16>(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
template <>
__device__ __forceinline__ uint32_t pack<F16>(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
}

constexpr uint32_t kNone = 0xffffffffu;

// A run of a range's rows that a block takes, and where its sums go: a slot of
// the workspace, or kNone: the gradient itself.
struct Run {
    uint32_t range, begin, end, slot;
};
// A range that was split: its slots are added up at the end.
struct Split {
    uint32_t range, slot, runs;
};
// What weight_plan_kernel makes of the offsets.
struct RunTable {
    uint32_t runs, splits;
};

struct WeightGrad {
    const void *dy;
    uint64_t dy_pitch;
    uint32_t rows, out_width, in_width, groups;
    const int8_t *codes;
    const uint8_t *scales;
    uint32_t tiles_o, tiles_i, accumulate;
    uint32_t of_one;               // without a table: runs of the one range
    const int32_t *offsets;        // its bounds, null: all rows
    const RunTable *table;
    const Run *runs;
    const Split *splits;
    void *grad;                    // [ranges][out_width][in_width]
    float *parts;                  // [slots][out_width][in_width]
};

// Word (4 rows' worth of banks) of rows [8 oct, 8 oct + 8) of an LDS column: columns are
// 128 bytes apart, so the place of an eight-row piece is mixed with the column's low bits (for
// readers: 8 neighbouring columns) and the next ones (for writers: 8 blocks of columns).
__device__ __forceinline__ uint32_t place(uint32_t col, uint32_t oct) {
    return col * 8 + ((oct ^ col ^ (col >> 3)) & 7);
}

// What a block computes.  Blocks go round the eight XCDs in turn, each with an L2 of
// its own, so an XCD takes a run of neighbouring tiles; a run goes through
// the tiles four high, so the 32 blocks that an XCD's CUs hold share 4 column ranges of dy and 8 of x
// (which has half the bytes) and an L2 fetches a twelfth to an eighth of what its blocks ask for.
struct Unit {
    uint32_t run, tile_o, tile_i;
};

__device__ __forceinline__ Unit unit_of(const WeightGrad &g) {
    const uint32_t tiles = g.tiles_o * g.tiles_i, all = g.table ? tiles : gridDim.x;
    const uint32_t before = blockIdx.x / all, at = blockIdx.x - before * all, xcd = at & 7;
    uint32_t id = xcd * (all / 8) + min(xcd, all & 7) + at / 8;
    Unit u;
    u.run = id / tiles;
    id -= u.run * tiles;
    u.run += before;
    const uint32_t band = id / (4 * g.tiles_i), high = min(4u, g.tiles_o - 4 * band);
    id -= band * 4 * g.tiles_i;
    u.tile_i = id / high;
    u.tile_o = 4 * band + id - u.tile_i * high;
    return u;
}

// The runs of ragged ranges: a range of more than `most` steps becomes several of about the
// same length, and of up to kRanked runs the longest come first, so that none is left for the
// end.  One block.  An empty range is a run too, which writes its zeros.
// It is one long chain of waits, so a run has a thread of its own, few runs get few waves, and the lengths that a run is
// compared with come sixteen at a time (64 ranges: 6 us; 25 ranges in about 100 runs 7 us, 54 with a thread per range).
constexpr uint32_t kPlanThreads = 1024, kRanked = 1024;

struct RunPlan {
    const int32_t *offsets;
    uint32_t rows, ranges, most;
    uint32_t max_runs, max_splits, max_slots;
    RunTable *table;
    Run *runs;
    Split *splits;
};

__global__ __launch_bounds__(kPlanThreads) void weight_plan_kernel(RunPlan p) {
    __shared__ uint32_t sums[3][kPlanThreads / 64];
    __shared__ uint4 lengths[kRanked / 4];
    uint32_t *const length = (uint32_t *)lengths;
    const uint32_t tid = threadIdx.x, waves = blockDim.x / 64, each = (p.ranges + blockDim.x - 1) / blockDim.x;
    const uint32_t first = min(tid * each, p.ranges), last = min(first + each, p.ranges);
    const auto read_bound = [&](uint32_t r) { return (uint32_t)min(max(p.offsets[r], 0), (int32_t)p.rows); };
    const uint32_t own[2] = {read_bound(first), read_bound(min(first + 1, p.ranges))};    // read once where a thread has one range
    const auto bound = [&](uint32_t r) { return r - first < 2 ? own[r - first] : read_bound(r); };
    const auto steps_of = [&](uint32_t begin, uint32_t end) { return end > begin ? (end - begin + kStep - 1) / kStep : 0u; };

    // how many runs, split ranges and slots the thread's ranges need, and those before it
    uint32_t need[3] = {}, at[3];
    for (uint32_t r = first; r < last; ++r) {
        const uint32_t n = max(1u, (steps_of(bound(r), bound(r + 1)) + p.most - 1) / p.most);
        need[0] += n;
        need[1] += n > 1;
        need[2] += n > 1 ? n : 0;
    }
    uint32_t sum[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        sum[i] = need[i];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t up = __shfl_up(sum[i], d, 64);
            if ((int)(tid & 63) >= d) sum[i] += up;
        }
        if ((tid & 63) == 63) sums[i][tid / 64] = sum[i];
    }
    __syncthreads();
    uint32_t total[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        total[i] = 0;
        uint32_t before = 0;
        for (uint32_t w = 0; w < waves; ++w) {
            before += w < tid / 64 ? sums[i][w] : 0;
            total[i] += sums[i][w];
        }
        at[i] = before + sum[i] - need[i];
    }

    // Ranges that overlap (offsets that do not ascend) can ask for more than there is room for: then none is split.
    const bool fits = total[0] <= p.max_runs && total[1] <= p.max_splits && total[2] <= p.max_slots;
    const uint32_t all = fits ? total[0] : p.ranges;
    if (tid == 0) *p.table = RunTable{all, fits ? total[1] : 0};
    const auto parts_of = [&](uint32_t begin, uint32_t end) { return fits ? max(1u, (steps_of(begin, end) + p.most - 1) / p.most) : 1u; };
    const auto run_of = [&](uint32_t r, uint32_t begin, uint32_t end, uint32_t n, uint32_t i, uint32_t slot) {
        const uint32_t part = (steps_of(begin, end) + n - 1) / n, from = min(begin + i * part * kStep, end);
        const uint32_t to = min(from + part * kStep, end);
        return Run{r, from, to, n > 1 ? slot + i : kNone};
    };

    if (all <= kRanked) {    // a thread has a range, then a run: the one that holds its place, and the place that its length takes
        __shared__ uint32_t run0[kRanked], begins[kRanked], ends[kRanked], slot0[kRanked];
        if (tid < p.ranges) {
            run0[tid] = fits ? at[0] : tid;
            begins[tid] = own[0];
            ends[tid] = max(own[0], own[1]);
            slot0[tid] = at[2];
            if (parts_of(own[0], own[1]) > 1) p.splits[at[1]] = Split{tid, at[2], need[0]};
        }
        if (tid < 16 && all + tid < kRanked) length[all + tid] = 0;
        __syncthreads();
        Run run = {};
        uint32_t mine = 0;
        if (tid < all) {
            uint32_t r = 0;    // the last range whose first run is not after this one
            for (uint32_t d = kRanked / 2; d; d >>= 1)
                if (r + d < p.ranges && run0[r + d] <= tid) r += d;
            run = run_of(r, begins[r], ends[r], parts_of(begins[r], ends[r]), tid - run0[r], slot0[r]);
            length[tid] = mine = run.end - run.begin;
        }
        __syncthreads();
        if (tid >= all) return;
        uint32_t rank = 0;
        for (uint32_t j = 0; j < all; j += 16) {    // past the last run: lengths of 0
            uint4 u[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) u[q] = lengths[j / 4 + q];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t l[4] = {u[q].x, u[q].y, u[q].z, u[q].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) rank += l[e] > mine || (l[e] == mine && j + 4 * q + e < tid);
            }
        }
        p.runs[rank] = run;
        return;
    }
    uint32_t n0 = fits ? at[0] : first, n1 = at[1], n2 = at[2];
    for (uint32_t r = first; r < last; ++r) {
        const uint32_t begin = bound(r), end = max(begin, bound(r + 1)), n = parts_of(begin, end);
        for (uint32_t i = 0; i < n; ++i) p.runs[n0++] = run_of(r, begin, end, n, i, n2);
        if (n > 1) {
            p.splits[n1++] = Split{r, n2, n};
            n2 += n;
        }
    }
}

template <int N>
struct Int {
    static constexpr int value = N;
};
// f(Int<0>), ..., f(Int<N - 1>)
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F &&f) {
    if constexpr (I < N) {
        f(Int<I>{});
        each<N, I + 1>(f);
    }
}

// Byte B of a word, signed, as a float: one instruction.
template <int B>
__device__ __forceinline__ float signed_byte(uint32_t w) {
    float v;
    if constexpr (B == 0)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(v) : "v"(w));
    else if constexpr (B == 1)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(v) : "v"(w));
    else if constexpr (B == 2)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(v) : "v"(w));
    else
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(v) : "v"(w));
    return v;
}

using Rsrc = __amdgpu_buffer_rsrc_t;

__device__ __forceinline__ Rsrc buffer(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00027000);
}

// Four waves on a tile of 32 C x 32 C, 16 C x 16 C a wave, in steps of 64 rows.
// A thread brings 8 rows of C columns of each operand.
//
// C = 8, 256 x 256: a wave reads 8 KB of LDS for 16 matrix instructions of 32 cycles, half of what LDS
// delivers, and a quarter more is written (by count, 8 waves of 128 x 64 would read three quarters; not measured).  With 256
// sums a lane there is one wave a SIMD, so nothing hides behind another wave: LDS holds two
// steps, and while the matrix instructions work on one, the rows of the next are turned and
// unpacked between them; those of the two after are on their way in registers (with only one of them the
// waits for memory took half of the time).
// C = 4, 128 x 128: 64 sums a lane and half of the LDS, so that two blocks share a CU.
//
// Measured: 16384 x 8192 x 4096 in 946 to 961 us (1150 TFLOP/s).  The matrix instructions are busy 58% of the cycles; beside
// each of them lie 22 cycles of issue of its 32, and LDS moves data in three quarters of the time that they would take
// alone: which of the two holds it is not shown.  64 ragged ranges of 2048 x 2048 over 65536 rows take 710 us.  There a unit
// has 16 steps on average and a start and an end that nothing hides; tried and slower or no faster: the next unit's rows asked for
// before the stores (705 us), 16 bytes a lane a store (760: pieces of 32 bytes of a line), a range's tiles all on one XCD
// (756), leaving out the zero step after an odd number (the registers no longer suffice).
//
// Rows past the end come back as zeros from the buffers' bounds.  ALIGNED: dy's rows begin on whole words, as
// buffer loads want, and are a multiple of 8 wide; else they are read with plain loads, which take any address, and
// masked.
template <class T, class G, int C, bool ALIGNED>
__global__ __launch_bounds__(256, C == 8 ? 1 : 2) void weight_gradient_kernel(WeightGrad g) {
    constexpr uint32_t kTile = 32 * C, kPad = 8;    // a tile's first block may begin up to 7 columns before it
    constexpr uint32_t kBuf = (kTile + kPad) * 8;
    constexpr int M = C / 2, kPieces = M * M;       // a wave's tiles of 32 x 32 along a side, and in all
    using Row = uint32_t __attribute__((ext_vector_type(C / 2)));    // C values of dy
    using Codes = uint32_t __attribute__((ext_vector_type(C / 4)));
    __shared__ Words4 lds[4 * kBuf];                // dy's two steps, then x's
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);

    const Unit unit = unit_of(g);
    Run run;
    if (g.table) {
        if (unit.run >= g.table->runs) return;
        run = g.runs[unit.run];
        if (run.begin == run.end && run.slot == kNone && g.accumulate) return;
    } else {
        uint32_t begin = 0, end = g.rows;
        if (g.offsets) {
            begin = (uint32_t)min(max(g.offsets[0], 0), (int32_t)g.rows);
            end = (uint32_t)min(max(g.offsets[1], (int32_t)begin), (int32_t)g.rows);
        }
        const uint32_t steps = (end - begin + kStep - 1) / kStep, each = (steps + g.of_one - 1) / g.of_one;
        run.range = 0;
        run.begin = min(begin + min(unit.run * each, steps) * kStep, end);
        run.end = min(run.begin + each * kStep, end);
        run.slot = g.of_one > 1 ? unit.run : kNone;
    }
    const uint32_t begin = run.begin, end = run.end;

    const uint32_t o0 = unit.tile_o * kTile, i0 = unit.tile_i * kTile;
    const uint32_t cb = tid % 32, oct = tid / 32;
    const uint32_t o_first = o0 + cb * C, i_first = i0 + cb * C;
    // not ALIGNED: the last block of dy's columns is moved back to end with the row
    const uint32_t o_from = ALIGNED ? o_first : g.out_width >= C ? min(o_first, g.out_width - C) : 0;
    const uint32_t dy_row = (uint32_t)g.dy_pitch * 2, x_row = g.groups * kGroup;    // bytes
    constexpr uint32_t kNowhere = 0x80000000u;
    const uint32_t dy_at = o_first < g.out_width ? oct * 8 * dy_row + o_from * 2 : kNowhere;
    const uint32_t x_at = i_first < x_row ? oct * 8 * x_row + i_first : kNowhere;
    const uint32_t s_at = i_first < x_row ? oct * 8 * g.groups + i_first / kGroup : kNowhere;
    const int32_t col0 = !ALIGNED && o_first < g.out_width ? (int32_t)o_from - (int32_t)o0 : (int32_t)(cb * C);
    // where a column's rows go in LDS: that of the block's column c is that of its column 0, xor c, 8 c further
    const uint32_t to = kPad * 8 + (place(cb * C, oct));

    // The rows from t0 on as buffers that end with the step or the range; a thread's rows are scalar offsets apart, which
    // the bounds check counts (a descriptor for each row took as long to make as the matrix instructions to run).
    Row dy[2][8];
    Codes x[2][8];
    uint32_t sc[2][8];
    Rsrc from_dy, from_codes, from_scales;
    const auto aim = [&](uint32_t t0) {
        const uint32_t n = t0 < end ? min(end - t0, kStep) : 0;
        const uint64_t t = n ? t0 : 0;
        if constexpr (ALIGNED) from_dy = buffer((const char *)g.dy + t * dy_row, n * dy_row);
        from_codes = buffer(g.codes + t * x_row, n * x_row);
        from_scales = buffer(g.scales + t * g.groups, n * g.groups);
    };
    const auto fetch_dy = [&](int set, uint32_t t0, uint32_t r) {
        if constexpr (C == 8) {
            static_assert(ALIGNED);
            dy[set][r] = __builtin_amdgcn_raw_buffer_load_b128(from_dy, dy_at, r * dy_row, 0);
        } else if constexpr (ALIGNED) {
            dy[set][r] = __builtin_amdgcn_raw_buffer_load_b64(from_dy, dy_at, r * dy_row, 0);
        } else {
            const uint32_t row = min(t0 + oct * 8 + r, end - 1);
            const uint16_t *p = (const uint16_t *)g.dy + row * g.dy_pitch + o_from;
            if (g.out_width >= C) {
                __builtin_memcpy(&dy[set][r], p, sizeof(Row));
            } else {
#pragma unroll
                for (int w = 0; w < C / 2; ++w)
                    dy[set][r][w] = (2 * w < g.out_width ? p[2 * w] : 0u) |
                                    (2 * w + 1 < g.out_width ? (uint32_t)p[2 * w + 1] << 16 : 0u);
            }
        }
    };
    const auto fetch_x = [&](int set, uint32_t r) {
        if constexpr (C == 8)
            x[set][r] = __builtin_amdgcn_raw_buffer_load_b64(from_codes, x_at, r * x_row, 0);
        else
            x[set][r][0] = __builtin_amdgcn_raw_buffer_load_b32(from_codes, x_at, r * x_row, 0);
        sc[set][r] = __builtin_amdgcn_raw_buffer_load_b8(from_scales, s_at, r * g.groups, 0);
    };
    // Column c of the thread's block, of the rows that begin at t0.
    const auto write_dy = [&](int set, uint32_t buf, uint32_t t0, int c) {
        Words4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint32_t lo = dy[set][2 * t][c / 2], hi = dy[set][2 * t + 1][c / 2];
            if constexpr (!ALIGNED) {
                lo = t0 + oct * 8 + 2 * t < end ? lo : 0u;
                hi = t0 + oct * 8 + 2 * t + 1 < end ? hi : 0u;
            }
            w[t] = __builtin_amdgcn_perm(hi, lo, c & 1 ? 0x07060302u : 0x05040100u);
        }
        if constexpr (ALIGNED)
            lds[buf * kBuf + (to ^ c) + c * 8] = w;
        else
            lds[buf * kBuf + kPad * 8 + (int32_t)place((uint32_t)(col0 + c), oct)] = w;
    };
    // Rows 2 t and 2 t + 1 of column c; with the last two the column is written.
    // A group of scale byte 255 has codes 0, and 0 times the infinity that its bits are as a float is NaN.
    Words4 turned;
    const auto unpack_x = [&](int set, uint32_t buf, auto column, int t) {
        constexpr int c = decltype(column)::value;
        float v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 2 * t + h;
            if constexpr (c == 0) sc[set][r] <<= 23;    // the scale as a float
            v[h] = signed_byte<c & 3>(x[set][r][c / 4]) * __uint_as_float(sc[set][r]);
        }
        turned[t] = pack<T>(v[0], v[1]);
        if (t == 3) lds[(2 + buf) * kBuf + (to ^ c) + c * 8] = turned;
    };

    // The words of column (wave's first + 32 m + lane % 32), rows [16 s + 8 (lane / 32), ...).
    const uint32_t c32 = lane % 32, key = (lane / 32 ^ c32 ^ c32 >> 3) & 7;
    const uint32_t at_o = kPad * 8 + (wave / 2 * (16 * C) + c32) * 8;
    const uint32_t at_i = 2 * kBuf + kPad * 8 + (wave % 2 * (16 * C) + c32) * 8;
    Words4 a[2][M], b[2][M];
    const auto read = [&](uint32_t buf, int s, int j) {    // one of the 2 M reads of quarter s
        const int m = j / 2;
        const uint32_t w = buf * kBuf + (key ^ (2 * (s ^ 2 * (m & 1)))) + m * 256;
        if (j & 1)
            b[s & 1][m] = lds[at_i + w];
        else
            a[s & 1][m] = lds[at_o + w];
    };
    Acc acc[M][M] = {};

    // A quarter of a step: M x M matrix instructions, and after each a little of the other work, which the
    // instruction's 32 cycles cover.  Quarters 0 and 1 unpack the next step's x, quarter 2 turns its dy,
    // quarter 3 reads from the next step's LDS words, written by then; the next rows are
    // asked for as soon as their registers are free.
    const auto quarter = [&](auto which, auto step, uint32_t t0) {
        constexpr int s = decltype(which)::value, buf = decltype(step)::value, set = buf ^ 1;
        const auto piece = [&](auto index) {
            constexpr int j = decltype(index)::value;
            acc[j / M][j % M] = mfma<T>(a[s & 1][j / M], b[s & 1][j % M], acc[j / M][j % M]);
            if constexpr (j < 2 * M) read(s < 3 ? buf : buf ^ 1, (s + 1) & 3, j);
            if constexpr (s < 2) {
                constexpr int kUnits = 2 * C / kPieces;    // of C columns of four, over two quarters
                each<kUnits>([&](auto part) {
                    constexpr int unit = s * 2 * C + j * kUnits + decltype(part)::value;
                    unpack_x(set, buf ^ 1, Int<unit / 4>{}, unit % 4);
                });
            }
            if constexpr (s == 2 && j < C) write_dy(set, buf ^ 1, t0 + kStep, j);
            if constexpr (s == 2 && C == 8 && j >= 8) fetch_x(set, j - 8);
            if constexpr (s == 2 && C == 4) each<2>([&](auto r) { fetch_x(set, 2 * j + decltype(r)::value); });
            if constexpr (s == 3 && C == 8 && j < 8) fetch_dy(set, t0 + 3 * kStep, j);
            if constexpr (s == 3 && C == 4) each<2>([&](auto r) { fetch_dy(set, t0 + 3 * kStep, 2 * j + decltype(r)::value); });
            __builtin_amdgcn_sched_barrier(0);
        };
        each<kPieces>(piece);
    };
    // Multiplies the step in LDS buffer `buf`, and writes the next one (set buf ^ 1) to the other.
    const auto step = [&](auto buf, uint32_t t0) {
        quarter(Int<0>{}, buf, t0);
        quarter(Int<1>{}, buf, t0);
        aim(t0 + 3 * kStep);
        quarter(Int<2>{}, buf, t0);
        __syncthreads();    // the other buffer is whole, and this one read
        quarter(Int<3>{}, buf, t0);
    };

    if (begin < end) {
        const auto fetch = [&](int set, uint32_t t0) {
            aim(t0);
            each<8>([&](auto r) {
                fetch_x(set, decltype(r)::value);
                fetch_dy(set, t0, decltype(r)::value);
            });
        };
        fetch(0, begin);
        fetch(1, begin + kStep);
        each<C>([&](auto c) {
            write_dy(0, 0, begin, decltype(c)::value);
            each<4>([&](auto t) { unpack_x(0, 0, c, decltype(t)::value); });
        });
        fetch(0, begin + 2 * kStep);
        __syncthreads();
        each<2 * M>([&](auto j) { read(0, 0, decltype(j)::value); });
        for (uint32_t t0 = begin; t0 < end; t0 += 2 * kStep) {
            step(Int<0>{}, t0);
            step(Int<1>{}, t0 + kStep);    // all zeros after an odd number of steps
        }
    }

    // Value e of a tile: row 8 (e / 4) + 4 (lane / 32) + e % 4, column lane % 32.  Rows and columns past the
    // gradient's are dropped by the buffer's bounds.
    const auto write = [&](auto type, void *result, uint32_t range, bool add) {
        using R = decltype(type);
        constexpr uint32_t kSize = sizeof(typename R::raw);
        const uint32_t row = g.in_width * kSize, o = o0 + wave / 2 * (16 * C);
        const uint32_t rows = o < g.out_width ? min(g.out_width - o, 16u * C) : 0;
        const Rsrc r = buffer((typename R::raw *)result + ((uint64_t)range * g.out_width + (rows ? o : 0)) * g.in_width, rows * row);
        each<kPieces>([&](auto index) {
            constexpr int m = decltype(index)::value / M, n = decltype(index)::value % M;
            const uint32_t i = i0 + wave % 2 * (16 * C) + n * 32 + lane % 32;
            const uint32_t at = i < g.in_width ? lane / 32 * 4 * row + i * kSize : kNowhere;
            each<16>([&](auto element) {
                constexpr int e = decltype(element)::value;
                const uint32_t down = (m * 32 + e / 4 * 8 + e % 4) * row;
                float v = acc[m][n][e];
                if constexpr (kSize == 4) {
                    if (add) v += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, at, down, 0));
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, at, down, 0);
                } else {
                    if (add)
                        v += R::up(__builtin_bit_cast(typename R::raw, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, at, down, 0)));
                    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, R::down(v)), r, at, down, 0);
                }
            });
        });
    };
    if (run.slot != kNone)
        write(F32{}, g.parts, run.slot, false);
    else if (g.accumulate)
        write(G{}, g.grad, run.range, true);
    else
        write(G{}, g.grad, run.range, false);
}

// Adds a split range's slots, in order: one pass over them, 5 us for 4 of 1024 x 1024.
template <class G>
__global__ __launch_bounds__(kBlock) void weight_join_kernel(WeightGrad g) {
    Split s = {0, 0, g.of_one};
    if (g.table) {
        if (blockIdx.y >= g.table->splits) return;
        s = g.splits[blockIdx.y];
    }
    const uint64_t size = (uint64_t)g.out_width * g.in_width;
    const float *parts = g.parts + s.slot * size;
    typename G::raw *grad = (typename G::raw *)g.grad + s.range * size;
    for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < size; i += (uint64_t)gridDim.x * kBlock) {
        float sum = g.accumulate ? G::up(grad[i]) : 0.0f;
        uint32_t r = 0;
        for (; r + 8 <= s.runs; r += 8) {    // eight loads on their way; 256 runs of 64 x 64: 46 us without, 18 with
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = parts[(r + j) * size + i];
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[j];
        }
        for (; r + 2 <= s.runs; r += 2) {
            const float a = parts[r * size + i], b = parts[(r + 1) * size + i];
            sum += a;
            sum += b;
        }
        if (r < s.runs) sum += parts[r * size + i];
        grad[i] = G::down(sum);
    }
}

// Rows of 16-bit values on a pitch of `padded` (a multiple of 8) values, zeros past the width.
__global__ __launch_bounds__(kBlock) void pack_rows_kernel(const __bf16 *x, uint64_t pitch, uint32_t total, Div per_row,
                                                           uint32_t width, uint4 *out) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row);
    const Slice<BF16> s = load_words<BF16>(x + row * pitch, (i - row * per_row.d) * kSlice, width);
    out[i] = make_uint4(s.w[0], s.w[1], s.w[2], s.w[3]);
}

struct WeightPlan {
    bool large, pack;
    uint32_t tiles_o, tiles_i;
    uint32_t each;                                // ragged: steps of a run at most
    uint64_t max_runs, max_splits, max_slots;     // one range: exact
    uint64_t packed, table, runs, splits, bytes;  // offsets of the workspace, after the slots
};

// Tiles of 256 x 256 where the 256 CUs get 16 steps or more each (1077 TFLOP/s on long sums, 686 with tiles of
// 128 x 128, which fill the chip with less).  One range: its rows are split until every CU has a block, of
// 16 (8) steps or more (small tiles with 4: 512 x 1024 x 1024 15 us, 11 with 8 or 16; with 16: 2048 x 512 x 512 19, 15 with 4 or 8;
// large tiles have 16 wherever they are taken), and a little more than 128 or 256 large tiles, which would leave most of the last round of the CUs
// idle, in two or three parts where that takes less (16000 x 4104 x 2048, 136 tiles: 316 us instead of 376; 8192 x
// 5120 x 3584, 280 tiles: 373 instead of 415) (two of the small tiles a CU take longer: 4096 x 1024 x 1024 31 us instead of 29).  Ragged ranges: runs
// of at most half of a CU's share, and the large tiles from 96 steps a CU on, as there are more units to even out: with
// 128 steps a CU 16 ranges of 2048 x 2048 take 333 us (382 with the small tiles), with 64 8 ranges 204 (182), with 34 34
// ranges of 520 x 1416 156 (113).
//
// Parts take 1 GB at most: without a bound a gradient of 32776 x 32776 asked for 12 GB.  A gradient that would need more is
// five rounds of the CUs and more, and of the last one there is little to win (131072 x 7424 x 13568 25.9 ms, 25.5 in three
// parts of 1.2 GB; 65536 x 8448 x 8192, two parts of 0.8 GB, 8.8 instead of 9.7).
//
// A dy that is no multiple of 8 wide is copied to one that is where that brings the large tiles: 8000 x 2001 x 2048 92 us
// instead of 133.  Not for an x of few columns (with 256 the copy loses, 65536 x 2001 180 us against 157; with 384 and 448 it would gain a
// tenth, 32768 x 2001 x 448 127 against 140; with 512 both take 126 for 16384 x 4001), nor for more than 8 GB, as that
// memory is the caller's.
constexpr uint64_t kPartsMost = 1ull << 30;

inline WeightPlan weight_plan(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges, bool whole) {
    WeightPlan p = {};
    const bool ragged = n_ranges > 1;
    const uint64_t steps = (rows + kStep - 1) / kStep;
    const auto tiles = [&](uint64_t side) { return ((out_width + side - 1) / side) * ((in_width + side - 1) / side); };
    const bool much = steps * tiles(256) >= 256 * (ragged ? 96 : 16);
    const uint64_t packed = rows * ((out_width + 7) / 8 * 16);
    p.pack = much && !whole && out_width % 8 && in_width >= 512 && packed <= 8ull << 30;
    p.large = much && (whole || p.pack);
    const uint64_t side = p.large ? 256 : 128, each = p.large ? 16 : 8, n = tiles(side);
    p.tiles_o = (uint32_t)((out_width + side - 1) / side);
    p.tiles_i = (uint32_t)((in_width + side - 1) / side);
    if (ragged) {
        const uint64_t half = steps * n / 512;
        p.each = (uint32_t)(half < each ? each : half);
        p.max_splits = steps / p.each;
        p.max_runs = n_ranges + p.max_splits;
        p.max_slots = 2 * p.max_splits;
    } else {
        uint64_t runs = 256 / n, most = steps / each;
        if (p.large && n > 128) {    // ns: rounds of the CUs, and the parts written and read
            uint64_t least = ~0ull;
            for (uint64_t r = 1; r <= 3 && (r == 1 || r * out_width * in_width * 4 <= kPartsMost); ++r) {
                const uint64_t time = (n * r + 255) / 256 * ((steps + r - 1) / r * 1850 + 14000) + (r > 1 ? r * n * 105 : 0);
                if (time < least) least = time, runs = r;
            }
        }
        runs = runs < most ? runs : most;
        p.max_runs = runs < 2 ? 1 : runs;
        p.max_splits = p.max_runs > 1;
        p.max_slots = p.max_runs > 1 ? p.max_runs : 0;
    }
    const auto up = [](uint64_t v) { return (v + 255) / 256 * 256; };
    p.bytes = up(p.max_slots * out_width * in_width * 4);
    if (ragged) {
        p.table = p.bytes;
        p.runs = p.table + up(sizeof(RunTable));
        p.splits = p.runs + up(p.max_runs * sizeof(Run));
        p.bytes = p.splits + up(p.max_splits * sizeof(Split));
    }
    p.packed = p.bytes;
    if (p.pack) p.bytes += up(packed);
    return p;
}

inline int check_weight(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges) {
    PL_TRY(check_sizes(rows, out_width));
    PL_TRY(check_sizes(rows, in_width));
    if (!n_ranges) return POSEIDON_E_INVAL;
    if (n_ranges > POSEIDON_RANGES_MAX) return POSEIDON_E_RANGE;
    // blocks of one launch
    const uint64_t tiles = ((out_width + 127) / 128) * ((in_width + 127) / 128);
    return tiles * n_ranges > POSEIDON_TILES_MAX ? POSEIDON_E_RANGE : POSEIDON_OK;
}

}  // namespace pl

using namespace pl;

extern "C" {

uint64_t poseidon_weight_gradient_workspace(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges) {
    if (check_weight(rows, out_width, in_width, n_ranges) != POSEIDON_OK) return UINT64_MAX;
    // the most that any layout of dy needs (it is copied by its width alone)
    const uint64_t a = weight_plan(rows, out_width, in_width, n_ranges, false).bytes;
    const uint64_t b = weight_plan(rows, out_width, in_width, n_ranges, true).bytes;
    return a < b ? b : a;
}

int poseidon_weight_gradient(const void *dy, uint64_t dy_pitch, uint32_t type, uint64_t rows, uint64_t out_width,
                             const int8_t *codes, const uint8_t *scales, uint64_t in_width, const int32_t *offsets,
                             uint32_t n_ranges, void *grad, uint32_t grad_type, uint32_t accumulate, void *workspace,
                             uint64_t workspace_bytes, void *hip_stream) {
    PL_TRY(check_weight(rows, out_width, in_width, n_ranges));
    PL_TRY(check_matrix(dy, dy_pitch, type, rows, out_width));
    PL_TRY(check_stash(codes, scales, rows));
    if (type == POSEIDON_F32 || !known(grad_type) || accumulate > 1 || !grad || !aligned(grad, size_of(grad_type)))
        return POSEIDON_E_INVAL;
    if (!offsets && n_ranges != 1) return POSEIDON_E_INVAL;
    PL_TRY(check_workspace(workspace, workspace_bytes,
                           poseidon_weight_gradient_workspace(rows, out_width, in_width, n_ranges)));
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool whole = out_width % 8 == 0 && aligned(dy, 4) && dy_pitch % 2 == 0;
    const WeightPlan p = weight_plan(rows, out_width, in_width, n_ranges, whole);
    char *base = (char *)workspace;
    WeightGrad g = {};
    g.dy = dy;
    g.dy_pitch = dy_pitch;
    g.rows = (uint32_t)rows;
    g.out_width = (uint32_t)out_width;
    g.in_width = (uint32_t)in_width;
    g.groups = groups_of(in_width);
    g.codes = codes;
    g.scales = scales;
    g.tiles_o = p.tiles_o;
    g.tiles_i = p.tiles_i;
    g.accumulate = accumulate;
    g.of_one = (uint32_t)p.max_runs;
    g.grad = grad;
    g.parts = (float *)base;
    g.offsets = offsets;
    if (p.pack) {
        const uint32_t per_row = (uint32_t)((out_width + 7) / 8);
        over_rows(rows, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
            pack_rows_kernel<<<blocks_for(n), kBlock, 0, stream>>>((const __bf16 *)dy + r * dy_pitch, dy_pitch, n,
                                                                   make_div(per_row), (uint32_t)out_width,
                                                                   (uint4 *)(base + p.packed) + r * per_row);
        });
        PL_TRY(launched());    // the next kernel reads it
        g.dy = base + p.packed;
        g.dy_pitch = per_row * 8ull;
    }
    if (n_ranges > 1) {
        RunPlan r = {offsets, (uint32_t)rows, n_ranges, p.each, (uint32_t)p.max_runs, (uint32_t)p.max_splits,
                     (uint32_t)p.max_slots, (RunTable *)(base + p.table), (Run *)(base + p.runs), (Split *)(base + p.splits)};
        g.table = r.table;
        g.runs = r.runs;
        g.splits = r.splits;
        const uint32_t threads = p.max_runs < kPlanThreads ? (uint32_t)(p.max_runs + 63) / 64 * 64 : kPlanThreads;
        weight_plan_kernel<<<1, threads, 0, stream>>>(r);
        PL_TRY(launched());    // the next kernel reads the table
    }
    const uint32_t blocks = (uint32_t)(p.tiles_o * p.tiles_i * p.max_runs);
    const uint64_t joins = (out_width * in_width + kBlock - 1) / kBlock;
    const dim3 join((uint32_t)(joins < 4096 ? joins : 4096), (uint32_t)p.max_splits);
    const auto run = [&](auto t) {
        using D = decltype(t);
        PL_TYPE(grad_type, if (p.large) weight_gradient_kernel<D, T, 8, true><<<blocks, 256, 0, stream>>>(g);
                else if (whole) weight_gradient_kernel<D, T, 4, true><<<blocks, 256, 0, stream>>>(g);
                else weight_gradient_kernel<D, T, 4, false><<<blocks, 256, 0, stream>>>(g);
                if (p.max_splits) weight_join_kernel<T><<<join, kBlock, 0, stream>>>(g));
    };
    if (type == POSEIDON_F16)
        run(F16{});
    else
        run(BF16{});
    return launched();
}

}  // extern "C"
