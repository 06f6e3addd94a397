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
// bytes to LDS, where a column's 64 rows of a step lie together.  Half of the
// waves bring dy, the other half the codes, which they also unpack and scale.
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

// Two values that the type holds exactly, as a pair.
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

struct WeightGrad {
    const void *dy;
    uint64_t dy_pitch;
    uint32_t rows, out_width, in_width, groups;
    const int8_t *codes;
    const uint8_t *scales;
    const int32_t *offsets;
    uint32_t tiles_o, tiles_i, splits, accumulate;
    void *grad;      // [ranges][out_width][in_width]
    float *parts;    // [splits][ranges][out_width][in_width] where splits > 1
    uint64_t size;   // ranges * out_width * in_width
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
    uint32_t range, split, tile_o, tile_i;
};

__device__ __forceinline__ Unit unit_of(const WeightGrad &g) {
    const uint32_t tiles = g.tiles_o * g.tiles_i, all = tiles * g.splits;
    Unit u;
    u.range = blockIdx.x / all;
    const uint32_t at = blockIdx.x - u.range * all, xcd = at & 7;
    uint32_t id = xcd * (all / 8) + min(xcd, all & 7) + at / 8;
    u.split = id / tiles;
    id -= u.split * tiles;
    const uint32_t band = id / (4 * g.tiles_i), high = min(4u, g.tiles_o - 4 * band);
    id -= band * 4 * g.tiles_i;
    u.tile_i = id / high;
    u.tile_o = 4 * band + id - u.tile_i * high;
    return u;
}

template <class G>
__device__ __forceinline__ void put(typename G::raw *grad, uint64_t at, float v, uint32_t accumulate) {
    grad[at] = G::down(accumulate ? G::up(grad[at]) + v : v);
}

// WO x WI waves of MO x MI tiles of 32 x 32 each.
template <class T, class G, int WO, int WI, int MO, int MI>
__global__ __launch_bounds__(WO *WI * 64) void weight_gradient_kernel(WeightGrad g) {
    constexpr uint32_t kTileO = WO * MO * 32, kTileI = WI * MI * 32, kWaves = WO * WI;
    static_assert(kTileO / 8 * 8 == kWaves / 2 * 64 && kTileI == kTileO, "an 8 x 8 block a thread");
    __shared__ Words4 lds_o[kTileO * 8], lds_i[kTileI * 8];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);

    const Unit unit = unit_of(g);
    const uint32_t split = unit.split, range = unit.range;
    const uint32_t o0 = unit.tile_o * kTileO, i0 = unit.tile_i * kTileI;
    uint32_t begin = 0, end = g.rows;
    if (g.offsets) {
        begin = (uint32_t)min(max(g.offsets[range], 0), (int32_t)g.rows);
        end = (uint32_t)min(max(g.offsets[range + 1], (int32_t)begin), (int32_t)g.rows);
    }
    {   // this split's steps
        const uint32_t steps = (end - begin + kStep - 1) / kStep, each = (steps + g.splits - 1) / g.splits;
        const uint32_t from = min(split * each, steps), to = min(from + each, steps);
        end = min(end, begin + to * kStep);
        begin += from * kStep;
    }

    // the thread's block: column block cb of the tile, rows [8 oct, 8 oct + 8) of a step
    const bool brings_dy = wave < kWaves / 2;
    const uint32_t block = (wave % (kWaves / 2)) * 64 + lane;
    const uint32_t cb = block % (kTileO / 8), oct = block / (kTileO / 8);
    const typename T::raw *dy = (const typename T::raw *)g.dy;
    const uint32_t o_first = o0 + cb * 8, i_first = i0 + cb * 8;
    // the last block of dy's columns is moved back to end with the row
    const uint32_t o_from = g.out_width >= 8 ? min(o_first, g.out_width - 8) : 0;
    const bool there = brings_dy ? o_first < g.out_width : i_first < g.groups * kGroup;
    const int32_t col0 = brings_dy ? (int32_t)o_from - (int32_t)o0 : (int32_t)(cb * 8);

    uint32_t st[8][4];    // dy: 8 rows of 4 words; codes: 8 rows of 2 words, and the scale byte in word 2
    const auto fetch = [&](uint32_t t0) {
        if (!there) return;
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) {
            const uint32_t row = min(t0 + oct * 8 + r, end - 1);
            if (brings_dy) {
                const typename T::raw *p = dy + (uint64_t)row * g.dy_pitch + o_from;
                if (g.out_width >= 8) {
                    __builtin_memcpy(st[r], p, 16);
                } else {
                    typename T::raw v[8];
#pragma unroll
                    for (uint32_t c = 0; c < 8; ++c) v[c] = c < g.out_width ? p[c] : T::down(0.0f);
                    __builtin_memcpy(st[r], v, 16);
                }
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(g.codes + (uint64_t)row * (g.groups * kGroup) + i_first);
                st[r][0] = w.x;
                st[r][1] = w.y;
                st[r][2] = g.scales[(uint64_t)row * g.groups + i_first / kGroup];
            }
        }
        if (t0 + kStep > end) {    // rows past the end count as zeros
#pragma unroll
            for (uint32_t r = 0; r < 8; ++r) {
                const bool in = t0 + oct * 8 + r < end;
#pragma unroll
                for (int w = 0; w < 4; ++w) st[r][w] = in ? st[r][w] : 0u;
            }
        }
    };
    const auto write = [&]() {
        if (!there) return;
        if (brings_dy) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                Words4 w;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    w[t] = __builtin_amdgcn_perm(st[2 * t + 1][c / 2], st[2 * t][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
                if (col0 + c >= 0) lds_o[place((uint32_t)(col0 + c), oct)] = w;
            }
        } else {
            float scale[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) scale[r] = scale_of(st[r][2]);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                float v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = (float)(int8_t)(st[r][c / 4] >> (8 * (c & 3))) * scale[r];
                Words4 w;
#pragma unroll
                for (int t = 0; t < 4; ++t) w[t] = pack<T>(v[2 * t], v[2 * t + 1]);
                lds_i[place((uint32_t)(col0 + c), oct)] = w;
            }
        }
    };

    const uint32_t wo = wave / WI * (MO * 32), wi = wave % WI * (MI * 32);
    Acc acc[MO][MI] = {};
    if (begin < end) fetch(begin);
    for (uint32_t t0 = begin; t0 < end; t0 += kStep) {
        __syncthreads();
        write();
        __syncthreads();
        if (t0 + kStep < end) fetch(t0 + kStep);
#pragma unroll
        for (uint32_t s = 0; s < kStep / 16; ++s) {
            Words4 a[MO], b[MI];
            const uint32_t oc = s * 2 + lane / 32;
#pragma unroll
            for (int m = 0; m < MO; ++m) a[m] = lds_o[place(wo + m * 32 + lane % 32, oc)];
#pragma unroll
            for (int n = 0; n < MI; ++n) b[n] = lds_i[place(wi + n * 32 + lane % 32, oc)];
#pragma unroll
            for (int m = 0; m < MO; ++m)
#pragma unroll
                for (int n = 0; n < MI; ++n) acc[m][n] = mfma<T>(a[m], b[n], acc[m][n]);
        }
    }

    // value 4 q + e of a tile: row 8 q + 4 (lane / 32) + e, column lane % 32
    const uint64_t base = (uint64_t)range * g.out_width * g.in_width;
#pragma unroll
    for (int m = 0; m < MO; ++m)
#pragma unroll
        for (int n = 0; n < MI; ++n) {
            const uint32_t i = i0 + wi + n * 32 + lane % 32;
            if (i >= g.in_width) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t o = o0 + wo + m * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4;
                if (o >= g.out_width) continue;
                const uint64_t at = base + (uint64_t)o * g.in_width + i;
                if (g.splits > 1)
                    g.parts[split * g.size + at] = acc[m][n][e];
                else
                    put<G>((typename G::raw *)g.grad, at, acc[m][n][e], g.accumulate);
            }
        }
}

// ---- tiles of 256 x 256 ----
//
// Four waves of 128 x 128 each: a wave reads 8 KB of LDS for 16 matrix
// instructions of 32 cycles, half of what LDS delivers, where 8 waves of 128 x 64 would ask for
// three quarters and the writes come on top.  With 256 sums a lane
// there is one wave a SIMD, so nothing hides behind another wave: LDS holds two
// steps, and while the matrix instructions work on one, the rows of
// the next are turned and unpacked between them and those of the one after are on
// their way.  Rows past the end come back as zeros from the buffers' bounds.

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

template <class T, class G>
__global__ __launch_bounds__(256, 1) void weight_gradient_wide_kernel(WeightGrad g) {
    constexpr uint32_t kTile = 256, kPad = 8;    // a tile's first block may begin up to 7 columns before it
    constexpr uint32_t kBuf = (kTile + kPad) * 8;
    __shared__ Words4 lds[4 * kBuf];             // dy's two steps, then x's
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);

    const Unit unit = unit_of(g);
    const uint32_t split = unit.split, range = unit.range;
    const uint32_t o0 = unit.tile_o * kTile, i0 = unit.tile_i * kTile;
    uint32_t begin = 0, end = g.rows;
    if (g.offsets) {
        begin = (uint32_t)min(max(g.offsets[range], 0), (int32_t)g.rows);
        end = (uint32_t)min(max(g.offsets[range + 1], (int32_t)begin), (int32_t)g.rows);
    }
    {   // this split's steps
        const uint32_t steps = (end - begin + kStep - 1) / kStep, each = (steps + g.splits - 1) / g.splits;
        const uint32_t from = min(split * each, steps), to = min(from + each, steps);
        end = min(end, begin + to * kStep);
        begin += from * kStep;
    }

    const uint32_t cb = tid % (kTile / 8), oct = tid / (kTile / 8);
    const uint32_t o_first = o0 + cb * 8, i_first = i0 + cb * 8;
    const uint32_t o_from = min(o_first, g.out_width - 8);
    const uint32_t dy_row = (uint32_t)g.dy_pitch * 2, x_row = g.groups * kGroup;    // bytes
    constexpr uint32_t kNowhere = 0x80000000u;
    const uint32_t dy_at = o_first < g.out_width ? oct * 8 * dy_row + o_from * 2 : kNowhere;
    const uint32_t x_at = i_first < x_row ? oct * 8 * x_row + i_first : kNowhere;
    const uint32_t s_at = i_first < x_row ? oct * 8 * g.groups + i_first / kGroup : kNowhere;
    const int32_t col0 = o_first < g.out_width ? (int32_t)o_from - (int32_t)o0 : (int32_t)(cb * 8);

    // Two steps' rows are on their way in registers while a third is in LDS.  A row's buffer begins at the row, so
    // the lanes' offsets are the same for all eight.
    Words4 dy[2][8];
    uint2 x[2][8];
    uint32_t sc[2][8];
    const auto rows_of = [&](const void *base, uint32_t row, uint32_t t0, uint32_t r) {
        const uint32_t n = t0 + r < end ? min(end - t0, kStep) - r : 0, t = n ? t0 + r : 0;
        return buffer((const char *)base + (uint64_t)t * row, n * row);
    };
    const auto fetch_dy = [&](int set, uint32_t t0, uint32_t r) {
        dy[set][r] = __builtin_amdgcn_raw_buffer_load_b128(rows_of(g.dy, dy_row, t0, r), dy_at, 0, 0);
    };
    const auto fetch_x = [&](int set, uint32_t t0, uint32_t r) {
        x[set][r] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rows_of(g.codes, x_row, t0, r), x_at, 0, 0));
        sc[set][r] = __builtin_amdgcn_raw_buffer_load_b8(rows_of(g.scales, g.groups, t0, r), s_at, 0, 0);
    };
    const auto write_dy = [&](int set, uint32_t buf, int c) {    // column c of the thread's block
        Words4 w;
#pragma unroll
        for (int t = 0; t < 4; ++t)
            w[t] = __builtin_amdgcn_perm(dy[set][2 * t + 1][c / 2], dy[set][2 * t][c / 2],
                                         c & 1 ? 0x07060302u : 0x05040100u);
        const uint32_t col = (uint32_t)(col0 + c);
        lds[buf * kBuf + kPad * 8 + (int32_t)place(col, oct)] = w;
    };
    // Rows 2 t and 2 t + 1 of column c; with the last two the column is written.
    // A group of scale byte 255 has codes 0, and 0 times the infinity that byte stands for is NaN.
    Words4 turned;
    const auto unpack_x = [&](int set, uint32_t buf, auto column, int t) {
        constexpr int c = decltype(column)::value;
        float v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 2 * t + h;
            v[h] = signed_byte<c & 3>(c < 4 ? x[set][r].x : x[set][r].y) * __uint_as_float(sc[set][r] << 23);
        }
        turned[t] = pack<T>(v[0], v[1]);
        if (t == 3) lds[(2 + buf) * kBuf + kPad * 8 + place(cb * 8 + c, oct)] = turned;
    };

    // word of column (wave's first + 32 m + lane % 32), rows [16 s + 8 (lane / 32), ...): off[s ^ 2 (m & 1)] + 256 m
    const uint32_t c32 = lane % 32, key = (lane / 32 ^ c32 ^ c32 >> 3) & 7;
    const uint32_t at_o = kPad * 8 + (wave / 2 * 128 + c32) * 8, at_i = 2 * kBuf + kPad * 8 + (wave % 2 * 128 + c32) * 8;
    Words4 a[2][4], b[2][4];
    const auto read = [&](uint32_t buf, int s, int j) {    // one of the eight reads of quarter s
        const int m = j / 2;
        const uint32_t w = buf * kBuf + (key ^ (2 * (s ^ 2 * (m & 1)))) + m * 256;
        if (j & 1)
            b[s & 1][m] = lds[at_i + w];
        else
            a[s & 1][m] = lds[at_o + w];
    };
    Acc acc[4][4] = {};

    // A quarter of a step: 16 matrix instructions, and after each a little of the
    // other work, which the instruction's 32 cycles cover.  Quarters 0 and 1 unpack the next step's x,
    // quarter 2 turns its dy, quarter 3 reads from the next step's LDS words, written by then.
    const auto quarter = [&](auto which, auto step, uint32_t t0) {
        constexpr int s = decltype(which)::value, buf = decltype(step)::value, set = buf ^ 1;
        const auto piece = [&](auto index) {
            constexpr int j = decltype(index)::value;
            acc[j / 4][j % 4] = mfma<T>(a[s & 1][j / 4], b[s & 1][j % 4], acc[j / 4][j % 4]);
            if constexpr (j < 8) read(s < 3 ? buf : buf ^ 1, (s + 1) & 3, j);
            if constexpr (s < 2) unpack_x(set, buf ^ 1, Int<s * 4 + j / 4>{}, j % 4);
            if constexpr (s == 2 && j < 8) write_dy(set, buf ^ 1, j);
            if constexpr (s == 2 && j >= 8) fetch_x(set, t0 + 3 * kStep, j - 8);
            if constexpr (s == 3 && j < 8) fetch_dy(set, t0 + 3 * kStep, j);
            __builtin_amdgcn_sched_barrier(0);
        };
        each<16>(piece);
    };
    // Multiplies the step in LDS buffer `buf`, and writes the next one (set buf ^ 1) to the other.
    const auto step = [&](auto buf, uint32_t t0) {
        quarter(Int<0>{}, buf, t0);
        quarter(Int<1>{}, buf, t0);
        quarter(Int<2>{}, buf, t0);
        __syncthreads();    // the other buffer is whole, and this one read
        quarter(Int<3>{}, buf, t0);
    };

    if (begin < end) {
        each<8>([&](auto r) {
            fetch_x(0, begin, decltype(r)::value);
            fetch_dy(0, begin, decltype(r)::value);
        });
        each<8>([&](auto r) {
            fetch_x(1, begin + kStep, decltype(r)::value);
            fetch_dy(1, begin + kStep, decltype(r)::value);
        });
        each<8>([&](auto c) {
            write_dy(0, 0, decltype(c)::value);
            each<4>([&](auto t) { unpack_x(0, 0, c, decltype(t)::value); });
        });
        each<8>([&](auto r) {
            fetch_x(0, begin + 2 * kStep, decltype(r)::value);
            fetch_dy(0, begin + 2 * kStep, decltype(r)::value);
        });
        __syncthreads();
        each<8>([&](auto j) { read(0, 0, decltype(j)::value); });
        for (uint32_t t0 = begin; t0 < end; t0 += 2 * kStep) {
            step(Int<0>{}, t0);
            step(Int<1>{}, t0 + kStep);    // all zeros after an odd number of steps
        }
    }

    const uint64_t base = (uint64_t)range * g.out_width * g.in_width;
    const uint32_t wo = wave / 2 * 128, wi = wave % 2 * 128;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t i = i0 + wi + n * 32 + lane % 32;
            if (i >= g.in_width) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t o = o0 + wo + m * 32 + e / 4 * 8 + lane / 32 * 4 + e % 4;
                if (o >= g.out_width) continue;
                const uint64_t at = base + (uint64_t)o * g.in_width + i;
                if (g.splits > 1)
                    g.parts[split * g.size + at] = acc[m][n][e];
                else
                    put<G>((typename G::raw *)g.grad, at, acc[m][n][e], g.accumulate);
            }
        }
}

// Adds the splits' parts, in order.
template <class G>
__global__ __launch_bounds__(kBlock) void weight_gradient_join_kernel(const float *parts, uint64_t size, uint32_t splits,
                                                                      uint32_t accumulate, typename G::raw *grad) {
    for (uint64_t i = (uint64_t)blockIdx.x * kBlock + threadIdx.x; i < size; i += (uint64_t)gridDim.x * kBlock) {
        float sum = 0.0f;
        for (uint32_t s = 0; s < splits; ++s) sum += parts[s * size + i];
        put<G>(grad, i, sum, accumulate);
    }
}

struct WeightPlan {
    bool large;
    uint32_t tiles_o, tiles_i, splits;
};

// Tiles of 256 x 256 where those give every second CU one, else tiles of 128 x 128; then the rows of each
// range are split until there are about 512 blocks, each with 8 steps or more if the ranges were equal.
inline WeightPlan weight_plan(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges) {
    WeightPlan p;
    const uint64_t at256 = ((out_width + 255) / 256) * ((in_width + 255) / 256) * n_ranges;
    p.large = at256 >= 128;
    const uint32_t side = p.large ? 256 : 128;
    p.tiles_o = (uint32_t)((out_width + side - 1) / side);
    p.tiles_i = (uint32_t)((in_width + side - 1) / side);
    const uint64_t units = (uint64_t)p.tiles_o * p.tiles_i * n_ranges;
    const uint64_t by_rows = rows / n_ranges / (8 * kStep);
    uint64_t s = (p.large ? 256 : 512) / units;
    s = s < by_rows ? s : by_rows;
    p.splits = (uint32_t)(s < 1 ? 1 : s);
    return p;
}

inline int check_weight(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges) {
    PL_TRY(check_sizes(rows, out_width));
    PL_TRY(check_sizes(rows, in_width));
    if (!n_ranges) return POSEIDON_E_INVAL;
    if (n_ranges > POSEIDON_RANGES_MAX) return POSEIDON_E_RANGE;
    const uint64_t tiles = ((out_width + 127) / 128) * ((in_width + 127) / 128);
    return tiles * n_ranges > POSEIDON_TILES_MAX ? POSEIDON_E_RANGE : POSEIDON_OK;    // blocks of one launch
}

}  // namespace pl

using namespace pl;

extern "C" {

uint64_t poseidon_weight_gradient_workspace(uint64_t rows, uint64_t out_width, uint64_t in_width, uint32_t n_ranges) {
    if (check_weight(rows, out_width, in_width, n_ranges) != POSEIDON_OK) return UINT64_MAX;
    const WeightPlan p = weight_plan(rows, out_width, in_width, n_ranges);
    return p.splits > 1 ? p.splits * (uint64_t)n_ranges * out_width * in_width * 4 : 0;
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
    WeightPlan p = weight_plan(rows, out_width, in_width, n_ranges);
    // The wide kernel's buffer loads want whole words of dy.
    const bool wide = p.large && aligned(dy, 4) && dy_pitch % 2 == 0 && out_width % 2 == 0 && out_width >= 8;
    if (p.large && !wide) {
        p.tiles_o = (uint32_t)((out_width + 127) / 128);
        p.tiles_i = (uint32_t)((in_width + 127) / 128);
    }
    WeightGrad g = {};
    g.dy = dy;
    g.dy_pitch = dy_pitch;
    g.rows = (uint32_t)rows;
    g.out_width = (uint32_t)out_width;
    g.in_width = (uint32_t)in_width;
    g.groups = groups_of(in_width);
    g.codes = codes;
    g.scales = scales;
    g.offsets = offsets;
    g.tiles_o = p.tiles_o;
    g.tiles_i = p.tiles_i;
    g.splits = p.splits;
    g.accumulate = accumulate;
    g.grad = grad;
    g.parts = (float *)workspace;
    g.size = (uint64_t)n_ranges * out_width * in_width;
    const uint32_t blocks = p.tiles_o * p.tiles_i * p.splits * n_ranges;
    const auto run = [&](auto t) {
        using D = decltype(t);
        PL_TYPE(grad_type, if (wide) weight_gradient_wide_kernel<D, T><<<blocks, 256, 0, stream>>>(g);
                else weight_gradient_kernel<D, T, 2, 2, 2, 2><<<blocks, 256, 0, stream>>>(g);
                if (p.splits > 1) {
                    const uint64_t n = (g.size + kBlock - 1) / kBlock;
                    weight_gradient_join_kernel<T><<<(uint32_t)(n < 4096 ? n : 4096), kBlock, 0, stream>>>(
                        g.parts, g.size, g.splits, g.accumulate, (T::raw *)grad);
                });
    };
    if (type == POSEIDON_F16)
        run(F16{});
    else
        run(BF16{});
    return launched();
}

}  // extern "C"
