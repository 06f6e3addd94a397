// Root-mean-square norm of poseidon_layers.h with the residual's addition, and its gradient:
//   h = x + r, n = h / sqrt(mean h^2 + eps), out = n w;
//   g = w dout, dx = dsum + rstd (g - n mean(n g)), dw = sum over the rows of dout n.
//
// A team of lanes holds a row in registers, so every operand is read once; memory bounds both directions.  Teams stay for
// many rows: they read the weights once, and the backward pass holds its sums for dw in registers until its last row.
// Widths of whole pieces of 16 bytes run at 4.5 to 5.8 TB/s forward and backward up to 8192 values, where a plain copy kernel
// reaches 6.2 at 1 GiB and the library's copy 5.2, wider ones at 3.3 to 5.2 (two slices a lane backward do not fit the registers), odd ones at 3.3 to 4.1.
#include "layers_device.h"

#include <type_traits>

namespace pl {

constexpr uint32_t kNormWidth = POSEIDON_NORM_WIDTH_MAX;
constexpr uint32_t kWhole = 0;    // a team of as many waves as its block has, which meet at barriers
template <uint32_t TEAM>
struct Team {
    static constexpr uint32_t kPerBlock = TEAM == kWhole ? 1 : kBlock / TEAM;
    static constexpr uint32_t kMost = TEAM == kWhole ? 1024 : kBlock;    // threads of a block
    static constexpr uint32_t kSlots = TEAM == kWhole ? 16 : 1;          // one for each wave that may meet
    static __device__ __forceinline__ uint32_t size() { return TEAM == kWhole ? blockDim.x : TEAM; }
};

// Waves that a SIMD has at a time: what their registers allow, but for a few that are kept in memory (forward in 16 bits with one
// slice 3 to 5, backward from the sum as it is 2 to 3).  Forward in 16 bits: 32768 x 8192 with the residual and the sum kept 438 us,
// with six or seven waves, which keep none in memory, 471; 21845 x 6144 without what is kept 191 and 186.  Forward in 32 bits
// eight would keep many there (32768 x 4096, the sum kept too: 569 us, with six 486).
// So would six waves backward from 8 bits (32768 x 8192: 528 us, with five 367); from the sum as it is 32768 x 4096 takes 193 us
// with six and 222 with five, in 32 bits 416 and 408.
template <class T, uint32_t N>
constexpr uint32_t kForwardWaves = N == 1 ? (T::kShort ? 8 : 6) : 4;
template <uint32_t TEAM, uint32_t N, bool KEPT>
constexpr uint32_t kBackwardWaves = N == 2 ? 4 : TEAM == kWhole && !KEPT ? 6 : 5;

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }

// `op` over the lanes of a team, in one order; `slots`: a word for each wave, 0 past the team's (which `op` leaves alone), not in use
// by an earlier call that a wave may still read.
template <uint32_t TEAM, class V, class F>
__device__ __forceinline__ V over_team(V v, F op, V *slots) {
#pragma unroll
    for (uint32_t d = (TEAM == kWhole ? 64 : TEAM) / 2; d; d >>= 1) v = op(v, __shfl_xor(v, (int)d, 64));
    if constexpr (TEAM == kWhole) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x / 64] = v;
        __syncthreads();
        v = slots[0];
#pragma unroll
        for (uint32_t w = 1; w < Team<TEAM>::kSlots; ++w) v = op(v, slots[w]);
    }
    return v;
}

__device__ __forceinline__ void load_weight(const void *weight, uint32_t type, uint32_t col, uint32_t width, float (&v)[8]) {
    if (type == POSEIDON_F32)
        load_slice<F32>((const float *)weight, col, width, v);
    else if (type == POSEIDON_F16)
        load_slice<F16>((const _Float16 *)weight, col, width, v);
    else
        load_slice<BF16>((const __bf16 *)weight, col, width, v);
}

struct NormForward {
    const void *x, *residual, *weight;
    uint64_t x_pitch, residual_pitch;
    uint32_t rows, width, padded, weight_type;    // padded: slices of a row with its last group filled up
    float eps;
    void *out, *sum;
    uint64_t out_pitch, sum_pitch;
    float *rstd;
    int8_t *out_codes, *sum_codes;
    uint8_t *out_scales, *sum_scales;
};

// Values as their type holds them: what is kept in 8 bits is the 8-bit form of what was written in 16.
template <class T>
__device__ __forceinline__ void as_written(const float (&v)[8], float (&r)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = T::up(T::down(v[i]));
}

template <class T, bool STREAM>
__device__ __forceinline__ void keep_slice(const float (&v)[8], uint64_t row, uint32_t s, uint32_t padded, int8_t *codes,
                                           uint8_t *scales) {
    const uint32_t byte = scale_byte<T>(v);
    uint32_t w[2];
    codes_of(v, byte, w);
    if (s < padded) {
        store_codes<STREAM>(codes, row * padded + s, w);
        if (!(s & 7)) scales[(row * padded + s) >> 3] = (uint8_t)byte;
    }
}

// 1 / sqrt(mean h^2 + eps) of a row whose squares leave the 32-bit range: of h 2^-e, where 2^e is about the largest value.
template <uint32_t TEAM, uint32_t N>
__device__ __forceinline__ float far_rstd(const float (&h)[N][8], float size, float eps, float plain, float *sums,
                                          uint32_t *most) {
    uint32_t m = 0;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(h[j][i]) & 0x7fffffffu);
    m = over_team<TEAM>(m, larger, most);
    if (m == 0 || m >= 0x7f800000u) return plain;
    const int e = __builtin_amdgcn_frexp_expf(__uint_as_float(m));
    float ss = 0.0f;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = ldexpf(h[j][i], -e);
            ss = fmaf(v, v, ss);
        }
    ss = over_team<TEAM>(ss, add, sums);
    const float scaled = ldexpf(eps, -2 * e);
    return scaled > 1e30f ? 1.0f / sqrtf(eps) : ldexpf(1.0f / sqrtf(ss / size + scaled), -e);
}

template <class T, uint32_t TEAM, uint32_t N, bool STREAM>
__global__ __launch_bounds__(Team<TEAM>::kMost, (kForwardWaves<T, N>)) void norm_forward_kernel(NormForward a) {
    __shared__ __attribute__((aligned(16))) float sums[3][Team<TEAM>::kSlots];
    __shared__ __attribute__((aligned(16))) uint32_t most[Team<TEAM>::kSlots];
    const uint32_t lanes = Team<TEAM>::size(), lane = TEAM == kWhole ? threadIdx.x : threadIdx.x % TEAM;
    const uint32_t first = blockIdx.x * Team<TEAM>::kPerBlock + (TEAM == kWhole ? 0 : threadIdx.x / lanes), step = gridDim.x * Team<TEAM>::kPerBlock;
    if constexpr (TEAM == kWhole) {
        if (threadIdx.x < 16) sums[0][threadIdx.x] = sums[1][threadIdx.x] = sums[2][threadIdx.x] = 0.0f, most[threadIdx.x] = 0;
        __syncthreads();
    }
    const float size = (float)a.width;
    float w[N][8];
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) load_weight(a.weight, a.weight_type, (lane + j * lanes) * kSlice, a.width, w[j]);
    uint32_t turn = 0;
    for (uint64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const typename T::raw *x = (const typename T::raw *)a.x + row * a.x_pitch;
        float h[N][8];
        Slice<T> in[N], more[N];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) in[j] = load_words<T, STREAM>(x, (lane + j * lanes) * kSlice, a.width);
        if (a.residual) {
            const typename T::raw *r = (const typename T::raw *)a.residual + row * a.residual_pitch;
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) more[j] = load_words<T, STREAM>(r, (lane + j * lanes) * kSlice, a.width);
        }
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) values<T>(in[j], h[j]);
        if (a.residual) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                float r[8];
                values<T>(more[j], r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[j][i] += r[i];
            }
        }
        float ss = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(h[j][i], h[j][i], ss);
        ss = over_team<TEAM>(ss, add, sums[turn]);
        float rstd = 1.0f / sqrtf(ss / size + a.eps);
        if (!(ss > 1e-24f && ss < 1e36f)) rstd = far_rstd<TEAM, N>(h, size, a.eps, rstd, sums[2], most);
        if (lane == 0 && a.rstd) a.rstd[row] = rstd;
        if (a.sum) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j)
                store_slice<T, STREAM>((typename T::raw *)a.sum + row * a.sum_pitch, (lane + j * lanes) * kSlice, a.width, h[j]);
        }
        if (a.sum_codes) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                float v[8];
                as_written<T>(h[j], v);
                keep_slice<T, STREAM>(v, row, lane + j * lanes, a.padded, a.sum_codes, a.sum_scales);
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] = h[j][i] * rstd * w[j][i];
        if (a.out) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j)
                store_slice<T, STREAM>((typename T::raw *)a.out + row * a.out_pitch, (lane + j * lanes) * kSlice, a.width, h[j]);
        }
        if (a.out_codes) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                float v[8];
                as_written<T>(h[j], v);
                keep_slice<T, STREAM>(v, row, lane + j * lanes, a.padded, a.out_codes, a.out_scales);
            }
        }
    }
}

struct NormBackward {
    const void *dout, *h, *dsum, *weight;
    uint64_t dout_pitch, h_pitch, dsum_pitch, dx_pitch;
    const int8_t *codes;
    const uint8_t *scales;
    const float *rstd;
    uint32_t rows, width, padded, weight_type;
    void *dx;
    float *parts;    // [gridDim.x][width] sums for dw, null: no weight gradient
};

template <class T, bool KEPT, uint32_t TEAM, uint32_t N, bool STREAM>
__global__ __launch_bounds__(Team<TEAM>::kMost, (kBackwardWaves<TEAM, N, KEPT>)) void norm_backward_kernel(NormBackward a) {
    __shared__ __attribute__((aligned(16))) float sums[2][Team<TEAM>::kSlots];
    const uint32_t lanes = Team<TEAM>::size(), lane = TEAM == kWhole ? threadIdx.x : threadIdx.x % TEAM;
    if constexpr (TEAM == kWhole) {
        if (threadIdx.x < 16) sums[0][threadIdx.x] = sums[1][threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const uint32_t team = TEAM == kWhole ? 0 : threadIdx.x / lanes, first = blockIdx.x * Team<TEAM>::kPerBlock + team, step = gridDim.x * Team<TEAM>::kPerBlock;
    const float size = (float)a.width;
    float w[N][8], dw[N][8] = {};
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) load_weight(a.weight, a.weight_type, (lane + j * lanes) * kSlice, a.width, w[j]);
    uint32_t turn = 0;
    for (uint64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const typename T::raw *dout = (const typename T::raw *)a.dout + row * a.dout_pitch;
        Slice<T> in[N], more[N], at[N];
        uint32_t code[N][2];
        float scale[N];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) in[j] = load_words<T, STREAM>(dout, (lane + j * lanes) * kSlice, a.width);
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            const uint32_t s = lane + j * lanes;
            if constexpr (KEPT) {
                const uint64_t i = row * a.padded + (s < a.padded ? s : 0);
                load_codes<STREAM>(a.codes, i, code[j]);
                scale[j] = scale_of(a.scales[i >> 3]);
            } else {
                at[j] = load_words<T, STREAM>((const typename T::raw *)a.h + row * a.h_pitch, s * kSlice, a.width);
            }
        }
        if (a.dsum) {
            const typename T::raw *d = (const typename T::raw *)a.dsum + row * a.dsum_pitch;
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) more[j] = load_words<T, STREAM>(d, (lane + j * lanes) * kSlice, a.width);
        }
        const float rstd = a.rstd[row];
        float g[N][8], n[N][8], dot = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            values<T>(in[j], g[j]);
            if constexpr (KEPT)
                values_of(code[j], lane + j * lanes < a.padded ? scale[j] : 0.0f, n[j]);
            else
                values<T>(at[j], n[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {    // past the row dout counts as 0
                n[j][i] *= rstd;
                dw[j][i] = fmaf(g[j][i], n[j][i], dw[j][i]);
                g[j][i] *= w[j][i];
                dot = fmaf(g[j][i], n[j][i], dot);
            }
        }
        dot = over_team<TEAM>(dot, add, sums[turn]) / size;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            float d[8] = {};
            if (a.dsum) values<T>(more[j], d);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, fmaf(-dot, n[j][i], g[j][i]), d[i]);
            store_slice<T, STREAM>((typename T::raw *)a.dx + row * a.dx_pitch, (lane + j * lanes) * kSlice, a.width, d);
        }
    }
    if (!a.parts) return;
    float *part = a.parts + (uint64_t)blockIdx.x * a.width;
    if constexpr (Team<TEAM>::kPerBlock > 1) {    // the block's teams, in order
        __shared__ float all[Team<TEAM>::kPerBlock][TEAM * N * 8];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) all[team][(lane + j * lanes) * kSlice + i] = dw[j][i];
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.width; c += kBlock) {
            float v = 0.0f;
#pragma unroll
            for (uint32_t t = 0; t < Team<TEAM>::kPerBlock; ++t) v += all[t][c];
            part[c] = v;
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t c = (lane + j * lanes) * kSlice + i;
                if (c < a.width) part[c] = dw[j][i];
            }
    }
}

// dw: 16 columns a block, sixteen lanes to each, which add every sixteenth part; then these, in order.
__global__ __launch_bounds__(kBlock) void norm_join_kernel(const float *parts, uint32_t n, uint32_t width, float *dweight,
                                                           uint32_t accumulate) {
    __shared__ float all[16][17];
    const uint32_t c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float v = 0.0f;
    if (col < width) {
#pragma unroll 8
        for (uint32_t p = r; p < n; p += 16) v += parts[(uint64_t)p * width + col];
    }
    all[r][c] = v;
    __syncthreads();
    if (r || col >= width) return;
    for (uint32_t t = 1; t < 16; ++t) v += all[t][c];
    dweight[col] = accumulate ? dweight[col] + v : v;
}

// Runs f(team size, slices a lane, threads of a block) for the smallest team that holds a row; a block that is a team has as
// many waves as that takes (26214 x 5120 with residual: 205 us, in eight waves of two slices 245).
template <class F>
inline void for_width(uint32_t padded, bool two, F f) {
    using std::integral_constant;
    const auto of = [&](auto n) {
        const uint32_t lanes = (padded + n.value - 1) / n.value;
        if (lanes <= 16)
            f(integral_constant<uint32_t, 16>{}, n, kBlock);
        else if (lanes <= 32)
            f(integral_constant<uint32_t, 32>{}, n, kBlock);
        else if (lanes <= 64)
            f(integral_constant<uint32_t, 64>{}, n, kBlock);
        else
            f(integral_constant<uint32_t, kWhole>{}, n, (lanes + 63) / 64 * 64);
    };
    if (two || padded > 1024)
        of(integral_constant<uint32_t, 2>{});
    else
        of(integral_constant<uint32_t, 1>{});
}
// Forward a lane has two slices where a team is a wave or less (262144 x 512: 98 us, in whole waves of one 169), one where it is
// a block: 64 registers a lane then and twice the waves (32768 x 4096 with residual: 194 us either way, 21845 x 6144 192 and
// 288, 65536 x 2048 195 and 221).  Backward it holds sums besides (65536 x 4096: 390 us with one, 523 with two).
template <class F>
inline void for_forward(uint32_t padded, F f) {
    for_width(padded, padded > 16 && padded <= 128, f);
}
template <class F>
inline void for_backward(uint32_t padded, F f) {
    for_width(padded, false, f);
}

// Blocks that the chip holds at a time, `waves` of their waves a SIMD, or fewer where the rows are: a block more a CU would begin
// when the others end (26214 x 5120 with two blocks of ten waves a CU 205 us, with three 245).  A block's waves go to the four SIMDs
// in turn, and blocks that fill 17 of 20 places have found theirs.
template <uint32_t TEAM>
inline uint32_t norm_blocks(uint64_t rows, uint32_t block, uint32_t waves) {
    const uint32_t w = block / 64, whole = w <= 4 ? 4 / w * waves : waves / ((w + 3) / 4), part = 17 * waves / (5 * w);
    const uint64_t n = (rows + Team<TEAM>::kPerBlock - 1) / Team<TEAM>::kPerBlock, most = 256 * (whole > part ? whole : part);
    return (uint32_t)(n < most ? n : most);
}
// Backward each is a row of sums for dw besides, so a team has four rows, where that leaves 512 blocks (4096 x 1024: 17 us, with as
// many as the chip holds 28, with 16 rows a team 25; 65536 x 128: 17 us, with eight rows 21).
template <uint32_t TEAM>
inline uint32_t norm_parts(uint64_t rows, uint32_t block, uint32_t waves) {
    const uint64_t most = rows / (4 * Team<TEAM>::kPerBlock), least = 512, n = norm_blocks<TEAM>(rows, block, waves);
    return (uint32_t)(n < least || n < most ? n : most < least ? least : most);
}
inline uint32_t norm_padded(uint64_t width) { return groups_of(width) * (kGroup / kSlice); }

}  // namespace pl

using namespace pl;

extern "C" {

int poseidon_norm_forward(const void *x, uint64_t x_pitch, const void *residual, uint64_t residual_pitch, uint32_t type,
                          uint64_t rows, uint64_t width, const void *weight, uint32_t weight_type, float eps, void *out,
                          uint64_t out_pitch, void *sum, uint64_t sum_pitch, float *rstd, int8_t *out_codes,
                          uint8_t *out_scales, int8_t *sum_codes, uint8_t *sum_scales, void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    if (width > kNormWidth) return POSEIDON_E_RANGE;
    if (!(eps >= 0.0f && eps < __builtin_inff())) return POSEIDON_E_INVAL;
    PL_TRY(check_matrix(x, x_pitch, type, rows, width));
    if (residual) PL_TRY(check_matrix(residual, residual_pitch, type, rows, width));
    PL_TRY(check_matrix(weight, width, weight_type, rows, width));
    const bool keep_out = out_codes || out_scales, keep_sum = sum_codes || sum_scales;
    if (rows && !out && !keep_out) return POSEIDON_E_INVAL;
    if (out) PL_TRY(check_matrix(out, out_pitch, type, rows, width));
    if (sum) PL_TRY(check_matrix(sum, sum_pitch, type, rows, width));
    if (keep_out) PL_TRY(check_stash(out_codes, out_scales, rows));
    if (keep_sum) PL_TRY(check_stash(sum_codes, sum_scales, rows));
    if (!aligned(rstd, 4)) return POSEIDON_E_INVAL;
    if (!rows) return POSEIDON_OK;
    const uint32_t padded = norm_padded(width);
    const NormForward a = {x,   residual, weight,    x_pitch,   residual_pitch, (uint32_t)rows, (uint32_t)width,
                           padded, weight_type, eps, out, sum, out_pitch, sum_pitch, rstd,
                           out_codes, sum_codes, out_scales, sum_scales};
    const uint32_t size = size_of(type);
    const uint64_t bytes = rows * width * (size * (1 + !!residual + !!out + !!sum) + keep_out + keep_sum);
    PL_STREAM(bytes, PL_TYPE(type, for_forward(padded, [&](auto team, auto n, uint32_t block) {
        if constexpr (n.value == 2 || team.value == 16 || team.value == kWhole)
            norm_forward_kernel<T, team.value, n.value, STREAM>
                <<<norm_blocks<team.value>(rows, block, kForwardWaves<T, n.value>), block, 0, (hipStream_t)hip_stream>>>(a);
    })));
    return launched();
}

uint64_t poseidon_norm_backward_workspace(uint64_t rows, uint64_t width) {
    if (check_sizes(rows, width) != POSEIDON_OK || width > kNormWidth) return UINT64_MAX;
    uint64_t parts = 0;    // of a sum that is not in 8 bits, which has more of them
    for_backward(norm_padded(width), [&](auto team, auto n, uint32_t block) {
        parts = norm_parts<team.value>(rows, block, kBackwardWaves<team.value, n.value, false>);
    });
    return parts * width * 4;
}

int poseidon_norm_backward(const void *dout, uint64_t dout_pitch, uint32_t type, uint64_t rows, uint64_t width,
                           const void *sum, uint64_t sum_pitch, const int8_t *codes, const uint8_t *scales,
                           const float *rstd, const void *weight, uint32_t weight_type, const void *dsum,
                           uint64_t dsum_pitch, void *dx, uint64_t dx_pitch, float *dweight, uint32_t accumulate,
                           void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    if (width > kNormWidth) return POSEIDON_E_RANGE;
    PL_TRY(check_matrix(dout, dout_pitch, type, rows, width));
    const bool kept = codes || scales;
    if (rows && kept == !!sum) return POSEIDON_E_INVAL;
    if (kept) PL_TRY(check_stash(codes, scales, rows));
    if (sum) PL_TRY(check_matrix(sum, sum_pitch, type, rows, width));
    PL_TRY(check_matrix(weight, width, weight_type, rows, width));
    if (dsum) PL_TRY(check_matrix(dsum, dsum_pitch, type, rows, width));
    PL_TRY(check_matrix(dx, dx_pitch, type, rows, width));
    if (rows && (!rstd || !aligned(rstd, 4))) return POSEIDON_E_INVAL;
    if (accumulate > 1 || !aligned(dweight, 4) || (accumulate && !dweight)) return POSEIDON_E_INVAL;
    if (dweight) PL_TRY(check_workspace(workspace, workspace_bytes, poseidon_norm_backward_workspace(rows, width)));
    const uint32_t padded = norm_padded(width);
    uint32_t blocks = 0;
    if (rows) {
        const NormBackward a = {dout, sum, dsum, weight, dout_pitch, sum_pitch, dsum_pitch, dx_pitch, codes, scales, rstd,
                                (uint32_t)rows, (uint32_t)width, padded, weight_type, dx, dweight ? (float *)workspace : nullptr};
        const uint32_t size = size_of(type);
        const uint64_t bytes = rows * width * (size * (2 + !kept + !!dsum) + kept);
        PL_STREAM(bytes, PL_TYPE(type, for_backward(padded, [&](auto team, auto n, uint32_t block) {
            if constexpr (n.value == 1 || team.value == kWhole) {
                const auto go = [&](auto kernel, uint32_t waves) {
                    blocks = norm_parts<team.value>(rows, block, waves);
                    kernel<<<blocks, block, 0, (hipStream_t)hip_stream>>>(a);
                };
                if (kept)
                    go(norm_backward_kernel<T, true, team.value, n.value, STREAM>, kBackwardWaves<team.value, n.value, true>);
                else
                    go(norm_backward_kernel<T, false, team.value, n.value, STREAM>, kBackwardWaves<team.value, n.value, false>);
            }
        })));
        PL_TRY(launched());
    }
    if (dweight && (rows || !accumulate)) {
        norm_join_kernel<<<(uint32_t)((width + 15) / 16), kBlock, 0, (hipStream_t)hip_stream>>>(
            (const float *)workspace, blocks, (uint32_t)width, dweight, accumulate);
        return launched();
    }
    return POSEIDON_OK;
}

}  // extern "C"
