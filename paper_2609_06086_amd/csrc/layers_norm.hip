// Root-mean-square norm of poseidon_layers.h with the residual's addition, and its gradient:
//   h = x + r, n = h / sqrt(mean h^2 + eps), out = n w;
//   g = w dout, dx = dsum + rstd (g - n mean(n g)), dw = sum over the rows of dout n.
//
// A team of lanes holds a row in registers, so every operand is read once; memory bounds both directions.  Teams stay for
// many rows: they read the weights once, and the backward pass holds its sums for dw in registers until its last row.
#include "layers_device.h"

#include <type_traits>

namespace pl {

constexpr uint32_t kNormWidth = POSEIDON_NORM_WIDTH_MAX;
template <uint32_t TEAM>
struct Team {
    static constexpr uint32_t kThreads = TEAM <= 64 ? kBlock : TEAM;    // teams that meet at barriers have a block each
    static constexpr uint32_t kPerBlock = kThreads / TEAM;
    static constexpr uint32_t kWaves = TEAM < 64 ? 1 : TEAM / 64;
};

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }

// `op` over the lanes of a team, in one order; `slots`: one word a wave, not in use by an earlier call that a wave may
// still read.
template <uint32_t TEAM, class V, class F>
__device__ __forceinline__ V over_team(V v, F op, V *slots) {
#pragma unroll
    for (uint32_t d = (TEAM < 64 ? TEAM : 64) / 2; d; d >>= 1) v = op(v, __shfl_xor(v, (int)d, 64));
    if constexpr (TEAM > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x / 64] = v;
        __syncthreads();
        v = slots[0];
#pragma unroll
        for (uint32_t w = 1; w < Team<TEAM>::kWaves; ++w) v = op(v, slots[w]);
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
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_forward_kernel(NormForward a) {
    __shared__ float sums[3][Team<TEAM>::kWaves];
    __shared__ uint32_t most[Team<TEAM>::kWaves];
    const uint32_t lane = threadIdx.x % TEAM;
    const uint32_t first = blockIdx.x * Team<TEAM>::kPerBlock + threadIdx.x / TEAM, step = gridDim.x * Team<TEAM>::kPerBlock;
    const float size = (float)a.width;
    float w[N][8];
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) load_weight(a.weight, a.weight_type, (lane + j * TEAM) * kSlice, a.width, w[j]);
    uint32_t turn = 0;
    for (uint64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const typename T::raw *x = (const typename T::raw *)a.x + row * a.x_pitch;
        float h[N][8];
        Slice<T> in[N], more[N];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) in[j] = load_words<T, STREAM>(x, (lane + j * TEAM) * kSlice, a.width);
        if (a.residual) {
            const typename T::raw *r = (const typename T::raw *)a.residual + row * a.residual_pitch;
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) more[j] = load_words<T, STREAM>(r, (lane + j * TEAM) * kSlice, a.width);
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
                store_slice<T, STREAM>((typename T::raw *)a.sum + row * a.sum_pitch, (lane + j * TEAM) * kSlice, a.width, h[j]);
        }
        if (a.sum_codes) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                float v[8];
                as_written<T>(h[j], v);
                keep_slice<T, STREAM>(v, row, lane + j * TEAM, a.padded, a.sum_codes, a.sum_scales);
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[j][i] = h[j][i] * rstd * w[j][i];
        if (a.out) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j)
                store_slice<T, STREAM>((typename T::raw *)a.out + row * a.out_pitch, (lane + j * TEAM) * kSlice, a.width, h[j]);
        }
        if (a.out_codes) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                float v[8];
                as_written<T>(h[j], v);
                keep_slice<T, STREAM>(v, row, lane + j * TEAM, a.padded, a.out_codes, a.out_scales);
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
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_backward_kernel(NormBackward a) {
    __shared__ float sums[2][Team<TEAM>::kWaves];
    const uint32_t lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const uint32_t first = blockIdx.x * Team<TEAM>::kPerBlock + team, step = gridDim.x * Team<TEAM>::kPerBlock;
    const float size = (float)a.width;
    float w[N][8], dw[N][8] = {};
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) load_weight(a.weight, a.weight_type, (lane + j * TEAM) * kSlice, a.width, w[j]);
    uint32_t turn = 0;
    for (uint64_t row = first; row < a.rows; row += step, turn ^= 1) {
        const typename T::raw *dout = (const typename T::raw *)a.dout + row * a.dout_pitch;
        Slice<T> in[N], more[N], at[N];
        uint32_t code[N][2];
        float scale[N];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) in[j] = load_words<T, STREAM>(dout, (lane + j * TEAM) * kSlice, a.width);
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            const uint32_t s = lane + j * TEAM;
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
            for (uint32_t j = 0; j < N; ++j) more[j] = load_words<T, STREAM>(d, (lane + j * TEAM) * kSlice, a.width);
        }
        const float rstd = a.rstd[row];
        float g[N][8], n[N][8], dot = 0.0f;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            values<T>(in[j], g[j]);
            if constexpr (KEPT)
                values_of(code[j], lane + j * TEAM < a.padded ? scale[j] : 0.0f, n[j]);
            else
                values<T>(at[j], n[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // past the row nothing counts, whatever its last group holds
                n[j][i] = (lane + j * TEAM) * kSlice + i < a.width ? n[j][i] * rstd : 0.0f;
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
            store_slice<T, STREAM>((typename T::raw *)a.dx + row * a.dx_pitch, (lane + j * TEAM) * kSlice, a.width, d);
        }
    }
    if (!a.parts) return;
    float *part = a.parts + (uint64_t)blockIdx.x * a.width;
    if constexpr (Team<TEAM>::kPerBlock > 1) {    // the block's teams, in order
        __shared__ float all[Team<TEAM>::kPerBlock][TEAM * N * 8];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) all[team][(lane + j * TEAM) * kSlice + i] = dw[j][i];
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.width; c += Team<TEAM>::kThreads) {
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
                const uint32_t c = (lane + j * TEAM) * kSlice + i;
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

// Runs f(team size, slices a lane) for the smallest team that holds a row.  Forward a lane has two slices (65536 x 4096 of 16
// bits, sum kept: 440 us, 5.5 TB/s, with one 452; 32768 x 8192 467 us and 532), but for the widths of whole blocks of one
// (131072 x 2048: 468 us, with two in blocks of 128 lanes 511).  Backward it holds sums besides, and one slice
// leaves room for the waves that keep memory busy (65536 x 4096: 356 us, 5.3 TB/s, with two 523).
template <class F>
inline void for_width(uint32_t padded, bool two, F f) {
    using std::integral_constant;
    using One = integral_constant<uint32_t, 1>;
    using Two = integral_constant<uint32_t, 2>;
    if (two || padded > 1024) {
        if (padded <= 32)
            f(integral_constant<uint32_t, 16>{}, Two{});
        else if (padded <= 128)
            f(integral_constant<uint32_t, 64>{}, Two{});
        else if (padded <= 256)
            f(integral_constant<uint32_t, 256>{}, One{});
        else if (padded <= 512)
            f(integral_constant<uint32_t, 256>{}, Two{});
        else if (padded <= 1024)
            f(integral_constant<uint32_t, 512>{}, Two{});
        else
            f(integral_constant<uint32_t, 1024>{}, Two{});
    } else {
        if (padded <= 16)
            f(integral_constant<uint32_t, 16>{}, One{});
        else if (padded <= 32)
            f(integral_constant<uint32_t, 32>{}, One{});
        else if (padded <= 64)
            f(integral_constant<uint32_t, 64>{}, One{});
        else if (padded <= 128)
            f(integral_constant<uint32_t, 128>{}, One{});
        else if (padded <= 256)
            f(integral_constant<uint32_t, 256>{}, One{});
        else if (padded <= 512)
            f(integral_constant<uint32_t, 512>{}, One{});
        else
            f(integral_constant<uint32_t, 1024>{}, One{});
    }
}

// Blocks that leave each CU `threads` threads, or fewer where the rows are.
template <uint32_t TEAM>
inline uint32_t norm_blocks(uint64_t rows, uint32_t threads) {
    const uint64_t n = (rows + Team<TEAM>::kPerBlock - 1) / Team<TEAM>::kPerBlock, most = 256 * threads / Team<TEAM>::kThreads;
    return (uint32_t)(n < most ? n : most);
}
// Backward each is a row of sums for dw besides: half as many (4096 x 4096: 32 us, with twice as many 40).
inline uint32_t norm_parts(uint64_t rows, uint32_t padded) {
    uint32_t n = 0;
    for_width(padded, false, [&](auto team, auto) { n = norm_blocks<team.value>(rows, 1024); });
    return n;
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
    PL_STREAM(bytes, PL_TYPE(type, for_width(padded, true, [&](auto team, auto n) {
        if constexpr (n.value == 2 || team.value == 256)
            norm_forward_kernel<T, team.value, n.value, STREAM>
                <<<norm_blocks<team.value>(rows, 2048), Team<team.value>::kThreads, 0, (hipStream_t)hip_stream>>>(a);
    })));
    return launched();
}

uint64_t poseidon_norm_backward_workspace(uint64_t rows, uint64_t width) {
    if (check_sizes(rows, width) != POSEIDON_OK || width > kNormWidth) return UINT64_MAX;
    return (uint64_t)norm_parts(rows, norm_padded(width)) * width * 4;
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
    const uint32_t padded = norm_padded(width), blocks = norm_parts(rows, padded);
    if (rows) {
        const NormBackward a = {dout, sum, dsum, weight, dout_pitch, sum_pitch, dsum_pitch, dx_pitch, codes, scales, rstd,
                                (uint32_t)rows, (uint32_t)width, padded, weight_type, dx, dweight ? (float *)workspace : nullptr};
        const uint32_t size = size_of(type);
        const uint64_t bytes = rows * width * (size * (2 + !kept + !!dsum) + kept);
        PL_STREAM(bytes, PL_TYPE(type, for_width(padded, false, [&](auto team, auto n) {
            if constexpr (n.value == 1 || team.value == 1024) {
                if (kept)
                    norm_backward_kernel<T, true, team.value, n.value, STREAM>
                        <<<blocks, Team<team.value>::kThreads, 0, (hipStream_t)hip_stream>>>(a);
                else
                    norm_backward_kernel<T, false, team.value, n.value, STREAM>
                        <<<blocks, Team<team.value>::kThreads, 0, (hipStream_t)hip_stream>>>(a);
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
