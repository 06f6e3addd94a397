// Row operators of poseidon_layers.h: the 8-bit form of activations, the gated
// activation, the experts' gather and combination, the embedding lookup.  Each
// reads its inputs once and writes its outputs once; memory bounds all of them.
#include "layers_device.h"

namespace pl {

// ---- activations kept in 8 bits ----

// e = ceil(log2(max |x| / 127)) over 64 values, code = round(x / 2^e).  Codes and scale bytes have no gaps, so a lane's
// slice is slice i of both.  Memory bounds both directions: 32768 x 8192 of 16 bits kept in 137 us (5.9 TB/s) and restored in
// 126 (6.4).
template <class T, bool STREAM>
__global__ __launch_bounds__(kBlock) void stash_kernel(const typename T::raw *x, uint64_t pitch, uint32_t total,
                                                       Div per_row, uint32_t width, int8_t *codes, uint8_t *scales) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;    // whole groups of 8 lanes: total is a multiple of 8
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    float v[8];
    load_slice<T, STREAM>(x + (uint64_t)row * pitch, s * kSlice, width, v);
    const uint32_t byte = scale_byte<T>(v);
    uint32_t w[2];
    codes_of(v, byte, w);
    store_codes<STREAM>(codes, i, w);
    if (!(i & 7)) scales[i >> 3] = (uint8_t)byte;
}

template <class T, bool STREAM>
__global__ __launch_bounds__(kBlock) void restore_kernel(const int8_t *codes, const uint8_t *scales, uint32_t total,
                                                         Div per_row, uint32_t width, typename T::raw *out,
                                                         uint64_t pitch) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    uint32_t w[2];
    load_codes<STREAM>(codes, i, w);
    float v[8];
    values_of(w, scale_of(scales[i >> 3]), v);
    store_slice<T, STREAM>(out + (uint64_t)row * pitch, s * kSlice, width, v);
}

// ---- gated activation ----

// 1 / (1 + exp(-z)) for z >= kFar.  16-bit outputs take the hardware's exponential and reciprocal (off by (2 + |z|) 2^-24
// of the value), 32-bit ones the exact-to-the-last-bits functions.  Below kFar exp(-z) soon overflows, at -88.7, and the
// reciprocal leaves the normal range.
constexpr float kFar = -80.0f;

template <class T>
__device__ __forceinline__ float sigmoid(float z) {
    if constexpr (T::kShort)
        return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
    else
        return 1.0f / (1.0f + expf(-z));
}

// a exp(z) b c for z < kFar, where 1 + exp(z) is 1 in 32 bits, so that the sigmoid is exp(z): what is left of it is still
// a normal value, or large factors make it one.  exp(z) = 2^n 2^part with a whole n; the factors' fractions are multiplied
// and the exponents added, so only the product itself can leave the range.  Below -1000 nothing is left of any product.
__device__ __forceinline__ float times_exp(float a, float z, float b, float c) {
    const float y = z * 1.44269504f, rest = fmaf(z, 1.44269504f, -y) + z * 1.92596303e-8f;    // z / ln 2 in two parts
    const bool gone = z < -1000.0f;
    const float n = gone ? 0.0f : rintf(y), part = gone ? 0.0f : __builtin_amdgcn_exp2f(y - n + rest);
    float product = part;
    int e = (int)n;
    for (const float f : {a, b, c}) {
        product *= __builtin_amdgcn_frexp_mantf(f);
        e += __builtin_amdgcn_frexp_expf(f);
    }
    return ldexpf(product, e);
}

__device__ __forceinline__ float least(const float (&v)[8]) {
    return fminf(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), fminf(fminf(v[4], v[5]), fminf(v[6], v[7])));
}

// silu(gate) * up and both kept, in one pass over gate and up; the backward pass reads them as they were kept.  Memory bounds
// both: 16384 x 12288 of 16 bits 258 us forward (6.3 TB/s), 259 backward (6.2).
template <class T, bool KEEP, bool STREAM>
__global__ __launch_bounds__(kBlock) void gated_forward_kernel(
    const typename T::raw *gate, uint64_t gate_pitch, const typename T::raw *up, uint64_t up_pitch, uint32_t total,
    Div per_row, uint32_t width, typename T::raw *out, uint64_t out_pitch, int8_t *gate_codes, uint8_t *gate_scales,
    int8_t *up_codes, uint8_t *up_scales) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    float g[8], u[8], h[8];
    load_slice<T, STREAM>(gate + (uint64_t)row * gate_pitch, s * kSlice, width, g);
    load_slice<T, STREAM>(up + (uint64_t)row * up_pitch, s * kSlice, width, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = g[j] * sigmoid<T>(g[j]) * u[j];
    if (least(g) < kFar) {
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = g[j] < kFar ? times_exp(g[j], g[j], u[j], 1.0f) : h[j];
    }
    store_slice<T, STREAM>(out + (uint64_t)row * out_pitch, s * kSlice, width, h);
    if constexpr (KEEP) {
        uint32_t w[2];
        const uint32_t bg = scale_byte<T>(g), bu = scale_byte<T>(u);
        codes_of(g, bg, w);
        store_codes<STREAM>(gate_codes, i, w);
        codes_of(u, bu, w);
        store_codes<STREAM>(up_codes, i, w);
        if (!(i & 7)) {
            gate_scales[i >> 3] = (uint8_t)bg;
            up_scales[i >> 3] = (uint8_t)bu;
        }
    }
}

template <class T, bool STREAM>
__global__ __launch_bounds__(kBlock) void gated_backward_kernel(
    const typename T::raw *dout, uint64_t dout_pitch, uint32_t total, Div per_row, uint32_t width,
    const int8_t *gate_codes, const uint8_t *gate_scales, const int8_t *up_codes, const uint8_t *up_scales,
    typename T::raw *dgate, uint64_t dgate_pitch, typename T::raw *dup, uint64_t dup_pitch) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    uint32_t wg[2], wu[2];
    load_codes<STREAM>(gate_codes, i, wg);
    load_codes<STREAM>(up_codes, i, wu);
    const float sg = scale_of(gate_scales[i >> 3]), su = scale_of(up_scales[i >> 3]);
    float d[8], g[8], u[8], a[8], b[8];
    load_slice<T, STREAM>(dout + (uint64_t)row * dout_pitch, s * kSlice, width, d);
    values_of(wg, sg, g);
    values_of(wu, su, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float sig = sigmoid<T>(g[j]), ds = d[j] * sig, slope = 1.0f + g[j] * (1.0f - sig);
        a[j] = ds * u[j] * slope;
        b[j] = ds * g[j];
    }
    if (least(g) < kFar) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] = g[j] < kFar ? times_exp(1.0f + g[j], g[j], d[j], u[j]) : a[j];
            b[j] = g[j] < kFar ? times_exp(g[j], g[j], d[j], 1.0f) : b[j];
        }
    }
    store_slice<T, STREAM>(dgate + (uint64_t)row * dgate_pitch, s * kSlice, width, a);
    store_slice<T, STREAM>(dup + (uint64_t)row * dup_pitch, s * kSlice, width, b);
}

// ---- experts ----

// Rows [*n_kept, rows) of `out` (and their 8-bit form) become zeros: a wave a row.
template <class T, bool WRITE, bool KEEP>
__device__ __forceinline__ void clear_rows(uint32_t wave, uint32_t waves, const int32_t *n_kept, uint64_t rows,
                                           uint32_t width, uint32_t groups, typename T::raw *out, int8_t *codes,
                                           uint8_t *scales) {
    const float zero[8] = {};
    const uint32_t lane = threadIdx.x & 63;
    for (uint64_t r = (uint64_t)max(*n_kept, 0) + wave; r < rows; r += waves)
        for (uint32_t s = lane; s < groups * 8; s += 64) {
            if constexpr (WRITE) store_slice<T>(out + r * width, s * kSlice, width, zero);
            if constexpr (KEEP) {
                const uint32_t none[2] = {};
                store_codes<false>(codes, r * (groups * 8) + s, none);
                if (!(s & 7)) scales[r * groups + (s >> 3)] = (uint8_t)T::kLow;
            }
        }
}

// A lane reads its slice of a token once and writes it to each of the token's
// places; the rounding to 8 bits is done once too.  Blocks from `main` on clear the places past the last choice.
// Writes bound it: 16384 tokens of 4096 values to 8 places each, kept too, 333 us (5.3 TB/s).  A lane per place, which
// writes in order and reads a token's row eight times from cache: 30 us more, with 2 choices 179 instead of 152 us.
template <class T, bool WRITE, bool KEEP, bool STREAM>
__global__ __launch_bounds__(kBlock) void gather_kernel(const typename T::raw *x, uint64_t pitch, uint32_t total,
                                                        Div per_row, uint32_t width, const int32_t *position,
                                                        uint32_t k, uint32_t main, const int32_t *n_kept,
                                                        uint32_t places, typename T::raw *xs, int8_t *codes,
                                                        uint8_t *scales) {
    if (blockIdx.x >= main) {
        const uint32_t waves = kBlock / 64;
        clear_rows<T, WRITE, KEEP>((blockIdx.x - main) * waves + threadIdx.x / 64, (gridDim.x - main) * waves, n_kept,
                                   places, width, per_row.d / 8, xs, codes, scales);
        return;
    }
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    float v[8];
    load_slice<T, STREAM>(x + (uint64_t)row * pitch, s * kSlice, width, v);
    uint32_t w[2] = {0, 0}, byte = 0;
    if constexpr (KEEP) {
        byte = scale_byte<T>(v);
        codes_of(v, byte, w);
    }
    const int32_t *at = position + (uint64_t)row * k;
    for (uint32_t j = 0; j < k; ++j) {
        const uint32_t p = (uint32_t)at[j];
        if (p >= places) continue;
        if constexpr (WRITE) store_slice<T, STREAM>(xs + (uint64_t)p * width, s * kSlice, width, v);
        if constexpr (KEEP) {
            store_codes<STREAM>(codes, (uint64_t)p * per_row.d + s, w);
            if (!(s & 7)) scales[((uint64_t)p * per_row.d + s) >> 3] = (uint8_t)byte;
        }
    }
}

// A lane sums its slice over the token's places, in the order of the choices; the
// rows of two choices are asked for before the first is added.  Memory bounds it: 16384 tokens of 4096 values from 8 places
// 200 us (6.0 TB/s).
template <class T, bool STREAM>
__global__ __launch_bounds__(kBlock) void combine_kernel(const typename T::raw *ys, uint32_t total, Div per_row,
                                                         uint32_t width, const int32_t *position, uint32_t k,
                                                         uint32_t places, const float *weights, typename T::raw *out,
                                                         uint64_t pitch) {
    constexpr uint32_t kAhead = 2;
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= total) return;
    const uint32_t row = quotient(i, per_row), s = i - row * per_row.d;
    const int32_t *at = position + (uint64_t)row * k;
    float sum[8] = {};
    for (uint32_t j0 = 0; j0 < k; j0 += kAhead) {
        uint32_t p[kAhead];
        float w[kAhead];
        Slice<T> y[kAhead];
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            if (j0 + j >= k) break;
            p[j] = (uint32_t)at[j0 + j];
            w[j] = weights ? weights[(uint64_t)row * k + j0 + j] : 1.0f;
        }
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            if (j0 + j >= k) break;
            y[j] = load_words<T, STREAM>(ys + (uint64_t)(p[j] < places ? p[j] : 0) * width, s * kSlice, width);
        }
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            if (j0 + j >= k) break;
            if (p[j] >= places) continue;
            float v[8];
            values<T>(y[j], v);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] = fmaf(w[j], v[c], sum[c]);
        }
    }
    store_slice<T, STREAM>(out + (uint64_t)row * pitch, s * kSlice, width, sum);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// A wave per place, so that ys is read and dys written in order; a token's row of dout comes from memory for the first of
// its places and from cache for the others.  8000 tokens of 4096 values by 8 choices: 222 us (4.8 TB/s), against 275 with a
// wave per token, whose rows of ys and dys lie anywhere.
template <class T, bool STREAM>
__global__ __launch_bounds__(kBlock) void combine_backward_kernel(const typename T::raw *dout, uint64_t pitch,
                                                                  const typename T::raw *ys, uint32_t width,
                                                                  const int32_t *order, Div k, const int32_t *n_kept,
                                                                  uint32_t first, uint32_t places, uint32_t choices,
                                                                  const float *weights, typename T::raw *dys,
                                                                  float *dweights) {
    constexpr uint32_t kAhead = 2;    // slices of a row asked for at a time
    const uint32_t i = blockIdx.x * (kBlock / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (i >= places) return;
    const uint64_t p = first + i;
    const uint32_t choice = (uint32_t)__builtin_amdgcn_readfirstlane(order[p]);
    if (choice >= choices) return;
    const bool kept = (int32_t)p < *n_kept;
    const float w = weights[choice];
    const typename T::raw *d = dout + quotient(choice, k) * pitch;
    float dot = 0.0f;
    for (uint32_t c0 = lane * kSlice; c0 < width; c0 += kAhead * 64 * kSlice) {
        Slice<T> dw[kAhead], yw[kAhead];
        if (kept) {
#pragma unroll
            for (uint32_t a = 0; a < kAhead; ++a) {    // past the row: zeros
                dw[a] = load_words<T>(d, c0 + a * 64 * kSlice, width);
                yw[a] = load_words<T, STREAM>(ys + p * width, c0 + a * 64 * kSlice, width);
            }
        }
#pragma unroll
        for (uint32_t a = 0; a < kAhead; ++a) {
            float y[8] = {};
            if (kept) {
                float v[8];
                values<T>(dw[a], v);
                values<T>(yw[a], y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dot = fmaf(v[e], y[e], dot);
                    y[e] = w * v[e];
                }
            }
            store_slice<T, STREAM>(dys + p * width, c0 + a * 64 * kSlice, width, y);
        }
    }
    dot = wave_sum(dot);
    if (lane == 0) dweights[choice] = dot;
}

// ---- embedding ----

// A lane's N slices are a grid apart: an id has to be there before its row can be asked for, and with one slice a lane
// these two waits in a row are most of a long call (65536 x 1024: 41 us with N = 4, 48 with 1).
template <class T, bool STREAM, uint32_t N>
__global__ __launch_bounds__(kBlock) void embed_kernel(const int32_t *ids, uint32_t total, Div per_row, uint32_t width,
                                                       const typename T::raw *table, uint64_t table_pitch,
                                                       uint32_t vocab, float scale, typename T::raw *out,
                                                       uint64_t pitch) {
    const uint32_t first = blockIdx.x * kBlock + threadIdx.x, step = gridDim.x * kBlock;
    uint32_t row[N], id[N];
    Slice<T> in[N];
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) {
        const uint32_t i = min(first + j * step, total - 1);
        row[j] = quotient(i, per_row);
        id[j] = (uint32_t)ids[row[j]];
    }
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) {
        const uint32_t s = min(first + j * step, total - 1) - row[j] * per_row.d;
        if (id[j] < vocab) in[j] = load_words<T>(table + (uint64_t)id[j] * table_pitch, s * kSlice, width);
    }
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) {
        const uint32_t i = first + j * step;
        if (i >= total) return;
        float v[8] = {};
        if (id[j] < vocab) {
            values<T>(in[j], v);
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c] *= scale;
        }
        store_slice<T, STREAM>(out + (uint64_t)row[j] * pitch, (i - row[j] * per_row.d) * kSlice, width, v);
    }
}

inline uint32_t slices_of(uint64_t width) { return (uint32_t)((width + kSlice - 1) / kSlice); }
inline uint32_t padded_slices_of(uint64_t width) { return groups_of(width) * (kGroup / kSlice); }

constexpr uint32_t kClearBlocks = 256;    // blocks that look for places past the last choice

}  // namespace pl

using namespace pl;

extern "C" {

int poseidon_stash(const void *x, uint64_t pitch, uint32_t type, uint64_t rows, uint64_t width, int8_t *codes,
                   uint8_t *scales, void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    PL_TRY(check_matrix(x, pitch, type, rows, width));
    PL_TRY(check_stash(codes, scales, rows));
    if (!rows) return POSEIDON_OK;
    const uint32_t per_row = padded_slices_of(width);
    PL_STREAM(rows * width * (size_of(type) + 1), PL_TYPE(type, over_rows(rows, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
        stash_kernel<T, STREAM><<<blocks_for(n), kBlock, 0, (hipStream_t)hip_stream>>>(
            (const T::raw *)x + r * pitch, pitch, n, make_div(per_row), (uint32_t)width, codes + r * per_row * kSlice,
            scales + r * (per_row / 8));
    })));
    return launched();
}

int poseidon_restore(const int8_t *codes, const uint8_t *scales, uint64_t rows, uint64_t width, void *out,
                     uint64_t out_pitch, uint32_t type, void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    PL_TRY(check_matrix(out, out_pitch, type, rows, width));
    PL_TRY(check_stash(codes, scales, rows));
    if (!rows) return POSEIDON_OK;
    const uint32_t per_row = padded_slices_of(width);
    PL_STREAM(rows * width * (size_of(type) + 1), PL_TYPE(type, over_rows(rows, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
        restore_kernel<T, STREAM><<<blocks_for(n), kBlock, 0, (hipStream_t)hip_stream>>>(
            codes + r * per_row * kSlice, scales + r * (per_row / 8), n, make_div(per_row), (uint32_t)width,
            (T::raw *)out + r * out_pitch, out_pitch);
    })));
    return launched();
}

int poseidon_gated_forward(const void *gate, uint64_t gate_pitch, const void *up, uint64_t up_pitch, uint32_t type,
                           uint64_t rows, uint64_t width, void *out, uint64_t out_pitch, int8_t *gate_codes,
                           uint8_t *gate_scales, int8_t *up_codes, uint8_t *up_scales, void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    PL_TRY(check_matrix(gate, gate_pitch, type, rows, width));
    PL_TRY(check_matrix(up, up_pitch, type, rows, width));
    PL_TRY(check_matrix(out, out_pitch, type, rows, width));
    const bool keep = gate_codes || gate_scales || up_codes || up_scales;
    if (keep) {
        PL_TRY(check_stash(gate_codes, gate_scales, rows));
        PL_TRY(check_stash(up_codes, up_scales, rows));
    }
    if (!rows) return POSEIDON_OK;
    const uint32_t per_row = padded_slices_of(width);
    const auto run = [&](auto kernel, auto t) {
        using T = decltype(t);
        over_rows(rows, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
            const uint64_t c = r * per_row * kSlice, b = r * (per_row / 8);
            kernel<<<blocks_for(n), kBlock, 0, (hipStream_t)hip_stream>>>(
                (const typename T::raw *)gate + r * gate_pitch, gate_pitch, (const typename T::raw *)up + r * up_pitch,
                up_pitch, n, make_div(per_row), (uint32_t)width, (typename T::raw *)out + r * out_pitch, out_pitch,
                keep ? gate_codes + c : nullptr, keep ? gate_scales + b : nullptr, keep ? up_codes + c : nullptr,
                keep ? up_scales + b : nullptr);
        });
    };
    PL_STREAM(rows * width * (3 * size_of(type) + 2), PL_TYPE(type, keep ? run(gated_forward_kernel<T, true, STREAM>, T{})
                                                                         : run(gated_forward_kernel<T, false, STREAM>, T{})));
    return launched();
}

int poseidon_gated_backward(const void *dout, uint64_t dout_pitch, uint32_t type, uint64_t rows, uint64_t width,
                            const int8_t *gate_codes, const uint8_t *gate_scales, const int8_t *up_codes,
                            const uint8_t *up_scales, void *dgate, uint64_t dgate_pitch, void *dup, uint64_t dup_pitch,
                            void *hip_stream) {
    PL_TRY(check_sizes(rows, width));
    PL_TRY(check_matrix(dout, dout_pitch, type, rows, width));
    PL_TRY(check_matrix(dgate, dgate_pitch, type, rows, width));
    PL_TRY(check_matrix(dup, dup_pitch, type, rows, width));
    PL_TRY(check_stash(gate_codes, gate_scales, rows));
    PL_TRY(check_stash(up_codes, up_scales, rows));
    if (!rows) return POSEIDON_OK;
    const uint32_t per_row = padded_slices_of(width);
    PL_STREAM(rows * width * (3 * size_of(type) + 2), PL_TYPE(type, over_rows(rows, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
        const uint64_t c = r * per_row * kSlice, b = r * (per_row / 8);
        gated_backward_kernel<T, STREAM><<<blocks_for(n), kBlock, 0, (hipStream_t)hip_stream>>>(
            (const T::raw *)dout + r * dout_pitch, dout_pitch, n, make_div(per_row), (uint32_t)width, gate_codes + c,
            gate_scales + b, up_codes + c, up_scales + b, (T::raw *)dgate + r * dgate_pitch, dgate_pitch,
            (T::raw *)dup + r * dup_pitch, dup_pitch);
    })));
    return launched();
}

int poseidon_expert_gather(const void *x, uint64_t pitch, uint32_t type, uint64_t tokens, uint64_t width,
                           const int32_t *position, uint32_t k, const int32_t *n_kept, void *xs, int8_t *codes,
                           uint8_t *scales, void *hip_stream) {
    if (!k) return POSEIDON_E_INVAL;
    if (tokens > POSEIDON_ROWS_MAX / k) return POSEIDON_E_RANGE;
    const uint64_t places = tokens * k;
    PL_TRY(check_sizes(places, width));
    PL_TRY(check_matrix(x, pitch, type, tokens, width));
    const bool keep = codes || scales;
    if (tokens && (!position || !n_kept || (!xs && !keep))) return POSEIDON_E_INVAL;
    if (xs) PL_TRY(check_matrix(xs, width, type, places, width));
    if (keep) PL_TRY(check_stash(codes, scales, places));
    if (!tokens) return POSEIDON_OK;
    const uint32_t per_row = padded_slices_of(width);
    const auto run = [&](auto kernel, auto t) {
        using T = decltype(t);
        over_rows(tokens, per_row, [&](uint64_t r, uint64_t n_rows, uint32_t n) {
            const bool last = r + n_rows == tokens;
            kernel<<<blocks_for(n) + (last ? kClearBlocks : 0), kBlock, 0, (hipStream_t)hip_stream>>>(
                (const typename T::raw *)x + r * pitch, pitch, n, make_div(per_row), (uint32_t)width,
                position + r * k, k, blocks_for(n), n_kept, (uint32_t)places, (typename T::raw *)xs, codes, scales);
        });
    };
    PL_STREAM(places * width * ((xs ? size_of(type) : 0) + keep),
              PL_TYPE(type, !keep ? run(gather_kernel<T, true, false, STREAM>, T{})
                            : xs  ? run(gather_kernel<T, true, true, STREAM>, T{})
                                  : run(gather_kernel<T, false, true, STREAM>, T{})));
    return launched();
}

int poseidon_expert_combine(const void *ys, uint32_t type, uint64_t tokens, uint64_t width, const int32_t *position,
                            uint32_t k, const float *weights, void *out, uint64_t out_pitch, void *hip_stream) {
    if (!k) return POSEIDON_E_INVAL;
    if (tokens > POSEIDON_ROWS_MAX / k) return POSEIDON_E_RANGE;
    PL_TRY(check_sizes(tokens * k, width));
    PL_TRY(check_matrix(ys, width, type, tokens, width));
    PL_TRY(check_matrix(out, out_pitch, type, tokens, width));
    if (tokens && !position) return POSEIDON_E_INVAL;
    if (!tokens) return POSEIDON_OK;
    const uint32_t per_row = slices_of(width);
    PL_STREAM(tokens * (k + 1) * width * size_of(type), PL_TYPE(type, over_rows(tokens, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
        combine_kernel<T, STREAM><<<blocks_for(n), kBlock, 0, (hipStream_t)hip_stream>>>(
            (const T::raw *)ys, n, make_div(per_row), (uint32_t)width, position + r * k, k,
            (uint32_t)(tokens * k), weights ? weights + r * k : nullptr, (T::raw *)out + r * out_pitch, out_pitch);
    })));
    return launched();
}

int poseidon_expert_combine_backward(const void *dout, uint64_t dout_pitch, const void *ys, uint32_t type,
                                     uint64_t tokens, uint64_t width, const int32_t *order, uint32_t k,
                                     const int32_t *n_kept, const float *weights, void *dys, float *dweights,
                                     void *hip_stream) {
    if (!k) return POSEIDON_E_INVAL;
    if (tokens > POSEIDON_ROWS_MAX / k) return POSEIDON_E_RANGE;
    const uint64_t places = tokens * k;
    PL_TRY(check_sizes(places, width));
    PL_TRY(check_matrix(dout, dout_pitch, type, tokens, width));
    PL_TRY(check_matrix(ys, width, type, places, width));
    PL_TRY(check_matrix(dys, width, type, places, width));
    if (tokens && (!order || !n_kept || !weights || !dweights)) return POSEIDON_E_INVAL;
    if (!tokens) return POSEIDON_OK;
    const uint64_t step = 1ull << 25;    // places of a launch
    PL_STREAM(tokens * (2 * k + 1) * width * size_of(type), PL_TYPE(type, for (uint64_t p = 0; p < places; p += step) {
        const uint32_t n = (uint32_t)(places - p < step ? places - p : step);
        combine_backward_kernel<T, STREAM><<<(n + kBlock / 64 - 1) / (kBlock / 64), kBlock, 0, (hipStream_t)hip_stream>>>(
            (const T::raw *)dout, dout_pitch, (const T::raw *)ys, (uint32_t)width, order, make_div(k), n_kept, (uint32_t)p, n,
            (uint32_t)places, weights, (T::raw *)dys, dweights);
    }));
    return launched();
}

int poseidon_embed(const int32_t *ids, uint64_t tokens, const void *table, uint64_t table_pitch, uint32_t type,
                   uint64_t vocab, uint64_t width, float scale, void *out, uint64_t out_pitch, void *hip_stream) {
    PL_TRY(check_sizes(tokens, width));
    if (vocab > POSEIDON_VOCAB_MAX) return POSEIDON_E_RANGE;
    PL_TRY(check_matrix(table, table_pitch, type, vocab, width));
    PL_TRY(check_matrix(out, out_pitch, type, tokens, width));
    if (tokens && !ids) return POSEIDON_E_INVAL;
    if (!tokens) return POSEIDON_OK;
    const uint32_t per_row = slices_of(width);
    const auto run = [&](auto kernel, auto t, uint32_t each) {
        using T = decltype(t);
        over_rows(tokens, per_row, [&](uint64_t r, uint64_t, uint32_t n) {
            kernel<<<blocks_for((n + each - 1) / each), kBlock, 0, (hipStream_t)hip_stream>>>(
                ids + r, n, make_div(per_row), (uint32_t)width, (const typename T::raw *)table, table_pitch, (uint32_t)vocab,
                scale, (typename T::raw *)out + r * out_pitch, out_pitch);
        });
    };
    // four slices a lane where that leaves every CU its 2048 lanes
    const bool four = tokens * per_row >= 4ull * 256 * 2048;
    PL_STREAM(tokens * width * 2 * size_of(type), PL_TYPE(type, four ? run(embed_kernel<T, STREAM, 4>, T{}, 4)
                                                                      : run(embed_kernel<T, STREAM, 1>, T{}, 1)));
    return launched();
}

}  // extern "C"
