#pragma once
// Device helpers of the layer operators: value types, slices of a row, the
// 8-bit form, and the host's argument checks.
//
// The row operators give one lane a slice of 8 neighbouring values (16 bytes of
// a 16-bit type), so a wave reads and writes 1 KB without gaps, and 8 lanes
// make a group of the 8-bit form, whose maximum takes three lane exchanges
// within a row of 16 lanes.  Rows may begin at any address that is a multiple of the
// value's size: global memory takes 16-byte accesses there, and only the last
// slice of a row whose width is no multiple of 8 goes value by value.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include "../../include/poseidon_layers.h"

namespace pl {

constexpr uint32_t kBlock = 256;    // threads of a row kernel
constexpr uint32_t kSlice = 8;      // values of a lane
constexpr uint32_t kGroup = POSEIDON_GROUP;

// Calls that move more than the 256 MB last-level cache holds mark what they read once and what they
// write as not worth keeping (STREAM): 5 to 10% faster there (a 1 GiB copy 6.5 instead of 6.1 TB/s);
// smaller outputs stay where the next kernel finds them.
constexpr uint64_t kStreamBytes = 256ull << 20;

// ---- value types ----

struct F32 {
    using raw = float;
    static constexpr uint32_t kLow = 1, kHigh = 248;       // scale bytes
    static constexpr bool kShort = false;
    static __device__ __forceinline__ float up(raw v) { return v; }
    static __device__ __forceinline__ raw down(float v) { return v; }
};
struct F16 {
    using raw = _Float16;
    static constexpr uint32_t kLow = 103, kHigh = 136;
    static constexpr bool kShort = true;
    static __device__ __forceinline__ float up(raw v) { return (float)v; }
    static __device__ __forceinline__ raw down(float v) { return (raw)v; }
};
struct BF16 {
    using raw = __bf16;
    static constexpr uint32_t kLow = 1, kHigh = 248;
    static constexpr bool kShort = true;
    static __device__ __forceinline__ float up(raw v) { return (float)v; }
    static __device__ __forceinline__ raw down(float v) { return (raw)v; }
};

// ---- exact division of n < 2^31 by a fixed d ----

struct Div {
    uint32_t d, m, s;
};

inline Div make_div(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    const uint64_t m = ((((1ull << s) - d) << 32) / d) + 1;
    return {d, (uint32_t)m, s};
}

__device__ __forceinline__ uint32_t quotient(uint32_t n, const Div &v) { return (__umulhi(v.m, n) + n) >> v.s; }

// ---- slices ----

// Four words at any even address.
typedef uint32_t AnyWords __attribute__((ext_vector_type(4), aligned(2)));

template <bool STREAM, int N>
__device__ __forceinline__ void get(uint32_t (&w)[N], const void *from) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const AnyWords *p = (const AnyWords *)from + i;
        const AnyWords u = STREAM ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = u[j];
    }
}

template <bool STREAM, int N>
__device__ __forceinline__ void put(void *to, const uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        AnyWords *p = (AnyWords *)to + i;
        const AnyWords u = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        if constexpr (STREAM)
            __builtin_nontemporal_store(u, p);
        else
            *p = u;
    }
}

// The words of a slice, as they lie in memory.
template <class T>
struct Slice {
    static constexpr int kWords = (int)sizeof(typename T::raw) * 2;
    uint32_t w[kWords];
};

// Values [col, col + 8) of a row of `width`; the ones past it are 0.  A slice that
// leaves the row is read from the row's last 8 values and moved down, so that
// every lane issues the same one or two 16-byte loads and none waits in a branch.
template <class T, bool STREAM = false>
__device__ __forceinline__ Slice<T> load_words(const typename T::raw *row, uint32_t col, uint32_t width) {
    constexpr int kWords = Slice<T>::kWords;
    Slice<T> s;
    if (width >= kSlice) {
        const uint32_t start = min(col, width - kSlice), gone = col - start;
        get<STREAM>(s.w, row + start);
        if (width % kSlice) {
            constexpr int kFour = kWords / 2, kTwo = kWords / 4;    // words of four and of two values
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t up = i + kFour < kWords ? s.w[i + kFour] : 0u;
                s.w[i] = gone & 4 ? up : s.w[i];
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t up = i + kTwo < kWords ? s.w[i + kTwo] : 0u;
                s.w[i] = gone & 2 ? up : s.w[i];
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t next = i + 1 < kWords ? s.w[i + 1] : 0u;
                const uint32_t up = T::kShort ? s.w[i] >> 16 | next << 16 : next;
                s.w[i] = gone & 1 ? up : s.w[i];
            }
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) s.w[i] = gone < kSlice ? s.w[i] : 0u;
    } else {
        typename T::raw r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = col + i < width ? row[col + i] : T::down(0.0f);
        __builtin_memcpy(s.w, r, sizeof s.w);
    }
    return s;
}

template <class T>
__device__ __forceinline__ void values(const Slice<T> &s, float (&v)[8]) {
    typename T::raw r[8];
    __builtin_memcpy(r, s.w, sizeof r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = T::up(r[i]);
}

template <class T, bool STREAM = false>
__device__ __forceinline__ void load_slice(const typename T::raw *row, uint32_t col, uint32_t width, float (&v)[8]) {
    values<T>(load_words<T, STREAM>(row, col, width), v);
}

template <class T, bool STREAM = false>
__device__ __forceinline__ void store_slice(typename T::raw *row, uint32_t col, uint32_t width, const float (&v)[8]) {
    typename T::raw r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = T::down(v[i]);
    if (col + kSlice <= width) {
        uint32_t w[Slice<T>::kWords];
        __builtin_memcpy(w, r, sizeof w);
        put<STREAM>(row + col, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < width) row[col + i] = r[i];
    }
}

// ---- the 8-bit form ----

template <int CTRL>
__device__ __forceinline__ uint32_t lanes(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// The scale byte of a group whose 8 lanes hold 8 values each.  The maximum is
// taken over the bits of |x|, which order as the values do, infinities and
// NaNs last.  a = 1.f 2^(x-127) needs e = x - 133 while 1.f <= 127/64.
template <class T>
__device__ __forceinline__ uint32_t scale_byte(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, lanes<0xB1>(m));     // lane ^ 1
    m = max(m, lanes<0x4E>(m));     // lane ^ 2
    m = max(m, lanes<0x141>(m));    // the other four of the eight lanes
    if (m >= 0x7f800000u) return 255u;
    const int b = (int)(m >> 23) - 6 + ((m & 0x7fffffu) > 0x7e0000u);
    return (uint32_t)min(max(b, (int)T::kLow), (int)T::kHigh);
}

// Codes of 8 values under a scale byte, four to a word.  x / 2^e is exact, and
// adding 1.5 * 2^23 rounds it to the nearest whole number, ties to even, whose
// low byte the sum's low byte is.
__device__ __forceinline__ void codes_of(const float (&v)[8], uint32_t byte, uint32_t (&w)[2]) {
    const float inv = __uint_as_float((254u - min(byte, 254u)) << 23);
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        q[i] = __float_as_uint(__builtin_amdgcn_fmed3f(v[i] * inv, -127.0f, 127.0f) + 12582912.0f);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(q[4 * h + 1], q[4 * h], 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(q[4 * h + 3], q[4 * h + 2], 0x04000c0cu);
        w[h] = byte == 255u ? 0u : lo | hi;
    }
}

__device__ __forceinline__ float scale_of(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23);
}

__device__ __forceinline__ void values_of(const uint32_t (&w)[2], float scale, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * scale;
}

using Codes8 = uint32_t __attribute__((ext_vector_type(2)));

template <bool STREAM>
__device__ __forceinline__ void load_codes(const int8_t *codes, uint64_t slice, uint32_t (&w)[2]) {
    const Codes8 *p = (const Codes8 *)codes + slice;
    const Codes8 u = STREAM ? __builtin_nontemporal_load(p) : *p;
    w[0] = u[0];
    w[1] = u[1];
}

template <bool STREAM>
__device__ __forceinline__ void store_codes(int8_t *codes, uint64_t slice, const uint32_t (&w)[2]) {
    Codes8 *p = (Codes8 *)codes + slice;
    if constexpr (STREAM)
        __builtin_nontemporal_store(Codes8{w[0], w[1]}, p);
    else
        *p = Codes8{w[0], w[1]};
}

// ---- host side ----

inline uint32_t size_of(uint32_t type) { return type == POSEIDON_F32 ? 4u : 2u; }
inline bool known(uint32_t type) { return type <= POSEIDON_BF16; }
inline uint32_t groups_of(uint64_t width) { return (uint32_t)((width + kGroup - 1) / kGroup); }
inline bool aligned(const void *p, uint64_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Sizes first (E_RANGE), then pointers: a matrix of no rows needs none.
inline int check_sizes(uint64_t rows, uint64_t width) {
    if (width == 0) return POSEIDON_E_INVAL;
    return rows > POSEIDON_ROWS_MAX || width > POSEIDON_WIDTH_MAX ? POSEIDON_E_RANGE : POSEIDON_OK;
}
inline int check_matrix(const void *p, uint64_t pitch, uint32_t type, uint64_t rows, uint64_t width) {
    if (!known(type) || pitch < width) return POSEIDON_E_INVAL;
    if (pitch > POSEIDON_PITCH_MAX) return POSEIDON_E_RANGE;
    return rows && (!p || !aligned(p, size_of(type))) ? POSEIDON_E_INVAL : POSEIDON_OK;
}
inline int check_stash(const void *codes, const void *scales, uint64_t rows) {
    return rows && (!codes || !scales || !aligned(codes, 16)) ? POSEIDON_E_INVAL : POSEIDON_OK;
}
inline int check_workspace(const void *p, uint64_t have, uint64_t need) {
    return need && (!p || have < need || !aligned(p, 256)) ? POSEIDON_E_INVAL : POSEIDON_OK;
}
inline int launched() { return hipGetLastError() == hipSuccess ? POSEIDON_OK : POSEIDON_E_DEVICE; }

// Calls f(first row, rows, slices) over row ranges of less than 2^31 slices each.
template <class F>
inline void over_rows(uint64_t rows, uint32_t slices_per_row, F f) {
    const uint64_t step = 0x7fffff00ull / slices_per_row;
    for (uint64_t r = 0; r < rows; r += step) {
        const uint64_t n = rows - r < step ? rows - r : step;
        f(r, n, (uint32_t)(n * slices_per_row));
    }
}

inline uint32_t blocks_for(uint32_t threads) { return (threads + kBlock - 1) / kBlock; }

}  // namespace pl

#define PL_TRY(expr)                         \
    do {                                     \
        const int rc_ = (expr);              \
        if (rc_ != POSEIDON_OK) return rc_;  \
    } while (0)

// Runs `...` with the constant STREAM for a call that moves `bytes`.
#define PL_STREAM(bytes, ...)                    \
    do {                                         \
        if ((bytes) > pl::kStreamBytes) {        \
            constexpr bool STREAM = true;        \
            __VA_ARGS__;                         \
        } else {                                 \
            constexpr bool STREAM = false;       \
            __VA_ARGS__;                         \
        }                                        \
    } while (0)

// Runs `...` with T as the value type that `type` names.
#define PL_TYPE(type, ...)              \
    do {                                \
        if ((type) == POSEIDON_F32) {   \
            using T = pl::F32;          \
            __VA_ARGS__;                \
        } else if ((type) == POSEIDON_F16) { \
            using T = pl::F16;          \
            __VA_ARGS__;                \
        } else {                        \
            using T = pl::BF16;         \
            __VA_ARGS__;                \
        }                               \
    } while (0)
