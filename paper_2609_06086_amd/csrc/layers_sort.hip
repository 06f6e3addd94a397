// Sort of tokens by expert, and the gradient of an embedding summed by token.
//
// Both sort whole keys stably with a counting sort of up to 9 bits a pass, the
// low bits first.  A block of eight waves takes up to 4096 neighbouring elements, a wave an eighth
// of them, 64 at a time in order; lanes with the same digit find each other with one
// ballot a bit, so an element's rank among the equal ones before it needs no
// atomics and the order is the same on every call.  Waits bound it, not bytes: 131072 choices of 64 experts take 5 us to count
// and 11 to place, up to 4096 elements 3 to 9 us in one block.
#include "layers_device.h"

namespace pl {

constexpr uint32_t kSortThreads = 512, kSortRounds = 8, kSortTile = kSortThreads * kSortRounds;
constexpr uint32_t kSortWaves = kSortThreads / 64, kMaxBits = 9, kMaxBins = 1u << kMaxBits;
// Up to this many blocks each block adds up the counts of the blocks before it by
// itself (a bin a thread); above it a kernel of its own turns them into sums once.
constexpr uint32_t kSelfScan = 128;

struct SortPass {
    const int32_t *keys;
    const int32_t *from;       // the elements' indexes, null: 0, 1, 2, ...
    uint32_t m, n_keys;        // elements; keys outside [0, n_keys) count as n_keys
    uint32_t shift, bins, bits;
    uint32_t blocks, rounds;   // of 64 elements a wave: a block takes 512 * rounds
    uint32_t *counts;          // [blocks][bins]
    uint32_t *totals;          // [bins], only where a kernel of its own scans
    int32_t *keys_out;         // null: not needed
    int32_t *order;            // the elements' indexes in their new order
    int32_t *position;         // null, or the new place of each element, -1 for key n_keys (single-pass sorts)
    int32_t *offsets;          // null, or the first place of each digit up to n_keys (single-pass sorts)
    uint32_t passes;           // of a sort of one block, which runs them all in LDS
};

// Memory to fill with zeros beside a sort, which keeps few CUs busy: `rows` rows of `bytes` (an even number).
struct Clear {
    char *to;
    uint64_t rows, bytes, pitch;
};

// Block `block` of `blocks`: a row, or of one row (a table without gaps) a piece of 16 bytes a thread, and what lies
// whole grids further.  Many blocks of one store a thread fill at 6.7 TB/s, blocks that go on through the memory in
// strides at 4.4 to 5.6: only above kClearMost blocks (32 GiB without gaps in a launch) do they go on.
constexpr uint64_t kClearPiece = (uint64_t)kSortThreads * 16, kClearMost = 1u << 22;

__device__ __forceinline__ void clear(const Clear &c, uint32_t block, uint32_t blocks) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const bool flat = c.rows == 1;
    const uint64_t step = flat ? blocks * kClearPiece : kClearPiece;
    for (uint64_t r = flat ? 0 : block; r < c.rows; r += flat ? 1 : blocks) {
        char *row = c.to + r * c.pitch;
        for (uint64_t at = (flat ? block * kClearPiece : 0) + threadIdx.x * 16u; at < c.bytes; at += step) {
            if (at + 16 <= c.bytes) {
                __builtin_memcpy(row + at, &zero, 16);
            } else {
                for (uint64_t i = at; i < c.bytes; i += 2) *(uint16_t *)(row + i) = 0;
            }
        }
    }
}

__device__ __forceinline__ uint32_t key_at(const SortPass &p, uint32_t i) {
    const uint32_t k = (uint32_t)p.keys[i];
    return min(k, p.n_keys);
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p, Clear c) {
    __shared__ uint32_t count[kMaxBins];
    if (blockIdx.x >= p.blocks) return clear(c, blockIdx.x - p.blocks, gridDim.x - p.blocks);
    for (uint32_t b = threadIdx.x; b < p.bins; b += kSortThreads) count[b] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * (kSortThreads * p.rounds);
    for (uint32_t r = 0; r < p.rounds; ++r) {
        const uint32_t i = first + r * kSortThreads + threadIdx.x;
        if (i < p.m) atomicAdd(&count[(key_at(p, i) >> p.shift) & (p.bins - 1)], 1u);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < p.bins; b += kSortThreads) p.counts[blockIdx.x * p.bins + b] = count[b];
}

// Exclusive sums over the blocks, a block of threads per bin.
__global__ __launch_bounds__(256) void sort_scan_kernel(SortPass p) {
    __shared__ uint32_t part[256];
    const uint32_t bin = blockIdx.x, tid = threadIdx.x;
    uint32_t carry = 0;
    for (uint32_t b0 = 0; b0 < p.blocks; b0 += 256) {
        const uint32_t b = b0 + tid;
        const uint32_t v = b < p.blocks ? p.counts[b * p.bins + bin] : 0u;
        part[tid] = v;
        __syncthreads();
        for (uint32_t d = 1; d < 256; d <<= 1) {
            const uint32_t add = tid >= d ? part[tid - d] : 0u;
            __syncthreads();
            part[tid] += add;
            __syncthreads();
        }
        if (b < p.blocks) p.counts[b * p.bins + bin] = carry + part[tid] - v;
        carry += part[255];
        __syncthreads();
    }
    if (tid == 0) p.totals[bin] = carry;
}

// Exclusive prefix over the 512 threads' values.
__device__ __forceinline__ uint32_t block_prefix(uint32_t v, uint32_t *wave_sums) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(s, d, 64);
        if ((int)lane >= d) s += up;
    }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t w = 0; w < wave; ++w) before += wave_sums[w];
    __syncthreads();
    return before + s - v;
}

// A pass.  SOLO: all of the elements are in one block, which runs every pass and
// passes keys and indexes on through LDS.
template <bool SOLO>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortPass p, Clear c) {
    __shared__ uint32_t count[kSortWaves][kMaxBins];
    __shared__ uint32_t wave_sums[kSortWaves];
    __shared__ uint32_t moved[SOLO ? 2 : 1][SOLO ? kSortTile : 1];
    if (blockIdx.x >= p.blocks) return clear(c, blockIdx.x - p.blocks, gridDim.x - p.blocks);
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
    const uint32_t first = (blockIdx.x * kSortWaves + wave) * (64 * p.rounds);
    const uint32_t rounds = first < p.m ? min((p.m - first + 63) / 64, p.rounds) : 0;    // of this wave
    const uint64_t below = (1ull << lane) - 1;
    uint32_t key[kSortRounds], index[kSortRounds];
#pragma unroll
    for (uint32_t r = 0; r < kSortRounds; ++r) {
        const uint32_t i = first + r * 64 + lane;
        const bool on = r < rounds && i < p.m;
        key[r] = on ? key_at(p, i) : 0xffffffffu;
        index[r] = on && p.from ? (uint32_t)p.from[i] : i;
    }
    for (uint32_t pass = 0; pass < (SOLO ? p.passes : 1u); ++pass) {
        const uint32_t shift = SOLO ? pass * p.bits : p.shift;
        const bool last = !SOLO || pass + 1 == p.passes;
        for (uint32_t w = 0; w < kSortWaves; ++w)
            if (tid < p.bins) count[w][tid] = 0;
        __syncthreads();

        // ranks within the wave's elements
        uint32_t rank[kSortRounds];
        volatile uint32_t *mine = count[wave];
#pragma unroll
        for (uint32_t r = 0; r < kSortRounds; ++r) {
            if (r >= rounds) break;
            const bool on = first + r * 64 + lane < p.m;
            const uint32_t digit = (key[r] >> shift) & (p.bins - 1);
            uint64_t same = __ballot(on);
            for (uint32_t b = 0; b < p.bits; ++b) {
                const uint64_t set = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? set : ~set;
            }
            const uint32_t old = mine[digit];
            const uint32_t before = (uint32_t)__popcll(same & below);
            rank[r] = old + before;
            __builtin_amdgcn_wave_barrier();
            if (on && before == 0) mine[digit] = old + (uint32_t)__popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();

        // a bin a thread: where the block's elements of this digit begin
        uint32_t before = 0, total = 0;
        if constexpr (SOLO) {
            if (tid < p.bins) {
#pragma unroll
                for (uint32_t w = 0; w < kSortWaves; ++w) total += count[w][tid];
            }
        } else if (p.totals) {
            if (tid < p.bins) {
                before = p.counts[blockIdx.x * p.bins + tid];
                total = p.totals[tid];
            }
        } else {    // the blocks' counts, shared by as many groups of threads as there is room for
            __shared__ uint32_t part[2][kSortThreads];
            const uint32_t bin = tid & (p.bins - 1), group = tid / p.bins, groups = kSortThreads / p.bins;
#pragma unroll 8
            for (uint32_t b = group; b < p.blocks; b += groups) {
                const uint32_t n = p.counts[b * p.bins + bin];
                before += b < blockIdx.x ? n : 0u;
                total += n;
            }
            part[0][tid] = before;
            part[1][tid] = total;
            __syncthreads();
            before = total = 0;
            if (tid < p.bins)
                for (uint32_t i = 0; i < groups; ++i) {
                    before += part[0][i * p.bins + tid];
                    total += part[1][i * p.bins + tid];
                }
        }
        const uint32_t start = block_prefix(total, wave_sums);
        if (tid < p.bins) {
            if (p.offsets && blockIdx.x == 0 && tid <= p.n_keys) p.offsets[tid] = (int32_t)start;
            uint32_t at = start + before;
#pragma unroll
            for (uint32_t w = 0; w < kSortWaves; ++w) {
                const uint32_t n = count[w][tid];
                count[w][tid] = at;
                at += n;
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < kSortRounds; ++r) {
            const uint32_t i = first + r * 64 + lane;
            if (r >= rounds || i >= p.m) continue;
            const uint32_t to = count[wave][(key[r] >> shift) & (p.bins - 1)] + rank[r];
            if (!last) {
                moved[0][to] = key[r];
                moved[SOLO][to] = index[r];
                continue;
            }
            p.order[to] = (int32_t)index[r];
            if (p.keys_out) p.keys_out[to] = (int32_t)key[r];
            if (p.position) p.position[i] = key[r] < p.n_keys ? (int32_t)to : -1;
        }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < kSortRounds; ++r) {
            const uint32_t i = first + r * 64 + lane;
            if (r >= rounds || i >= p.m) continue;
            key[r] = moved[0][i];
            index[r] = moved[SOLO][i];
        }
    }
}

// Few elements are spread over the eight waves of one block; then over blocks, of more elements each as they
// get many.
inline uint32_t sort_rounds(uint64_t m) {
    if (m <= kSortTile) return m ? (uint32_t)((m + kSortThreads - 1) / kSortThreads) : 1;
    return m <= 1u << 15 ? 2 : m <= 1u << 17 ? 4 : kSortRounds;
}
inline uint32_t sort_blocks(uint64_t m) {
    const uint64_t each = kSortThreads * sort_rounds(m);
    return (uint32_t)((m + each - 1) / each);
}
inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
// counts, then totals
inline uint64_t sort_counts_bytes(uint64_t m) { return round_up(((uint64_t)sort_blocks(m) + 1) * kMaxBins * 4, 256); }

// Blocks that clear beside a sort's, and part i of n of a clear.
inline uint32_t clear_blocks(const Clear &c) {
    const uint64_t n = c.rows == 1 ? (c.bytes + kClearPiece - 1) / kClearPiece : c.rows;
    return (uint32_t)(n < kClearMost ? n : kClearMost);
}
inline Clear part_of(const Clear &c, uint64_t i, uint64_t n) {
    Clear p = c;
    if (c.rows == 1) {
        const uint64_t units = c.bytes / 256, from = units * i / n * 256;
        p.to += from;
        p.bytes = (i + 1 == n ? c.bytes : units * (i + 1) / n * 256) - from;
    } else {
        const uint64_t from = c.rows * i / n;
        p.to += from * c.pitch;
        p.rows = c.rows * (i + 1) / n - from;
    }
    return p;
}

// Passes of `bits` bits over p.keys, with the clear spread over their launches.  lists: where passes but
// the last leave keys and indexes, and the last one its keys.
struct SortLists {
    int32_t *keys[2], *order[2];
};

// A launch that fails ends the sort: the next one would take its counts from memory that nothing wrote.
inline int sort(SortPass p, const SortLists &lists, const Clear &c, hipStream_t stream) {
    if (p.blocks == 1) {
        sort_place_kernel<true><<<1 + clear_blocks(c), kSortThreads, 0, stream>>>(p, c);
        return launched();
    }
    const bool scan = p.blocks > kSelfScan;
    uint32_t *const totals = p.counts + (uint64_t)p.blocks * p.bins;
    p.totals = scan ? totals : nullptr;
    int32_t *const order = p.order, *const keys = p.keys_out;
    for (uint32_t i = 0; i < p.passes; ++i) {
        const bool last = i + 1 == p.passes;
        if (i) {
            p.keys = lists.keys[(i - 1) & 1];
            p.from = lists.order[(i - 1) & 1];
        }
        p.keys_out = last ? keys : lists.keys[i & 1];
        p.order = last ? order : lists.order[i & 1];
        p.shift = i * p.bits;
        const Clear a = part_of(c, 2 * i, 2 * p.passes), b = part_of(c, 2 * i + 1, 2 * p.passes);
        sort_count_kernel<<<p.blocks + clear_blocks(a), kSortThreads, 0, stream>>>(p, a);
        PL_TRY(launched());
        if (scan) {
            SortPass q = p;
            q.totals = totals;
            sort_scan_kernel<<<p.bins, 256, 0, stream>>>(q);
            PL_TRY(launched());
        }
        sort_place_kernel<false><<<p.blocks + clear_blocks(b), kSortThreads, 0, stream>>>(p, b);
        PL_TRY(launched());
    }
    return POSEIDON_OK;
}

// ---- gradient of an embedding ----

// Sorted places in chunks of `chunk`; a block takes one chunk and 512 columns
// (64 lanes of 8).  Four rows of dout are on their way while four are added, in sorted order; it writes the sum
// of every token whose places all lie in the chunk.  A token that comes from the chunk
// before leaves its part in slot 0 of the chunk, one that only goes on into the
// next chunk in slot 1; embed_join_kernel adds those up in order.
// Rows lie anywhere, and the waits for them bound it: 32768 tokens of 2048 values 82 us (134 MB read, about 100
// written); eight rows on their way cost registers and 15 us more, chunks of 16 places 16 us more.
struct EmbedGrad {
    const int32_t *keys, *order;
    uint32_t m, vocab, width, chunk, chunks, accumulate;
    float scale;
    const void *dout;
    uint64_t dout_pitch;
    void *dtable;
    uint64_t dtable_pitch;
    float *parts;              // [chunks][2][padded], padded = width in whole slices
    uint32_t padded;
};

template <class G>
__device__ __forceinline__ void write_sum(const EmbedGrad &e, uint32_t key, uint32_t col, const float (&sum)[8]) {
    typename G::raw *row = (typename G::raw *)e.dtable + (uint64_t)key * e.dtable_pitch;
    float v[8] = {};
    if (e.accumulate) load_slice<G>(row, col, e.width, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e.accumulate ? fmaf(e.scale, sum[i], v[i]) : e.scale * sum[i];
    store_slice<G>(row, col, e.width, v);
}

template <class T, class G, bool STREAM>
__global__ __launch_bounds__(64) void embed_sum_kernel(EmbedGrad e) {
    constexpr uint32_t kAhead = 4;    // rows asked for at a time
    const uint32_t lane = threadIdx.x, chunk = blockIdx.x, col = (blockIdx.y * 64 + lane) * kSlice;
    const uint32_t lo = chunk * e.chunk, hi = min(lo + e.chunk, e.m);
    const typename T::raw *dout = (const typename T::raw *)e.dout;
    const uint32_t before = lo > 0 ? (uint32_t)e.keys[lo - 1] : e.vocab, after = hi < e.m ? (uint32_t)e.keys[hi] : e.vocab;
    float *parts = e.parts + (uint64_t)chunk * 2 * e.padded + col;
    const bool inside = col < e.width;
    float sum[8] = {};
    uint32_t key = (uint32_t)__builtin_amdgcn_readfirstlane(e.keys[lo]);
    bool from = before == key;    // the token comes from the chunk before
    const auto flush = [&](bool on) {
        if (key < e.vocab && inside) {
            if (from || on) {
                float *part = parts + (from ? 0 : e.padded);
#pragma unroll
                for (int i = 0; i < 8; ++i) part[i] = sum[i];
            } else {
                write_sum<G>(e, key, col, sum);
            }
        }
        from = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    };
    for (uint32_t a = lo; a < hi; a += 64) {    // a lane holds one of 64 places
        const uint32_t here = min(a + lane, hi - 1);
        const int32_t keys = e.keys[here], rows = e.order[here];
        const uint32_t n = min(hi - a, 64u);
        Slice<T> next[kAhead];
        const auto fetch = [&](uint32_t first) {
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                const uint32_t row = (uint32_t)__builtin_amdgcn_readlane(rows, min(first + j, n - 1));
                next[j] = load_words<T, STREAM>(dout + (uint64_t)row * e.dout_pitch, col, e.width);
            }
        };
        fetch(0);
        for (uint32_t first = 0; first < n; first += kAhead) {
            Slice<T> now[kAhead];
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) now[j] = next[j];
            if (first + kAhead < n) fetch(first + kAhead);
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                if (first + j >= n) break;
                const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(keys, first + j);
                if (k != key) {
                    flush(false);
                    key = k;
                }
                float v[8];
                values<T>(now[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[i];
            }
        }
    }
    flush(after == key);
}

// A block of four waves per chunk and 512 columns; it has work where a token
// begins in the chunk and goes on past it.  The waves take every fourth of the
// chunks that follow, and the first adds the four sums.  A few dependent waits: 9 us for 1024 chunks.
template <class G>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedGrad e) {
    __shared__ float share[3][64][kSlice + 1];
    const uint32_t chunk = blockIdx.x, lo = chunk * e.chunk, hi = min(lo + e.chunk, e.m);
    if (hi >= e.m) return;
    const uint32_t key = (uint32_t)e.keys[hi - 1];
    if (key >= e.vocab || (uint32_t)e.keys[hi] != key) return;
    if ((uint32_t)e.keys[lo] == key && lo > 0 && (uint32_t)e.keys[lo - 1] == key) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint32_t last = chunk + 1;    // one past the last chunk that begins with the token
    for (;;) {
        const uint32_t c = last + lane;
        const uint64_t same = __ballot(c < e.chunks && (uint32_t)e.keys[min(c, e.chunks - 1) * e.chunk] == key);
        last += same == ~0ull ? 64u : (uint32_t)__ffsll((unsigned long long)~same) - 1u;
        if (same != ~0ull) break;
    }
    const uint32_t col = (blockIdx.y * 64 + lane) * kSlice;
    const bool inside = col < e.width;
    float sum[8] = {};
    if (inside)
        for (uint32_t c = chunk + wave; c < last; c += 4) {
            const float *part = e.parts + ((uint64_t)c * 2 + (c == chunk)) * e.padded + col;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += part[i];
        }
    if (wave) {
#pragma unroll
        for (int i = 0; i < 8; ++i) share[wave - 1][lane][i] = sum[i];
    }
    __syncthreads();
    if (wave || !inside) return;
#pragma unroll
    for (int w = 0; w < 3; ++w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += share[w][lane][i];
    }
    write_sum<G>(e, key, col, sum);
}

// Places a block adds up: as many as leave 4096 waves, which fill the chip, from 8 to 32 (past 2^25 tokens more, so that there
// are at most 2^20 chunks).
inline uint32_t chunk_of(uint64_t tokens, uint64_t width) {
    const uint64_t columns = (width + 64 * kSlice - 1) / (64 * kSlice);
    uint32_t chunk = 8;
    while (chunk < 32 && chunk * 4096ull < tokens * columns) chunk *= 2;
    return tokens <= 1ull << 25 ? chunk : (uint32_t)round_up((tokens + (1u << 20) - 1) >> 20, 8);
}

struct EmbedWorkspace {
    uint64_t counts, keys[2], order[2], parts, bytes;    // offsets and size
};

inline EmbedWorkspace embed_workspace(uint64_t m, uint64_t width) {
    EmbedWorkspace w;
    const uint64_t list = round_up(m * 4, 256), padded = (width + kSlice - 1) / kSlice * kSlice;
    const uint64_t chunk = chunk_of(m, width), chunks = (m + chunk - 1) / chunk;
    w.counts = 0;
    w.keys[0] = sort_counts_bytes(m);
    w.keys[1] = w.keys[0] + list;
    w.order[0] = w.keys[1] + list;
    w.order[1] = w.order[0] + list;
    w.parts = w.order[1] + list;
    w.bytes = w.parts + round_up(chunks * 2 * padded * 4, 256);
    return w;
}

}  // namespace pl

using namespace pl;

extern "C" {

uint64_t poseidon_expert_sort_workspace(uint64_t tokens, uint32_t k, uint32_t n_experts) {
    if (!k || !n_experts || n_experts > POSEIDON_EXPERTS_MAX || tokens > POSEIDON_ROWS_MAX / k) return UINT64_MAX;
    return sort_blocks(tokens * k) > 1 ? sort_counts_bytes(tokens * k) : 0;
}

int poseidon_expert_sort(const int32_t *choice, uint64_t tokens, uint32_t k, uint32_t n_experts, int32_t *order,
                         int32_t *position, int32_t *offsets, void *workspace, uint64_t workspace_bytes,
                         void *hip_stream) {
    if (!k || !n_experts) return POSEIDON_E_INVAL;
    if (n_experts > POSEIDON_EXPERTS_MAX || tokens > POSEIDON_ROWS_MAX / k) return POSEIDON_E_RANGE;
    if (!offsets || (tokens && (!choice || !order || !position))) return POSEIDON_E_INVAL;
    PL_TRY(check_workspace(workspace, workspace_bytes, poseidon_expert_sort_workspace(tokens, k, n_experts)));
    const uint32_t m = (uint32_t)(tokens * k);
    SortPass p = {};
    p.keys = choice;
    p.m = m;
    p.n_keys = n_experts;
    while ((1u << p.bits) < n_experts + 1) ++p.bits;
    p.bins = 1u << p.bits;
    p.blocks = m ? sort_blocks(m) : 1;    // no choices: one block writes the offsets
    p.rounds = sort_rounds(m);
    p.passes = 1;
    p.counts = (uint32_t *)workspace;
    p.order = order;
    p.position = position;
    p.offsets = offsets;
    return sort(p, {}, {}, (hipStream_t)hip_stream);
}

uint64_t poseidon_embed_backward_workspace(uint64_t tokens, uint64_t vocab, uint64_t width) {
    if (check_sizes(tokens, width) != POSEIDON_OK || vocab > POSEIDON_VOCAB_MAX) return UINT64_MAX;
    return tokens ? embed_workspace(tokens, width).bytes : 0;
}

int poseidon_embed_backward(const int32_t *ids, uint64_t tokens, const void *dout, uint64_t dout_pitch, uint32_t type,
                            uint64_t vocab, uint64_t width, float scale, void *dtable, uint64_t dtable_pitch,
                            uint32_t dtable_type, uint32_t accumulate, void *workspace, uint64_t workspace_bytes,
                            void *hip_stream) {
    PL_TRY(check_sizes(tokens, width));
    if (vocab > POSEIDON_VOCAB_MAX) return POSEIDON_E_RANGE;
    PL_TRY(check_matrix(dout, dout_pitch, type, tokens, width));
    PL_TRY(check_matrix(dtable, dtable_pitch, dtable_type, vocab, width));
    if (accumulate > 1 || (tokens && !ids)) return POSEIDON_E_INVAL;
    PL_TRY(check_workspace(workspace, workspace_bytes, poseidon_embed_backward_workspace(tokens, vocab, width)));
    const hipStream_t stream = (hipStream_t)hip_stream;
    const uint32_t slices = (uint32_t)((width + kSlice - 1) / kSlice);
    if (!vocab || (!tokens && accumulate)) return POSEIDON_OK;
    const uint64_t size = size_of(dtable_type);
    Clear c = {(char *)dtable, vocab, width * size, dtable_pitch * size};
    if (accumulate) c.rows = 0;
    if (c.rows && dtable_pitch == width) {
        c.bytes *= c.rows;
        c.rows = 1;
    }

    const uint32_t m = (uint32_t)tokens;
    const EmbedWorkspace w = embed_workspace(tokens, width);
    char *base = (char *)workspace;
    uint32_t bits = 1;
    while ((1u << bits) < vocab + 1) ++bits;
    SortPass p = {};
    p.keys = ids;
    p.m = m;
    p.n_keys = (uint32_t)vocab;
    p.passes = (bits + kMaxBits - 1) / kMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.bins = 1u << p.bits;
    p.blocks = m ? sort_blocks(m) : 1;
    p.rounds = sort_rounds(m);
    p.counts = (uint32_t *)(base + w.counts);
    SortLists lists;
    for (uint32_t i = 0; i < 2; ++i) {
        lists.keys[i] = (int32_t *)(base + w.keys[i]);
        lists.order[i] = (int32_t *)(base + w.order[i]);
    }
    p.keys_out = lists.keys[(p.passes - 1) & 1];
    p.order = lists.order[(p.passes - 1) & 1];
    PL_TRY(sort(p, lists, c, stream));
    if (!m) return POSEIDON_OK;

    EmbedGrad e = {};
    e.keys = p.keys_out;
    e.order = p.order;
    e.m = m;
    e.vocab = (uint32_t)vocab;
    e.width = (uint32_t)width;
    e.chunk = chunk_of(tokens, width);
    e.chunks = (m + e.chunk - 1) / e.chunk;
    e.accumulate = accumulate;
    e.scale = scale;
    e.dout = dout;
    e.dout_pitch = dout_pitch;
    e.dtable = dtable;
    e.dtable_pitch = dtable_pitch;
    e.parts = (float *)(base + w.parts);
    e.padded = slices * kSlice;
    const dim3 grid(e.chunks, (slices + 63) / 64);
    const auto run = [&](auto t) {
        using D = decltype(t);
        PL_STREAM(tokens * width * size_of(type), PL_TYPE(dtable_type, embed_sum_kernel<D, T, STREAM><<<grid, 64, 0, stream>>>(e);
                                                          if (e.chunks > 1) embed_join_kernel<T><<<grid, 256, 0, stream>>>(e)));
    };
    PL_TYPE(type, run(T{}));
    return launched();
}

}  // extern "C"
