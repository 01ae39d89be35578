// token_embedding.cu -- a scaled row of one table for every token, and the dense
// gradient of the table.
//
//   out[i, :]   = scale * E[token_i, :]
//   dE[v, :] (+)= scale * sum over the positions i with token_i = v of grad_out[i, :]
//
// Both move rows and do an operation or two per value: HBM's bandwidth is their bound,
// launches and dependent loads at a few tokens.
#include <cmath>

#include "token_rows.cuh"
#include "tbe_launch.h"

namespace cbtbe {
namespace {

// ---------------------------------------------------------------- lookup

// 128 threads of up to 64 bytes each and 16 blocks per SM (32 registers a thread, every warp
// that an SM holds): a block is a chain of a token's load, a row's load and a store, so bytes
// in flight decide. 262144 rows of 8 KB: 444 us, 5.7 TB/s. In pieces of 16 bytes: 450 us, and
// 504 with 6 blocks of 256 threads, 462 with 8, 530 with 2 or 8 pieces a thread, 526 with 32
// blocks of 64, 655 with resident blocks that load the next tokens ahead (more registers,
// fewer warps). Pieces of 32 bytes on the wider side halve the arithmetic on indices per byte:
// 131072 rows of 1024 bf16 into fp32 135 -> 125 us, 8192 of 2048 bf16 18.4 -> 16.4.
constexpr int kLookupThreads = 128;
constexpr int kLookupBlocks = 16;
// Pieces in flight per thread.
template <int IN, int V> constexpr int kLookupPieces = V * (IN == CB_F32 ? 4 : 2) == 32 ? 2 : 4;

struct LookupArgs {
    Tokens tokens;
    const void* table;
    int64_t row_stride;  // values
    Positions out_at;
    void* out;
    uint32_t pieces;     // per row
    float scale;
    int* error;
};

// A block takes kLookupThreads * kLookupPieces consecutive pieces (of V values) of the
// output, a thread every kLookupThreads-th: rows of any length fill the threads, stores
// are consecutive, and each thread has its loads in flight together.
template <int IN, int OUT, int V>
__global__ void __launch_bounds__(kLookupThreads, kLookupBlocks) token_lookup_kernel(const LookupArgs P) {
    constexpr int kPieces = kLookupPieces<IN, V>;
    begin_kernel();
    const uint64_t first = static_cast<uint64_t>(blockIdx.x) * (kLookupThreads * kPieces);
    const uint32_t row0 = static_cast<uint32_t>(first / P.pieces);
    const uint32_t within = static_cast<uint32_t>(first - static_cast<uint64_t>(row0) * P.pieces) + threadIdx.x;
    Piece<IN, V> x[kPieces];
    uint32_t row[kPieces], piece[kPieces];
    int64_t token[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        const uint32_t k = within + u * kLookupThreads;
        const uint32_t r = k / P.pieces;
        row[u] = row0 + r;
        piece[u] = k - r * P.pieces;
        token[u] = row[u] < P.tokens.n ? P.tokens.load(row[u]) : 0;
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        const bool valid = token[u] >= 0 && token[u] < P.tokens.rows;
        x[u] = zero_piece<IN, V>();
        if (row[u] < P.tokens.n) {
            if (valid)
                x[u] = load_piece<IN, V>(static_cast<const char*>(P.table) +
                                         (token[u] * P.row_stride + static_cast<int64_t>(piece[u]) * V) *
                                             dtype_bytes(IN));
            else if (P.error && piece[u] == 0) set_error(P.error, CB_ERR_INDEX_OOB);
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        if (row[u] < P.tokens.n) {
            float f[V];
            widen<IN, V>(x[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] *= P.scale;
            store_piece<OUT, V>(static_cast<char*>(P.out) +
                                    (P.out_at.at(row[u]) + static_cast<int64_t>(piece[u]) * V) * dtype_bytes(OUT), f);
        }
    }
}

// Rows that no vector of 4 values fits (a length or an address that is odd, or twice an odd
// number: V = 1 or 2): a warp takes 256 V consecutive values of a row, a lane every 32nd piece
// of V, so that loads of 2 or 4 bytes a lane are still whole lines, and a row's index is worked
// out once for 8 pieces a lane. (One value at a time in the kernel above: 131072 rows of 1613
// halves 600 us, most of it arithmetic on indices, and 233 so.)
constexpr int kOddPieces = 8;
template <int IN, int OUT, int V>
__global__ void __launch_bounds__(kLookupThreads) token_lookup_odd_kernel(const LookupArgs P, int32_t dim) {
    begin_kernel();
    const uint64_t w = (static_cast<uint64_t>(blockIdx.x) * kLookupThreads + threadIdx.x) / 32;
    const uint64_t row = w / P.pieces;
    if (row >= P.tokens.n) return;
    const int lane = threadIdx.x & 31, col = (static_cast<int>(w - row * P.pieces) * 32 * kOddPieces + lane) * V;
    const int64_t token = P.tokens.load(static_cast<uint32_t>(row));
    const bool valid = token >= 0 && token < P.tokens.rows;
    if (!valid && P.error && col == 0) set_error(P.error, CB_ERR_INDEX_OOB);
    const char* from = static_cast<const char*>(P.table) + (token * P.row_stride + col) * dtype_bytes(IN);
    char* to = static_cast<char*>(P.out) + (P.out_at.at(static_cast<uint32_t>(row)) + col) * dtype_bytes(OUT);
    const float scale = valid ? P.scale : 0.f;  // zeros for no row of the table, whatever the scale
    Piece<IN, V> x[kOddPieces];
#pragma unroll
    for (int k = 0; k < kOddPieces; ++k)
        x[k] = valid && col + 32 * V * k < dim ? load_piece<IN, V>(from + 32 * V * k * dtype_bytes(IN)) : zero_piece<IN, V>();
#pragma unroll
    for (int k = 0; k < kOddPieces; ++k) {
        if (col + 32 * V * k < dim) {
            float f[V];
            widen<IN, V>(x[k], f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] *= scale;
            store_piece<OUT, V>(to + 32 * V * k * dtype_bytes(OUT), f);
        }
    }
}
template <int IN, int OUT, int V>
void launch_lookup_odd(LookupArgs P, int32_t dim, cudaStream_t s) {
    P.pieces = static_cast<uint32_t>((dim + 32 * V * kOddPieces - 1) / (32 * V * kOddPieces));
    const uint64_t warps = static_cast<uint64_t>(P.tokens.n) * P.pieces, per = kLookupThreads / 32;
    launch(token_lookup_odd_kernel<IN, OUT, V>, dim3(static_cast<unsigned>((warps + per - 1) / per)), dim3(kLookupThreads),
           0, s, P, dim);
}

template <int IN, int OUT, int V>
void launch_lookup(LookupArgs P, int32_t dim, cudaStream_t s) {
    P.pieces = static_cast<uint32_t>(dim / V);
    const uint64_t total = static_cast<uint64_t>(P.tokens.n) * P.pieces;
    const uint64_t per = kLookupThreads * kLookupPieces<IN, V>;
    launch(token_lookup_kernel<IN, OUT, V>, dim3(static_cast<unsigned>((total + per - 1) / per)), dim3(kLookupThreads), 0,
           s, P);
}
template <int IN, int OUT>
void launch_lookup(const LookupArgs& P, int32_t dim, int v, cudaStream_t s) {
    if constexpr (IN != CB_F32 && OUT != CB_F32) {
        if (v == 16) {
            launch_lookup<IN, OUT, 16>(P, dim, s);
            return;
        }
    }
    if (v == 8) launch_lookup<IN, OUT, 8>(P, dim, s);
    else if (v == 4) launch_lookup<IN, OUT, 4>(P, dim, s);
    else if (v == 2) launch_lookup_odd<IN, OUT, 2>(P, dim, s);
    else launch_lookup_odd<IN, OUT, 1>(P, dim, s);
}
template <int IN>
void launch_lookup(const LookupArgs& P, int32_t dim, int v, int out_dtype, cudaStream_t s) {
    if (out_dtype == CB_F32) launch_lookup<IN, CB_F32>(P, dim, v, s);
    else if (out_dtype == CB_F16) launch_lookup<IN, CB_F16>(P, dim, v, s);
    else launch_lookup<IN, CB_BF16>(P, dim, v, s);
}

// ---------------------------------------------------------------- gradient

struct GradArgs {
    Tokens tokens;
    int64_t padding;      // the token that gets no gradient, or -1
    const void* grad_out;
    Positions go_at;
    int32_t dim;
    float scale;
    void* grad;           // [rows, dim]
    int64_t grad_stride;  // values
    int32_t grad_dtype;
    int32_t accumulate;
    int* error;
};

// The columns of a lane in a slab of a row: J pieces of V values, 32 pieces apart.
template <int V> constexpr int kLanePieces = V <= 2 ? 4 : 1;
template <int V> constexpr int kSlab = 32 * V * kLanePieces<V>;
template <int DT, int V>
struct LanePieces {
    Piece<DT, V> x[kLanePieces<V>];
};
template <int DT, int V>
__device__ __forceinline__ LanePieces<DT, V> load_go(const GradArgs& P, uint32_t position, int col) {
    LanePieces<DT, V> r;
    const char* p = static_cast<const char*>(P.grad_out) + (P.go_at.at(position) + col) * dtype_bytes(DT);
#pragma unroll
    for (int j = 0; j < kLanePieces<V>; ++j)
        r.x[j] = col + j * 32 * V < P.dim ? load_piece<DT, V>(p + j * 32 * V * dtype_bytes(DT)) : zero_piece<DT, V>();
    return r;
}
template <int V>
struct Sum {
    float f[kLanePieces<V>][V];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < kLanePieces<V>; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) f[j][i] = 0.f;
    }
    template <int DT>
    __device__ __forceinline__ void add(const LanePieces<DT, V>& r) {
#pragma unroll
        for (int j = 0; j < kLanePieces<V>; ++j) {
            float y[V];
            widen<DT, V>(r.x[j], y);
#pragma unroll
            for (int i = 0; i < V; ++i) f[j][i] += y[i];
        }
    }
    __device__ __forceinline__ void add(const Sum& o) {
#pragma unroll
        for (int j = 0; j < kLanePieces<V>; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) f[j][i] += o.f[j][i];
    }
    // The lane's sums at columns col, .. of an fp32 row of `dim` values (16-byte aligned).
    __device__ __forceinline__ void put(float* row, int col, int dim) const {
#pragma unroll
        for (int j = 0; j < kLanePieces<V>; ++j) {
            float* p = row + col + j * 32 * V;
            if (col + j * 32 * V >= dim) break;
            if constexpr (V == 1) {
                *p = f[j][0];
            } else if constexpr (V == 2) {
                *reinterpret_cast<float2*>(p) = make_float2(f[j][0], f[j][1]);
            } else {
#pragma unroll
                for (int i = 0; i < V; i += 4)
                    *reinterpret_cast<float4*>(p + i) = make_float4(f[j][i], f[j][i + 1], f[j][i + 2], f[j][i + 3]);
            }
        }
    }
    __device__ __forceinline__ void add(const float* row, int col, int dim) {
#pragma unroll
        for (int j = 0; j < kLanePieces<V>; ++j) {
            const float* p = row + col + j * 32 * V;
            if (col + j * 32 * V >= dim) break;
            if constexpr (V == 1) {
                f[j][0] += *p;
            } else if constexpr (V == 2) {
                const float2 x = *reinterpret_cast<const float2*>(p);
                f[j][0] += x.x;
                f[j][1] += x.y;
            } else {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float4 x = *reinterpret_cast<const float4*>(p + i);
                    f[j][i] += x.x;
                    f[j][i + 1] += x.y;
                    f[j][i + 2] += x.z;
                    f[j][i + 3] += x.w;
                }
            }
        }
    }
};

template <int DT, int V>
__device__ __forceinline__ void add_stored(const void* p, float (&f)[V]) {
    const Piece<DT, V> x = load_piece<DT, V, false>(p);  // written by this kernel: not through the read-only path
    float y[V];
    widen<DT, V>(x, y);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] += y[i];
}

// The finished sum of a table row: scaled, added to what is there or not, rounded once.
template <int V>
__device__ __forceinline__ void finish_row(const GradArgs& P, int64_t row, int col, const Sum<V>& s) {
    char* p = static_cast<char*>(P.grad) + (row * P.grad_stride + col) * dtype_bytes(P.grad_dtype);
#pragma unroll
    for (int j = 0; j < kLanePieces<V>; ++j) {
        if (col + j * 32 * V >= P.dim) break;
        char* q = p + j * 32 * V * dtype_bytes(P.grad_dtype);
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = s.f[j][i] * P.scale;
        if (P.grad_dtype == CB_F32) {
            if (P.accumulate) add_stored<CB_F32, V>(q, f);
            store_piece<CB_F32, V>(q, f);
        } else if (P.grad_dtype == CB_F16) {
            if (P.accumulate) add_stored<CB_F16, V>(q, f);
            store_piece<CB_F16, V>(q, f);
        } else {
            if (P.accumulate) add_stored<CB_BF16, V>(q, f);
            store_piece<CB_BF16, V>(q, f);
        }
    }
}
// Zeros to `bytes` (even) of a span that starts at any even address, by a warp: 32 bytes a
// lane between the edges of whole sectors.
__device__ __forceinline__ void zero_span(char* p, int64_t bytes, int lane) {
    const int64_t head = min64(bytes, -reinterpret_cast<uintptr_t>(p) & 31), body = (bytes - head) / 32;
    const int tail = static_cast<int>(bytes - head - body * 32);
    if (2 * lane < head) *reinterpret_cast<uint16_t*>(p + 2 * lane) = 0;
    p += head;
#pragma unroll 4
    for (int64_t i = lane; i < body; i += 32)
        asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(p + 32 * i), "r"(0) : "memory");
    if (2 * lane < tail) *reinterpret_cast<uint16_t*>(p + body * 32 + 2 * lane) = 0;
}
// Zeros to the rows r0 + k (k < 8) whose bit is set in `empty`: neighbours without a gap as one
// span, so that short rows and rows of odd lengths fill a warp's stores too. (A row at a time in
// stores of its own alignment, 64 rows a block: 28 tokens into 88621 rows of 1998 fp32 124
// us and 98 so, 20 into 59384 of 3688 halves 74 and 63, 8192 into 100000 of 1001 bf16 100 and 83,
// 16384 into 65536 of 1024 fp32 80 and 76. Where single rows of 8 KB are to be zeroed among many with
// tokens it is no gain: 262144 into 131072 of 4096 bf16 563 and 570.)
constexpr int kFillWarpRows = 8;
struct Rows {
    char* data;
    int64_t pitch, used;  // bytes
};
__device__ __forceinline__ void zero_rows(const Rows& g, int64_t r0, uint32_t empty, int lane) {
    while (empty) {
        const int k = __ffs(empty) - 1, count = g.pitch == g.used ? __ffs(~(empty >> k)) - 1 : 1;
        zero_span(g.data + (r0 + k) * g.pitch, count * g.used, lane);
        empty &= ~(((1u << count) - 1u) << k);
    }
}

// The sort key of a token: its row, or `rows` (after all rows) for one without gradient.
__device__ __forceinline__ uint32_t token_key(const GradArgs& P, int64_t token, bool report) {
    const bool valid = token >= 0 && token < P.tokens.rows;
    if (!valid && report && P.error) set_error(P.error, CB_ERR_INDEX_OOB);
    return valid && token != P.padding ? static_cast<uint32_t>(token) : static_cast<uint32_t>(P.tokens.rows);
}

// ---------------------------------------------------------------- few tokens: by matching

constexpr int kMatchThreads = 256;
constexpr int kMatchWarps = kMatchThreads / 32;
constexpr uint32_t kMatchTokens = 2048;  // most tokens of a call without a sort
constexpr int kMatchSlabs = 8;           // slabs of a row per block
constexpr int kFillRows = 512;           // most rows of the gradient per zeroing block

// One block per (token, group of slabs): the first position of its token sums all of the
// token's positions, in order; other blocks end at once. The blocks after those write zeros
// to the rows that no token names. n is at most kMatchTokens, so that a block reads all
// tokens in a few loads, and the call is one launch.
template <int DT, int V>
__global__ void __launch_bounds__(kMatchThreads) token_match_kernel(const GradArgs P, uint32_t token_blocks,
                                                                    int slab_groups, Rows grad, int fill_rows) {
    __shared__ uint16_t list[kMatchTokens];
    __shared__ int counts[kMatchWarps];
    __shared__ uint8_t touched[kFillRows];
    __shared__ __align__(16) float part[kMatchWarps][kSlab<V>];
    begin_kernel();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t n = P.tokens.n;
    if (blockIdx.x >= token_blocks) {
        const int64_t r0 = static_cast<int64_t>(blockIdx.x - token_blocks) * fill_rows;
        for (int r = threadIdx.x; r < fill_rows; r += kMatchThreads) touched[r] = 0;
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < n; j += kMatchThreads) {
            const int64_t r = static_cast<int64_t>(token_key(P, P.tokens.load(j), false)) - r0;
            if (r >= 0 && r < fill_rows) touched[r] = 1;
        }
        __syncthreads();
        const int mine = min(fill_rows / kMatchWarps, kFillWarpRows);  // of a warp at a time
        for (int r = wid * mine; r < fill_rows; r += kMatchWarps * mine) {
            const bool zero = lane < mine && r0 + r + lane < P.tokens.rows && !touched[r + min(lane, mine - 1)];
            zero_rows(grad, r0 + r, __ballot_sync(kFull, zero), lane);
        }
        return;
    }
    const uint32_t i = blockIdx.x / slab_groups;
    const int group = blockIdx.x % slab_groups;
    const uint32_t key = token_key(P, P.tokens.load(i), threadIdx.x == 0 && group == 0);
    if (key == static_cast<uint32_t>(P.tokens.rows)) return;
    bool earlier = false;
    for (uint32_t j = threadIdx.x; j < i; j += kMatchThreads) earlier |= token_key(P, P.tokens.load(j), false) == key;
    if (__syncthreads_or(earlier)) return;
    // The token's positions in order: every warp a part of the positions from i on.
    const uint32_t per = (n - i + kMatchWarps - 1) / kMatchWarps;
    const uint32_t lo = min(i + wid * per, n), hi = min(lo + per, n);
    int mine = 0;
    for (uint32_t j0 = lo; j0 < hi; j0 += 32) {
        const uint32_t j = j0 + lane;
        const bool same = j < hi && token_key(P, P.tokens.load(j), false) == key;
        const uint32_t mask = __ballot_sync(kFull, same);
        if (same) list[lo - i + mine + __popc(mask & ((1u << lane) - 1u))] = static_cast<uint16_t>(j);
        mine += __popc(mask);
    }
    if (lane == 0) counts[wid] = mine;
    __syncthreads();
    int count = 0, before = 0;
    for (int w = 0; w < kMatchWarps; ++w) {
        before += w < wid ? counts[w] : 0;
        count += counts[w];
    }
    uint16_t moved[kMatchTokens / kMatchWarps / 32];
#pragma unroll
    for (int k = 0; k < static_cast<int>(kMatchTokens / kMatchWarps / 32); ++k)
        moved[k] = k * 32 + lane < mine ? list[lo - i + k * 32 + lane] : 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < static_cast<int>(kMatchTokens / kMatchWarps / 32); ++k)
        if (k * 32 + lane < mine) list[before + k * 32 + lane] = moved[k];
    __syncthreads();
    // Short lists: a warp per slab. Long ones: all warps on each slab, a part of the list each.
    constexpr int U = 4;
    const bool split = count > 2 * kMatchWarps;
    const int a = split ? count * wid / kMatchWarps : 0, b = split ? count * (wid + 1) / kMatchWarps : count;
    for (int k = split ? 0 : wid; k < kMatchSlabs; k += split ? 1 : kMatchWarps) {
        const int slab = (group * kMatchSlabs + k) * kSlab<V>;
        if (slab >= P.dim) break;
        const int col = slab + lane * V;
        Sum<V> sum;
        sum.clear();
        for (int j = a; j < b; j += U) {
            LanePieces<DT, V> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u < b) x[u] = load_go<DT, V>(P, list[j + u], col);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (j + u < b) sum.add(x[u]);
        }
        if (split) {
            sum.put(part[wid], lane * V, P.dim - slab);
            __syncthreads();
            if (wid == 0) {
                sum.clear();
                for (int w = 0; w < kMatchWarps; ++w) sum.add(part[w], lane * V, P.dim - slab);
                finish_row<V>(P, key, col, sum);
            }
            __syncthreads();
        } else {
            finish_row<V>(P, key, col, sum);
        }
    }
}

// ---------------------------------------------------------------- many tokens: sorted

constexpr int kRadixDigits = 256;
constexpr int kKeyThreads = 1024;
constexpr int kKeysPerThread = static_cast<int>(kSortTileKeys) / kKeyThreads;
static_assert(kKeysPerThread * kKeyThreads == kSortTileKeys && kKeyThreads >= kRadixDigits, "tiles of the sort");

// Pairs (key, position), a tile of the sort per block, with the first pass's digit counts of
// the tile; the later passes' counts are cleared, and the sort's description of its one
// "table" (keys from 0) and tiles written. `touched` (cleared before, or null) gets a 1 for
// every row with a token: a table of the tile's latest keys keeps most of a hot token's stores
// from being made, which all go to one place (131072 skewed tokens: 16 -> 6 us).
struct SortBuffers {
    uint32_t *keys[2], *positions[2];
    Chunk* tiles;
    uint32_t* digits;  // [passes][tiles][256]
    TableDev* table;
    int64_t *first_tile, *num_tiles, *table_pos;  // [2], [1], [2]
    uint8_t* touched;  // [rows], padded to 8
    uint32_t* keyed;   // with `touched`: blocks that have set their flags (cleared before)
};
__global__ void __launch_bounds__(kKeyThreads) token_keys_kernel(const GradArgs P, const SortBuffers S, int passes) {
    constexpr int kSeen = 4096;
    __shared__ uint32_t sh[kRadixDigits], seen[kSeen];
    if (threadIdx.x < kRadixDigits) sh[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < kSeen; i += kKeyThreads) seen[i] = ~0u;
    begin_kernel();
    const uint32_t n = P.tokens.n, tile = blockIdx.x, tiles = gridDim.x;
    const uint32_t first = tile * static_cast<uint32_t>(kSortTileKeys);
    const uint32_t count = min(static_cast<uint32_t>(kSortTileKeys), n - first);
    int64_t token[kKeysPerThread];
#pragma unroll
    for (int u = 0; u < kKeysPerThread; ++u) {
        const uint32_t k = threadIdx.x + u * kKeyThreads;
        token[u] = k < count ? P.tokens.load(first + k) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kKeysPerThread; ++u) {
        const uint32_t k = threadIdx.x + u * kKeyThreads;
        if (k < count) {
            const uint32_t key = token_key(P, token[u], true);
            S.keys[0][first + k] = key;
            S.positions[0][first + k] = first + k;
            atomicAdd(&sh[key & (kRadixDigits - 1)], 1u);
            if (S.touched && key < P.tokens.rows) {
                volatile uint32_t* last = seen + (key & (kSeen - 1));
                if (*last != key) {
                    *last = key;
                    S.touched[key] = 1;  // by any number of threads: one value
                }
            }
        }
    }
    __syncthreads();
    // This block's flags, and what its launch waited for, before the count: see token_fill_kernel.
    if (S.touched && threadIdx.x == 0)
        asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(S.keyed) : "memory");
    if (threadIdx.x < kRadixDigits) {
        S.digits[tile * kRadixDigits + threadIdx.x] = sh[threadIdx.x];
        for (int p = 1; p < passes; ++p)
            S.digits[(static_cast<int64_t>(p) * tiles + tile) * kRadixDigits + threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) {
        Chunk c{};
        c.k0 = first;
        c.len = count;
        S.tiles[tile] = c;
        if (tile == 0) {
            TableDev t{};
            t.rows = P.tokens.rows;
            *S.table = t;
            S.first_tile[0] = S.table_pos[0] = 0;
            S.first_tile[1] = *S.num_tiles = tiles;
            S.table_pos[1] = n;
        }
    }
}

__global__ void __launch_bounds__(256) token_clear_kernel(uint2* words, int64_t n) {
    begin_kernel();
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += gridDim.x * 256ll)
        words[i] = make_uint2(0, 0);
}

// Zeros to every row without a token. Writes alone, while the sort between the keys and the
// sums is a chain of short kernels of few blocks: this kernel needs the flags of
// token_keys_kernel only, is launched after the sort's last pass without waiting for it, and
// waits at its end for those after it. Blocks stay for the whole kernel (a block that waited
// at its end would keep a later one from starting).
// The sort's first pass lets the next kernels launch once it has waited for the keys, so these are done
// when this kernel begins; that their stores are visible here too, without a wait of its own, rests on
// the key blocks' count, released after the flags and acquired before they are read. A thread that
// does not find all of them waits for the whole chain first.
__global__ void __launch_bounds__(256) token_fill_kernel(Rows grad, int64_t rows, const uint8_t* touched,
                                                         const uint32_t* keyed, uint32_t key_blocks) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint32_t done;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(done) : "l"(keyed) : "memory");
    if (done != key_blocks) asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncwarp();
    const int lane = threadIdx.x & 31;
    const int64_t step = gridDim.x * 8ll * kFillWarpRows;
    for (int64_t r0 = (blockIdx.x * 8ll + threadIdx.x / 32) * kFillWarpRows; r0 < rows; r0 += step) {
        const bool zero = lane < kFillWarpRows && r0 + lane < rows && !__ldcg(touched + r0 + min(lane, kFillWarpRows - 1));
        zero_rows(grad, r0, __ballot_sync(kFull, zero), lane);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

struct Sorted {
    const uint32_t *keys, *positions;
    uint32_t chunk, chunks;  // positions per chunk
    float *head, *tail;      // [chunks, dim] sums of runs that began before / end after a chunk
};

constexpr int kReduceThreads = 256;
constexpr int kReduceWarps = kReduceThreads / 32;
constexpr int kReduceRows = 8;       // rows in flight per warp

// A warp takes a chunk of the sorted positions and a slab of columns: it adds the rows of a
// run of equal keys and finishes the table row at the run's end. Runs cut by the chunk's ends
// leave their sums for token_join_kernel.
template <int DT, int V>
__global__ void __launch_bounds__(kReduceThreads) token_reduce_kernel(const GradArgs P, const Sorted S, int slabs) {
    begin_kernel();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t n = P.tokens.n, none = static_cast<uint32_t>(P.tokens.rows);
    const uint64_t w = static_cast<uint64_t>(blockIdx.x) * kReduceWarps + wid;
    const uint32_t chunk = static_cast<uint32_t>(w / slabs);
    if (chunk >= S.chunks) return;
    const int col = static_cast<int>(w - static_cast<uint64_t>(chunk) * slabs) * kSlab<V> + lane * V;
    const uint32_t first = chunk * S.chunk, last = min(first + S.chunk, n);
    bool begun = first == 0 || S.keys[first - 1] != S.keys[first];
    Sum<V> sum;
    sum.clear();
    for (uint32_t k0 = first; k0 < last; k0 += 32) {
        const uint32_t k = k0 + lane;
        const uint32_t key = k < last ? S.keys[k] : none;
        const uint32_t position = k < last ? S.positions[k] : 0;
        // The lane's position ends a run (the end of the keys does too).
        const uint32_t after = k + 1 < n ? S.keys[min(k + 1, n - 1)] : ~0u;
        const uint32_t ends = __ballot_sync(kFull, k < last && after != key);
        const int count = static_cast<int>(min(last - k0, 32u));
        if (__shfl_sync(kFull, key, 0) == none) return;  // keys from here on have no row
        for (int j0 = 0; j0 < count; j0 += kReduceRows) {
            LanePieces<DT, V> x[kReduceRows];
#pragma unroll
            for (int u = 0; u < kReduceRows; ++u) {
                const uint32_t at = __shfl_sync(kFull, position, j0 + u);
                if (j0 + u < count) x[u] = load_go<DT, V>(P, at, col);
            }
            if (P.accumulate) {  // the rows that the runs ending here are added to, on their way too
                const uint32_t here = ends >> j0 & ((1u << kReduceRows) - 1u);
#pragma unroll
                for (int u = 0; u < kReduceRows; ++u) {
                    const uint32_t row = __shfl_sync(kFull, key, j0 + u);
                    if (here >> u & 1 && row != none && col < P.dim)  // a slab may reach past the row, and the tensor
                        prefetch_l1(static_cast<const char*>(P.grad) + (row * P.grad_stride + col) * dtype_bytes(P.grad_dtype));
                }
            }
#pragma unroll
            for (int u = 0; u < kReduceRows; ++u) {
                const uint32_t row = __shfl_sync(kFull, key, j0 + u);
                if (j0 + u < count && row != none) {
                    sum.add(x[u]);
                    const bool end = ends >> (j0 + u) & 1;
                    if (end) {
                        if (begun) finish_row<V>(P, row, col, sum);
                        else sum.put(S.head + static_cast<int64_t>(chunk) * P.dim, col, P.dim);
                        sum.clear();
                        begun = true;
                    } else if (k0 + j0 + u + 1 == last) {  // goes on in the next chunk
                        sum.put((begun ? S.tail : S.head) + static_cast<int64_t>(chunk) * P.dim, col, P.dim);
                    }
                }
            }
        }
    }
}

// The rows whose runs cross chunks: the sum left at the end of the chunk in which a run
// begins, and those of the chunks after it, in order. A block takes kJoinChunks chunks and a slab: a
// lane finds out whether a run crosses its chunk's end and how far it goes; then each warp
// joins short runs, and all warps a long one, a part of its chunks each.
constexpr uint32_t kJoinChunks = 32;  // a lane each
constexpr uint32_t kJoinShort = 8;  // most chunks after the first of a run joined by one warp
constexpr int kJoinLoads = 4;

template <int V>
__global__ void __launch_bounds__(kReduceThreads) token_join_kernel(const GradArgs P, const Sorted S, int slabs) {
    __shared__ __align__(16) float part[kReduceWarps][kSlab<V>];
    begin_kernel();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t chunk0 = blockIdx.x / slabs * kJoinChunks;
    const int slab = static_cast<int>(blockIdx.x % slabs), base = slab * kSlab<V>, col = base + lane * V;
    const uint32_t mine = chunk0 + lane;
    uint32_t key = 0, pieces = 0;  // chunks after `mine` of the run that begins in it and crosses its end
    if (mine + 1 < S.chunks) {
        const uint32_t first = mine * S.chunk, next = first + S.chunk;
        key = S.keys[next - 1];
        if (key != static_cast<uint32_t>(P.tokens.rows) && S.keys[next] == key && (first == 0 || S.keys[first - 1] != key)) {
            // The last chunk that begins with the key: steps that double, then bisection.
            uint32_t lo = mine + 1, hi = S.chunks;
            for (uint32_t step = 1; lo + step < hi; step *= 2) {
                if (S.keys[(lo + step) * S.chunk] != key) hi = lo + step;
                else lo += step;
            }
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (S.keys[mid * S.chunk] == key) lo = mid;
                else hi = mid;
            }
            pieces = lo - mine;
        }
    }
    auto add_pieces = [&](Sum<V>& sum, uint32_t chunk, uint32_t a, uint32_t b) {
        for (uint32_t k = a; k < b; k += kJoinLoads) {
            Sum<V> x[kJoinLoads];
#pragma unroll
            for (int u = 0; u < kJoinLoads; ++u) {
                x[u].clear();
                if (k + u < b) x[u].add(S.head + static_cast<int64_t>(chunk + 1 + k + u) * P.dim, col, P.dim);
            }
#pragma unroll
            for (int u = 0; u < kJoinLoads; ++u) sum.add(x[u]);
        }
    };
    uint32_t shorts = __ballot_sync(kFull, pieces > 0 && pieces <= kJoinShort);
    for (int k = 0; shorts; ++k, shorts &= shorts - 1) {
        const int l = __ffs(shorts) - 1;
        const uint32_t count = __shfl_sync(kFull, pieces, l), row = __shfl_sync(kFull, key, l);
        if (k % kReduceWarps != wid) continue;
        Sum<V> sum;
        sum.clear();
        sum.add(S.tail + static_cast<int64_t>(chunk0 + l) * P.dim, col, P.dim);
        add_pieces(sum, chunk0 + l, 0, count);
        finish_row<V>(P, row, col, sum);
    }
    uint32_t longs = __ballot_sync(kFull, pieces > kJoinShort);  // the same in every warp
    for (; longs; longs &= longs - 1) {
        const int l = __ffs(longs) - 1;
        const uint32_t count = __shfl_sync(kFull, pieces, l), row = __shfl_sync(kFull, key, l);
        Sum<V> sum;
        sum.clear();
        if (wid == 0) sum.add(S.tail + static_cast<int64_t>(chunk0 + l) * P.dim, col, P.dim);
        add_pieces(sum, chunk0 + l, static_cast<uint32_t>(static_cast<uint64_t>(count) * wid / kReduceWarps),
                   static_cast<uint32_t>(static_cast<uint64_t>(count) * (wid + 1) / kReduceWarps));
        sum.put(part[wid], lane * V, P.dim - base);
        __syncthreads();
        if (wid == 0) {
            sum.clear();
            for (int w = 0; w < kReduceWarps; ++w) sum.add(part[w], lane * V, P.dim - base);
            finish_row<V>(P, row, col, sum);
        }
        __syncthreads();
    }
}

// Sorted positions per chunk: short enough for the chunks and slabs of a call to give every
// SM some 32 warps, long enough for the sums that chunks leave (two rows in fp32 at most) to
// be few beside the rows that they read.
uint32_t grad_chunk(int64_t n, int32_t dim) {
    const int64_t warps = 152 * 32, slabs = (dim + 255) / 256;
    uint32_t chunk = 128;
    while (chunk > 16 && n * slabs / chunk < warps) chunk /= 2;
    return chunk;
}

int key_bits(int64_t rows) {  // keys are 0 .. rows
    int bits = 1;
    while (bits < 32 && (rows >> bits) != 0) ++bits;
    return bits;
}

struct GradWorkspace {
    size_t keys[2], positions[2], tiles, digits, table, scalars, touched, head, tail, bytes;
    int64_t num_tiles, touched_words;
    uint32_t chunk;
    int passes;
};
GradWorkspace grad_layout(int64_t n, int64_t rows, int32_t dim) {
    GradWorkspace w{};
    if (n <= kMatchTokens) return w;
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += static_cast<size_t>((bytes + 255) / 256 * 256);
        return here;
    };
    w.num_tiles = (n + kSortTileKeys - 1) / kSortTileKeys;
    w.passes = (key_bits(rows) + 7) / 8;
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = take(n * 4);
        w.positions[i] = take(n * 4);
    }
    w.tiles = take(w.num_tiles * static_cast<int64_t>(sizeof(Chunk)));
    w.digits = take((w.num_tiles + 1) * w.passes * kRadixDigits * 4);
    w.table = take(sizeof(TableDev));
    w.scalars = take(5 * 8);
    w.touched_words = (rows + 7) / 8;
    w.touched = take((w.touched_words + 1) * 8);  // and the count of key blocks
    w.chunk = grad_chunk(n, dim);
    const int64_t chunks = (n + w.chunk - 1) / w.chunk;
    w.head = take(chunks * dim * 4);
    w.tail = take(chunks * dim * 4);
    w.bytes = at;
    return w;
}

Rows grad_rows(const GradArgs& P) {
    const int64_t elem = dtype_bytes(P.grad_dtype);
    return {static_cast<char*>(P.grad), P.grad_stride * elem, P.dim * elem};
}

// A zeroing block of a match takes 8 to 512 rows: at most these bytes, so that blocks many more
// than run at once share them evenly, of short rows as few blocks as fill the GPU, since each
// looks at all tokens.
constexpr int64_t kFillBytes = 128 << 10, kFillBlocks = 304;
template <int DT, int V>
void launch_match(const GradArgs& P, cudaStream_t s) {
    const int groups = (P.dim + kSlab<V> * kMatchSlabs - 1) / (kSlab<V> * kMatchSlabs);
    const uint32_t token_blocks = P.tokens.n * groups;
    const Rows grad = grad_rows(P);
    int fill_rows = kFillRows;
    while (fill_rows > kMatchWarps && (fill_rows * grad.used > kFillBytes || P.tokens.rows < kFillBlocks * fill_rows))
        fill_rows /= 2;
    const int64_t fill = P.accumulate ? 0 : (P.tokens.rows + fill_rows - 1) / fill_rows;
    if (token_blocks + fill == 0) return;
    launch(token_match_kernel<DT, V>, dim3(static_cast<unsigned>(token_blocks + fill)), dim3(kMatchThreads), 0, s, P,
           token_blocks, groups, grad, fill_rows);
}

void launch_fill(const GradArgs& P, const SortBuffers& B, uint32_t key_blocks, int sms, cudaStream_t s) {
    const int64_t warps = (P.tokens.rows + kFillWarpRows - 1) / kFillWarpRows;
    static const int resident = resident_blocks(token_fill_kernel, 256);
    const int64_t most = static_cast<int64_t>(sms) * resident;
    launch(token_fill_kernel, dim3(static_cast<unsigned>(min64((warps + 7) / 8, most))), dim3(256), 0, s, grad_rows(P),
           P.tokens.rows, static_cast<const uint8_t*>(B.touched), static_cast<const uint32_t*>(B.keyed), key_blocks);
}

template <int DT, int V>
void launch_sorted(const GradArgs& P, const GradWorkspace& w, char* base, int sms, cudaStream_t s) {
    SortBuffers B{};
    for (int i = 0; i < 2; ++i) {
        B.keys[i] = reinterpret_cast<uint32_t*>(base + w.keys[i]);
        B.positions[i] = reinterpret_cast<uint32_t*>(base + w.positions[i]);
    }
    B.tiles = reinterpret_cast<Chunk*>(base + w.tiles);
    B.digits = reinterpret_cast<uint32_t*>(base + w.digits);
    B.table = reinterpret_cast<TableDev*>(base + w.table);
    int64_t* scalars = reinterpret_cast<int64_t*>(base + w.scalars);
    B.first_tile = scalars;
    B.table_pos = scalars + 2;
    B.num_tiles = scalars + 4;
    const bool few = w.num_tiles <= kFewSortTiles, fill = !P.accumulate && P.tokens.rows > 0;
    if (fill) {
        B.touched = reinterpret_cast<uint8_t*>(base + w.touched);
        B.keyed = reinterpret_cast<uint32_t*>(B.touched + w.touched_words * 8);
        const int64_t words = w.touched_words + 1;
        launch(token_clear_kernel, dim3(static_cast<unsigned>(min64(sms, (words + 255) / 256))), dim3(256), 0, s,
               reinterpret_cast<uint2*>(B.touched), words);
    }
    launch(token_keys_kernel, dim3(static_cast<unsigned>(w.num_tiles)), dim3(kKeyThreads), 0, s, P, B, w.passes);
    const int64_t words = w.num_tiles * kRadixDigits;
    // With many tiles every pass counts its own digits, per tile (one array) and in total.
    uint32_t* totals = B.digits + words;
    if (!few) cudaMemsetAsync(totals, 0, static_cast<size_t>(w.passes) * kRadixDigits * 4, s);
    for (int p = 0; p < w.passes; ++p) {
        SortPass S{};
        S.keys_in = B.keys[p & 1];
        S.vals_in = B.positions[p & 1];
        S.keys_out = B.keys[(p + 1) & 1];
        S.vals_out = B.positions[(p + 1) & 1];
        S.tiles = B.tiles;
        S.num_tiles = B.num_tiles;
        S.table_first_tile = B.first_tile;
        S.tables = B.table;
        S.n = P.tokens.n;
        S.shift = 8 * p;
        S.table_pos = B.table_pos;
        S.tile_digits = few ? B.digits + p * words : B.digits;
        S.next_digits = few && p + 1 < w.passes ? S.tile_digits + words : nullptr;
        S.table_digits = few ? nullptr : totals + p * kRadixDigits;
        S.T = 1;
        // All but the first pass let the kernels after them launch at once: token_fill_kernel
        // then runs beside the sort, behind the first pass's wait for the keys.
        S.release = few && fill && p > 0;
        launch_radix_pass(S, w.num_tiles, s);
    }
    if (fill) launch_fill(P, B, static_cast<uint32_t>(w.num_tiles), sms, s);
    Sorted R{};
    R.keys = B.keys[w.passes & 1];
    R.positions = B.positions[w.passes & 1];
    R.chunk = w.chunk;
    R.chunks = (P.tokens.n + R.chunk - 1) / R.chunk;
    R.head = reinterpret_cast<float*>(base + w.head);
    R.tail = reinterpret_cast<float*>(base + w.tail);
    const int slabs = (P.dim + kSlab<V> - 1) / kSlab<V>;
    const uint64_t warps = static_cast<uint64_t>(R.chunks) * slabs;
    launch(token_reduce_kernel<DT, V>, dim3(static_cast<unsigned>((warps + kReduceWarps - 1) / kReduceWarps)),
           dim3(kReduceThreads), 0, s, P, R, slabs);
    if (R.chunks > 1)
        launch(token_join_kernel<V>, dim3((R.chunks + kJoinChunks - 1) / kJoinChunks * slabs), dim3(kReduceThreads), 0, s,
               P, R, slabs);
}

template <int DT, int V>
void launch_grad(const GradArgs& P, const GradWorkspace& w, char* base, int sms, cudaStream_t s) {
    if (P.tokens.n <= kMatchTokens) launch_match<DT, V>(P, s);
    else launch_sorted<DT, V>(P, w, base, sms, s);
}
template <int DT>
void launch_grad(const GradArgs& P, const GradWorkspace& w, char* base, int v, int sms, cudaStream_t s) {
    if (v == 8) launch_grad<DT, 8>(P, w, base, sms, s);
    else if (v == 4) launch_grad<DT, 4>(P, w, base, sms, s);
    else if (v == 2) launch_grad<DT, 2>(P, w, base, sms, s);
    else launch_grad<DT, 1>(P, w, base, sms, s);
}

// ---------------------------------------------------------------- arguments

bool current_sms(int* sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess &&
        cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && *sms > 0)
        return true;
    cudaGetLastError();
    return false;
}
bool valid_dtype(int d) { return d == CB_F32 || d == CB_F16 || d == CB_BF16; }

// A row-major operand whose rows are taken in pieces of v values: v divides its dim and
// strides, and a piece is aligned to its size.
bool takes(const void* p, int dtype, int64_t dim, int64_t s0, int64_t s1, int v) {
    const int64_t bytes = static_cast<int64_t>(v) * dtype_bytes(dtype);
    return dim % v == 0 && s0 % v == 0 && s1 % v == 0 && reinterpret_cast<uintptr_t>(p) % bytes == 0;
}

// Sizes come in 64 bits, so that one past 32 is refused and not cut off on its way here.
constexpr int64_t kTokensBelow = int64_t(1) << 30, kRowsBelow = int64_t(1) << 31, kDimMost = int64_t(1) << 20;
bool valid_sizes(int64_t rows, int64_t dim) { return rows >= 0 && rows < kRowsBelow && dim >= 0 && dim <= kDimMost; }
bool valid_tokens(const void* tokens, int idx_dtype, int64_t sequences, int64_t length) {
    return (idx_dtype == CB_I32 || idx_dtype == CB_I64) && sequences >= 0 && length >= 0 &&
           (sequences == 0 || length <= (kTokensBelow - 1) / sequences) &&
           (sequences == 0 || length == 0 ||
            (tokens && reinterpret_cast<uintptr_t>(tokens) % (idx_dtype == CB_I32 ? 4 : 8) == 0));
}
bool aligned_to(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % dtype_bytes(dtype) == 0; }

}  // namespace
}  // namespace cbtbe

extern "C" cb_status cb_token_forward(const void* table, cb_dtype table_dtype, int64_t rows, int64_t dim,
                                      int64_t row_stride, const void* tokens, cb_index_dtype idx_dtype, int64_t sequences,
                                      int64_t length, int64_t token_sequence_stride, int64_t token_stride, float scale,
                                      void* out, cb_dtype out_dtype, int64_t out_sequence_stride, int64_t out_stride,
                                      int* error, cudaStream_t stream) {
    using namespace cbtbe;
    if (!valid_tokens(tokens, idx_dtype, sequences, length) || !valid_dtype(table_dtype) || !valid_dtype(out_dtype) ||
        !valid_sizes(rows, dim) || !(scale == scale) || reinterpret_cast<uintptr_t>(error) % 4)
        return CB_ERR_INVALID_ARG;
    const int64_t n = sequences * length;
    if (n == 0 || dim == 0) return CB_OK;
    if (!out || (rows > 0 && !table) || (rows > 1 && row_stride < dim) || !aligned_to(table, table_dtype) ||
        !aligned_to(out, out_dtype) || !rows_apart(sequences, out_sequence_stride, length, out_stride, dim))
        return CB_ERR_INVALID_ARG;
    LookupArgs P{};
    P.tokens = {tokens, positions(sequences, length, token_sequence_stride, token_stride), static_cast<uint32_t>(n),
                idx_dtype == CB_I32, rows};
    P.table = table;
    P.row_stride = row_stride;
    P.out_at = positions(sequences, length, out_sequence_stride, out_stride);
    P.out = out;
    P.scale = scale;
    P.error = error;
    // Pieces of 32 bytes on the wider side, and of half as many values until they fit the
    // row, the strides and the addresses.
    const int64_t s1 = length > 1 ? out_stride : 0, s0 = sequences > 1 ? out_sequence_stride : 0;
    const int64_t table_stride = rows > 1 ? row_stride : 0;
    int v = table_dtype == CB_F32 || out_dtype == CB_F32 ? 8 : 16;
    while (v > 1 && !(takes(table, table_dtype, dim, table_stride, 0, v) && takes(out, out_dtype, dim, s0, s1, v)))
        v /= 2;
    // The zeros of a token out of range times infinity: the kernel for odd rows leaves them zeros (the
    // other has no register to spare for it).
    if (std::isinf(scale)) v = static_cast<int>(min64(v, 2));
    const int32_t d = static_cast<int32_t>(dim);
    if (table_dtype == CB_F32) launch_lookup<CB_F32>(P, d, v, out_dtype, stream);
    else if (table_dtype == CB_F16) launch_lookup<CB_F16>(P, d, v, out_dtype, stream);
    else launch_lookup<CB_BF16>(P, d, v, out_dtype, stream);
    return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA;
}

extern "C" int64_t cb_token_backward_workspace_bytes(int64_t num_tokens, int64_t rows, int64_t dim) {
    using namespace cbtbe;
    if (num_tokens <= 0 || num_tokens >= kTokensBelow || !valid_sizes(rows, dim) || dim == 0) return 0;
    return static_cast<int64_t>(grad_layout(num_tokens, rows, static_cast<int32_t>(dim)).bytes);
}

extern "C" cb_status cb_token_backward(const void* grad_out, cb_dtype go_dtype, int64_t go_sequence_stride,
                                       int64_t go_stride, const void* tokens, cb_index_dtype idx_dtype, int64_t sequences,
                                       int64_t length, int64_t token_sequence_stride, int64_t token_stride, int64_t rows,
                                       int64_t dim, float scale, int64_t padding_idx, int accumulate, void* grad,
                                       cb_dtype grad_dtype, int64_t grad_stride, void* workspace, int64_t workspace_bytes,
                                       int* error, cudaStream_t stream) {
    using namespace cbtbe;
    if (!valid_tokens(tokens, idx_dtype, sequences, length) || !valid_dtype(go_dtype) || !valid_dtype(grad_dtype) ||
        !valid_sizes(rows, dim) || !(scale == scale) || reinterpret_cast<uintptr_t>(error) % 4)
        return CB_ERR_INVALID_ARG;
    const int64_t n = sequences * length;
    if (dim == 0 || (n == 0 && (accumulate || rows == 0))) return CB_OK;
    if ((rows > 0 && !grad) || (n > 0 && !grad_out) || (rows > 1 && grad_stride < dim) ||
        !aligned_to(grad_out, go_dtype) || !aligned_to(grad, grad_dtype) ||
        (length > 1 && go_stride < 0) || (sequences > 1 && go_sequence_stride < 0))
        return CB_ERR_INVALID_ARG;
    const GradWorkspace w = grad_layout(n, rows, static_cast<int32_t>(dim));
    if (w.bytes > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 ||
                        workspace_bytes < static_cast<int64_t>(w.bytes)))
        return CB_ERR_CAPACITY;
    GradArgs P{};
    P.tokens = {tokens, positions(sequences, length, token_sequence_stride, token_stride), static_cast<uint32_t>(n),
                idx_dtype == CB_I32, rows};
    P.padding = padding_idx;
    P.grad_out = grad_out;
    P.go_at = positions(sequences, length, go_sequence_stride, go_stride);
    P.dim = static_cast<int32_t>(dim);
    P.scale = scale;
    P.grad = grad;
    P.grad_stride = grad_stride;
    P.grad_dtype = grad_dtype;
    P.accumulate = accumulate;
    P.error = error;
    const int64_t s1 = length > 1 ? go_stride : 0, s0 = sequences > 1 ? go_sequence_stride : 0;
    const int64_t row_stride = rows > 1 ? grad_stride : 0;
    int v = go_dtype == CB_F32 && grad_dtype == CB_F32 ? 4 : 8;
    while (v > 1 && !(takes(grad_out, go_dtype, dim, s0, s1, v) && takes(grad, grad_dtype, dim, row_stride, 0, v)))
        v /= 2;
    int sms = 0;
    if (!current_sms(&sms)) return CB_ERR_CUDA;
    char* base = static_cast<char*>(workspace);
    if (go_dtype == CB_F32) launch_grad<CB_F32>(P, w, base, v, sms, stream);
    else if (go_dtype == CB_F16) launch_grad<CB_F16>(P, w, base, v, sms, stream);
    else launch_grad<CB_BF16>(P, w, base, v, sms, stream);
    return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA;
}
