// window_attention_tc.cuh -- what the tensor-core kernels of windowed attention share: tiles of
// 128 rows by TMA, products with an operand in TMEM, what a tile of rows sees, and its masks.
#pragma once

#include "tensor_core.cuh"
#include "window_attention.cuh"

namespace cbtbe {
namespace attention {

constexpr int kTile = 128;                       // rows (tokens) of a tile
constexpr uint32_t kBoxBytes = kTile * 64 * 2;   // 64 values of each, as TMA copies them
template <int D> constexpr uint32_t kRowsBytes = D / 64 * kBoxBytes;

// ---------------------------------------------------------------- instructions

// D (+)= A B over 16 values of K, A of 128 rows in TMEM (two values a column).
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(shape), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// tc::mma_shape of bf16 operands.
template <bool BF16>
__host__ __device__ constexpr uint32_t mma_shape(int m, int n, bool b_mn_major) {
    return tc::mma_shape(m, n, b_mn_major) | (BF16 ? 1u << 7 | 1u << 10 : 0u);
}

#define CB_R8(r, i) \
    "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define CB_R32(r, i) CB_R8(r, i), CB_R8(r, i + 8), CB_R8(r, i + 16), CB_R8(r, i + 24)

// 64 columns of the warp's 32 lanes; they have arrived when the call returns.
__device__ __forceinline__ void tmem_load64(uint32_t addr, uint32_t (&r)[64]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : CB_R32(r, 0), CB_R32(r, 32)
        : "r"(addr)
        : "memory");
}
// 16 columns, without the wait for them (tmem_store_wait).
__device__ __forceinline__ void tmem_store16_begin(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
// 32 columns, without the wait for them (tmem_store_wait).
__device__ __forceinline__ void tmem_store32_begin(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}
// 8 columns times f.
__device__ __forceinline__ void scale8(uint32_t addr, float f) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : CB_R8(r, 0)
                 : "r"(addr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};\n\t"
                 "tcgen05.wait::st.sync.aligned;" ::"r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The largest of three.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// a * b + c and a + b of two values at once.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Registers of a thread from here on, by all warps of a group of four.
template <int N>
__device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// This thread's stores to shared memory, before TMA reads them (and a barrier between). Only those: the fence over all
// memory waits for the thread's stores to global memory too, 1500 clocks.
__device__ __forceinline__ void fence_to_tma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t src, int32_t x, int32_t y, int32_t z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(src), "r"(x), "r"(y), "r"(z)
                 : "memory");
}
__device__ __forceinline__ void tma_store_done() {  // read from shared memory
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// A tile of `D` columns: head `head`, tokens from `token` on.
template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int token) {
#pragma unroll
    for (int x = 0; x < D / 64; ++x) tc::tma_load(dst + x * kBoxBytes, map, bar, x * 64, head, token);
}

// Byte of columns 8 c .. 8 c + 7 (16 bytes) of row r in a tile as TMA lays it out.
__device__ __forceinline__ uint32_t tile_byte(int r, int c) {
    return static_cast<uint32_t>(c >> 3) * kBoxBytes + static_cast<uint32_t>(r) * 128 +
           static_cast<uint32_t>(((c & 7) ^ (r & 7)) << 4);
}

// ---------------------------------------------------------------- whole warps

// A whole warp waits, and is together again after it: instructions that want the warp converged may follow.
//
// Products are issued by one lane of a warp that is together before and after (an `if` and __syncwarp): what they take is
// then in registers that the warp shares; a thread in a branch of its own moves each value there first and could not keep the
// tensor cores busy. Without the __syncwarp the other lanes would poll the next barrier while the one issues: they
// can change the shared registers under it, and fall two phases of a barrier behind.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) {
    return __all_sync(kFull, tc::barrier_wait(tc::smem_addr(bar), parity & 1));
}
// One arrival for the warp, behind what its lanes did.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) tc::barrier_arrive(tc::smem_addr(bar));
    __syncwarp();
}

// Zeros in rows `from` .. 127 of a tile, by a whole warp, before the tile's products.
//
// The last block of an item holds tokens that none of its rows sees: of the next session, or of none. Their infinities and NaNs
// would survive the zeros by which they are multiplied, and all of the item's rows would have to be computed again (a session of
// 32768 tokens x 8 heads over 1 beside one of NaNs: backward 1730 ms, 10 with the rows cleared, 4.5 beside one of numbers).
//
// Such a tile lands on a barrier of its own (`landed`); a warp that has little else to do, the one that stores or over
// keys the one that brings lse and delta, waits for it there, clears the rows and arrives where the tile's products wait for
// any other's copy. (By the warp that issues the products these took 5 to 14 % longer in the backward pass, cleared tiles
// or not; by the one that looks ahead 41 against 36 us where all sessions are short.)
template <int D>
__device__ __forceinline__ void clear_rows(unsigned char* tile, int from, int lane) {
    for (int r = from + lane / 8; r < kTile; r += 4)  // a lane 16 bytes
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
            *reinterpret_cast<uint4*>(tile + x * kBoxBytes + r * 128 + lane % 8 * 16) = make_uint4(0u, 0u, 0u, 0u);
    fence_to_tma();
}
// For a warp: the barriers on which tiles to be cleared land, one for each place of a tile. `turns` has the phase of each.
template <int D>
__device__ __forceinline__ bool clear_landed(uint64_t* landed, uint64_t* full, uint32_t place, uint32_t& turns, unsigned char* tile,
                                             int from, int lane) {
    if (!warp_wait(landed + place, turns >> place)) return false;
    turns ^= 1u << place;
    clear_rows<D>(tile, from, lane);
    warp_arrive(full + place);
    return true;
}

// ---------------------------------------------------------------- what rows see

// Bits i of columns [a, b) among the 32 from `first` on. (The instruction's shifts by 32 and more give 0.)
__device__ __forceinline__ uint32_t ones_from(int bit) {
    uint32_t r;
    asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(~0u), "r"(max(bit, 0)));
    return r;
}
__device__ __forceinline__ uint32_t range_bits(int a, int b, int first) { return ones_from(a - first) & ~ones_from(b - first); }

// Two intervals of positions: a row's tokens in sight, or (for a key) the rows that see it.
struct TwoRanges {
    int a0, a1, b0, b1;
    __device__ __forceinline__ uint32_t bits(int first) const { return range_bits(a0, a1, first) | range_bits(b0, b1, first); }
};

// The keys that the rows of a tile see: [lo, hi), and before that the first tokens of the
// session that the tile begins in, [s0, s1). All empty where the tile has no token of a session.
struct Sight {
    int lo, hi, s0, s1;
};
struct Row {
    int start, first;  // of the session, and of the window; both t + 1 where t is of no session
    bool real;
};
__device__ __forceinline__ Row row_of(const Shape& S, int64_t t) {
    Row r{0, 0, false};
    if (t < S.tokens && S.end[t] > t) {
        r.start = S.start[t];
        r.first = static_cast<int>(max64(r.start, t - S.window + 1));
        r.real = true;
    }
    return r;
}
// From the least `first`, the end of the last real row and the least `start` of a tile.
__device__ __forceinline__ Sight sight_of(int lo, int hi, int start, int sinks) {
    Sight s{hi == 0 ? 0 : lo, hi, 0, 0};
    if (hi > 0 && start < lo) {
        s.s0 = start;
        s.s1 = static_cast<int>(min64(static_cast<int64_t>(start) + sinks, lo));
    }
    return s;
}
__host__ __device__ __forceinline__ int tiles_of(int n) { return (n + kTile - 1) / kTile; }

// ---------------------------------------------------------------- two tiles of queries and their keys

// Two tiles that read one head of keys and values: the same tokens of two heads that share it,
// where heads share in twos (then their keys are the same); else 256 tokens of one head.
inline bool pairs_heads(const Shape& S) { return S.group % 2 == 0; }
inline int64_t work_items(const Shape& S) {
    const int64_t tiles = (S.tokens + kTile - 1) / kTile;
    return pairs_heads(S) ? tiles * (S.heads / 2) : (tiles + 1) / 2 * S.heads;
}
struct Work {
    int token[2], head[2], kv;
};
__device__ __forceinline__ Work work_of(const Shape& S, unsigned item, bool pair_heads) {
    Work W;
    const unsigned per = static_cast<unsigned>(pair_heads ? S.heads / 2 : S.heads), tile = item / per;
    const int p = static_cast<int>(item - tile * per);
    W.head[0] = pair_heads ? 2 * p : p;
    W.head[1] = pair_heads ? 2 * p + 1 : p;
    W.token[0] = static_cast<int>(tile) * (pair_heads ? kTile : 2 * kTile);
    W.token[1] = pair_heads ? W.token[0] : W.token[0] + kTile;
    W.kv = W.head[0] / S.group;
    return W;
}

// The blocks of keys of a work item, in order: first tokens of tile 0's session, of tile 1's (or of both
// at once), then what the windows reach.
struct Blocks {
    Sight x[2];
    int sinks0, sinks1, base, count;
    bool shared;
    struct Block {
        int at;          // first key
        bool use[2];
        int from[2], to[2];  // keys of it that count, for each tile
    };
    __device__ __forceinline__ Blocks(const Sight& a, const Sight& b) {
        x[0] = a;
        x[1] = b;
        shared = a.s0 == b.s0 && a.s1 == b.s1;
        sinks0 = tiles_of(a.s1 - a.s0);
        sinks1 = shared ? 0 : tiles_of(b.s1 - b.s0);
        base = a.hi == 0 ? b.lo : (b.hi == 0 ? a.lo : min(a.lo, b.lo));
        count = sinks0 + sinks1 + tiles_of(max(max(a.hi, b.hi) - base, 0));
    }
    // Keys of block i, from its first on, that some row may see. Fewer than 128 only in the last of each kind.
    __device__ __forceinline__ int counted(int i) const {
        if (i < sinks0) return x[0].s1 - x[0].s0 - i * kTile;
        i -= sinks0;
        if (i < sinks1) return x[1].s1 - x[1].s0 - i * kTile;
        return max(x[0].hi, x[1].hi) - base - (i - sinks1) * kTile;
    }
    // f(i, counted(i)) of the blocks i, from `from` to `to` - 1, that hold keys which no row sees.
    template <class F>
    __device__ __forceinline__ bool to_clear(int from, int to, F f) const {
        const int last[3] = {sinks0 - 1, sinks0 + sinks1 - 1, count - 1};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int i = last[k], keys = counted(i);
            if (i < from || i >= to || (k && i == last[k - 1]) || keys >= kTile) continue;
            if (!f(i, keys)) return false;
        }
        return true;
    }
    __device__ __forceinline__ Block at(int i) const {
        Block k;
        if (i < sinks0 + sinks1) {
            const int t = i < sinks0 ? 0 : 1;
            k.at = x[t].s0 + (i - (t ? sinks0 : 0)) * kTile;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                k.use[u] = u == t || shared;
                k.from[u] = x[u].s0;
                k.to[u] = x[u].s1;
            }
            return k;
        }
        k.at = base + (i - sinks0 - sinks1) * kTile;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            k.use[u] = k.at < x[u].hi && k.at + kTile > x[u].lo;
            k.from[u] = x[u].lo;
            k.to[u] = x[u].hi;
        }
        return k;
    }
};

// What a block's warps need to know of an item, found out ahead by one of them.
struct Item {
    Work W;
    Sight sight[2];
    int begin[2];                // of the session that the tile begins in
    unsigned char row[2][kTile];  // where a row's session begins: that many tokens into the tile, or kBefore, or kNowhere
};
constexpr int kBefore = 254, kNowhere = 255;
__device__ __forceinline__ void look_ahead(const Shape& S, Item& it, int x, int token, int lane) {
    int lo = INT32_MAX, hi = 0, s0 = INT32_MAX;
#pragma unroll
    for (int k = 0; k < kTile / 32; ++k) {
        const int t = token + k * 32 + lane;
        const Row r = row_of(S, t);
        it.row[x][k * 32 + lane] = static_cast<unsigned char>(!r.real ? kNowhere : (r.start < token ? kBefore : r.start - token));
        if (!r.real) continue;
        lo = min(lo, r.first);
        hi = max(hi, t + 1);
        s0 = min(s0, r.start);
    }
    lo = __reduce_min_sync(kFull, lo);
    hi = __reduce_max_sync(kFull, hi);
    s0 = __reduce_min_sync(kFull, s0);
    if (lane == 0) {
        it.sight[x] = sight_of(lo, hi, s0, S.sinks);
        it.begin[x] = s0;
    }
}
__device__ __forceinline__ Row row_in(const Shape& S, const Item& it, int x, int row) {
    const int code = it.row[x][row];
    Row r{0, 0, code != kNowhere};
    if (r.real) {
        const int t = it.W.token[x] + row;
        r.start = code == kBefore ? it.begin[x] : it.W.token[x] + code;
        r.first = static_cast<int>(max64(r.start, t - S.window + 1));
    }
    return r;
}

// A tensor's tiles for TMA.
bool tile_map(CUtensorMap* map, const Heads& h, int64_t tokens, int32_t heads, int32_t dim, int32_t dtype);

}  // namespace attention
}  // namespace cbtbe
