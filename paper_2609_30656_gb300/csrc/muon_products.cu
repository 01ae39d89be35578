// muon_products.cu -- the products of Newton-Schulz steps on the tensor cores (tcgen05, fp16 into
// fp32): tiles by one block, by a pair of blocks on two SMs, and by a cluster over a long K, with
// what follows a product in its epilogue.
#include "muon_internal.cuh"

namespace cbtbe {
namespace muon {
namespace {

constexpr int kTileM = 128, kTileK = 64;
constexpr int kEpilogueWarps = 8;  // two for each quarter of TMEM's lanes, every other 32 columns each
// Two warps copy, every other stage each: waiting for a stage, arming its barrier and issuing its
// copies takes a thread 107 + 58 + 66 clocks a copy. The multiplying warp's loop counts as much:
// it runs as a whole and elects a lane to issue, so that operands are in registers that the warp
// shares, adds to descriptors built once, and tests the next stage's barrier while it issues. With
// one lane in a branch that built them (250 clocks to issue four products, 98 to see a barrier,
// 85 to commit) a step of 64 of K took 600 clocks at any width: five steps of 1024 x 1024 137
// us and 110 so, of 2048 x 2048 257 and 219, of 4 x 1024 x 4096 386 and 333.
constexpr int kCopyWarps = 2, kMultiplyWarp = kEpilogueWarps + kCopyWarps;
constexpr int kProductThreads = (kMultiplyWarp + 1) * 32;
constexpr uint32_t kBoxBytes = 64 * 64 * 2;                 // 64 rows of 64 fp16
template <int BN> constexpr int kStages = BN == 128 ? 6 : 8;
// Sums of a tile in TMEM: two of its width, or of every part's.
template <int BN, Product WHAT> constexpr int kSumColumns = WHAT == kGram && BN == 64 ? kPartsMost * BN : BN;
template <int BN> constexpr uint32_t kStageBytes = (kTileM + BN) * kTileK * 2;

struct Tile {
    int32_t b, i, j;
};

// Column tiles of `width` of row tile i (of `height`) that reach the lower triangle.
__host__ __device__ __forceinline__ int lower_tiles(int i, int height, int width, int col_tiles) {
    const int need = ((i + 1) * height + width - 1) / width;
    return need < col_tiles ? need : col_tiles;
}

template <int HEIGHT, Product WHAT>
__device__ __forceinline__ Tile tile_at(const ProductArgs& P, int64_t t) {
    Tile T;
    T.b = static_cast<int>(t / P.tiles);
    int r = static_cast<int>(t - T.b * P.tiles);
    if constexpr (kSymmetric<WHAT>) {
        T.i = 0;
        while (true) {
            const int c = lower_tiles(T.i, HEIGHT, P.width, P.col_tiles);
            if (r < c) break;
            r -= c;
            ++T.i;
        }
        T.j = r;
    } else {
        // Eight row tiles at a time, so that concurrent tiles share operands in L2.
        constexpr int G = 8;
        const int group = r / (G * P.col_tiles), first = group * G;
        const int rows = P.row_tiles - first < G ? P.row_tiles - first : G;
        r -= group * G * P.col_tiles;
        T.i = first + r % rows;
        T.j = r / rows;
    }
    return T;
}

// 32 bytes, a whole sector, of one lane: halves of them would be fetched twice (the shared
// memory of these kernels leaves little for L1) and written in two.
__device__ __forceinline__ void load_sector(const void* p, uint32_t* w) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store_sector(void* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p)
                 : "memory");
}

// 32 halves of a lane's row.
struct Halves {
    uint32_t w[16];
};
__device__ __forceinline__ Halves load_halves(const __half* p) {
    Halves h;
    load_sector(p, h.w);
    load_sector(p + 16, h.w + 8);
    return h;
}
__device__ __forceinline__ void unpack_halves(const Halves& h, float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        __half2 x;
        memcpy(&x, &h.w[k], 4);
        const float2 f = __half22float2(x);
        v[2 * k] = f.x;
        v[2 * k + 1] = f.y;
    }
}
__device__ __forceinline__ void store_halves(__half* p, const float (&v)[32]) {
    uint32_t w[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        memcpy(&w[k], &h, 4);
    }
    store_sector(p, w);
    store_sector(p + 16, w + 8);
}

// Two values rounded to 16 bits.
template <int DT>
__device__ __forceinline__ uint32_t pack(float x, float y) {
    uint32_t w;
    if constexpr (DT == CB_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        memcpy(&w, &h, 4);
    } else {
        const __half2 h = __floats2half2_rn(x, y);
        memcpy(&w, &h, 4);
    }
    return w;
}

// 32 columns of a lane's row into the caller's matrix where its rows are whole sectors: no
// exchange between lanes. (Through shared memory, 16 columns at a time: bf16 weights, of which
// four lanes then share a sector, a step of 4 x 1024 x 4096 398 us, and 365 so; fp32 ones 389
// and 386, 8 x 512 x 2048 239 and 234.)
template <int DT>
__device__ __forceinline__ void finish_row(const ProductArgs& P, int batch, int row, int col, float (&v)[32]) {
    constexpr int kBytes = DT == CB_F32 ? 4 : 2, V = 32 / kBytes;  // values of a sector
    if (row >= P.m) return;
    char* p = static_cast<char*>(P.user) + (batch * P.user_batch + row * P.user_row + col) * kBytes;
#pragma unroll
    for (int c = 0; c < 32; c += 2 * V) {  // two sectors at a time: all four of fp32 take registers that there are not
        uint32_t w[16];
        if (P.weights) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (col + c + k * V < P.n) load_sector(p + (c + k * V) * kBytes, w + 8 * k);
        }
#pragma unroll
        for (int k = 0; k < 2 * V; ++k) {
            float x = v[c + k] * (1.f / kScaleX);
            if (P.weights) {
                float old;
                if constexpr (DT == CB_F32) {
                    old = __uint_as_float(w[k]);
                } else {
                    const uint32_t half = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu;
                    if constexpr (DT == CB_BF16) {
                        old = __uint_as_float(half << 16);
                    } else {
                        const uint16_t bits = static_cast<uint16_t>(half);
                        __half h;
                        memcpy(&h, &bits, 2);
                        old = __half2float(h);
                    }
                }
                x = fmaf(-P.rate, x, P.keep * old);
            }
            v[c + k] = x;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            if constexpr (DT == CB_F32) w[k] = __float_as_uint(v[c + k]);
            else w[k] = pack<DT>(v[2 * k], v[2 * k + 1]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (col + c + k * V < P.n) store_sector(p + (c + k * V) * kBytes, w + 8 * k);
    }
}

// 16 columns of a warp's 32 rows into the caller's matrix, through shared memory so that
// lanes run along the caller's rows, V values each: loads (of weights) first, then stores. 16 bytes
// a lane where rows allow them: a step of 4 x 4096 x 1024 in bf16 387 us, and 413 with 8.
constexpr int kStageFloats = 32 * 20;  // rows of 16 (or, transposed, 32) values padded to 20 (36)
template <int DT, int V>
__device__ __forceinline__ void finish_result(const ProductArgs& P, int batch, int row, int col, const float* v,
                                              float* stage, int lane) {
    char* user = static_cast<char*>(P.user) + batch * P.user_batch * dtype_bytes(DT);
    __syncwarp();
    if (P.transposed) {
#pragma unroll
        for (int k = 0; k < 16; ++k) stage[k * 36 + lane] = v[k];
    } else {
#pragma unroll
        for (int k = 0; k < 16; k += 4)
            *reinterpret_cast<float4*>(stage + lane * 20 + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    }
    __syncwarp();
    const int row0 = P.transposed ? col : row - lane, col0 = P.transposed ? row - lane : col;
    const int rows = P.transposed ? P.n : P.m, cols = P.transposed ? P.m : P.n;  // of the caller's matrix
    constexpr int N = 16 / V;                                                     // pieces of V values a lane
    const int wide = (P.transposed ? 32 : 16) / V, pitch = P.transposed ? 36 : 20;  // lanes per row
    const int c = lane % wide * V, r = lane / wide, step = 32 / wide;
    const int64_t at = static_cast<int64_t>(row0 + r) * P.user_row + col0 + c, down = step * P.user_row;
    float w[N][V] = {};
    if (P.weights) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (row0 + r + k * step >= rows) break;
            if (P.user_vector) {
                if (col0 + c < cols) load_values<V>(user, at + k * down, DT, w[k]);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (col0 + c + e < cols) w[k][e] = load_value(user, at + k * down + e, DT);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (row0 + r + k * step >= rows) break;
        float x[V];
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 s = *reinterpret_cast<const float4*>(stage + (r + k * step) * pitch + c + e);
            x[e] = s.x, x[e + 1] = s.y, x[e + 2] = s.z, x[e + 3] = s.w;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            x[e] *= 1.f / kScaleX;
            if (P.weights) x[e] = fmaf(-P.rate, x[e], P.keep * w[k][e]);
        }
        if (P.user_vector) {
            if (col0 + c < cols) {
                if constexpr (V == 4) store_values4<DT>(user, at + k * down, x);
                else *reinterpret_cast<uint4*>(user + 2 * (at + k * down)) =
                    make_uint4(pack<DT>(x[0], x[1]), pack<DT>(x[2], x[3]), pack<DT>(x[4], x[5]), pack<DT>(x[6], x[7]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (col0 + c + e < cols) store_value(user, at + k * down + e, x[e], DT);
        }
    }
}

// What the result at a lane's 32 columns has added to it: loaded a turn ahead of its use.
struct Term {
    Halves hi, lo;
};
template <Product WHAT>
__device__ __forceinline__ void load_term(const ProductArgs& P, int batch, int row, int col, Term& t) {
    if (row >= P.m || col >= P.n || WHAT == kGram) return;
    const int64_t at = batch * P.term_batch + static_cast<int64_t>(row) * P.term_ld + col;
    t.hi = load_halves(P.term_hi + at);
    if (WHAT != kPoly) t.lo = load_halves(P.term_lo + at);
}

// 32 columns [col, col + 32) of row `row` of a tile's result: `v` holds the products' sums.
template <Product WHAT>
__device__ __forceinline__ void finish(const ProductArgs& P, int batch, int row, int col, float (&v)[32],
                                       const Term& term, float* stage, int lane) {
    const bool live = row < P.m;
    if constexpr (WHAT == kGram) {
        constexpr float s = kScaleA / (kScaleX * kScaleX);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= s;
    } else if constexpr (WHAT == kPoly) {
        float t[32];
        unpack_halves(term.hi, t);
        const float c = P.c / kScaleA, diagonal = P.shift * kScaleA;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            v[k] = fmaf(c, v[k], P.b * t[k]);
            if (row == col + k) v[k] += diagonal;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= 1.f / kScaleA;
        float t[32];
        unpack_halves(term.lo, t);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = fmaf(P.a, t[k], v[k]);
        unpack_halves(term.hi, t);
        const float a = P.a - P.shift;
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = fmaf(a, t[k], v[k]);
    }
    if constexpr (kSymmetric<WHAT>) {
        __half* out = P.out_hi + batch * P.out_batch;
        const int block = col / kTileM, row_block = row / kTileM;
        if (live && block <= row_block) store_halves(out + static_cast<int64_t>(row) * P.out_ld + col, v);
        if (live && block < row_block) {  // whole blocks of columns below the diagonal: all within the matrix
#pragma unroll
            for (int k = 0; k < 32; ++k) out[static_cast<int64_t>(col + k) * P.out_ld + row] = __float2half_rn(v[k]);
        }
    } else if constexpr (WHAT == kUpdate) {
        if (live) {
            const int64_t at = batch * P.out_batch + static_cast<int64_t>(row) * P.out_ld + col;
            store_halves(P.out_hi + at, v);
#pragma unroll
            for (int k = 0; k < 32; k += 2) {  // two conversions at once, the same as those stored
                const float2 hi = __half22float2(__floats2half2_rn(v[k], v[k + 1]));
                v[k] -= hi.x;
                v[k + 1] -= hi.y;
            }
            store_halves(P.out_lo + at, v);
        }
    } else if (P.user_sectors) {
        if (P.user_dtype == CB_F32) finish_row<CB_F32>(P, batch, row, col, v);
        else if (P.user_dtype == CB_BF16) finish_row<CB_BF16>(P, batch, row, col, v);
        else finish_row<CB_F16>(P, batch, row, col, v);
    } else {
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            const bool wide = P.user_vector == 8;
            if (P.user_dtype == CB_F32) finish_result<CB_F32, 4>(P, batch, row, col + h, v + h, stage, lane);
            else if (P.user_dtype == CB_BF16 && wide) finish_result<CB_BF16, 8>(P, batch, row, col + h, v + h, stage, lane);
            else if (P.user_dtype == CB_BF16) finish_result<CB_BF16, 4>(P, batch, row, col + h, v + h, stage, lane);
            else if (wide) finish_result<CB_F16, 8>(P, batch, row, col + h, v + h, stage, lane);
            else finish_result<CB_F16, 4>(P, batch, row, col + h, v + h, stage, lane);
        }
    }
}

// Brings the caller's weights at a warp's columns of a tile into L2 while the tile before it
// is finished. Only transposed ones, of which a warp reads 16 short rows at a time: a step of
// 4 x 4096 x 1024 in bf16 392 us without and 383 with; others are no faster for it.
__device__ __forceinline__ void fetch_weights(const ProductArgs& P, int batch, int row0, int col0, int width, int warp,
                                              int lane) {
    if (row0 >= P.m) return;
    const char* user = static_cast<const char*>(P.user) + (batch * P.user_batch + row0) * dtype_bytes(P.user_dtype);
    for (int c = col0 + warp / 4 * 32 + lane; c < min(col0 + width, P.n); c += 64)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(user + c * P.user_row * dtype_bytes(P.user_dtype)));
}

// The epilogue of a tile: a warp's rows row0 .. row0 + 31, every other 32 columns. Those that no
// row of C has, or that the other triangle gives, are skipped.
template <Product WHAT>
__device__ __forceinline__ void finish_tile(const ProductArgs& P, int batch, int row0, int col0, int width, uint32_t tmem,
                                            uint32_t ready, uint32_t parity, float* stage, int warp, int lane, bool& ok,
                                            bool write = true, int parts = 1) {
    const int row = row0 + lane;
    auto skip = [&](int c) { return c >= width || col0 + c >= P.n || (kSymmetric<WHAT> && (col0 + c) / kTileM > row0 / kTileM); };
    int c = warp / 4 * 32;
    Term next{};
    if (!skip(c)) load_term<WHAT>(P, batch, row, col0 + c, next);
    ok = __all_sync(kFull, tc::barrier_wait(ready, parity));
    if (!ok) return;
    tc::fence_after();
    for (; !skip(c); c += 64) {
        const Term term = next;
        float v[32];
        const uint32_t at = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16) + c;
        tc::tmem_load32(at, v);
        if constexpr (WHAT == kGram) {
            for (int k = 1; k < parts; ++k) {
                float more[32];
                tc::tmem_load32(at + k * width, more);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += more[i];
            }
        }
        if (!skip(c + 64)) load_term<WHAT>(P, batch, row, col0 + c + 64, next);
        if (write) finish<WHAT>(P, batch, row, col0 + c, v, term, stage, lane);
    }
    tc::fence_before();
    __syncwarp();
}

// A wait of this thread ran out. Products after this one go on with what is there, but the last one finds the
// call's word set and leaves the caller's matrix as it is.
__device__ __forceinline__ void report_timeout(const ProductArgs& P) {
    set_error(P.fault, CB_ERR_TIMEOUT);
    if (P.error) set_error(P.error, CB_ERR_TIMEOUT);
}
template <Product WHAT>
__device__ __forceinline__ bool may_write(const ProductArgs& P) {  // a whole warp
    if constexpr (WHAT != kResult) return true;
    return __all_sync(kFull, __ldcg(P.fault) == 0);
}

// C = A B in tiles of 128 x BN, tile after tile by each block. Operand A is K-major; B is
// K-major for the symmetric products (A's own rows), and X as it lies (MN-major) for B X.
// One warp copies tiles of 64 of K into a ring of stages, one issues the products into
// one of two accumulators in TMEM, eight take the other through the epilogue.
template <int BN, Product WHAT>
__global__ void __launch_bounds__(kProductThreads, 1)
muon_product_kernel(const __grid_constant__ CUtensorMap left, const __grid_constant__ CUtensorMap right,
                    const ProductArgs P) {
    constexpr int S = kStages<BN>;
    constexpr int kSums = kSumColumns<BN, WHAT>;
    constexpr uint32_t kColumns = 2 * kSums;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[S], empty[S], ready[2], drained[2];
    __shared__ uint32_t tmem_at;
    __shared__ __align__(16) float stage[WHAT == kResult ? kEpilogueWarps * kStageFloats : 4];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            tc::barrier_init(tc::smem_addr(ready + s), 1);
            tc::barrier_init(tc::smem_addr(drained + s), kEpilogueWarps);
        }
        tc::barrier_init_fence();
        tc::tma_prefetch(&left);
        tc::tma_prefetch(&right);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), kColumns);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int64_t total = P.tiles * P.batch;
    const int ksteps = (P.k + kTileK - 1) / kTileK;
    const int per = kSums > BN ? (ksteps + P.parts - 1) / P.parts : ksteps;  // of a part
    bool ok = true;

    if (warp >= kEpilogueWarps && warp < kMultiplyWarp) {
        if (tc::elect()) {  // copies
            int s = warp - kEpilogueWarps, first = s;  // stage, and step of K, of the block's next tile
            uint32_t phase = 0;
            for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
                const Tile T = tile_at<kTileM, WHAT>(P, t);
                int k = first;
                for (; k < ksteps; k += kCopyWarps) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                    const uint32_t bar = tc::smem_addr(full + s);
                    uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>;
                    tc::barrier_expect(bar, kStageBytes<BN>);
#pragma unroll
                    for (int x = 0; x < kTileM / 64; ++x, at += kBoxBytes)
                        tc::tma_load(at, &left, bar, k * kTileK, T.i * kTileM + x * 64, T.b);
#pragma unroll
                    for (int x = 0; x < BN / 64; ++x, at += kBoxBytes) {
                        if constexpr (kSymmetric<WHAT>) tc::tma_load(at, &right, bar, k * kTileK, T.j * BN + x * 64, T.b);
                        else tc::tma_load(at, &right, bar, T.j * BN + x * 64, k * kTileK, T.b);
                    }
                    if ((s += kCopyWarps) >= S) s -= S, phase ^= 1;
                }
                first = k - ksteps;
            }
            // Copies in flight land before the block's shared memory goes away: those of
            // stages that were never multiplied, after a wait that ran out.
            if (!ok)
                for (int x = 0; x < S; x += kCopyWarps) {
                    if ((s -= kCopyWarps) < 0) s += S, phase ^= 1;
                    if (!tc::barrier_wait(tc::smem_addr(full + s), phase)) break;
                }
        }
    } else if (warp == kMultiplyWarp) {
        // products
        constexpr uint32_t shape = tc::mma_shape(kTileM, BN, !kSymmetric<WHAT>);
        constexpr uint32_t step_b = kSymmetric<WHAT> ? 32 : 2048;  // of 16 of K
        const uint32_t base = tc::smem_addr(ring);
        const uint64_t first_a = tc::operand_k_major(base);
        const uint64_t first_b = kSymmetric<WHAT> ? tc::operand_k_major(base + kTileM * kTileK * 2)
                                                  : tc::operand_mn_major(base + kTileM * kTileK * 2, kBoxBytes);
        const bool one = tc::elect();
        int s = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool here = false;  // the next stage's copies, polled while this one's products are issued
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            if (!(ok = tc::barrier_wait(tc::smem_addr(drained + acc), acc_phase ^ 1))) break;
            tc::fence_after();
            uint32_t sums = tmem + acc * kSums;
            int within = 0;  // steps done of a part
            for (int k = 0; k < ksteps; ++k) {
                if (!here && !(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                tc::fence_after();
                if (kSums > BN && within == per) within = 0, sums += BN;
                const uint64_t da = tc::advance(first_a, s * kStageBytes<BN>), db = tc::advance(first_b, s * kStageBytes<BN>);
                const uint32_t done = tc::smem_addr(empty + s);
                if (++s == S) s = 0, phase ^= 1;
                here = tc::barrier_test(tc::smem_addr(full + s), phase);
                if (one) {
#pragma unroll
                    for (int x = 0; x < kTileK / 16; ++x)
                        tc::mma_f16<1>(sums, tc::advance(da, x * 32), tc::advance(db, x * step_b), shape, within > 0 || x > 0);
                    tc::mma_commit<1>(done);
                    if (k + 1 == ksteps) tc::mma_commit<1>(tc::smem_addr(ready + acc));
                }
                ++within;
            }
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    } else {  // epilogue
        int acc = 0;
        uint32_t acc_phase = 0;
        const bool write = may_write<WHAT>(P);
        auto fetch = [&](int64_t t) {
            if (WHAT != kResult || !P.weights || !P.transposed || t >= total) return;
            const Tile T = tile_at<kTileM, WHAT>(P, t);
            fetch_weights(P, T.b, T.i * kTileM + warp % 4 * 32, T.j * BN, BN, warp, lane);
        };
        fetch(blockIdx.x);
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            fetch(t + gridDim.x);
            const Tile T = tile_at<kTileM, WHAT>(P, t);
            finish_tile<WHAT>(P, T.b, T.i * kTileM + warp % 4 * 32, T.j * BN, BN, tmem + acc * kSums,
                              tc::smem_addr(ready + acc), acc_phase, stage + (WHAT == kResult ? warp * kStageFloats : 0), warp,
                              lane, ok, write, kSums > BN ? (ksteps + per - 1) / per : 1);
            if (!ok) break;
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(drained + acc));
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    }
    if (!ok) report_timeout(P);  // the copying lane, or a whole warp
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<1>(tmem, kColumns);
}

// The same in tiles of 256 x P.width by pairs of blocks on two SMs: each block copies and
// keeps 128 rows of A and half of the columns of B, one lane of the first block issues the
// products of both, and each block has 128 rows of the sums in its TMEM. At the tensor cores' rate
// a 128 x 128 tile wants 128 bytes of copies a clock into its SM, which takes 100 (330 clocks for a
// step of 64 of K instead of 256); a pair's 256 x 256 tile wants 64 (522 instead of 512). P.width is
// a multiple of 32 (a block's half of the columns, of 16; 128 are copied) so that a few rounds
// of tiles can be made to fill the GPU. Operands that are K-major come in boxes of 128 rows,
// fewer copies than of 64. X of 4096 x 4096: 93 us, 70 % of the tensor pipe's cycles (81 and 82 % without lo).
constexpr int kPairM = 256, kPairWidth = 256, kPairStages = 6;
constexpr uint32_t kPairStageBytes = (128 + kPairWidth / 2) * kTileK * 2;

template <Product WHAT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
muon_pair_kernel(const __grid_constant__ CUtensorMap left, const __grid_constant__ CUtensorMap right,
                 const ProductArgs P) {
    constexpr int S = kPairStages;
    constexpr uint32_t kColumns = 2 * kPairWidth;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    // full, drained: those of the first block count for both; empty, ready: each block's own.
    __shared__ uint64_t full[S], empty[S], ready[2], drained[2];
    __shared__ uint32_t tmem_at;
    __shared__ __align__(16) float stage[WHAT == kResult ? kEpilogueWarps * kStageFloats : 4];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = static_cast<int>(tc::cluster_rank());
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            tc::barrier_init(tc::smem_addr(ready + s), 1);
            tc::barrier_init(tc::smem_addr(drained + s), 2 * kEpilogueWarps);
        }
        tc::barrier_init_fence();
        tc::tma_prefetch(&left);
        tc::tma_prefetch(&right);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<2>(tc::smem_addr(&tmem_at), kColumns);
    tc::fence_before();
    tc::cluster_sync();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int64_t total = P.tiles * P.batch;
    const int64_t first = blockIdx.x / 2, step = gridDim.x / 2;
    const int ksteps = (P.k + kTileK - 1) / kTileK, half = P.width / 2;
    bool ok = true;

    if (warp >= kEpilogueWarps && warp < kMultiplyWarp) {
        if (tc::elect()) {  // copies
            int s = warp - kEpilogueWarps, k0 = s;  // stage, and step of K, of the pair's next tile
            uint32_t phase = 0;
            for (int64_t t = first; t < total && ok; t += step) {
                const Tile T = tile_at<kPairM, WHAT>(P, t);
                const int row = T.i * kPairM + rank * 128, col = T.j * P.width + rank * half;
                int k = k0;
                for (; k < ksteps; k += kCopyWarps) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                    const uint32_t bar = tc::in_first_block(tc::smem_addr(full + s));
                    uint32_t at = tc::smem_addr(ring) + s * kPairStageBytes;
                    if (rank == 0) tc::barrier_expect(tc::smem_addr(full + s), 2 * kPairStageBytes);
                    tc::tma_load_pair(at, &left, bar, k * kTileK, row, T.b);
                    at += 2 * kBoxBytes;
                    if constexpr (kSymmetric<WHAT>) {
                        tc::tma_load_pair(at, &right, bar, k * kTileK, col, T.b);
                    } else {
                        tc::tma_load_pair(at, &right, bar, col, k * kTileK, T.b);
                        tc::tma_load_pair(at + kBoxBytes, &right, bar, col + 64, k * kTileK, T.b);
                    }
                    if ((s += kCopyWarps) >= S) s -= S, phase ^= 1;
                }
                k0 = k - ksteps;
            }
            if (!ok && rank == 0)  // copies in flight land before the blocks' shared memory goes away
                for (int x = 0; x < S; x += kCopyWarps) {
                    if ((s -= kCopyWarps) < 0) s += S, phase ^= 1;
                    if (!tc::barrier_wait(tc::smem_addr(full + s), phase)) break;
                }
        }
    } else if (warp == kMultiplyWarp) {
        if (rank == 0) {  // products of both blocks
            const uint32_t shape = tc::mma_shape(kPairM, P.width, !kSymmetric<WHAT>);
            constexpr uint32_t step_b = kSymmetric<WHAT> ? 32 : 2048;  // of 16 of K
            const uint32_t base = tc::smem_addr(ring);
            const uint64_t first_a = tc::operand_k_major(base);
            const uint64_t first_b = kSymmetric<WHAT> ? tc::operand_k_major(base + 2 * kBoxBytes)
                                                      : tc::operand_mn_major(base + 2 * kBoxBytes, kBoxBytes);
            const bool one = tc::elect();
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool here = false;  // the next stage's copies, polled while this one's products are issued
            for (int64_t t = first; t < total && ok; t += step) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(drained + acc), acc_phase ^ 1))) break;
                tc::fence_after();
                for (int k = 0; k < ksteps; ++k) {
                    if (!here && !(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                    tc::fence_after();
                    const uint64_t da = tc::advance(first_a, s * kPairStageBytes), db = tc::advance(first_b, s * kPairStageBytes);
                    const uint32_t done = tc::smem_addr(empty + s);
                    if (++s == S) s = 0, phase ^= 1;
                    here = tc::barrier_test(tc::smem_addr(full + s), phase);
                    if (one) {
#pragma unroll
                        for (int x = 0; x < kTileK / 16; ++x)
                            tc::mma_f16<2>(tmem + acc * kPairWidth, tc::advance(da, x * 32), tc::advance(db, x * step_b), shape,
                                           k > 0 || x > 0);
                        tc::mma_commit<2>(done);
                        if (k + 1 == ksteps) tc::mma_commit<2>(tc::smem_addr(ready + acc));
                    }
                }
                if (++acc == 2) acc = 0, acc_phase ^= 1;
            }
        }
    } else {  // epilogue
        int acc = 0;
        uint32_t acc_phase = 0;
        const bool write = may_write<WHAT>(P);
        auto fetch = [&](int64_t t) {
            if (WHAT != kResult || !P.weights || !P.transposed || t >= total) return;
            const Tile T = tile_at<kPairM, WHAT>(P, t);
            fetch_weights(P, T.b, T.i * kPairM + rank * 128 + warp % 4 * 32, T.j * P.width, P.width, warp, lane);
        };
        fetch(first);
        for (int64_t t = first; t < total && ok; t += step) {
            fetch(t + step);
            const Tile T = tile_at<kPairM, WHAT>(P, t);
            finish_tile<WHAT>(P, T.b, T.i * kPairM + rank * 128 + warp % 4 * 32, T.j * P.width, P.width,
                              tmem + acc * kPairWidth, tc::smem_addr(ready + acc), acc_phase,
                              stage + (WHAT == kResult ? warp * kStageFloats : 0), warp, lane, ok, write);
            if (!ok) break;
            if (lane == 0) tc::barrier_arrive_cluster(tc::in_first_block(tc::smem_addr(drained + acc)));
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    }
    if (!ok) report_timeout(P);  // the copying lane, or a whole warp
    __syncwarp();
    tc::fence_before();
    tc::cluster_sync();  // neither block ends while the other may signal its barriers
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<2>(tmem, kColumns);
}

// A = X X^T of few tiles and a long K: a cluster of P.parts blocks takes a tile of 128 x 64, a
// part of K each, and every block adds up a share of the tile's rows over all of them, in
// order, from their shared memory.

__global__ void __launch_bounds__(kProductThreads, 1)
muon_split_kernel(const __grid_constant__ CUtensorMap rows, const ProductArgs P) {
    constexpr int BN = 64, S = kStages<BN>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    float* sums = reinterpret_cast<float*>(ring);  // [128][64], once the products are done
    __shared__ uint64_t full[S], empty[S], ready;
    __shared__ uint32_t tmem_at;
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        tc::barrier_init(tc::smem_addr(&ready), 1);
        tc::barrier_init_fence();
        tc::tma_prefetch(&rows);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), BN);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int rank = static_cast<int>(tc::cluster_rank());
    const Tile T = tile_at<kTileM, kGram>(P, blockIdx.x / P.parts);
    const int all = (P.k + kTileK - 1) / kTileK, per = (all + P.parts - 1) / P.parts;
    const int first = rank * per, count = max(0, min(per, all - first));
    bool ok = true;

    if (warp >= kEpilogueWarps && warp < kMultiplyWarp) {
        if (tc::elect()) {  // copies
            int k = warp - kEpilogueWarps;
            for (; k < count; k += kCopyWarps) {
                const int s = k % S;
                if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), (k / S & 1) ^ 1))) break;
                const uint32_t bar = tc::smem_addr(full + s);
                const uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>;
                const int x = (first + k) * kTileK;
                tc::barrier_expect(bar, kStageBytes<BN>);
                tc::tma_load(at, &rows, bar, x, T.i * kTileM, T.b);
                tc::tma_load(at + kBoxBytes, &rows, bar, x, T.i * kTileM + 64, T.b);
                tc::tma_load(at + 2 * kBoxBytes, &rows, bar, x, T.j * BN, T.b);
            }
            if (!ok)  // copies in flight land before the block's shared memory goes away
                for (int x = k - S; x < k; x += kCopyWarps)
                    if (x >= 0 && !tc::barrier_wait(tc::smem_addr(full + x % S), x / S & 1)) break;
        }
    } else if (warp == kMultiplyWarp) {
        // products
        constexpr uint32_t shape = tc::mma_shape(kTileM, BN, false);
        const uint64_t first_a = tc::operand_k_major(tc::smem_addr(ring)), first_b = tc::advance(first_a, 2 * kBoxBytes);
        const bool one = tc::elect();
        for (int k = 0; k < count && ok; ++k) {
            const int s = k % S;
            if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), k / S & 1))) break;
            tc::fence_after();
            const uint64_t da = tc::advance(first_a, s * kStageBytes<BN>), db = tc::advance(first_b, s * kStageBytes<BN>);
            if (one) {
#pragma unroll
                for (int x = 0; x < kTileK / 16; ++x)
                    tc::mma_f16<1>(tmem, tc::advance(da, x * 32), tc::advance(db, x * 32), shape, k > 0 || x > 0);
                tc::mma_commit<1>(tc::smem_addr(empty + s));
                if (k + 1 == count) tc::mma_commit<1>(tc::smem_addr(&ready));
            }
        }
    } else {
        const int row = warp % 4 * 32 + lane, c = warp / 4 * 32;
        float v[32] = {};
        if (count > 0) {
            ok = __all_sync(kFull, tc::barrier_wait(tc::smem_addr(&ready), 0));
            tc::fence_after();
            tc::tmem_load32(tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16) + c, v);
        }
        // After a wait that ran out copies may still be on their way into the ring: the sums
        // then stay unwritten (the result is reported as incomplete).
        if (ok) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)  // 16-byte pieces of a row, swizzled over the banks
                *reinterpret_cast<float4*>(sums + row * BN + (((c + k) / 4 ^ (row & 15)) << 2)) =
                    make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        }
    }
    if (!ok) report_timeout(P);  // the copying lane, or a whole warp
    __syncwarp();
    tc::fence_before();
    tc::cluster_sync();
    if (warp < kEpilogueWarps) {
        const int share = kTileM / P.parts, columns = BN / 4;
        constexpr float scale = kScaleA / (kScaleX * kScaleX);
        __half* out = P.out_hi + T.b * P.out_batch;
        for (int i = threadIdx.x; i < share * columns; i += kEpilogueWarps * 32) {
            const int r = rank * share + i % share, c4 = i / share;  // lanes along the rows
            const uint32_t at = tc::smem_addr(sums + r * BN + ((c4 ^ (r & 15)) << 2));
            float4 part[kPartsMost];
#pragma unroll
            for (int k = 0; k < kPartsMost; ++k)
                part[k] = k < P.parts ? tc::load_cluster(tc::in_block(at, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            float4 t = part[0];
#pragma unroll
            for (int k = 1; k < kPartsMost; ++k) {
                t.x += part[k].x;
                t.y += part[k].y;
                t.z += part[k].z;
                t.w += part[k].w;
            }
            const int row = T.i * kTileM + r, col = T.j * BN + c4 * 4, block = col / kTileM;
            if (row >= P.m || col >= P.n || block > T.i) continue;
            const __half2 h0 = __floats2half2_rn(t.x * scale, t.y * scale), h1 = __floats2half2_rn(t.z * scale, t.w * scale);
            uint2 w;
            memcpy(&w.x, &h0, 4);
            memcpy(&w.y, &h1, 4);
            *reinterpret_cast<uint2*>(out + static_cast<int64_t>(row) * P.out_ld + col) = w;  // rows are padded to 64
            if (block < T.i) {
                const __half h[4] = {__low2half(h0), __high2half(h0), __low2half(h1), __high2half(h1)};
#pragma unroll
                for (int e = 0; e < 4; ++e) out[static_cast<int64_t>(col + e) * P.out_ld + row] = h[e];
            }
        }
    }
    tc::cluster_sync();  // no block ends while others read its sums
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<1>(tmem, BN);
}

// ---------------------------------------------------------------- launches

template <Product WHAT>
int64_t tiles_of(int32_t m, int32_t n, int height, int width) {
    const int row_tiles = (m + height - 1) / height, col_tiles = (n + width - 1) / width;
    if (!kSymmetric<WHAT>) return static_cast<int64_t>(row_tiles) * col_tiles;
    int64_t t = 0;
    for (int i = 0; i < row_tiles; ++i) t += lower_tiles(i, height, width, col_tiles);
    return t;
}
template <Product WHAT>
void set_tiles(ProductArgs& P, int height, int width) {
    P.row_tiles = (P.m + height - 1) / height;
    P.col_tiles = (P.n + width - 1) / width;
    P.width = width;
    P.tiles = tiles_of<WHAT>(P.m, P.n, height, width);
}

bool launch_split(const CUtensorMap& rows, ProductArgs P, cudaStream_t s) {
    set_tiles<kGram>(P, kTileM, 64);
    constexpr size_t smem = kStages<64> * kStageBytes<64> + 1024;
    static std::atomic<uint64_t> devices{0};
    return shared_memory(muon_split_kernel, smem, devices) &&
           launch_clusters(muon_split_kernel, P.parts, P.tiles * P.batch * P.parts, kProductThreads, smem, s, rows, P);
}

template <int BN, Product WHAT>
bool launch_tiles(const CUtensorMap& left, const CUtensorMap& right, ProductArgs P, int sms, cudaStream_t s) {
    set_tiles<WHAT>(P, kTileM, BN);
    constexpr size_t smem = kStages<BN> * kStageBytes<BN> + 1024;
    static std::atomic<uint64_t> devices{0};
    if (!shared_memory(muon_product_kernel<BN, WHAT>, smem, devices)) return false;
    launch(muon_product_kernel<BN, WHAT>, dim3(static_cast<unsigned>(min64(P.tiles * P.batch, sms))),
           dim3(kProductThreads), smem, s, left, right, P);
    return true;
}
template <Product WHAT>
bool launch_pairs(const CUtensorMap& left, const CUtensorMap& right, ProductArgs P, int width, int sms, cudaStream_t s) {
    set_tiles<WHAT>(P, kPairM, width);
    constexpr size_t smem = kPairStages * kPairStageBytes + 1024;
    static std::atomic<uint64_t> devices{0};
    if (!shared_memory(muon_pair_kernel<WHAT>, smem, devices)) return false;
    launch(muon_pair_kernel<WHAT>, dim3(static_cast<unsigned>(2 * min64(P.tiles * P.batch, sms / 2))),
           dim3(kProductThreads), smem, s, left, right, P);
    return true;
}

// The tiles with the least time, in clocks: rounds of tiles over the GPU, each the steps of 64
// of K that it takes, and what a kernel takes besides (launch, first copies, last epilogue).
// Fitted to all three products at 16 sizes of 200 to 4096, each with tiles of one kind forced: a
// step is 320 clocks at 128 x 64 and 330 at 128 x 128 (the tensor cores need 192 and 256), and
// two a column by pairs, which is what the tensor cores need. The choice was within 1.5 us of
// the best kind for each of the products in nearly all. What another would cost, in five steps: 1024 x 1024
// 110 us (64 wide; 128 in any one product 4 to 8 more, pairs of 256 17 to 25), 4 x 1024 x 1024 162 (128,
// the update by pairs of 256; 64 in any one 6 to 20 more), 2048 x 2048 222 (the same; 64 18 to 55 more).
template <Product WHAT>
bool launch_best(const Operand& left, const Operand& right, const ProductArgs& P, int sms, cudaStream_t s) {
    const int64_t ksteps = (P.k + kTileK - 1) / kTileK;
    auto time = [&](int height, int width, int at_once, int64_t step, int64_t fixed) {
        return (tiles_of<WHAT>(P.m, P.n, height, width) * P.batch + at_once - 1) / at_once * ksteps * step + fixed;
    };
    int64_t best = time(kTileM, 64, sms, 320, 6500);
    if constexpr (WHAT == kGram) {
        if (P.parts > 1) {
            const int64_t blocks = tiles_of<kGram>(P.m, P.n, kTileM, 64) * P.batch * P.parts;
            const int64_t split = (blocks + sms - 1) / sms * ((ksteps + P.parts - 1) / P.parts * 320 + 10500);
            return split < best ? launch_split(left.box64, P, s)
                                : launch_tiles<64, WHAT>(left.box64, right.box64, P, sms, s);
        }
    }
    int width = 64;
    const int64_t t128 = time(kTileM, 128, sms, 330, 8000);
    if (t128 < best) best = t128, width = 128;
    bool pair = false;
    for (int w = 160; w <= kPairWidth; w += 32) {
        const int64_t t = time(kPairM, w, sms / 2, 2 * w + 10, 6200 + 20 * w);
        if (t < best) best = t, width = w, pair = true;
    }
    if (pair) return launch_pairs<WHAT>(left.box128, kSymmetric<WHAT> ? right.box128 : right.box64, P, width, sms, s);
    if (width == 128) return launch_tiles<128, WHAT>(left.box64, right.box64, P, sms, s);
    return launch_tiles<64, WHAT>(left.box64, right.box64, P, sms, s);
}

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
                cudaSuccess || q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    return encode;
}

// [batch][rows][cols] of fp16 with rows of `ld` values, in boxes of 64 values of box_rows rows;
// values past a row or past the rows read as zeros.
bool tensor_map(CUtensorMap* map, const void* data, int64_t cols, int64_t rows, int64_t batch, int64_t ld,
                uint32_t box_rows) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                                static_cast<cuuint64_t>(batch)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * rows * 2};
    const cuuint32_t box[3] = {64, box_rows, 1};
    const cuuint32_t step[3] = {1, 1, 1};
    return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(data), dims, strides, box,
                                step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool tensor_maps_work() { return tensor_map_encoder() != nullptr; }

bool Operand::set(const void* data, int64_t cols, int64_t rows, int64_t batch, int64_t ld) {
    return tensor_map(&box64, data, cols, rows, batch, ld, 64) && tensor_map(&box128, data, cols, rows, batch, ld, 128);
}

bool launch_product(Product what, const Operand& left, const Operand& right, const ProductArgs& P, int sms,
                    cudaStream_t s) {
    switch (what) {
        case kGram: return launch_best<kGram>(left, right, P, sms, s);
        case kPoly: return launch_best<kPoly>(left, right, P, sms, s);
        case kUpdate: return launch_best<kUpdate>(left, right, P, sms, s);
        default: return launch_best<kResult>(left, right, P, sms, s);
    }
}

}  // namespace muon
}  // namespace cbtbe
