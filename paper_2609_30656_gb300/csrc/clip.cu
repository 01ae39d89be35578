// clip.cu -- the 2-norm over all gradients of a model, and clipping to it (include/cb_tbe.h).
//
//   norm = sqrt(sum over all tensors of x^2),  f = min(1, max_norm / (norm + eps)),  x <- f x
//
// The factor is known only after every value has been read, so clipping reads twice and writes once, and
// where nothing is clipped in place the second pass ends at once. The copy rate bounds both. The tensors
// come as a table in the kernels' parameters (no copy to the device, so a call can be captured);
// all of them are one sequence of chunks that the blocks take in turn. The second pass goes through
// the chunks backwards: what the first read last is still in L2. 217 tensors of 384 M values, 1.04 GB: 150 us for the norm
// (6.9 TB/s) and 337 for the products (6.0 TB/s), 501 a call.
//
// Squares are summed in fp32 by thread over a chunk's values, those sums with what their additions round
// off, by magnitude (SquareSum), and the blocks' sums in fp64 in one order: the same bits every time, no
// overflow or underflow that the norm itself does not have.
#include "muon_internal.cuh"
#include "token_rows.cuh"

#include <algorithm>
#include <exception>
#include <utility>
#include <vector>

namespace cbtbe {
namespace clip {
namespace {

constexpr int kThreads = 256;
template <int DT> constexpr int kPieces = DT == CB_F32 ? 4 : 8;       // of 8 values a thread has in flight: 128 bytes
template <int DT> constexpr int kChunk = kThreads * kPieces<DT> * 8;  // values: 32 KB
__host__ __device__ constexpr int chunk_values(int dtype) { return dtype == CB_F32 ? kChunk<CB_F32> : kChunk<CB_BF16>; }
// Resident, of both passes: a second round of blocks would leave most SMs idle.
constexpr int kBlocksAnSm = 4;
constexpr int64_t kMostValues = int64_t{1} << 40;       // of a tensor
constexpr int64_t kMostTensors = 1 << 20;

// One tensor: rows of `cols` values. One with dense values is one row.
struct Entry {
    const void* in;
    void* out;               // where the clipped values go; may be in
    const int64_t* count;    // how many of the values there are, on the device; or null: all
    int64_t n, cols;         // values; of a row
    int64_t in_row, out_row;
    int64_t chunk;           // the first of its chunks
    int32_t in_dtype, out_dtype;
};
template <int N>
struct Table {
    Entry e[N];
    int32_t tensors;
    int64_t chunks;
};
// Tables of two sizes: the parameters of a launch are copied whole (24 small tensors 41 us a call, 25 tensors 44).
constexpr int kSmallTable = 24, kLargeTable = 400;
static_assert(sizeof(Table<kLargeTable>) < 32000, "kernel parameters are limited to 32764 bytes");

template <int N>
__device__ __forceinline__ int find_entry(const Table<N>& T, int64_t chunk) {
    int lo = 0, hi = T.tensors - 1;  // the last entry whose first chunk is not above it
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (T.e[mid].chunk <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Pieces of 8 values begin where the tensor has a multiple of 8 values' bytes (16 or 32) behind it in
// memory: `lead` values come before the first of them, value by value, as do those behind the last whole piece. A
// thread has pieces kStep values apart.
constexpr int kStep = kThreads * 8;
__device__ __forceinline__ int lead_of(const void* p, int dtype) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return dtype == CB_F32 ? static_cast<int>((32 - a % 32) % 32 / 4) : static_cast<int>((16 - a % 16) % 16 / 2);
}
__device__ __forceinline__ int64_t count_of(const Entry& e) {
    if (!e.count) return e.n;
    const int64_t c = *e.count;
    return c < 0 ? 0 : (c < e.n ? c : e.n);
}
// Whole pieces of a thread with `left` values from its first one on.
template <int DT>
__device__ __forceinline__ int whole_pieces(int64_t left) {
    return left < 8 ? 0 : static_cast<int>(min64(kPieces<DT>, (left - 8) / kStep + 1));
}
__device__ __forceinline__ int64_t place(int64_t i, int64_t cols, int64_t row, bool dense) {
    if (dense) return i;
    const int64_t r = i / cols;
    return r * row + (i - r * cols);
}

template <int DT>
__device__ __forceinline__ void piece_squares(const Piece<DT, 8>& x, muon::SquareSum& s) {
    float f[8], sum = 0.f;
    widen<DT, 8>(x, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
    // In this range neither an overflow nor squares below fp32's normal numbers matter. Else (zeros, an
    // infinity or a NaN too) by magnitude.
    if (sum >= 0x1p-110f && sum < 0x1p83f) {
        s.add_mid(sum);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (f[i] != 0.f) s.add(f[i]);
    }
}
template <int DT>
__device__ __forceinline__ void chunk_squares(const Entry& e, int64_t chunk, muon::SquareSum& s) {
    const int64_t n = count_of(e), first = (chunk - e.chunk) * kChunk<DT>;
    const bool dense = e.cols >= e.n;
    const char* in = static_cast<const char*>(e.in);
    constexpr int kSize = DT == CB_F32 ? 4 : 2;
    const int lead = lead_of(in, DT);
    if (!dense) {
        for (int64_t i = first + threadIdx.x; i < first + kChunk<DT> && i < n; i += kThreads)
            s.add(muon::load_value(in, place(i, e.cols, e.in_row, false), DT));
        return;
    }
    if (first == 0 && static_cast<int>(threadIdx.x) < lead && static_cast<int64_t>(threadIdx.x) < n)
        s.add(muon::load_value(in, threadIdx.x, DT));
    const int64_t at = first + lead + threadIdx.x * 8;
    const int pieces = whole_pieces<DT>(n - at);
    const char* mine = in + at * kSize;
    if (pieces == kPieces<DT>) {  // all on their way at once
        Piece<DT, 8> x[kPieces<DT>];
#pragma unroll
        for (int p = 0; p < kPieces<DT>; ++p) x[p] = load_piece<DT, 8, false>(mine + p * kStep * kSize);
#pragma unroll
        for (int p = 0; p < kPieces<DT>; ++p) piece_squares<DT>(x[p], s);
    } else {
#pragma unroll 1
        for (int p = 0; p < pieces; ++p) piece_squares<DT>(load_piece<DT, 8, false>(mine + p * kStep * kSize), s);
    }
    // The values behind the last whole piece, in the tensor's last chunk.
    const int64_t end = min64(first + lead + kChunk<DT>, n);
    const int64_t rest = end - (end - lead) % 8 + threadIdx.x;
    if (end == n && threadIdx.x < 8 && rest < n && rest >= first + lead) s.add(muon::load_value(in, rest, DT));
}

// First pass: a block's sums of its chunks.
template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksAnSm)
clip_norm_kernel(const __grid_constant__ Table<N> T, float4* partial) {
    __shared__ float4 joined[kThreads / 32];
    begin_kernel();
    muon::SquareSum s;
    for (int64_t c = blockIdx.x; c < T.chunks; c += gridDim.x) {
        const Entry& e = T.e[find_entry(T, c)];
        if (e.in_dtype == CB_F32) chunk_squares<CB_F32>(e, c, s);
        else if (e.in_dtype == CB_BF16) chunk_squares<CB_BF16>(e, c, s);
        else chunk_squares<CB_F16>(e, c, s);
    }
    s.add_lanes();
    if ((threadIdx.x & 31) == 0) joined[threadIdx.x / 32] = make_float4(s.mid, s.rest, s.big, s.small);
    __syncthreads();
    if (threadIdx.x) return;
    muon::SquareSum t;
    for (int w = 0; w < kThreads / 32; ++w) {
        muon::SquareSum o;
        o.mid = joined[w].x;
        o.rest = joined[w].y;
        o.big = joined[w].z;
        o.small = joined[w].w;
        t.add(o);
    }
    partial[blockIdx.x] = make_float4(t.mid, t.rest, t.big, t.small);
}

// The norm from the blocks' sums, by a whole block; every block that asks gets the same bits.
__device__ double total_norm(const float4* partial, int parts) {
    __shared__ double joined[kThreads / 32];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) {
        const float4 p = __ldcg(partial + i);
        sum += static_cast<double>(p.x) + static_cast<double>(p.y) + static_cast<double>(p.z) * 0x1p160 +
               static_cast<double>(p.w) * 0x1p-160;
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(kFull, sum, off);
    if ((threadIdx.x & 31) == 0) joined[threadIdx.x / 32] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kThreads / 32; ++w) sum += joined[w];
    return sqrt(sum);
}

__global__ void __launch_bounds__(kThreads)
clip_finish_kernel(const float4* partial, int parts, float* norm) {
    begin_kernel();
    const double n = total_norm(partial, parts);
    if (threadIdx.x == 0) *norm = static_cast<float>(n);
}

template <int DT>
__device__ __forceinline__ void store_scaled(const Piece<DT, 8>& x, float f, char* to, int dtype) {
    float v[8];
    widen<DT, 8>(x, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f;
    if (dtype == CB_F32) store_piece<CB_F32, 8>(to, v);
    else if (dtype == CB_BF16) store_piece<CB_BF16, 8>(to, v);
    else store_piece<CB_F16, 8>(to, v);
}
template <int DT>
__device__ __forceinline__ void chunk_scaled(const Entry& e, int64_t chunk, float f) {
    const int64_t n = count_of(e), first = (chunk - e.chunk) * kChunk<DT>;
    const char* in = static_cast<const char*>(e.in);
    char* out = static_cast<char*>(e.out);
    const int to = e.out_dtype;
    constexpr int kIn = DT == CB_F32 ? 4 : 2;
    const int lead = lead_of(in, DT);
    const bool dense = e.cols >= e.n;
    if (!dense || lead != lead_of(out, to)) {
        for (int64_t i = first + threadIdx.x; i < first + kChunk<DT> && i < n; i += kThreads)
            muon::store_value(out, place(i, e.cols, e.out_row, dense),
                              muon::load_value(in, place(i, e.cols, e.in_row, dense), DT) * f, to);
        return;
    }
    if (first == 0 && static_cast<int>(threadIdx.x) < lead && static_cast<int64_t>(threadIdx.x) < n)
        muon::store_value(out, threadIdx.x, muon::load_value(in, threadIdx.x, DT) * f, to);
    const int64_t at = first + lead + threadIdx.x * 8;
    const int pieces = whole_pieces<DT>(n - at);
    const char* mine = in + at * kIn;
    const int size = to == CB_F32 ? 4 : 2;
    char* target = out + at * size;
    if (pieces == kPieces<DT>) {  // all on their way at once
        Piece<DT, 8> x[kPieces<DT>];
#pragma unroll
        for (int p = 0; p < kPieces<DT>; ++p) x[p] = load_piece<DT, 8, false>(mine + p * kStep * kIn);
#pragma unroll
        for (int p = 0; p < kPieces<DT>; ++p) store_scaled<DT>(x[p], f, target + p * kStep * size, to);
    } else {
#pragma unroll 1
        for (int p = 0; p < pieces; ++p)
            store_scaled<DT>(load_piece<DT, 8, false>(mine + p * kStep * kIn), f, target + p * kStep * size, to);
    }
    // The values behind the last whole piece, in the tensor's last chunk.
    const int64_t end = min64(first + lead + kChunk<DT>, n);
    const int64_t rest = end - (end - lead) % 8 + threadIdx.x;
    if (end == n && threadIdx.x < 8 && rest < n && rest >= first + lead)
        muon::store_value(out, rest, muon::load_value(in, rest, DT) * f, to);
}

// Second pass: the norm, the factor, and the values times it.
template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksAnSm)
clip_scale_kernel(const __grid_constant__ Table<N> T, const float4* partial, int parts, float max_norm, float eps,
                  float* norm) {
    begin_kernel();
    const double n = total_norm(partial, parts);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(n);
    const double over = n + static_cast<double>(eps);
    const double ratio = over == 0.0 ? 1.0 : static_cast<double>(max_norm) / over;  // all zeros stay that
    const float f = ratio >= 1.0 ? 1.f : static_cast<float>(ratio);  // a NaN stays one
    for (int64_t k = blockIdx.x; k < T.chunks; k += gridDim.x) {
        const int64_t c = T.chunks - 1 - k;
        const Entry& e = T.e[find_entry(T, c)];
        if (f == 1.f && e.in == e.out) continue;
        if (e.in_dtype == CB_F32) chunk_scaled<CB_F32>(e, c, f);
        else if (e.in_dtype == CB_BF16) chunk_scaled<CB_BF16>(e, c, f);
        else chunk_scaled<CB_F16>(e, c, f);
    }
}

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 152;
    return sms;
}
int grid_blocks(int64_t chunks) {
    return static_cast<int>(std::min<int64_t>(chunks, static_cast<int64_t>(sm_count()) * kBlocksAnSm));
}

bool type_ok(int t) { return t == CB_F32 || t == CB_F16 || t == CB_BF16; }
int size_of(int t) { return t == CB_F32 ? 4 : 2; }

// Memory that a call reads or writes.
struct Range {
    uintptr_t begin, end;
    int64_t row, width;  // bytes from a row to the next, of a row; row = 0: one row
    int64_t tensor;
    bool written;
};
bool share(const Range& a, const Range& b) {  // their bounds do
    if (a.row == 0 && b.row == 0) return true;
    const int64_t row = a.row ? a.row : b.row;
    if ((a.row && b.row && a.row != b.row) || a.width > row || b.width > row) return true;
    // Columns of one matrix: apart if their places within a row are.
    const int64_t off = static_cast<int64_t>((b.begin - a.begin) % static_cast<uintptr_t>(row));
    return off < a.width || off + b.width > row;
}
// No value that is written is in a second tensor, or read in another place than its own.
bool apart(std::vector<Range>& r) {
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = i + 1; j < r.size() && r[j].begin < r[i].end; ++j)
            if ((r[i].written || r[j].written) && share(r[i], r[j])) return false;
    return true;
}

// `ranges`: what else a call writes.
cb_status check(const cb_grad_tensor* t, int64_t tensors, bool scale, std::vector<Entry>& entries, std::vector<Range> ranges) {
    if (tensors < 0 || (tensors > 0 && !t)) return CB_ERR_INVALID_ARG;
    entries.reserve(static_cast<size_t>(tensors));
    for (int64_t i = 0; i < tensors; ++i) {
        const cb_grad_tensor& g = t[i];
        if (!type_ok(g.dtype) || g.rows < 0 || g.cols < 0 || g.rows > kMostValues || g.cols > kMostValues)
            return CB_ERR_INVALID_ARG;
        if (g.rows > 0 && g.cols > kMostValues / g.rows) return CB_ERR_INVALID_ARG;
        if (g.rows > 1 && (g.row_stride < g.cols || g.row_stride > kMostValues / g.rows)) return CB_ERR_INVALID_ARG;
        if (scale && (!type_ok(g.out_dtype) ||
                      (g.rows > 1 && (g.out_row_stride < g.cols || g.out_row_stride > kMostValues / g.rows))))
            return CB_ERR_INVALID_ARG;
        if (g.count && (g.rows > 1 || reinterpret_cast<uintptr_t>(g.count) % 8)) return CB_ERR_INVALID_ARG;
        if (g.rows == 0 || g.cols == 0) continue;
        const uintptr_t in = reinterpret_cast<uintptr_t>(g.data), out = reinterpret_cast<uintptr_t>(g.out);
        if (!in || in % size_of(g.dtype) || (scale && (!out || out % size_of(g.out_dtype)))) return CB_ERR_INVALID_ARG;
        Entry e{};
        e.in = g.data;
        e.out = g.out;
        e.count = g.count;
        e.n = g.rows * g.cols;
        const bool dense = g.rows == 1 || (g.row_stride == g.cols && (!scale || g.out_row_stride == g.cols));
        e.cols = dense ? e.n : g.cols;
        e.in_row = g.row_stride;
        e.out_row = g.out_row_stride;
        e.in_dtype = g.dtype;
        e.out_dtype = scale ? g.out_dtype : g.dtype;
        entries.push_back(e);
        if (!scale) continue;
        auto range = [&](uintptr_t p, int64_t row, int size, bool written) {
            const bool one = g.rows == 1 || row == g.cols;
            ranges.push_back({p, p + static_cast<uintptr_t>(one ? e.n : (g.rows - 1) * row + g.cols) * size,
                              one ? 0 : row * size, (one ? e.n : g.cols) * size, i, written});
        };
        const bool in_place = in == out && g.dtype == g.out_dtype && (g.rows == 1 || g.row_stride == g.out_row_stride);
        range(out, g.out_row_stride, size_of(e.out_dtype), true);
        if (g.count) ranges.push_back({reinterpret_cast<uintptr_t>(g.count), reinterpret_cast<uintptr_t>(g.count + 1), 0, 8, i, false});
        if (!in_place) range(in, g.row_stride, size_of(g.dtype), false);
    }
    return apart(ranges) ? CB_OK : CB_ERR_INVALID_ARG;
}

template <int N>
void launch_pass(const Entry* e, int tensors, const float4* partial, int at, int parts, bool scale, float max_norm, float eps,
                 float* norm, int* blocks, cudaStream_t s) {
    Table<N> T;
    T.tensors = tensors;
    T.chunks = 0;
    for (int i = 0; i < tensors; ++i) {
        T.e[i] = e[i];
        T.e[i].chunk = T.chunks;
        T.chunks += (e[i].n + chunk_values(e[i].in_dtype) - 1) / chunk_values(e[i].in_dtype);
    }
    const int grid = grid_blocks(T.chunks);
    if (blocks) *blocks = grid;
    if (scale) launch(clip_scale_kernel<N>, dim3(grid), dim3(kThreads), 0, s, T, partial, parts, max_norm, eps, norm);
    else launch(clip_norm_kernel<N>, dim3(grid), dim3(kThreads), 0, s, T, const_cast<float4*>(partial) + at);
}

cb_status run(const cb_grad_tensor* t, int64_t tensors, bool scale, float max_norm, float eps, float* norm, void* workspace,
              int64_t workspace_bytes, cudaStream_t stream) {
    std::vector<Entry> entries;
    std::vector<Range> also;
    const int64_t need = cb_grad_norm_workspace_bytes(tensors);
    for (const auto& [p, bytes] : {std::pair<const void*, int64_t>{norm, 4}, {workspace, need}})
        if (scale && p && bytes > 0)
            also.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, 0, bytes, -1, true});
    const cb_status status = check(t, tensors, scale, entries, std::move(also));
    if (status != CB_OK) return status;
    if (reinterpret_cast<uintptr_t>(norm) % 4 || (!scale && !norm)) return CB_ERR_INVALID_ARG;
    if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < need)) return CB_ERR_CAPACITY;
    const float4* partial = static_cast<const float4*>(workspace);
    const int total = static_cast<int>(entries.size());
    int parts = 0;
    auto pass = [&](int first, bool second, float* out) {
        const int n = std::min(total - first, kLargeTable);
        int blocks = 0;
        if (n <= kSmallTable)
            launch_pass<kSmallTable>(entries.data() + first, n, partial, parts, parts, second, max_norm, eps, out, &blocks, stream);
        else
            launch_pass<kLargeTable>(entries.data() + first, n, partial, parts, parts, second, max_norm, eps, out, &blocks, stream);
        return blocks;
    };
    for (int first = 0; first < total; first += kLargeTable) parts += pass(first, false, nullptr);
    if (scale && total > 0) {
        for (int first = 0; first < total; first += kLargeTable) pass(first, true, first ? nullptr : norm);
    } else if (norm) {
        launch(clip_finish_kernel, dim3(1), dim3(kThreads), 0, stream, partial, parts, norm);
    }
    return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA;
}

}  // namespace
}  // namespace clip
}  // namespace cbtbe

extern "C" int64_t cb_grad_norm_workspace_bytes(int64_t tensors) {
    using namespace cbtbe::clip;
    if (tensors <= 0 || tensors > kMostTensors) return 0;
    return (tensors + kLargeTable - 1) / kLargeTable * sm_count() * kBlocksAnSm * static_cast<int64_t>(sizeof(float4));
}

extern "C" cb_status cb_grad_norm(const cb_grad_tensor* tensors, int64_t num_tensors, float* norm, void* workspace,
                                  int64_t workspace_bytes, cudaStream_t stream) {
    if (num_tensors > cbtbe::clip::kMostTensors) return CB_ERR_INVALID_ARG;
    try {
        return cbtbe::clip::run(tensors, num_tensors, false, 0.f, 0.f, norm, workspace, workspace_bytes, stream);
    } catch (const std::exception&) {  // no memory for the table
        return CB_ERR_OOM;
    }
}

extern "C" cb_status cb_grad_clip(const cb_grad_tensor* tensors, int64_t num_tensors, float max_norm, float eps, float* norm,
                                  void* workspace, int64_t workspace_bytes, cudaStream_t stream) {
    if (num_tensors > cbtbe::clip::kMostTensors || !(max_norm >= 0.f) || !(eps >= 0.f)) return CB_ERR_INVALID_ARG;
    try {
        return cbtbe::clip::run(tensors, num_tensors, true, max_norm, eps, norm, workspace, workspace_bytes, stream);
    } catch (const std::exception&) {
        return CB_ERR_OOM;
    }
}
