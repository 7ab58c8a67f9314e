// Embedding lookup with scaling, and every node's gradient of the embedding by sorted tokens.
//
// The gradient of row v is scale times the sum of the rows of dY whose token is v, in the order of the rows, so its result
// does not depend on what runs when.  Three steps: the tokens of up to kChunk consecutive rows of a node are sorted, stably, by a
// CTA (least significant digits first, a warp's rank among equal digits by matching lanes); where each tile of kTileRows
// vocabulary rows begins in a chunk is written beside them; then a CTA takes a tile's rows of 256 columns, finds each row's
// occurrences in the chunks and adds them up, one warp a row, or all its warps where there are many.  A token outside the
// vocabulary is sorted behind all others and is nobody's.
// Bound by HBM: the gradient of the whole vocabulary is written for every node.
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kLookupThreads = 256;

template <class T>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const __grid_constant__ Lookup a, int shift, bool wide_e, bool wide_y) {
    chain_begin();
    const int per = 1 << shift;
    const int64_t step = static_cast<int64_t>(gridDim.x) * (kLookupThreads >> shift);
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * (kLookupThreads >> shift) + (threadIdx.x >> shift); i < a.rows; i += step) {
        const int64_t t = a.tokens.at(i);
        const bool in = t >= 0 && t < a.vocab;
        const T* e = static_cast<const T*>(a.E) + (in ? t : 0) * a.lde;
        T* y = static_cast<T*>(a.Y) + i * a.ldy;
        for (int64_t j = (threadIdx.x & (per - 1)) * 8; j < a.d; j += per * 8) {
            const int n = static_cast<int>(min(static_cast<int64_t>(8), a.d - j));
            float v[8];
            load8(e + j, in ? n : 0, wide_e, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = in ? v[q] * a.scale : 0.f;
            store8(y + j, n, wide_y, v);
        }
    }
}

// ---- the tokens in order ---------------------------------------------------------------------------------------
constexpr int kChunk = 4096, kSortThreads = 512, kSortWarps = kSortThreads / 32, kMine = kChunk / kSortThreads;
constexpr int kTileRows = 64;
constexpr int kDigit = 8, kDigits = 1 << kDigit;

// A chunk's sorted tokens, the rows (of its node) that they come from, and where each tile's begin.
struct Sorted {
    int32_t* token; int32_t* row; int32_t* start;
    int64_t chunks, tiles;                           // a node's
    __host__ __device__ int64_t at(int64_t node, int64_t chunk) const { return node * chunks + chunk; }
};
Sorted sorted_of(int64_t nodes, int64_t rows, int64_t vocab, void* workspace) {
    Sorted s{};
    s.chunks = (rows + kChunk - 1) / kChunk;
    s.tiles = (vocab + kTileRows - 1) / kTileRows;
    const int64_t all = nodes * s.chunks;
    s.token = static_cast<int32_t*>(workspace);
    s.row = s.token + all * kChunk;
    s.start = s.row + all * kChunk;
    return s;
}

__global__ void __launch_bounds__(kSortThreads) sort_kernel(Index tokens, int64_t rows, int vocab, int bits, Sorted out) {
    chain_begin();
    extern __shared__ int32_t mem[];
    int32_t* key[2] = {mem, mem + kChunk};
    uint16_t* from[2] = {reinterpret_cast<uint16_t*>(mem + 2 * kChunk), reinterpret_cast<uint16_t*>(mem + 2 * kChunk) + kChunk};
    __shared__ uint16_t count[kSortWarps][kDigits];
    __shared__ int total[kDigits];
    __shared__ int carry[kSortWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t chunk = blockIdx.x, node = blockIdx.y, first = chunk * kChunk;
    const int n = static_cast<int>(min(static_cast<int64_t>(kChunk), rows - first));
    for (int q = threadIdx.x; q < n; q += kSortThreads) {
        const int64_t t = tokens.at(node * rows + first + q);
        key[0][q] = t >= 0 && t < vocab ? static_cast<int32_t>(t) : vocab;
        from[0][q] = static_cast<uint16_t>(q);
    }
    // each warp ranks the keys of its own stretch, 32 at a time
    const int stretch = (n + kSortWarps * 32 - 1) / (kSortWarps * 32);       // of 32 keys; at most kMine
    int b = 0;
    for (int low = 0; low < bits; low += kDigit, b ^= 1) {
        for (int q = threadIdx.x; q < kSortWarps * kDigits; q += kSortThreads) (&count[0][0])[q] = 0;
        __syncthreads();
        int digit[kMine], rank[kMine];
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int q = (warp * stretch + u) * 32 + lane;
            const bool in = u < stretch && q < n;
            digit[u] = in ? (key[b][q] >> low) & (kDigits - 1) : kDigits;
            rank[u] = 0;
            if (u < stretch) {                       // the same for the whole warp
                const uint32_t same = __match_any_sync(0xffffffffu, digit[u]);
                const uint32_t before = same & ((1u << lane) - 1);
                if (in) rank[u] = count[warp][digit[u]] + __popc(before);
                __syncwarp();
                if (in && before == 0) count[warp][digit[u]] += static_cast<uint16_t>(__popc(same));
                __syncwarp();
            }
        }
        __syncthreads();
        // where each (digit, warp) begins: over the warps, then over the digits
        int sum = 0;
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kSortWarps; ++w) { const int c = count[w][threadIdx.x]; count[w][threadIdx.x] = static_cast<uint16_t>(sum); sum += c; }
        int scan = sum;
        for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, scan, o); if (lane >= o) scan += y; }
        if (lane == 31) carry[warp] = scan;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < warp; ++w) before += carry[w];
        if (threadIdx.x < kDigits) total[threadIdx.x] = before + scan - sum;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int q = (warp * stretch + u) * 32 + lane;
            if (u < stretch && q < n) {
                const int to = total[digit[u]] + count[warp][digit[u]] + rank[u];
                key[b ^ 1][to] = key[b][q];
                from[b ^ 1][to] = from[b][q];
            }
        }
        __syncthreads();
    }
    const int64_t at = out.at(node, chunk);
    int32_t* start = out.start + at * (out.tiles + 1);
    for (int q = threadIdx.x; q < n; q += kSortThreads) {
        out.token[at * kChunk + q] = key[b][q];
        out.row[at * kChunk + q] = static_cast<int32_t>(first + from[b][q]);
    }
    // start[t] = the first place whose token lies in tile t or behind it
    for (int q = threadIdx.x; q <= n; q += kSortThreads) {
        const int64_t tile = q < n ? min(out.tiles, static_cast<int64_t>(key[b][q] == vocab ? out.tiles : key[b][q] / kTileRows)) : out.tiles;
        const int64_t last = q == 0 ? -1 : key[b][q - 1] == vocab ? out.tiles : key[b][q - 1] / kTileRows;
        for (int64_t t = last + 1; t <= tile; ++t) start[t] = q;
    }
}

// ---- the sums ----------------------------------------------------------------------------------------------------
constexpr int kGradWarps = 8, kSlice = 256;          // columns a CTA
constexpr int kMany = 64;                            // occurrences from which on all warps share a row

// The lane's eight columns of a slice: neighbouring ones, or 32 apart where rows are not on 16 bytes.
template <class T, bool WIDE>
__device__ __forceinline__ void add_row(const T* row, int lane, int left, float (&sum)[8]) {
    if (WIDE) {
        float v[8];
        load8(row + lane * 8, left - lane * 8, true, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e * 32 + lane < left) sum[e] += to_f(row[e * 32 + lane]);
    }
}
template <class G, bool WIDE>
__device__ __forceinline__ void finish_row(G* to, int lane, int left, bool accumulate, const float (&sum)[8], float scale) {
    float v[8];
    if (WIDE) {
        if (accumulate) load8(static_cast<const G*>(to) + lane * 8, left - lane * 8, true, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = accumulate ? fmaf(sum[e], scale, v[e]) : sum[e] * scale;
        store8(to + lane * 8, left - lane * 8, true, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e * 32 + lane < left) {
                G* p = to + e * 32 + lane;
                put(p, accumulate ? fmaf(sum[e], scale, to_f(*p)) : sum[e] * scale);
            }
    }
}

// Where token v lies in the part [s, e) of a chunk.
__device__ __forceinline__ int2 find(const int32_t* token, int s, int e, int v) {
    int lo = s, hi = e;
    while (lo < hi) { const int m = (lo + hi) >> 1; if (token[m] < v) lo = m + 1; else hi = m; }
    const int from = lo;
    hi = e;
    while (lo < hi) { const int m = (lo + hi) >> 1; if (token[m] <= v) lo = m + 1; else hi = m; }
    return make_int2(from, lo);
}

// Adds up the rows of token v in the order of their chunks; `part` of `parts` takes every parts-th group of kGroup
// occurrences (of each chunk's).  Returns how many there are.
constexpr int kGroup = 8;
template <class T, bool WIDE>
__device__ __forceinline__ int64_t add_token(const EmbeddingGrad& a, const Sorted& s, int64_t node, int64_t tile, int v, const T* dy, int left,
                                             bool count_only, int part, int parts, float (&sum)[8]) {
    const int lane = threadIdx.x & 31;
    int64_t n = 0;
    for (int64_t c0 = 0; c0 < s.chunks; c0 += 32) {
        int2 mine = make_int2(0, 0);
        if (c0 + lane < s.chunks) {
            const int64_t at = s.at(node, c0 + lane);
            const int32_t* start = s.start + at * (s.tiles + 1) + tile;
            mine = find(s.token + at * kChunk, start[0], start[1], v);
        }
        for (uint32_t some = __ballot_sync(0xffffffffu, mine.x < mine.y); some; some &= some - 1) {
            const int c = __ffs(some) - 1;
            const int from = __shfl_sync(0xffffffffu, mine.x, c), to = __shfl_sync(0xffffffffu, mine.y, c);
            n += to - from;
            if (count_only) continue;
            const int32_t* row = s.row + s.at(node, c0 + c) * kChunk;
            for (int q = from + part * kGroup; q < to; q += parts * kGroup) {
                const int32_t* r = row + q;
                const int m = min(kGroup, to - q);
                if (m == kGroup) {
#pragma unroll
                    for (int u = 0; u < kGroup; ++u) add_row<T, WIDE>(dy + r[u] * a.lddy, lane, left, sum);
                } else {
                    for (int u = 0; u < m; ++u) add_row<T, WIDE>(dy + r[u] * a.lddy, lane, left, sum);
                }
            }
        }
    }
    return n;
}

template <class T, class G, bool WIDE>
__global__ void __launch_bounds__(kGradWarps * 32) embedding_grad_kernel(const __grid_constant__ EmbeddingGrad a, const Sorted s) {
    chain_begin();
    __shared__ float part[kGradWarps][kSlice];
    __shared__ uint8_t many[kTileRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile = blockIdx.x, node = blockIdx.z, col = static_cast<int64_t>(blockIdx.y) * kSlice;
    const int left = static_cast<int>(min(static_cast<int64_t>(kSlice), a.d - col));
    const T* dy = static_cast<const T*>(a.dY) + node * a.rows * a.lddy + col;
    G* de = static_cast<G*>(a.dE[node]) + col;
    const int rows = static_cast<int>(min(static_cast<int64_t>(kTileRows), a.vocab - tile * kTileRows));
    for (int r = warp; r < rows; r += kGradWarps) {
        const int v = static_cast<int>(tile * kTileRows) + r;
        float sum[8] = {};
        const int64_t n = add_token<T, WIDE>(a, s, node, tile, v, dy, left, true, 0, 1, sum);
        if (lane == 0) many[r] = n >= kMany;
        if (n >= kMany || (n == 0 && a.accumulate)) continue;
        if (n > 0) add_token<T, WIDE>(a, s, node, tile, v, dy, left, false, 0, 1, sum);
        finish_row<G, WIDE>(de + v * a.d, lane, left, a.accumulate, sum, a.scale);
    }
    __syncthreads();
    for (int r = 0; r < rows; ++r) {
        if (!many[r]) continue;                      // the same for the whole CTA
        const int v = static_cast<int>(tile * kTileRows) + r;
        float sum[8] = {};
        add_token<T, WIDE>(a, s, node, tile, v, dy, left, false, warp, kGradWarps, sum);
#pragma unroll
        for (int e = 0; e < 8; ++e) part[warp][e * 32 + lane] = sum[e];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int w = 1; w < kGradWarps; ++w) sum[e] += part[w][e * 32 + lane];
            finish_row<G, WIDE>(de + v * a.d, lane, left, a.accumulate, sum, a.scale);
        }
        __syncthreads();
    }
}

bool on16(const void* p, int64_t ld_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld_bytes % 16 == 0; }

template <class T, class G>
cudaError_t launch_grad(const EmbeddingGrad& a, const Sorted& s, bool wide, cudaStream_t st) {
    const int64_t slices = (a.d + kSlice - 1) / kSlice;
    const dim3 grid(static_cast<unsigned>(s.tiles), static_cast<unsigned>(slices), static_cast<unsigned>(a.nodes));
    return wide ? launch_chain(embedding_grad_kernel<T, G, true>, grid, kGradWarps * 32, 0, st, a, s)
                : launch_chain(embedding_grad_kernel<T, G, false>, grid, kGradWarps * 32, 0, st, a, s);
}

}  // namespace

cudaError_t lookup(const Lookup& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.d == 0) return cudaSuccess;
    int shift = 0;
    while (shift < 8 && (8LL << shift) < a.d) ++shift;
    const int64_t per = kLookupThreads >> shift, es = dtype == GLR_BF16 ? 2 : 4;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.rows + per - 1) / per, 152 * 32)));
    const bool wide_e = on16(a.E, a.vocab > 1 ? a.lde * es : 0), wide_y = on16(a.Y, a.rows > 1 ? a.ldy * es : 0);
    return dtype == GLR_BF16 ? launch_chain(lookup_kernel<__nv_bfloat16>, grid, kLookupThreads, 0, st, a, shift, wide_e, wide_y)
                             : launch_chain(lookup_kernel<float>, grid, kLookupThreads, 0, st, a, shift, wide_e, wide_y);
}

int64_t embedding_grad_bytes(int64_t nodes, int64_t rows, int64_t vocab) {
    const Sorted s = sorted_of(nodes, rows, vocab, nullptr);
    return nodes * s.chunks * (2 * kChunk + s.tiles + 1) * 4;
}

cudaError_t embedding_grad(const EmbeddingGrad& a, int dtype, int grad_dtype, cudaStream_t st) {
    if (a.vocab == 0 || a.d == 0) return cudaSuccess;
    const Sorted s = sorted_of(a.nodes, a.rows, a.vocab, a.workspace);
    if (s.chunks > 0) {
        int bits = 0;
        while ((int64_t{1} << bits) <= a.vocab) ++bits;          // of the largest key, vocab
        constexpr int kBytes = kChunk * 2 * (4 + 2);
        cudaError_t e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e == cudaSuccess)
            e = launch_chain(sort_kernel, dim3(static_cast<unsigned>(s.chunks), static_cast<unsigned>(a.nodes)), kSortThreads, kBytes, st,
                             a.tokens, a.rows, static_cast<int>(a.vocab), bits, s);
        if (e != cudaSuccess) return e;
    } else if (a.accumulate) {
        return cudaSuccess;
    }
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, gs = grad_dtype == GLR_BF16 ? 2 : 4;
    bool wide = on16(a.dY, a.nodes * a.rows > 1 ? a.lddy * es : 0) && a.d % 8 == 0;
    for (int64_t i = 0; i < a.nodes; ++i) wide = wide && on16(a.dE[i], a.d * gs);
    if (dtype == GLR_BF16)
        return grad_dtype == GLR_BF16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(a, s, wide, st) : launch_grad<__nv_bfloat16, float>(a, s, wide, st);
    return grad_dtype == GLR_BF16 ? launch_grad<float, __nv_bfloat16>(a, s, wide, st) : launch_grad<float, float>(a, s, wide, st);
}

}  // namespace rows
}  // namespace glr
