// Embedding lookup with scaling, and every node's gradient of the embedding by sorted tokens.
//
// The gradient of row v is scale times the sum of the rows of dY whose token is v, in the order of the rows, so its result
// does not depend on what runs when.  A CTA takes kTileRows rows of the vocabulary and up to 512 columns, puts the rows of dY that
// belong to them in order of (token, row), and adds them up, one warp a row, or all its warps where there are many.
// Where it finds them depends on the node's rows: up to kScan, among all of the node's tokens; beyond, in chunks of kChunk rows that a
// kernel before has sorted by their tokens, stably, with the place where each tile begins.  Both order by ranks among equal
// digits (warps take consecutive stretches; lanes with the same digit are matched).  A token outside the vocabulary is nobody's.
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
    for (int64_t t = threadIdx.x; t <= out.tiles; t += kSortThreads) {
        const int64_t least = min(t * kTileRows, static_cast<int64_t>(vocab));
        int lo = 0, hi = n;
        while (lo < hi) { const int m = (lo + hi) >> 1; if (key[b][m] < least) lo = m + 1; else hi = m; }
        start[t] = lo;
    }
}

// ---- the sums ----------------------------------------------------------------------------------------------------
constexpr int kGradWarps = 8, kGradThreads = kGradWarps * 32, kSlice = 256;          // columns at a time
constexpr int kMany = 64;                            // occurrences from which on all warps share a row
constexpr int kScan = 1024;                          // a node's rows up to which its tokens are looked through
constexpr int kBatches = 4, kPlaces = kBatches * kGradThreads;       // entries of a tile in shared memory
constexpr int kChunksAtOnce = kGradThreads;

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

// Adds up the rows `row[0 .. n)` of dY: every parts-th group of kGroup of them, in their order.
constexpr int kGroup = 8;
template <class T, bool WIDE>
__device__ __forceinline__ void add_rows(const T* dy, int64_t lddy, const int32_t* row, int n, int part, int parts, int left, float (&sum)[8]) {
    const int lane = threadIdx.x & 31;
    for (int q = part * kGroup; q < n; q += parts * kGroup) {
        if (n - q >= kGroup) {
#pragma unroll
            for (int u = 0; u < kGroup; ++u) add_row<T, WIDE>(dy + row[q + u] * lddy, lane, left, sum);
        } else {
            for (int u = q; u < n; ++u) add_row<T, WIDE>(dy + row[u] * lddy, lane, left, sum);
        }
    }
}
// ... of token v in the chunks, one after the other, for tiles whose entries do not fit in shared memory.  Returns how many.
template <class T, bool WIDE>
__device__ __noinline__ int64_t add_token(const Sorted& s, int64_t node, int64_t tile, int v, const T* dy, int64_t lddy, int left, bool count_only,
                                          int part, int parts, float (&sum)[8]) {
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
            if (!count_only) add_rows<T, WIDE>(dy, lddy, s.row + s.at(node, c0 + c) * kChunk + from, to - from, part, parts, left, sum);
        }
    }
    return n;
}

// A whole tile whose entries do not fit in shared memory, each row's looked for in all chunks.
template <class T, class G, bool WIDE>
__device__ __noinline__ void add_tile(const EmbeddingGrad& a, const Sorted& s, int64_t node, int64_t tile, int rows, int64_t col0, int slices,
                                      float (*part)[kSlice]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t col = col0; col < col0 + slices * kSlice && col < a.d; col += kSlice) {
        const int left = static_cast<int>(min(static_cast<int64_t>(kSlice), a.d - col));
        const T* dy = static_cast<const T*>(a.dY) + node * a.rows * a.lddy + col;
        G* de = static_cast<G*>(a.dE[node]) + col;
        for (int r = 0; r < rows; ++r) {
            const int v = static_cast<int>(tile * kTileRows) + r;
            float sum[8] = {};
            const int64_t c = add_token<T, WIDE>(s, node, tile, v, dy, a.lddy, left, false, warp, kGradWarps, sum);
            if (c == 0 && a.accumulate) continue;    // the same for the whole CTA
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
}

// The sum over the CTA's threads before this one, and over all of them.
__device__ __forceinline__ int2 scan_threads(int v, int* carry) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int sum = v;
    for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += y; }
    if (lane == 31) carry[warp] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kGradWarps; ++w) { before += w < warp ? carry[w] : 0; all += carry[w]; }
    return make_int2(before + sum - v, all);
}

template <class T, class G, bool WIDE>
__global__ void __launch_bounds__(kGradThreads, 5) embedding_grad_kernel(const __grid_constant__ EmbeddingGrad a, const Sorted s, bool scan, int slices) {
    chain_begin();
    __shared__ float part[kGradWarps][kSlice];
    __shared__ int32_t list[kPlaces];
    __shared__ int off[kTileRows + 1];
    __shared__ uint16_t count[kGradWarps][kTileRows];
    __shared__ int2 chunk_part[kChunksAtOnce];       // of the chunks' entries: the tile's first place, the entries before it
    __shared__ int carry[kGradWarps];
    __shared__ uint8_t many[kTileRows];              // rows that all warps share
    __shared__ int some;                             // their number
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t tile = blockIdx.x, node = blockIdx.z;
    const int rows = static_cast<int>(min(static_cast<int64_t>(kTileRows), a.vocab - tile * kTileRows));
    const int64_t v0 = tile * kTileRows;
    const T* dy0 = static_cast<const T*>(a.dY) + node * a.rows * a.lddy;
    // the tile's entries: the node's tokens, or those of the chunks one after the other
    int n = static_cast<int>(a.rows);
    bool fits = true;
    if (!scan) {
        fits = s.chunks <= kChunksAtOnce;
        int mine = 0, from = 0;
        if (fits && threadIdx.x < s.chunks) {
            const int32_t* start = s.start + s.at(node, threadIdx.x) * (s.tiles + 1) + tile;
            from = start[0];
            mine = start[1] - from;
        }
        const int2 sum = scan_threads(mine, carry);
        chunk_part[threadIdx.x] = make_int2(from, sum.x);
        n = sum.y;
        fits = fits && n <= kPlaces;
    }
    for (int q = threadIdx.x; q < kGradWarps * kTileRows; q += kGradThreads) (&count[0][0])[q] = 0;
    if (threadIdx.x == 0) some = 0;
    __syncthreads();
    if (!fits) {                                     // the same for the whole CTA
        add_tile<T, G, WIDE>(a, s, node, tile, rows, static_cast<int64_t>(blockIdx.y) * slices * kSlice, slices, part);
        return;
    }
    {
        // each warp ranks a stretch of entries; what it knows of them stays in registers
        const int stretch = (n + kGradThreads - 1) / kGradThreads;
        int32_t row[kBatches];
        uint32_t rank[kBatches];                     // the token's row of the tile, and its rank among the warp's
#pragma unroll
        for (int u = 0; u < kBatches; ++u) {
            rank[u] = kTileRows << 16;
            row[u] = 0;
            if (u < stretch) {                       // the same for the whole CTA
                const int x = (warp * stretch + u) * 32 + lane;
                int r = kTileRows;
                if (x < n) {
                    if (scan) {
                        const int64_t t = a.tokens.at(node * a.rows + x) - v0;
                        row[u] = x;
                        if (t >= 0 && t < rows) r = static_cast<int>(t);
                    } else {
                        int c = 0, end = static_cast<int>(s.chunks);         // the last chunk that begins at x or before
                        while (end - c > 1) { const int m = (c + end) >> 1; if (chunk_part[m].y <= x) c = m; else end = m; }
                        const int64_t at = s.at(node, c) * kChunk + chunk_part[c].x + (x - chunk_part[c].y);
                        row[u] = s.row[at];
                        r = static_cast<int>(s.token[at] - v0);
                    }
                }
                if (__any_sync(0xffffffffu, r < kTileRows)) {
                    const uint32_t same = __match_any_sync(0xffffffffu, r), before = same & ((1u << lane) - 1);
                    if (r < kTileRows) rank[u] = static_cast<uint32_t>(r) << 16 | (count[warp][r] + __popc(before));
                    __syncwarp();
                    if (r < kTileRows && before == 0) count[warp][r] += static_cast<uint16_t>(__popc(same));
                    __syncwarp();
                }
            }
        }
        __syncthreads();
        int sum = 0;
        if (threadIdx.x < kTileRows)
            for (int w = 0; w < kGradWarps; ++w) { const int c = count[w][threadIdx.x]; count[w][threadIdx.x] = static_cast<uint16_t>(sum); sum += c; }
        const int2 place = scan_threads(sum, carry);
        if (threadIdx.x < kTileRows) off[threadIdx.x] = place.x;
        if (threadIdx.x == 0) off[kTileRows] = place.y;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kBatches; ++u) {
            const int r = static_cast<int>(rank[u] >> 16);
            if (r < kTileRows) list[off[r] + count[warp][r] + (rank[u] & 0xffffu)] = row[u];
        }
        __syncthreads();
    }
    const int64_t col0 = static_cast<int64_t>(blockIdx.y) * slices * kSlice;
    const int width = static_cast<int>(min(static_cast<int64_t>(slices) * kSlice, a.d - col0));
    const T* dy = dy0 + col0;
    G* de = static_cast<G*>(a.dE[node]) + v0 * a.d + col0;
    const auto rows_of = [&](int r, int from, int parts, int c0) {
        float sum[8] = {};
        add_rows<T, WIDE>(dy + c0, a.lddy, list + off[r], off[r + 1] - off[r], from, parts, width - c0, sum);
        if (parts == 1) { finish_row<G, WIDE>(de + r * a.d + c0, lane, width - c0, a.accumulate, sum, a.scale); return; }
#pragma unroll
        for (int e = 0; e < 8; ++e) part[warp][e * 32 + lane] = sum[e];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int w = 1; w < kGradWarps; ++w) sum[e] += part[w][e * 32 + lane];
            finish_row<G, WIDE>(de + r * a.d + c0, lane, width - c0, a.accumulate, sum, a.scale);
        }
        __syncthreads();
    };
    for (int r = warp; r < rows; r += kGradWarps) {
        const int n_r = off[r + 1] - off[r];
        if (n_r == 0) {
            if (a.accumulate) continue;
            if (WIDE) {
                constexpr int kPer = 16 / sizeof(G);
                for (int j = lane * kPer; j < width; j += 32 * kPer) *reinterpret_cast<uint4*>(de + r * a.d + j) = make_uint4(0, 0, 0, 0);
            } else {
                for (int j = lane; j < width; j += 32) put(de + r * a.d + j, 0.f);
            }
        } else if (n_r >= kMany) {
            if (lane == 0) many[atomicAdd(&some, 1)] = static_cast<uint8_t>(r);
        } else {
            for (int c0 = 0; c0 < width; c0 += kSlice) rows_of(r, 0, 1, c0);
        }
    }
    __syncthreads();
    for (int q = 0; q < some; ++q)
        for (int c0 = 0; c0 < width; c0 += kSlice) rows_of(many[q], warp, kGradWarps, c0);
}

bool on16(const void* p, int64_t ld_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld_bytes % 16 == 0; }

template <class T, class G>
cudaError_t launch_grad(const EmbeddingGrad& a, const Sorted& s, bool scan, bool wide, cudaStream_t st) {
    // columns a CTA: one slice where that takes all, or where two would leave SMs idle
    const int64_t all = (a.d + kSlice - 1) / kSlice;
    const int slices = all > 1 && s.tiles * a.nodes * ((all + 1) / 2) >= 152 * 8 ? 2 : 1;
    const dim3 grid(static_cast<unsigned>(s.tiles), static_cast<unsigned>((all + slices - 1) / slices), static_cast<unsigned>(a.nodes));
    return wide ? launch_chain(embedding_grad_kernel<T, G, true>, grid, kGradThreads, 0, st, a, s, scan, slices)
                : launch_chain(embedding_grad_kernel<T, G, false>, grid, kGradThreads, 0, st, a, s, scan, slices);
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
    if (rows <= kScan) return 0;
    const Sorted s = sorted_of(nodes, rows, vocab, nullptr);
    return nodes * s.chunks * (2 * kChunk + s.tiles + 1) * 4;
}

cudaError_t embedding_grad(const EmbeddingGrad& a, int dtype, int grad_dtype, cudaStream_t st) {
    if (a.vocab == 0 || a.d == 0) return cudaSuccess;
    const Sorted s = sorted_of(a.nodes, a.rows, a.vocab, a.workspace);
    const bool scan = a.rows <= kScan;
    if (!scan) {
        int bits = 0;
        while ((int64_t{1} << bits) <= a.vocab) ++bits;          // of the largest key, vocab
        constexpr int kBytes = kChunk * 2 * (4 + 2);
        cudaError_t e = cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e == cudaSuccess)
            e = launch_chain(sort_kernel, dim3(static_cast<unsigned>(s.chunks), static_cast<unsigned>(a.nodes)), kSortThreads, kBytes, st,
                             a.tokens, a.rows, static_cast<int>(a.vocab), bits, s);
        if (e != cudaSuccess) return e;
    } else if (a.rows == 0 && a.accumulate) {
        return cudaSuccess;
    }
    const int64_t es = dtype == GLR_BF16 ? 2 : 4, gs = grad_dtype == GLR_BF16 ? 2 : 4;
    bool wide = on16(a.dY, a.nodes * a.rows > 1 ? a.lddy * es : 0) && a.d % 8 == 0;
    for (int64_t i = 0; i < a.nodes; ++i) wide = wide && on16(a.dE[i], a.d * gs);
    if (dtype == GLR_BF16)
        return grad_dtype == GLR_BF16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(a, s, scan, wide, st) : launch_grad<__nv_bfloat16, float>(a, s, scan, wide, st);
    return grad_dtype == GLR_BF16 ? launch_grad<float, __nv_bfloat16>(a, s, scan, wide, st) : launch_grad<float, float>(a, s, scan, wide, st);
}

}  // namespace rows
}  // namespace glr
