// Embedding lookup with scaling, and every node's gradient of the embedding by sorted tokens.
//
// The gradient of row v is scale times the sum of the rows of dY whose token is v.  They are put in the order of the rows and
// added up in partial sums that the sizes and the tokens fix (a warp's groups of lanes take rows in turn, and from kMany rows on
// the warps groups of 32), so that the result does not depend on what runs when.  A CTA takes 64 or 256 rows of the vocabulary
// and 64 or 256 columns and adds up the rows of dY that belong to them, one warp a row, or all its warps where there are many.
// Where it finds them depends on the node's rows: up to kScan it looks through the node's tokens and puts its own in order of
// (token, row); beyond, chunks of kChunk rows have been sorted by their tokens, stably, by a kernel before, with the place where each
// tile begins.  Both order by ranks among equal digits: warps take consecutive stretches, lanes with the same digit are matched.
// A token outside the vocabulary is nobody's.
// Bound by HBM: the gradient of the whole vocabulary is written for every node (8 nodes x 1024 rows, 32768 x 2048 bf16, 1.1 GB:
// 179 us, 6.2 TB/s; lookups of 16384 rows of 4096 bf16 34 us).  Tiles of 64 rows instead of 256 took 256 us: what a CTA does before
// it writes costs as much as its writes.  Eight rows of dY are loaded before the first is added (one at a time: 200 us).
#include <algorithm>

#include "glr_rows.cuh"

namespace glr {
namespace rows {

namespace {

constexpr int kLookupThreads = 256;

template <class T>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const __grid_constant__ Lookup a, int shift) {
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
            load8(e + j, in ? n : 0, true, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] *= a.scale;        // (0 for padding)
            store8(y + j, n, true, v);
        }
    }
}

// Rows off 16 bytes: 256 columns a warp.
template <class T>
__global__ void __launch_bounds__(kLookupThreads) lookup_apart_kernel(const __grid_constant__ Lookup a, int64_t parts) {
    chain_begin();
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kLookupThreads / 32);
    for (int64_t q = static_cast<int64_t>(blockIdx.x) * (kLookupThreads / 32) + (threadIdx.x >> 5); q < a.rows * parts; q += warps) {
        const int64_t i = q / parts, first = (q - i * parts) * 256, t = a.tokens.at(i);
        const bool in = t >= 0 && t < a.vocab;
        float v[8];
        load_apart(static_cast<const T*>(a.E) + (in ? t : 0) * a.lde, first, in ? a.d : 0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        store_apart(static_cast<T*>(a.Y) + i * a.ldy, first, a.d, v);
    }
}

// ---- the tokens in order ---------------------------------------------------------------------------------------
constexpr int kChunk = 4096, kSortThreads = 512, kSortWarps = kSortThreads / 32, kMine = kChunk / kSortThreads;
constexpr int kDigit = 9, kDigits = 1 << kDigit;        // two passes for up to 2^18 - 1 tokens

// A chunk's sorted tokens, the rows (of its node) that they come from, and where each tile's begin.
struct Sorted {
    int32_t* token; int32_t* row; int32_t* start;
    int64_t chunks, tiles;                           // a node's
    int tile_rows;
    __host__ __device__ int64_t at(int64_t node, int64_t chunk) const { return node * chunks + chunk; }
};
// A tile's rows: few where the tiles would leave SMs idle, and where a table of many would not have room for the chunks.
constexpr int kFewRows = 64, kManyRows = 256;
int tile_rows(int64_t nodes, int64_t rows, int64_t vocab, int64_t d) {
    return rows <= 8 * kChunk && (vocab + kManyRows - 1) / kManyRows * nodes * ((d + 255) / 256) >= 152 * 5 ? kManyRows : kFewRows;
}
Sorted sorted_of(int64_t nodes, int64_t rows, int64_t vocab, int64_t d, void* workspace) {
    Sorted s{};
    s.chunks = (rows + kChunk - 1) / kChunk;
    s.tile_rows = tile_rows(nodes, rows, vocab, d);
    s.tiles = (vocab + s.tile_rows - 1) / s.tile_rows;
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
        const int64_t least = min(t * out.tile_rows, static_cast<int64_t>(vocab));
        int lo = 0, hi = n;
        while (lo < hi) { const int m = (lo + hi) >> 1; if (key[b][m] < least) lo = m + 1; else hi = m; }
        start[t] = lo;
    }
}

// ---- the sums ----------------------------------------------------------------------------------------------------
constexpr int kGradWarps = 8, kGradThreads = kGradWarps * 32;
constexpr int kMany = 64;                            // occurrences from which on all warps share a row
constexpr int kScan = 1024;                          // a node's rows up to which its tokens are looked through

// L lanes take a row of dY, 8 L columns of it; with L = 8 a warp adds up four rows at once.
// The lane's eight columns of a slice of a row, as they lie in memory (0 beyond the last one): neighbouring ones (WIDE 1), also
// where dE's rows are on 16 bytes and only dY's are not (2: 8 x 1024 rows with a stride of 2049, 32768 x 2048 bf16 188 us; as 0
// 251), else L apart (0).  Of rows off 16 bytes four are loaded at once (two: 4 x 6639 rows into 3062 x 989 bf16 100 us, now 79).
template <class T, int WIDE, int L> struct Columns;
template <int L> struct Columns<__nv_bfloat16, 1, L> {
    static constexpr int kAhead = 8;                 // rows loaded before the first one is added
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int lane, int left) {
        u = lane * 8 < left ? *reinterpret_cast<const uint4*>(row + lane * 8) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void add(float (&sum)[8]) const {
        float v[8];
        widen8(u, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
};
template <int L> struct Columns<float, 1, L> {
    static constexpr int kAhead = 4;
    float4 a, b;
    __device__ __forceinline__ void load(const float* row, int lane, int left) {
        const float4* p = reinterpret_cast<const float4*>(row + lane * 8);
        const bool in = lane * 8 < left;
        a = in ? p[0] : make_float4(0.f, 0.f, 0.f, 0.f);
        b = in ? p[1] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void add(float (&sum)[8]) const {
        sum[0] += a.x; sum[1] += a.y; sum[2] += a.z; sum[3] += a.w; sum[4] += b.x; sum[5] += b.y; sum[6] += b.z; sum[7] += b.w;
    }
};
template <class T, int L> struct Columns<T, 0, L> {
    static constexpr int kAhead = 4;
    T x[8];
    __device__ __forceinline__ void load(const T* row, int lane, int left) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e * L + lane < left ? row[e * L + lane] : T(0.f);
    }
    __device__ __forceinline__ void add(float (&sum)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += to_f(x[e]);
    }
};
template <class T, int L> struct Columns<T, 2, L> {
    static constexpr int kAhead = 4;
    T x[8];
    __device__ __forceinline__ void load(const T* row, int lane, int left) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = lane * 8 < left ? row[lane * 8 + e] : T(0.f);
    }
    __device__ __forceinline__ void add(float (&sum)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += to_f(x[e]);
    }
};
template <class G, int WIDE, int L>
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
            if (e * L + lane < left) {
                G* p = to + e * L + lane;
                put(p, accumulate ? fmaf(sum[e], scale, to_f(*p)) : sum[e] * scale);
            }
    }
}

// The first place of [s, e) whose token is v or a later one.
__device__ __forceinline__ int first_at(const int32_t* token, int s, int e, int v) {
    while (s < e) { const int m = (s + e) >> 1; if (token[m] < v) s = m + 1; else e = m; }
    return s;
}

// Adds up the rows `row[0 .. n)` of dY: every parts-th group of 32 of them, in their order; the lanes have a sum for each of
// their 32 / L groups.
template <class T, int WIDE, int L>
__device__ __forceinline__ void add_rows(const T* dy, int64_t lddy, const int32_t* row, int n, int part, int parts, int left, float (&sum)[8]) {
    using C = Columns<T, WIDE, L>;
    constexpr int kAtOnce = 32 / L;
    const int lane = threadIdx.x & 31, own = lane & (L - 1), group = lane / L;
    for (int q = part * 32; q < n; q += parts * 32) {
        const int mine = q + lane < n ? row[q + lane] : 0, m = min(32, n - q);
        int u = 0;
        for (; u + C::kAhead * kAtOnce <= m; u += C::kAhead * kAtOnce) {
            C c[C::kAhead];
#pragma unroll
            for (int k = 0; k < C::kAhead; ++k) c[k].load(dy + __shfl_sync(0xffffffffu, mine, u + k * kAtOnce + group) * lddy, own, left);
#pragma unroll
            for (int k = 0; k < C::kAhead; ++k) c[k].add(sum);
        }
        for (; u < m; u += 2 * kAtOnce) {
            C c[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int x = u + k * kAtOnce + group;
                c[k].load(dy + __shfl_sync(0xffffffffu, mine, min(x, 31)) * lddy, own, x < m ? left : 0);
            }
            c[0].add(sum);
            c[1].add(sum);
        }
    }
}

// A tile's rows, one warp each, then those that all warps share.  of(r) is how many rows of dY the tile's row r has;
// add(r, part, parts, sum) adds up every parts-th group of them.
template <class G, int WIDE, int L, class Of, class Add>
__device__ __forceinline__ void sum_rows(const EmbeddingGrad& a, G* de, int rows, int left, float (*part)[8 * L], uint16_t* many, int* some,
                                         const Of& of, const Add& add) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const auto total = [&](int r, int from, int parts, float (&sum)[8]) {
        add(r, from, parts, sum);
#pragma unroll
        for (int o = L; o < 32; o *= 2)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], o);
    };
    for (int r = warp; r < rows; r += kGradWarps) {
        const int n = of(r);
        if (n == 0) {
            if (a.accumulate) continue;
            if (WIDE) {
                constexpr int kPer = 16 / sizeof(G);
#pragma unroll
                for (int j = lane * kPer; j < 8 * L; j += 32 * kPer)
                    if (j < left) *reinterpret_cast<uint4*>(de + r * a.d + j) = make_uint4(0, 0, 0, 0);
            } else {
                for (int j = lane; j < left; j += 32) put(de + r * a.d + j, 0.f);
            }
        } else if (n >= kMany) {
            if (lane == 0) many[atomicAdd(some, 1)] = static_cast<uint16_t>(r);
        } else {
            float sum[8] = {};
            total(r, 0, 1, sum);
            if (lane < L) finish_row<G, WIDE, L>(de + r * a.d, lane, left, a.accumulate, sum, a.scale);
        }
    }
    __syncthreads();
    for (int q = 0; q < *some; ++q) {
        const int r = many[q];
        float sum[8] = {};
        total(r, warp, kGradWarps, sum);
        if (lane < L) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[warp][e * L + lane] = sum[e];
        }
        __syncthreads();
        if (warp == 0 && lane < L) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int w = 1; w < kGradWarps; ++w) sum[e] += part[w][e * L + lane];
            finish_row<G, WIDE, L>(de + r * a.d, lane, left, a.accumulate, sum, a.scale);
        }
        __syncthreads();
    }
}

// Up to kScan rows a node: the CTA looks through the node's tokens.
template <class T, class G, int WIDE, int R, int L>
__global__ void __launch_bounds__(kGradThreads, 4) scan_grad_kernel(const __grid_constant__ EmbeddingGrad a) {
    chain_begin();
    __shared__ float part[kGradWarps][8 * L];
    __shared__ int32_t list[kScan];                  // the tile's rows of dY in order of (token, row)
    __shared__ int off[R + 1];                       // where each of its tokens begins
    __shared__ uint16_t count[kGradWarps][R];
    __shared__ int carry[kGradWarps];
    __shared__ uint16_t many[R];
    __shared__ int some;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t node = blockIdx.z, v0 = static_cast<int64_t>(blockIdx.x) * R, col = static_cast<int64_t>(blockIdx.y) * (8 * L);
    const int rows = static_cast<int>(min(static_cast<int64_t>(R), a.vocab - v0)), left = static_cast<int>(min(static_cast<int64_t>(8 * L), a.d - col));
    // each warp takes a stretch of rows: their tokens' places in the tile (R: none), then the ranks among the warp's too
    constexpr int kBatches = kScan / kGradThreads;
    const int n = static_cast<int>(a.rows), stretch = (n + kGradThreads - 1) / kGradThreads;
    uint32_t rank[kBatches];
#pragma unroll
    for (int u = 0; u < kBatches; ++u) {
        const int x = (warp * stretch + u) * 32 + lane;
        rank[u] = R;
        if (u < stretch && x < n) {
            const int64_t t = a.tokens.at(node * a.rows + x) - v0;
            if (t >= 0 && t < rows) rank[u] = static_cast<uint32_t>(t);
        }
    }
    for (int q = threadIdx.x; q < kGradWarps * R / 2; q += kGradThreads) reinterpret_cast<uint32_t*>(&count[0][0])[q] = 0;
    if (threadIdx.x == 0) some = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kBatches; ++u) {
        const int r = static_cast<int>(rank[u]);
        rank[u] = static_cast<uint32_t>(r) << 16;
        if (__any_sync(0xffffffffu, r < R)) {
            const uint32_t same = __match_any_sync(0xffffffffu, r), before = same & ((1u << lane) - 1);
            if (r < R) rank[u] |= count[warp][r] + __popc(before);
            __syncwarp();
            if (r < R && before == 0) count[warp][r] += static_cast<uint16_t>(__popc(same));
            __syncwarp();
        }
    }
    __syncthreads();
    int sum = 0;
    if (threadIdx.x < R)
        for (int w = 0; w < kGradWarps; ++w) { const int c = count[w][threadIdx.x]; count[w][threadIdx.x] = static_cast<uint16_t>(sum); sum += c; }
    int before = sum;                                // of the threads up to this one, then before it
    for (int o = 1; o < 32; o *= 2) { const int y = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += y; }
    if (lane == 31) carry[warp] = before;
    __syncthreads();
    before -= sum;
    for (int w = 0; w < warp; ++w) before += carry[w];
    if (threadIdx.x < R) off[threadIdx.x] = before;
    if (threadIdx.x == R - 1) off[R] = before + sum;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kBatches; ++u) {
        const int r = static_cast<int>(rank[u] >> 16);
        if (r < R) list[off[r] + count[warp][r] + (rank[u] & 0xffffu)] = (warp * stretch + u) * 32 + lane;
    }
    __syncthreads();
    const T* dy = static_cast<const T*>(a.dY) + node * a.rows * a.lddy + col;
    sum_rows<G, WIDE, L>(a, static_cast<G*>(a.dE[node]) + v0 * a.d + col, rows, left, part, many, &some,
                      [&](int r) { return off[r + 1] - off[r]; },
                      [&](int r, int from, int parts, float (&s)[8]) { add_rows<T, WIDE, L>(dy, a.lddy, list + off[r], off[r + 1] - off[r], from, parts, left, s); });
}

// Beyond: the tile's part of every sorted chunk, with a table of where each row begins in each chunk (TABLE), or, of more
// chunks than it has room for, looked for row by row.
constexpr int kTable = 2080;
template <class T, class G, int WIDE, int R, int L, bool TABLE>
__global__ void __launch_bounds__(kGradThreads, 4) sorted_grad_kernel(const __grid_constant__ EmbeddingGrad a, const Sorted s) {
    chain_begin();
    __shared__ float part[kGradWarps][8 * L];
    __shared__ int32_t table[TABLE ? kTable : 1];
    __shared__ uint16_t many[R];
    __shared__ int some;
    const int lane = threadIdx.x & 31;
    const int64_t tile = blockIdx.x, node = blockIdx.z, v0 = tile * R, col = static_cast<int64_t>(blockIdx.y) * (8 * L);
    const int rows = static_cast<int>(min(static_cast<int64_t>(R), a.vocab - v0)), left = static_cast<int>(min(static_cast<int64_t>(8 * L), a.d - col));
    const auto part_of = [&](int64_t chunk) {
        const int32_t* start = s.start + s.at(node, chunk) * (s.tiles + 1) + tile;
        return make_int2(start[0], start[1]);
    };
    if (threadIdx.x == 0) some = 0;
    if (TABLE)
        for (int q = threadIdx.x; q < static_cast<int>(s.chunks) * (R + 1); q += kGradThreads) {
            const int chunk = q / (R + 1), r = q % (R + 1);
            const int2 p = part_of(chunk);
            table[q] = r == 0 ? p.x : r == R ? p.y : first_at(s.token + s.at(node, chunk) * kChunk, p.x, p.y, static_cast<int>(v0) + r);
        }
    __syncthreads();
    const T* dy = static_cast<const T*>(a.dY) + node * a.rows * a.lddy + col;
    // the part of chunk c0 + lane that is row r's
    const auto mine = [&](int64_t c0, int r) {
        if (c0 + lane >= s.chunks) return make_int2(0, 0);
        if (TABLE) return make_int2(table[lane * (R + 1) + r], table[lane * (R + 1) + r + 1]);
        const int2 p = part_of(c0 + lane);
        const int32_t* token = s.token + s.at(node, c0 + lane) * kChunk;
        return make_int2(first_at(token, p.x, p.y, static_cast<int>(v0) + r), first_at(token, p.x, p.y, static_cast<int>(v0) + r + 1));
    };
    sum_rows<G, WIDE, L>(a, static_cast<G*>(a.dE[node]) + v0 * a.d + col, rows, left, part, many, &some,
        [&](int r) {
            int n = 0;
            for (int64_t c0 = 0; c0 < s.chunks; c0 += 32) { const int2 m = mine(c0, r); n += m.y - m.x; }
            return __reduce_add_sync(0xffffffffu, n);
        },
        [&](int r, int from, int parts, float (&sum)[8]) {
            for (int64_t c0 = 0; c0 < s.chunks; c0 += 32) {
                const int2 m = mine(c0, r);
                for (uint32_t some_of = __ballot_sync(0xffffffffu, m.x < m.y); some_of; some_of &= some_of - 1) {
                    const int c = __ffs(some_of) - 1;
                    const int begin = __shfl_sync(0xffffffffu, m.x, c), end = __shfl_sync(0xffffffffu, m.y, c);
                    add_rows<T, WIDE, L>(dy, a.lddy, s.row + s.at(node, c0 + c) * kChunk + begin, end - begin, from, parts, left, sum);
                }
            }
        });
}

bool on16(const void* p, int64_t ld_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld_bytes % 16 == 0; }

template <class T, class G, int WIDE, int R, int L>
cudaError_t launch_tiles(const EmbeddingGrad& a, const Sorted& s, cudaStream_t st) {
    const dim3 grid(static_cast<unsigned>(s.tiles), static_cast<unsigned>((a.d + 8 * L - 1) / (8 * L)), static_cast<unsigned>(a.nodes));
    if (a.rows <= kScan) return launch_chain(scan_grad_kernel<T, G, WIDE, R, L>, grid, kGradThreads, 0, st, a);
    return s.chunks * (R + 1) <= kTable ? launch_chain(sorted_grad_kernel<T, G, WIDE, R, L, true>, grid, kGradThreads, 0, st, a, s)
                                        : launch_chain(sorted_grad_kernel<T, G, WIDE, R, L, false>, grid, kGradThreads, 0, st, a, s);
}
template <class T, class G, int WIDE>
cudaError_t launch_wide(const EmbeddingGrad& a, const Sorted& s, cudaStream_t st) {
    if (s.tile_rows == kManyRows) return launch_tiles<T, G, WIDE, kManyRows, 32>(a, s, st);
    // narrow slices where wide ones would leave SMs idle: a token of many rows then keeps fewer columns waiting
    return s.tiles * a.nodes * ((a.d + 255) / 256) < 152 * 4 ? launch_tiles<T, G, WIDE, kFewRows, 8>(a, s, st)
                                                             : launch_tiles<T, G, WIDE, kFewRows, 32>(a, s, st);
}
template <class T, class G>
cudaError_t launch_grad(const EmbeddingGrad& a, const Sorted& s, int wide, cudaStream_t st) {
    return wide == 0 ? launch_wide<T, G, 0>(a, s, st) : wide == 1 ? launch_wide<T, G, 1>(a, s, st) : launch_wide<T, G, 2>(a, s, st);
}

}  // namespace

cudaError_t lookup(const Lookup& a, int dtype, cudaStream_t st) {
    if (a.rows == 0 || a.d == 0) return cudaSuccess;
    const int64_t es = dtype == GLR_BF16 ? 2 : 4;
    if (!on16(a.E, a.vocab > 1 ? a.lde * es : 0) || !on16(a.Y, a.rows > 1 ? a.ldy * es : 0)) {
        const int64_t parts = (a.d + 255) / 256, warps = kLookupThreads / 32;
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.rows * parts + warps - 1) / warps, 152 * 32)));
        return dtype == GLR_BF16 ? launch_chain(lookup_apart_kernel<__nv_bfloat16>, grid, kLookupThreads, 0, st, a, parts)
                                 : launch_chain(lookup_apart_kernel<float>, grid, kLookupThreads, 0, st, a, parts);
    }
    int shift = 0;
    while (shift < 8 && (8LL << shift) < a.d) ++shift;
    const int64_t per = kLookupThreads >> shift;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((a.rows + per - 1) / per, 152 * 32)));
    return dtype == GLR_BF16 ? launch_chain(lookup_kernel<__nv_bfloat16>, grid, kLookupThreads, 0, st, a, shift)
                             : launch_chain(lookup_kernel<float>, grid, kLookupThreads, 0, st, a, shift);
}

int64_t embedding_grad_bytes(int64_t nodes, int64_t rows, int64_t vocab, int64_t d) {
    if (rows <= kScan) return 0;
    const Sorted s = sorted_of(nodes, rows, vocab, d, nullptr);
    return nodes * s.chunks * (2 * kChunk + s.tiles + 1) * 4;
}

cudaError_t embedding_grad(const EmbeddingGrad& a, int dtype, int grad_dtype, cudaStream_t st) {
    if (a.vocab == 0 || a.d == 0) return cudaSuccess;
    const Sorted s = sorted_of(a.nodes, a.rows, a.vocab, a.d, a.workspace);
    if (a.rows > kScan) {
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
    bool whole = a.d % 8 == 0;
    for (int64_t i = 0; i < a.nodes; ++i) whole = whole && on16(a.dE[i], a.d * gs);
    const int wide = !whole ? 0 : on16(a.dY, a.nodes * a.rows > 1 ? a.lddy * es : 0) ? 1 : 2;
    if (dtype == GLR_BF16)
        return grad_dtype == GLR_BF16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(a, s, wide, st) : launch_grad<__nv_bfloat16, float>(a, s, wide, st);
    return grad_dtype == GLR_BF16 ? launch_grad<float, __nv_bfloat16>(a, s, wide, st) : launch_grad<float, float>(a, s, wide, st);
}

}  // namespace rows
}  // namespace glr
