// Embedding lookup with scaling and its gradient (gfx950): the node that turns the tokens of a batch into rows.
//
//   y[t]      = scale * table[id[t]]                       for 0 <= id[t] < vocab, else +0
//   dtable[v] = scale * sum over t with id[t] = v of dy[t]  (ascending t, fp32)
#include "rows.h"

namespace ngc {

// Bound: HBM (32768 rows of 4096 bf16 out of 50257: 59 us, 4.5 TB/s written; 143 MB of the 268 read come from it, frequent rows from the caches).
// GL lanes per token, as many as a row has vectors, so that every lane has work and a long row's loads are under way together; 16 bytes a lane and
// step.  Rows of no multiple of 16 bytes end in a vector that overlaps the one before it (both hold the same values), rows below 16 bytes go element
// by element.
template <typename T, int GL>
__global__ __launch_bounds__(256) void embedding_rows(const T *__restrict__ table, const int64_t *__restrict__ ids, T *__restrict__ y, int64_t tokens,
                                                      int vocab, int width, float scale, int whole)
{
    constexpr int E = SmElem<T>::E;
    const int lane = threadIdx.x & (GL - 1);
    const unsigned nvec = ((unsigned)width + E - 1) / E;
    for (int64_t t = (int64_t)blockIdx.x * (256 / GL) + threadIdx.x / GL; t < tokens; t += (int64_t)gridDim.x * (256 / GL)) {
        const int64_t id = ids[t];
        const bool live = id >= 0 && id < vocab;
        const T *src = table + (size_t)(live ? id : 0) * width;
        T *dst = y + (size_t)t * width;
        if (width < E) {
            if (lane < width) SmElem<T>::store(dst + lane, live ? SmElem<T>::load(src + lane) * scale : 0.f);
            continue;
        }
        for (unsigned i = lane; i < nvec; i += GL) {
            const unsigned at = i * E + E <= (unsigned)width ? i * E : width - E;
            float f[E];
            SmElem<T>::unpack(load16_any(src + at), f);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = live ? f[e] * scale : 0.f;
            if (whole) store16_result(dst + at, SmElem<T>::pack(f), true);
            else store16_any(dst + at, SmElem<T>::pack(f));
        }
    }
}

template <typename T>
static hipError_t launch_embedding_t(int64_t tokens, int vocab, int width, float scale, const T *table, const int64_t *ids, T *y, hipStream_t st)
{
    constexpr int E = SmElem<T>::E;
    const int nvec = width / E + (width % E != 0), whole = width % E == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0;
    // a grid holds fewer than 2^32 threads: its workgroups go on with later tokens
#define NGC_EMB(GL)                                                                                                                                \
    do {                                                                                                                                           \
        const int64_t need = (tokens + 256 / (GL) - 1) / (256 / (GL)), grid = need < (1 << 23) ? need : 1 << 23;                                   \
        NGC_LAUNCH((embedding_rows<T, GL>), dim3((unsigned)grid), dim3(256), 0, st, table, ids, y, tokens, vocab, width, scale, whole);             \
    } while (0)
    if (nvec <= 8) NGC_EMB(8);
    else if (nvec <= 32) NGC_EMB(32);
    else if (nvec <= 256) NGC_EMB(64);
    else NGC_EMB(256);
#undef NGC_EMB
    return launch_result();
}

hipError_t launch_embedding(int dtype, int64_t tokens, int vocab, int width, float scale, const void *table, const int64_t *ids, void *y, hipStream_t st)
{
    if (dtype == NGC_BF16) return launch_embedding_t(tokens, vocab, width, scale, static_cast<const uint16_t *>(table), ids, static_cast<uint16_t *>(y), st);
    return launch_embedding_t(tokens, vocab, width, scale, static_cast<const float *>(table), ids, static_cast<float *>(y), st);
}

// ---- gradient ---------------------------------------------------------------------------------------------------------------
//
// The tokens are sorted by id, stably, so that a row of the gradient is the sum over a run of the sorted tokens in ascending order; ids outside
// the table drop out.  Four launches, whose order of additions the sizes alone fix:
//   1  a block of tokens per workgroup: sorted by range (a range is 2^shift neighbouring ids, at most 2048 of them); where each range begins
//   2  a workgroup per range: its tokens of all blocks, sorted by id; where each id begins.  Where a range begins among all tokens is the sum
//      over the blocks of where it begins there, so no scan over ranges is needed.  Rows without tokens are zeroed here, under the latency of
//      the ranges that have many
//   3  chunks of the sorted tokens that belong to one id: their sums (frequent ids only: padding, articles)
//   4  the rows that have tokens: tokens up to the first chunk, chunks, tokens behind the last, times scale
// Both sorts rank a wave's 64 tokens among each other with one ballot per bit of the bin, and waves own consecutive tokens.
// Up to 8192 tokens take three launches: each range looks through all tokens itself (from the L2), which costs less than a launch that sorts
// blocks (5001 tokens, 10007 rows of 777, fp32, all launches: 31.8 -> 27 us; 18935 tokens: 7.6 us for launch 1 alone).  Above,
// the looking grows with tokens x ranges.
// Bound: HBM, dy read once and dtable written once (16384 tokens of 2048 bf16 over 32000 rows: 88 us for 329 MB; launches, timed each by itself, 11, 48 with the
// zeros of 25000 rows, 6 and 30 us).
constexpr int EMB_RANGES = 2048, EMB_BLOCKS = 512, EMB_TILE = 2048, EMB_SCAN = 8192;
// Waves of a range's workgroup: the range of the frequent ids may hold a third of the tokens (18935 tokens, 18913 rows of 64: launch 2 takes 26 us
// with four, 17 with eight)
constexpr int EMB_WAVES = 8;
constexpr int EMB_MOST = 1 << 10;                        // ids of a range at most

struct EmbPlan {
    bool scan;
    int shift, ranges, blocks, chunk;
    int64_t per_block, chunks;                           // tokens of a block (a multiple of EMB_TILE)
    size_t starts, byrange, byid, rowstart, sums, total; // offsets in the workspace
};

static EmbPlan emb_plan(int64_t tokens, int vocab, int width)
{
    EmbPlan p{};
    p.scan = tokens <= EMB_SCAN;
    while (((vocab - 1) >> p.shift) >= (p.scan && vocab < EMB_MOST * 1024 ? 1024 : EMB_RANGES)) ++p.shift;
    p.ranges = ((vocab - 1) >> p.shift) + 1;
    p.per_block = (tokens + EMB_BLOCKS - 1) / EMB_BLOCKS;
    p.per_block = p.per_block < EMB_TILE ? EMB_TILE : (p.per_block + EMB_TILE - 1) / EMB_TILE * EMB_TILE;
    p.blocks = (int)((tokens + p.per_block - 1) / p.per_block);
    // A row adds up to two chunks' worth of tokens and all of its chunks one after the other: a chunk of a quarter of the root keeps both short
    p.chunk = 32;
    while ((int64_t)p.chunk * p.chunk < tokens / 16 && p.chunk < 4096) p.chunk *= 2;
    p.chunks = tokens / p.chunk;
    if (tokens < 256) {                                  // one launch less; a row of all tokens takes 32 steps
        p.chunk = 1 << 30;
        p.chunks = 0;
    }
    size_t at = 0;
    auto take = [&](size_t &where, size_t bytes) { where = at; at += (bytes + 255) & ~(size_t)255; };
    take(p.starts, p.scan ? 0 : (size_t)(p.ranges + 1) * p.blocks * 4);
    take(p.byrange, p.scan ? 0 : (size_t)tokens * 8);
    take(p.byid, (size_t)tokens * 4);
    take(p.rowstart, ((size_t)vocab + 1) * 4);
    take(p.sums, (size_t)p.chunks * width * 4);
    p.total = at;
    return p;
}

// lanes of this wave with the same bin (of `bits` bits) among the live ones
__device__ __forceinline__ uint64_t same_bin(unsigned bin, int bits, bool live)
{
    uint64_t mask = __ballot(live);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((bin >> b) & 1);
        mask &= (bin >> b) & 1 ? set : ~set;
    }
    return mask;
}

// where the next token of `bin` goes, tokens of lower lanes first; next: the wave's counters.  Called by whole waves.
__device__ __forceinline__ unsigned place_in_order(unsigned *next, unsigned bin, int bits, bool live, int lane)
{
    const uint64_t mask = same_bin(bin, bits, live);
    unsigned at = 0;
    if (live) {
        at = next[bin] + (unsigned)__popcll(mask & ((1ull << lane) - 1));
        asm volatile("" ::: "memory");                   // a wave's LDS accesses are carried out in order
        if ((mask >> lane) == 1) next[bin] = at + 1;     // the last of them
    }
    asm volatile("" ::: "memory");
    return at;
}

// exclusive sum over the 64 NW threads of a workgroup; sm: NW words.  total: of all
template <int NW>
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned *sm, unsigned &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned sum = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned t = __shfl_up(sum, o, 64);
        if (lane >= o) sum += t;
    }
    __syncthreads();
    if (lane == 63) sm[wave] = sum;
    __syncthreads();
    unsigned before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? sm[w] : 0;
        total += sm[w];
    }
    return before + sum - v;
}

// First column of a lane's group of four; false past the end (the column is then 0).  The last group overlaps the one before it (both hold the
// same sums).  ONE: a group is one column (widths below four).
template <bool ONE>
__device__ __forceinline__ bool column_of(int group, int width, int &col)
{
    const bool in = ONE ? group < width : group < (width >> 2) + ((width & 3) != 0);
    col = !in ? 0 : ONE ? group : group < (width >> 2) ? 4 * group : width - 4;
    return in;
}
template <bool ONE, typename T>
__device__ __forceinline__ float4 load_group(const T *p)
{
    if constexpr (ONE) return make_float4(SmElem<T>::load(p), 0.f, 0.f, 0.f);
    else return load4_any(p);
}
template <bool ONE>
__device__ __forceinline__ void store_group(float *p, float4 v)
{
    if constexpr (ONE) *p = v.x;
    else store16_any(p, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
}

__global__ __launch_bounds__(512) void embedding_sort_blocks(const int64_t *__restrict__ ids, uint2 *__restrict__ byrange, unsigned *__restrict__ starts,
                                                             int64_t tokens, int vocab, int shift, int bits, int ranges, int64_t per_block)
{
    extern __shared__ unsigned cnt[];                    // [8][ranges], 8 words of the scan
    unsigned *const sm = cnt + 8 * ranges;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * per_block, mine = first + wave * (per_block / 8);
    for (int i = threadIdx.x; i < 8 * ranges; i += 512) cnt[i] = 0;
    __syncthreads();
    // four steps' ids at a time (per_block / 8 is a multiple of 256)
    for (int64_t i = 0; i < per_block / 8; i += 256) {
        int64_t id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = mine + i + 64 * k + lane < tokens ? ids[mine + i + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (id[k] >= 0 && id[k] < vocab) atomicAdd(&cnt[wave * ranges + (int)(id[k] >> shift)], 1u);
    }
    __syncthreads();
    // ranges 4 tid .. 4 tid + 3: what lies in front of each, wave by wave
    unsigned own[EMB_RANGES / 512], sum = 0, total;
#pragma unroll
    for (int k = 0; k < EMB_RANGES / 512; ++k) {
        const int r = threadIdx.x * (EMB_RANGES / 512) + k;
        own[k] = 0;
        if (r < ranges)
            for (int w = 0; w < 8; ++w) own[k] += cnt[w * ranges + r];
        sum += own[k];
    }
    unsigned at = block_scan<8>(sum, sm, total);
#pragma unroll
    for (int k = 0; k < EMB_RANGES / 512; ++k) {
        const int r = threadIdx.x * (EMB_RANGES / 512) + k;
        if (r < ranges) {
            starts[(size_t)r * gridDim.x + blockIdx.x] = at;
            unsigned w0 = at;
            for (int w = 0; w < 8; ++w) {
                const unsigned c = cnt[w * ranges + r];
                cnt[w * ranges + r] = w0;
                w0 += c;
            }
        }
        at += own[k];
    }
    if (threadIdx.x == 0) starts[(size_t)ranges * gridDim.x + blockIdx.x] = total;
    __syncthreads();
    for (int64_t i = 0; i < per_block / 8; i += 256) {
        int64_t id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = mine + i + 64 * k + lane < tokens ? ids[mine + i + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool live = id[k] >= 0 && id[k] < vocab;
            const unsigned to = place_in_order(cnt + wave * ranges, live ? (unsigned)(id[k] >> shift) : 0u, bits, live, lane);
            if (live) byrange[first + to] = make_uint2((unsigned)(mine + i + 64 * k + lane), (unsigned)id[k] & ((1u << shift) - 1));
        }
    }
}

// Second half of the sort, by a workgroup of NW waves: the tokens of a range, of which wave w holds entries lo .. hi - 1 (token, id within the range), all
// waves' in the tokens' order; base: tokens of lower ids.  cnt: NW x size words, none: size bytes, sm: NW words of LDS.
template <int NW, class F>
__device__ __forceinline__ void sort_range(unsigned lo, unsigned hi, F entry, unsigned base, unsigned all, int range, bool last, int shift, unsigned *cnt, uint8_t *none,
                                           unsigned *sm, unsigned *__restrict__ byid, unsigned *__restrict__ rowstart, float *__restrict__ dtable, int vocab, int width)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, size = 1 << shift;
    for (int i = threadIdx.x; i < NW * size; i += 64 * NW) cnt[i] = 0;
    __syncthreads();
    if (size > 1) {
        for (unsigned e = lo + lane; e < hi; e += 256) {
            unsigned id[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) id[k] = e + 64 * k < hi ? entry(e + 64 * k).y : 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (e + 64 * k < hi) atomicAdd(&cnt[wave * size + id[k]], 1u);
        }
    } else if (lane == 0) {
        cnt[wave] = hi > lo ? hi - lo : 0;
    }
    __syncthreads();
    unsigned sum = 0, total;
    const int rows = (size + 64 * NW - 1) / (64 * NW);                 // ids of a thread
    for (int k = 0; k < rows; ++k) {
        const int r = threadIdx.x * rows + k;
        if (r < size)
            for (int w = 0; w < NW; ++w) sum += cnt[w * size + r];
    }
    unsigned at = block_scan<NW>(sum, sm, total);
    for (int k = 0; k < rows; ++k) {
        const int r = threadIdx.x * rows + k;
        if (r >= size) break;
        const int64_t v = ((int64_t)range << shift) + r;
        if (v <= vocab) rowstart[v] = base + at;         // v = vocab: the end of the last row, if it falls inside the last range
        const unsigned begin = at;
        for (int w = 0; w < NW; ++w) {
            const unsigned c = cnt[w * size + r];
            cnt[w * size + r] = at;
            at += c;
        }
        none[r] = at == begin && v < vocab;
    }
    if (last && threadIdx.x == 0) rowstart[vocab] = base + all;
    __syncthreads();
    for (unsigned e = lo; e < hi; e += 256) {
        uint2 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = e + 64 * k + lane < hi ? entry(e + 64 * k + lane) : make_uint2(0, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool live = e + 64 * k + lane < hi;
            const unsigned to = place_in_order(cnt + wave * size, v[k].y, shift, live, lane);
            if (live) byid[base + to] = v[k].x;
        }
    }
    // Zeros of a row as whole 16 bytes of memory, wherever it begins, by as many lanes as it has of them (62700 rows of 19 columns: 28 -> 11 us
    // against all lanes on a row).  Rows of whole 128-byte lines are streamed past the cache, which keeps dy there (16384 tokens bf16, 32000 rows
    // of 2048, all launches: 98 -> 91 us); lines that two rows share are not (206 MB of rows of 2209: 60 us streamed, 32 us through the cache)
    const bool lines = (width & 31) == 0 && (reinterpret_cast<uintptr_t>(dtable) & 127) == 0;
    const int lanes = width <= 32 ? 8 : width <= 1024 ? 64 : 256;
    const uint64_t skew = (reinterpret_cast<uintptr_t>(dtable) >> 2) & 3;
    float *const grid16 = dtable - skew;
    for (int r = threadIdx.x / lanes; r < size; r += 64 * NW / lanes) {
        if (!none[r]) continue;
        const uint64_t from = (uint64_t)(((int64_t)range << shift) + r) * width + skew, to = from + width, q0 = (from + 3) >> 2, q1 = to >> 2;
        const int l = threadIdx.x & (lanes - 1);
        for (uint64_t q = q0 + l; q < q1; q += lanes) store16_result(grid16 + 4 * q, make_uint4(0, 0, 0, 0), lines);
        if (l < 8) {                                     // up to three floats in front and behind (or all of a row inside one 16 bytes)
            const uint64_t i = l < 4 ? from + l : (q1 >= q0 ? 4 * q1 : to) + (l - 4);
            if (l < 4 ? i < to && i < 4 * q0 : i < to) grid16[i] = 0.f;
        }
    }
}

__global__ __launch_bounds__(64 * EMB_WAVES) void embedding_sort_ranges(const uint2 *__restrict__ byrange, const unsigned *__restrict__ starts, unsigned *__restrict__ byid,
                                                             unsigned *__restrict__ rowstart, float *__restrict__ dtable, int vocab, int width, int shift, int blocks,
                                                             int64_t per_block)
{
    __shared__ unsigned pre[EMB_BLOCKS + 1], from[EMB_BLOCKS], cnt[EMB_WAVES * EMB_MOST], sm[EMB_WAVES];
    __shared__ uint8_t none[EMB_MOST];
    const int wave = threadIdx.x >> 6, range = blockIdx.x;
    unsigned base = 0, all = 0;
    static_assert(EMB_BLOCKS == 64 * EMB_WAVES, "a block a thread");
    // segments of this range: a block a thread
    const int b = threadIdx.x;
    unsigned s0 = 0, len = 0;
    if (b < blocks) {
        s0 = starts[(size_t)range * blocks + b];
        len = starts[(size_t)(range + 1) * blocks + b] - s0;
    }
    pre[b] = block_scan<EMB_WAVES>(len, sm, all);
    from[b] = s0;
    if (b == 0) pre[EMB_BLOCKS] = all;
    (void)block_scan<EMB_WAVES>(s0, sm, base);           // base: tokens of lower ids
    const unsigned per_wave = (all + 64 * EMB_WAVES - 1) / (64 * EMB_WAVES) * 64, lo = wave * per_wave, hi = lo + per_wave < all ? lo + per_wave : all;
    auto entry = [&](unsigned e) {                       // the block whose segment holds entry e
        int a = 0, b = blocks;
        while (b - a > 1) {
            const int m = (a + b) >> 1;
            if (pre[m] <= e) a = m;
            else b = m;
        }
        return byrange[a * per_block + from[a] + (e - pre[a])];
    };
    sort_range<EMB_WAVES>(lo, hi, entry, base, all, range, range == (int)gridDim.x - 1, shift, cnt, none, sm, byid, rowstart, dtable, vocab, width);
}

static unsigned scan_lds(int tokens, int shift) { return ((tokens + 255) / 256 * 256 + (4 << shift) + 4) * 4 + (1 << shift); }

// SCAN: a wave looks through a quarter of the tokens, keeps those of the range in their order and counts those of lower ids
__global__ __launch_bounds__(256) void embedding_sort_scan(const int64_t *__restrict__ ids, unsigned *__restrict__ byid, unsigned *__restrict__ rowstart,
                                                           float *__restrict__ dtable, int tokens, int vocab, int width, int shift)
{
    // as much LDS as the sizes need: few tokens leave room for eight workgroups on a compute unit
    extern __shared__ unsigned space[];                  // scan_lds words
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, range = blockIdx.x, size = 1 << shift;
    const int share = (tokens + 255) / 256 * 64;
    unsigned *const list = space + wave * share, *const cnt = space + 4 * share, *const sm = cnt + 4 * size;
    uint8_t *const none = reinterpret_cast<uint8_t *>(sm + 4);
    const int t0 = wave * share, t1 = t0 + share < tokens ? t0 + share : tokens;
    unsigned mine = 0, lower = 0;
    for (int t = t0; t < t1; t += 512) {
        int64_t id[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) id[k] = t + 64 * k + lane < t1 ? ids[t + 64 * k + lane] : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool live = id[k] >= 0 && id[k] < vocab;
            const int r = live ? (int)(id[k] >> shift) : -1;
            const uint64_t here = __ballot(r == range);
            if (r == range) list[mine + __popcll(here & ((1ull << lane) - 1))] = (unsigned)(t + 64 * k + lane) << 16 | ((unsigned)id[k] & ((1u << shift) - 1));
            mine += __popcll(here);
            lower += __popcll(__ballot(live && r < range));
        }
    }
    unsigned base, all;
    (void)block_scan<4>(lane == 0 ? lower : 0, sm, base);
    (void)block_scan<4>(lane == 0 ? mine : 0, sm, all);
    auto entry = [&](unsigned e) { return make_uint2(list[e] >> 16, list[e] & 0xFFFFu); };
    sort_range<4>(0, mine, entry, base, all, range, range == (int)gridDim.x - 1, shift, cnt, none, sm, byid, rowstart, dtable, vocab, width);
}

// sum[u] += rows row(lo) .. row(hi - 1) of dy, columns col[u] ..; U groups per lane.  lo and hi are the same in all lanes.  The loads of B rows are
// under way at a time (past the end: the last row again, not added), their additions are in that order.
template <bool ONE, int U, int B, typename T, typename F>
__device__ __forceinline__ void add_rows(float4 (&sum)[U], const T *__restrict__ dy, F row, unsigned lo, unsigned hi, int width, const int (&col)[U])
{
    for (unsigned i = lo; i < hi; i += B) {
        unsigned t[B];
        float4 v[B][U];
#pragma unroll
        for (int k = 0; k < B; ++k) t[k] = row(i + k < hi ? i + k : hi - 1);
#pragma unroll
        for (int k = 0; k < B; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u) v[k][u] = load_group<ONE>(dy + (size_t)t[k] * width + col[u]);
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const bool in = i + k < hi;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                sum[u].x += in ? v[k][u].x : 0.f;
                sum[u].y += in ? v[k][u].y : 0.f;
                sum[u].z += in ? v[k][u].z : 0.f;
                sum[u].w += in ? v[k][u].w : 0.f;
            }
        }
    }
}

template <bool ONE, typename T>
__global__ __launch_bounds__(256) void embedding_sum_chunks(const T *__restrict__ dy, const int64_t *__restrict__ ids, const unsigned *__restrict__ byid,
                                                            const unsigned *__restrict__ rowstart, float *__restrict__ sums, int vocab, int width, int chunk)
{
    const unsigned lo = blockIdx.x * (unsigned)chunk, hi = lo + chunk;
    if (hi > rowstart[vocab] || ids[byid[lo]] != ids[byid[hi - 1]]) return;         // uniform
    for (int g0 = blockIdx.y * 256; 4 * (int64_t)g0 < width; g0 += gridDim.y * 256) {
        float4 sum[1] = {make_float4(0.f, 0.f, 0.f, 0.f)};
        int col[1];
        const bool in = column_of<ONE>(g0 + threadIdx.x, width, col[0]);
        add_rows<ONE, 1, 16>(sum, dy, [&](unsigned i) { return byid[i]; }, lo, hi, width, col);
        if (in) store_group<ONE>(sums + (size_t)blockIdx.x * width + col[0], sum[0]);
    }
}

// A unit of UW waves goes through rows unit, unit + units, ...: it looks at 64 of them at a time and adds up those that have tokens.  Neighbouring
// ids, of which the low ones are often the frequent ones, fall to different units.
template <bool ONE, int UW, int U, typename T>
__global__ __launch_bounds__(256) void embedding_sum_rows(const T *__restrict__ dy, const unsigned *__restrict__ byid, const unsigned *__restrict__ rowstart,
                                                          const float *__restrict__ sums, float *__restrict__ dtable, int vocab, int width, int chunk,
                                                          float scale)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int unit = blockIdx.x * (4 / UW) + wave / UW, units = gridDim.x * (4 / UW), at = (wave % UW) * 64 + lane;
    for (int64_t v0 = unit; v0 < vocab; v0 += (int64_t)units * 64) {
        const int64_t mine = v0 + (int64_t)lane * units;
        unsigned first = 0, last = 0;
        if (mine < vocab) {
            first = rowstart[mine];
            last = rowstart[mine + 1];
        }
        for (uint64_t todo = __ballot(last > first); todo; todo &= todo - 1) {
            const int k = __ffsll((unsigned long long)todo) - 1;
            const unsigned lo = __builtin_amdgcn_readlane(first, k), hi = __builtin_amdgcn_readlane(last, k);
            const unsigned c0 = (lo + chunk - 1) / chunk, c1 = hi / chunk;          // chunks inside, if c0 < c1
            const auto token = [&](unsigned i) { return byid[i]; };
            float *out = dtable + (size_t)(v0 + (int64_t)k * units) * width;
            for (int g0 = 0; 4 * (int64_t)g0 < width; g0 += UW * 64 * U) {
                float4 sum[U];
                int col[U];
                bool in[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    sum[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                    in[u] = column_of<ONE>(g0 + u * UW * 64 + at, width, col[u]);
                }
                add_rows<ONE, U, 8>(sum, dy, token, lo, c0 < c1 ? c0 * chunk : hi, width, col);
                if (c0 < c1) {
                    add_rows<ONE, U, 8>(sum, sums, [](unsigned c) { return c; }, c0, c1, width, col);
                    add_rows<ONE, U, 8>(sum, dy, token, c1 * chunk, hi, width, col);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (in[u]) store_group<ONE>(out + col[u], make_float4(sum[u].x * scale, sum[u].y * scale, sum[u].z * scale, sum[u].w * scale));
            }
        }
    }
}

size_t embedding_bwd_workspace(int64_t tokens, int vocab, int width) { return emb_plan(tokens, vocab, width).total; }

template <typename T>
static hipError_t launch_embedding_bwd_t(int64_t tokens, int vocab, int width, float scale, const T *dy, const int64_t *ids, float *dtable, char *ws, hipStream_t st)
{
    const EmbPlan p = emb_plan(tokens, vocab, width);
    unsigned *starts = reinterpret_cast<unsigned *>(ws + p.starts), *byid = reinterpret_cast<unsigned *>(ws + p.byid), *rowstart = reinterpret_cast<unsigned *>(ws + p.rowstart);
    uint2 *byrange = reinterpret_cast<uint2 *>(ws + p.byrange);
    float *sums = reinterpret_cast<float *>(ws + p.sums);
    hipError_t e;
    if (p.scan) {
        NGC_LAUNCH(embedding_sort_scan, dim3(p.ranges), dim3(256), scan_lds((int)tokens, p.shift), st, ids, byid, rowstart, dtable, (int)tokens, vocab, width, p.shift);
    } else {
        int bits = 0;
        while ((1 << bits) < p.ranges) ++bits;
        static LdsLimitOnce lds;
        if ((e = lds.raise(reinterpret_cast<const void *>(&embedding_sort_blocks))) != hipSuccess) return e;
        NGC_LAUNCH(embedding_sort_blocks, dim3(p.blocks), dim3(512), (p.ranges + 1) * 8 * 4, st, ids, byrange, starts, tokens, vocab, p.shift, bits, p.ranges, p.per_block);
        if ((e = launch_result()) != hipSuccess) return e;
        NGC_LAUNCH(embedding_sort_ranges, dim3(p.ranges), dim3(64 * EMB_WAVES), 0, st, byrange, starts, byid, rowstart, dtable, vocab, width, p.shift, p.blocks, p.per_block);
    }
    if ((e = launch_result()) != hipSuccess) return e;
    const int groups = width < 4 ? width : width / 4 + (width % 4 != 0);
    if (p.chunks) {
        int64_t slices = ((int64_t)groups + 255) / 256;
        if (slices > (1 << 23) / p.chunks + 1) slices = (1 << 23) / p.chunks + 1;   // a grid holds fewer than 2^32 threads
        const auto kernel = width < 4 ? embedding_sum_chunks<true, T> : embedding_sum_chunks<false, T>;
        NGC_LAUNCH(kernel, dim3((unsigned)p.chunks, (unsigned)(slices < 65535 ? slices : 65535)), dim3(256), 0, st, dy, ids, byid, rowstart, sums, vocab, width, p.chunk);
        if ((e = launch_result()) != hipSuccess) return e;
    }
#define NGC_EMB_ROWS(ONE, UW, U)                                                                                                                       \
    do {                                                                                                                                           \
        const int need = (vocab + 4 / (UW) - 1) / (4 / (UW));                                                                                       \
        NGC_LAUNCH((embedding_sum_rows<ONE, UW, U, T>), dim3(need < 2048 ? need : 2048), dim3(256), 0, st, dy, byid, rowstart, sums, dtable, vocab, width,  \
                   p.chunk, scale);                                                                                                                \
    } while (0)
    if (width < 4) NGC_EMB_ROWS(true, 1, 1);
    else if (groups <= 64) NGC_EMB_ROWS(false, 1, 1);
    else if (groups <= 128) NGC_EMB_ROWS(false, 2, 1);
    else if (groups <= 256) NGC_EMB_ROWS(false, 4, 1);
    else NGC_EMB_ROWS(false, 4, 2);
#undef NGC_EMB_ROWS
    return launch_result();
}

hipError_t launch_embedding_bwd(int dtype, int64_t tokens, int vocab, int width, float scale, const void *dy, const int64_t *ids, float *dtable, void *ws,
                                hipStream_t st)
{
    if (dtype == NGC_BF16) return launch_embedding_bwd_t(tokens, vocab, width, scale, static_cast<const uint16_t *>(dy), ids, dtable, static_cast<char *>(ws), st);
    return launch_embedding_bwd_t(tokens, vocab, width, scale, static_cast<const float *>(dy), ids, dtable, static_cast<char *>(ws), st);
}

}  // namespace ngc
