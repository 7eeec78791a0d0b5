// Layer norm over the last axis of a [rows, cols] tensor and its backprop (gfx950).
//
//   mean = sum_j x[j] / cols,  rstd = (sum_j (x[j] - mean)^2 / cols + eps)^(-1/2)
//   y[j] = (x[j] - mean) rstd gamma[j] + beta[j]
//   g = dy gamma, xh = (x - mean) rstd:  dx[j] = rstd (g[j] - sum_k g[k] / cols - xh[j] sum_k g[k] xh[k] / cols)
//   dgamma[j] = sum over the rows of dy[j] xh[j],  dbeta[j] = sum over the rows of dy[j]
//
// Bound: HBM (forward one read and one write of the tensor, backprop two reads and one write).  A row lives in the registers of a group of
// lanes, 8 to 64 of a wave or a workgroup, as vectors of 16 bytes; the variance is the sum of squared differences from the mean that the same
// registers gave, not a difference of sums.  A group goes through several rows: gamma and beta stay in registers (read for every row they are
// twice the traffic of a bf16 row out of the caches) and the next row is on its way while the current one is reduced.  In the backprop the
// same lanes add up their columns' dgamma and dbeta over the group's rows; the groups' sums are joined by a second launch in a fixed order.
// Rows that are no multiple of 16 bytes end in a vector that overlaps the one before it, as softmax's.  Rows beyond the registers take a
// workgroup each and three passes (backprop two, and the columns' sums a pass of their own); rows below 16 bytes a thread each.
// 16384 x 4096 bf16: forward 43 us, 6.2 TB/s; backprop 76 us, 5.3 TB/s, and 5 us for the second launch.  8 rows: 3.5 us.  Backprop of 4096 fp32 rows: 8192
// columns, in registers, 78 + 5 us, 5.2 TB/s; 16384, beyond them, 191 + 98 + 5 us, as x and dy are read three times.
#include "rows.h"

namespace ngc {

// sum over the 64 NW threads of a workgroup, fixed order; slot: a pair of NW words, another one than in the call before
template <int NW>
__device__ __forceinline__ float2 block_sum2(float2 v, float2 *slot)
{
    v.x = group_sum<64>(v.x);
    v.y = group_sum<64>(v.y);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) v.x += slot[w].x, v.y += slot[w].y;
    return v;
}

// E fp32 values at any 4-byte address
template <int E>
__device__ __forceinline__ void load_floats(const float *p, float (&f)[E])
{
#pragma unroll
    for (int k = 0; k < E; k += 4) {
        const uint4 v = load16_any(p + k);
        f[k] = __uint_as_float(v.x); f[k + 1] = __uint_as_float(v.y); f[k + 2] = __uint_as_float(v.z); f[k + 3] = __uint_as_float(v.w);
    }
}

// The vectors of a row in a group of GL lanes: vector vi begins at first(vi); of the last one only the elements that the vector before it does
// not hold count.
template <typename T, int GL, bool TAIL>
struct RowVectors {
    static constexpr int E = SmElem<T>::E;
    int cols, nvec, lane;
    __device__ __forceinline__ RowVectors(int c) : cols(c), nvec(TAIL ? (int)(((unsigned)c + E - 1) / E) : c / E), lane(threadIdx.x & (GL - 1)) {}
    __device__ __forceinline__ int index(int j) const { return j * GL + lane; }
    __device__ __forceinline__ bool has(int j) const { return index(j) < nvec; }
    __device__ __forceinline__ int first(int j) const { return TAIL && (index(j) + 1) * E > cols ? cols - E : index(j) * E; }
    __device__ __forceinline__ bool counts(int j, int e) const { return has(j) && (!TAIL || e >= (index(j) + 1) * E - cols); }
};

template <typename T, int V, int GL, bool TAIL>
__global__ __launch_bounds__(GL <= 64 ? 256 : GL) void layer_norm_reg(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd,
                                                                      int rows, int cols, float eps)
{
    constexpr int E = SmElem<T>::E, RPW = GL <= 64 ? 256 / GL : 1, NW = GL <= 64 ? 1 : GL / 64;
    constexpr bool KEEP = V * E <= 16 || GL < 1024;      // gamma and beta in registers
    __shared__ float2 sm[2][NW];
    const RowVectors<T, GL, TAIL> at(cols);
    const int group = threadIdx.x / GL;
    float ga[V][E], be[V][E];
    auto affine = [&](int j) {
#pragma unroll
        for (int e = 0; e < E; ++e) ga[j][e] = 1.f, be[j][e] = 0.f;
        if (gamma && at.has(j)) load_floats<E>(gamma + at.first(j), ga[j]);
        if (beta && at.has(j)) load_floats<E>(beta + at.first(j), be[j]);
    };
    if (KEEP)
#pragma unroll
        for (int j = 0; j < V; ++j) affine(j);
    uint4 next[V];
    auto load = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            next[j] = make_uint4(0, 0, 0, 0);
            if (row < rows && at.has(j)) next[j] = load16_any(x + (size_t)row * cols + at.first(j));
        }
    };
    const float inv = 1.0f / (float)cols;
    auto total = [&](float v, int slot) {
        if constexpr (GL <= 64) return group_sum<GL>(v);
        else return block_sum2<NW>(make_float2(v, 0.f), sm[slot]).x;
    };
    load((int64_t)blockIdx.x * RPW + group);
    for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < rows; r0 += (int64_t)gridDim.x * RPW) {
        const int64_t row = r0 + group;
        uint4 cur[V];
        float f[E], s = 0.f, q = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) cur[j] = next[j];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            SmElem<T>::unpack(cur[j], f);
#pragma unroll
            for (int e = 0; e < E; ++e) s += !TAIL || at.counts(j, e) ? f[e] : 0.f;                 // zeros past the end
        }
        const float mu = total(s, 0) * inv;
        load(row + (int64_t)gridDim.x * RPW);            // behind the wait for this row
#pragma unroll
        for (int j = 0; j < V; ++j) {
            SmElem<T>::unpack(cur[j], f);
#pragma unroll
            for (int e = 0; e < E; ++e) q += at.counts(j, e) ? (f[e] - mu) * (f[e] - mu) : 0.f;
        }
        const float rs = 1.0f / sqrtf(total(q, 1) * inv + eps);
        if (row >= rows) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!at.has(j)) continue;
            if (!KEEP) affine(j);
            SmElem<T>::unpack(cur[j], f);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = fmaf((f[e] - mu) * rs, ga[j][e], be[j][e]);
            if (TAIL) store16_any(y + (size_t)row * cols + at.first(j), SmElem<T>::pack(f));
            else store16_result(y + (size_t)row * cols + at.first(j), SmElem<T>::pack(f), true);
        }
        if (at.lane == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = rs;
        }
    }
}

// part: [workgroups][2][cols], dgamma's sums and dbeta's; NULL: not asked for
template <typename T, int V, int GL, bool TAIL>
__global__ __launch_bounds__(GL <= 64 ? 256 : GL) void layer_norm_bwd_reg(const T *x, const float *gamma, const float *mean, const float *rstd, const T *dy,
                                                                          T *dx, float *part, int rows, int cols)
{
    constexpr int E = SmElem<T>::E, RPW = GL <= 64 ? 256 / GL : 1, NW = GL <= 64 ? 1 : GL / 64;
    __shared__ float2 sm[2][NW];
    __shared__ float sums[RPW > 1 ? RPW - 1 : 1][RPW > 1 ? GL * E : 1];
    const RowVectors<T, GL, TAIL> at(cols);
    const int group = threadIdx.x / GL;
    float ga[V][E], dg[V][E], db[V][E];
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int e = 0; e < E; ++e) ga[j][e] = 1.f, dg[j][e] = db[j][e] = 0.f;
        if (gamma && at.has(j)) load_floats<E>(gamma + at.first(j), ga[j]);
    }
    uint4 nx[V], ny[V];
    float nmu = 0.f, nrs = 0.f;
    auto load = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            nx[j] = ny[j] = make_uint4(0, 0, 0, 0);
            if (row < rows && at.has(j)) {
                nx[j] = load16_any(x + (size_t)row * cols + at.first(j));
                ny[j] = load16_any(dy + (size_t)row * cols + at.first(j));
            }
        }
        if (row < rows) nmu = mean[row], nrs = rstd[row];
    };
    const float inv = 1.0f / (float)cols;
    constexpr bool AHEAD = V * E <= 16;                  // the next row is loaded under this one's sums (else the registers do not hold it)
    if (AHEAD) load((int64_t)blockIdx.x * RPW + group);
    int slot = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * RPW; r0 < rows; r0 += (int64_t)gridDim.x * RPW, slot ^= 1) {
        const int64_t row = r0 + group;
        if (!AHEAD) load(row);
        const float mu = nmu, rs = nrs;
        uint4 cx[V], cy[V];
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < V; ++j) cx[j] = nx[j], cy[j] = ny[j];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float a[E], b[E];
            SmElem<T>::unpack(cx[j], a);
            SmElem<T>::unpack(cy[j], b);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float xh = (a[e] - mu) * rs, d = row < rows && at.counts(j, e) ? b[e] : 0.f, g = d * ga[j][e];
                s.x += g;
                s.y = fmaf(g, xh, s.y);
                dg[j][e] = fmaf(d, xh, dg[j][e]);
                db[j][e] += d;
            }
        }
        if (!AHEAD) {
            keep_packed(cx);
            keep_packed(cy);
        }
        if constexpr (GL <= 64) s = make_float2(group_sum<GL>(s.x), group_sum<GL>(s.y));
        else s = block_sum2<NW>(s, sm[slot]);
        if (AHEAD) load(row + (int64_t)gridDim.x * RPW);                 // behind the wait for this row
        if (row >= rows) continue;
        const float ma = s.x * inv, mb = s.y * inv;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!at.has(j)) continue;
            float a[E], b[E];
            SmElem<T>::unpack(cx[j], a);
            SmElem<T>::unpack(cy[j], b);
#pragma unroll
            for (int e = 0; e < E; ++e) b[e] = rs * (b[e] * ga[j][e] - ma - (a[e] - mu) * rs * mb);
            if (TAIL) store16_any(dx + (size_t)row * cols + at.first(j), SmElem<T>::pack(b));
            else store16_result(dx + (size_t)row * cols + at.first(j), SmElem<T>::pack(b), true);
        }
    }
    if (!part) return;
    // the groups of a workgroup hold the same columns
    float *out = part + (size_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            float (&mine)[E] = w ? db[j] : dg[j];
            if constexpr (RPW > 1) {
                __syncthreads();
                if (group)
#pragma unroll
                    for (int e = 0; e < E; ++e) sums[group - 1][e * GL + at.lane] = mine[e];
                __syncthreads();
                if (group) continue;
                for (int o = 0; o < RPW - 1; ++o)
#pragma unroll
                    for (int e = 0; e < E; ++e) mine[e] += sums[o][e * GL + at.lane];
            }
            // an element that two vectors hold is stored by the one that counted it
            if (at.has(j))
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at.counts(j, e)) out[(size_t)w * cols + at.first(j) + e] = mine[e];
        }
}

// Rows of any length >= E: a workgroup of 1024 per row.  The last elements, less than a vector, go one by one.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_long(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd, int cols,
                                                        float eps)
{
    constexpr int E = SmElem<T>::E;
    __shared__ float2 sm[2][16];
    const size_t base = (size_t)blockIdx.x * cols;
    const int nvec = cols / E;
    const int64_t rest = (int64_t)nvec * E + threadIdx.x;
    const float inv = 1.0f / (float)cols, tail = rest < cols ? SmElem<T>::load(x + base + rest) : 0.f;
    float s = tail, q = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x; i < nvec; i += 1024) {
        float f[E];
        SmElem<T>::unpack(load16_any(x + base + (size_t)i * E), f);
#pragma unroll
        for (int e = 0; e < E; ++e) s += f[e];
    }
    const float mu = block_sum2<16>(make_float2(s, 0.f), sm[0]).x * inv;
    if (rest < cols) q = (tail - mu) * (tail - mu);
#pragma unroll 4
    for (int i = threadIdx.x; i < nvec; i += 1024) {
        float f[E];
        SmElem<T>::unpack(load16_any(x + base + (size_t)i * E), f);
#pragma unroll
        for (int e = 0; e < E; ++e) q += (f[e] - mu) * (f[e] - mu);
    }
    const float rs = 1.0f / sqrtf(block_sum2<16>(make_float2(q, 0.f), sm[1]).x * inv + eps);
#pragma unroll 2
    for (int i = threadIdx.x; i < nvec; i += 1024) {
        float f[E], ga[E], be[E];
        SmElem<T>::unpack(load16_any(x + base + (size_t)i * E), f);
#pragma unroll
        for (int e = 0; e < E; ++e) ga[e] = 1.f, be[e] = 0.f;
        if (gamma) load_floats<E>(gamma + (size_t)i * E, ga);
        if (beta) load_floats<E>(beta + (size_t)i * E, be);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = fmaf((f[e] - mu) * rs, ga[e], be[e]);
        store16_any(y + base + (size_t)i * E, SmElem<T>::pack(f));
    }
    if (rest < cols) SmElem<T>::store(y + base + rest, fmaf((tail - mu) * rs, gamma ? gamma[rest] : 1.f, beta ? beta[rest] : 0.f));
    if (threadIdx.x == 0) {
        if (mean) mean[blockIdx.x] = mu;
        if (rstd) rstd[blockIdx.x] = rs;
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_bwd_long(const T *x, const float *gamma, const float *mean, const float *rstd, const T *dy, T *dx,
                                                            int cols)
{
    constexpr int E = SmElem<T>::E;
    __shared__ float2 sm[16];
    const size_t base = (size_t)blockIdx.x * cols;
    const int nvec = cols / E;
    const int64_t rest = (int64_t)nvec * E + threadIdx.x;
    const float mu = mean[blockIdx.x], rs = rstd[blockIdx.x], inv = 1.0f / (float)cols;
    float2 s = make_float2(0.f, 0.f);
    float tg = 0.f, tx = 0.f;
    if (rest < cols) {
        tg = SmElem<T>::load(dy + base + rest) * (gamma ? gamma[rest] : 1.f);
        tx = (SmElem<T>::load(x + base + rest) - mu) * rs;
        s = make_float2(tg, tg * tx);
    }
    auto vec = [&](int i, float (&g)[E], float (&xh)[E]) {
        float ga[E];
        SmElem<T>::unpack(load16_any(dy + base + (size_t)i * E), g);
        SmElem<T>::unpack(load16_any(x + base + (size_t)i * E), xh);
        if (gamma) load_floats<E>(gamma + (size_t)i * E, ga);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (gamma) g[e] *= ga[e];
            xh[e] = (xh[e] - mu) * rs;
        }
    };
#pragma unroll 2
    for (int i = threadIdx.x; i < nvec; i += 1024) {
        float g[E], xh[E];
        vec(i, g, xh);
#pragma unroll
        for (int e = 0; e < E; ++e) s.x += g[e], s.y = fmaf(g[e], xh[e], s.y);
    }
    s = block_sum2<16>(s, sm);
    const float ma = s.x * inv, mb = s.y * inv;
#pragma unroll 2
    for (int i = threadIdx.x; i < nvec; i += 1024) {
        float g[E], xh[E];
        vec(i, g, xh);
#pragma unroll
        for (int e = 0; e < E; ++e) g[e] = rs * (g[e] - ma - xh[e] * mb);
        store16_any(dx + base + (size_t)i * E, SmElem<T>::pack(g));
    }
    if (rest < cols) SmElem<T>::store(dx + base + rest, rs * (tg - ma - tx * mb));
}

// Rows below one vector: a thread per row.
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_tiny(const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd, int rows, int cols,
                                                       float eps)
{
    constexpr int E = SmElem<T>::E;
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= rows) return;
    float f[E], s = 0.f, q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += f[e] = e < cols ? SmElem<T>::load(x + (size_t)row * cols + e) : 0.f;
    const float mu = s / (float)cols;
#pragma unroll
    for (int e = 0; e < E; ++e) q += e < cols ? (f[e] - mu) * (f[e] - mu) : 0.f;
    const float rs = 1.0f / sqrtf(q / (float)cols + eps);
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < cols) SmElem<T>::store(y + (size_t)row * cols + e, fmaf((f[e] - mu) * rs, gamma ? gamma[e] : 1.f, beta ? beta[e] : 0.f));
    if (mean) mean[row] = mu;
    if (rstd) rstd[row] = rs;
}

template <typename T>
__global__ __launch_bounds__(256) void layer_norm_bwd_tiny(const T *x, const float *gamma, const float *mean, const float *rstd, const T *dy, T *dx,
                                                           int rows, int cols)
{
    constexpr int E = SmElem<T>::E;
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= rows) return;
    const float mu = mean[row], rs = rstd[row];
    float g[E], xh[E], a = 0.f, b = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        g[e] = e < cols ? SmElem<T>::load(dy + (size_t)row * cols + e) * (gamma ? gamma[e] : 1.f) : 0.f;
        xh[e] = e < cols ? (SmElem<T>::load(x + (size_t)row * cols + e) - mu) * rs : 0.f;
        a += g[e];
        b = fmaf(g[e], xh[e], b);
    }
    a /= (float)cols;
    b /= (float)cols;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < cols) SmElem<T>::store(dx + (size_t)row * cols + e, rs * (g[e] - a - xh[e] * b));
}

// Columns' sums over a chunk of rows, for the rows of the last two kinds; 64 columns, four rows at a time
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_bwd_cols(const T *__restrict__ x, const float *__restrict__ mean, const float *__restrict__ rstd,
                                                           const T *__restrict__ dy, float *__restrict__ part, int rows, int cols, int chunk)
{
    __shared__ float2 sm[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * chunk, r1 = rows - r0 < chunk ? rows : r0 + chunk;
    float *out = part + (size_t)blockIdx.x * 2 * cols;
    for (int64_t j0 = (int64_t)blockIdx.y * 64; j0 < cols; j0 += (int64_t)gridDim.y * 64) {
        const int64_t j = j0 + lane;
        float2 s = make_float2(0.f, 0.f);
        if (j < cols)
#pragma unroll 4
            for (int64_t r = r0 + wave; r < r1; r += 4) {
                const float d = SmElem<T>::load(dy + (size_t)r * cols + j);
                s.x = fmaf(d, (SmElem<T>::load(x + (size_t)r * cols + j) - mean[r]) * rstd[r], s.x);
                s.y += d;
            }
        __syncthreads();
        if (wave) sm[wave - 1][lane] = s;
        __syncthreads();
        if (wave || j >= cols) continue;
#pragma unroll
        for (int w = 0; w < 3; ++w) s.x += sm[w][lane].x, s.y += sm[w][lane].y;
        out[j] = s.x;
        out[cols + j] = s.y;
    }
}

// dgamma (blockIdx.y = 0) or dbeta of 32 columns from the parts, eight threads a column
__global__ __launch_bounds__(256) void layer_norm_bwd_join(const float *__restrict__ part, float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                           int parts, int cols)
{
    __shared__ float sm[8][32];
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    for (int64_t j0 = (int64_t)blockIdx.x * 32; j0 < cols; j0 += (int64_t)gridDim.x * 32) {
        const int64_t j = j0 + c;
        float s = 0.f;
        if (j < cols)
#pragma unroll 8
            for (int p = q; p < parts; p += 8) s += part[((size_t)p * 2 + blockIdx.y) * cols + j];
        __syncthreads();
        sm[q][c] = s;
        __syncthreads();
        if (q || j >= cols) continue;
#pragma unroll
        for (int w = 1; w < 8; ++w) s += sm[w][c];
        out[j] = s;
    }
}

// How rows of this length are taken: below one vector a thread per row; else the smallest group of lanes and the fewest vectors per lane that
// hold the row; else a workgroup per row that walks it several times.
enum NormKernel { LN_TINY, LN_REG, LN_LONG };
struct NormPlan {
    NormKernel kernel;
    int V, GL, grid;             // vectors per lane, lanes per row, workgroups
};

static NormPlan norm_plan(int dtype, int rows, int cols, bool bwd)
{
    const int E = dtype == NGC_BF16 ? 8 : 4, nvec = cols / E + (cols % E != 0);
    if (cols < E) return {LN_TINY, 1, 1, (int)(((int64_t)rows + 255) / 256)};
    // {vectors per lane, lanes}.  The backprop holds five values per element: more than 16 elements a lane leave one wave a SIMD (taken for the
    // longest rows only), and the 128 registers a lane of a workgroup of 1024 do not hold 16.
    static const int forward[][2] = {{1, 8}, {1, 16}, {1, 32}, {1, 64}, {2, 64}, {4, 64}, {2, 256}, {4, 256}, {2, 1024}, {4, 1024}, {0, 0}};
    static const int backprop[][2] = {{1, 8}, {1, 16}, {1, 32}, {1, 64}, {2, 64}, {4, 64}, {1, 256}, {2, 256}, {2, 512}, {4, 512}, {0, 0}};
    for (const int (*q)[2] = bwd ? backprop : forward; (*q)[0]; ++q) {
        const int *g = *q;
        if (nvec > g[0] * g[1] || (bwd && g[0] * E > 16 && g[1] < 512)) continue;
        const int rpw = g[1] <= 64 ? 256 / g[1] : 1, need = (int)(((int64_t)rows + rpw - 1) / rpw);
        // Forward: what the compute units hold at a time.  Backprop: every workgroup leaves 2 cols partial sums, and reads of them cost as much
        // as writes: at most two workgroups of 256 per compute unit, and four rows per group where there are enough rows for that.
        int most = g[1] == 1024 ? 512 : 2048;
        if (bwd) {
            most = g[1] == 512 ? 256 : 512;
            if (need < 4 * most) most = need / 4 < 256 ? 256 : need / 4;
        }
        const int per = (need + most - 1) / most;
        return {LN_REG, g[0], g[1], (need + per - 1) / per};
    }
    return {LN_LONG, 1, 1024, rows};
}

// parts of the columns' sums
static int norm_parts(int dtype, int rows, int cols)
{
    const NormPlan p = norm_plan(dtype, rows, cols, true);
    if (p.kernel == LN_REG) return p.grid;
    return rows < 64 ? 1 : rows < 64 * 256 ? rows / 64 : 256;
}

size_t layer_norm_bwd_workspace(int dtype, int rows, int cols) { return (size_t)norm_parts(dtype, rows, cols) * 2 * cols * sizeof(float); }

#define NGC_LN_CASE(KERNEL, V, GL, ARGS)                                                                                                           \
    case (GL) * 16 + (V): NGC_LAUNCH((KERNEL<T, V, GL, TAIL>), dim3(p.grid), dim3((GL) <= 64 ? 256 : (GL)), 0, st, NGC_LN_ARGS ARGS); break;
#define NGC_LN_ARGS(...) __VA_ARGS__

template <typename T, bool TAIL>
static hipError_t launch_norm_reg(const NormPlan &p, int rows, int cols, float eps, const T *x, const float *gamma, const float *beta, T *y, float *mean,
                                  float *rstd, hipStream_t st)
{
#define NGC_LN(V, GL) NGC_LN_CASE(layer_norm_reg, V, GL, (x, gamma, beta, y, mean, rstd, rows, cols, eps))
    switch (p.GL * 16 + p.V) {
        NGC_LN(1, 8) NGC_LN(1, 16) NGC_LN(1, 32) NGC_LN(1, 64) NGC_LN(2, 64) NGC_LN(4, 64) NGC_LN(2, 256) NGC_LN(4, 256) NGC_LN(2, 1024) NGC_LN(4, 1024)
    default: return hipErrorInvalidValue;
    }
#undef NGC_LN
    return launch_result();
}

template <typename T, bool TAIL>
static hipError_t launch_norm_bwd_reg(const NormPlan &p, int rows, int cols, const T *x, const float *gamma, const float *mean, const float *rstd,
                                      const T *dy, T *dx, float *part, hipStream_t st)
{
#define NGC_LN(V, GL) NGC_LN_CASE(layer_norm_bwd_reg, V, GL, (x, gamma, mean, rstd, dy, dx, part, rows, cols))
    switch (p.GL * 16 + p.V) {
        NGC_LN(1, 8) NGC_LN(1, 16) NGC_LN(1, 32) NGC_LN(1, 64) NGC_LN(2, 64) NGC_LN(1, 256) NGC_LN(2, 256) NGC_LN(2, 512) NGC_LN(4, 512)
    case 64 * 16 + 4:
        if constexpr (sizeof(T) == 4) NGC_LAUNCH((layer_norm_bwd_reg<T, 4, 64, TAIL>), dim3(p.grid), dim3(256), 0, st, x, gamma, mean, rstd, dy, dx, part, rows, cols);
        break;
    default: return hipErrorInvalidValue;
    }
#undef NGC_LN
    return launch_result();
}

template <typename T>
static bool whole_vectors(int cols, const void *a, const void *b, const void *c)
{
    return cols % SmElem<T>::E == 0 && ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c)) & 15) == 0;
}

template <typename T>
static hipError_t launch_norm_t(int rows, int cols, float eps, const T *x, const float *gamma, const float *beta, T *y, float *mean, float *rstd,
                                hipStream_t st)
{
    const NormPlan p = norm_plan(sizeof(T) == 2 ? NGC_BF16 : NGC_F32, rows, cols, false);
    if (p.kernel == LN_REG)
        return whole_vectors<T>(cols, x, y, nullptr) ? launch_norm_reg<T, false>(p, rows, cols, eps, x, gamma, beta, y, mean, rstd, st)
                                                     : launch_norm_reg<T, true>(p, rows, cols, eps, x, gamma, beta, y, mean, rstd, st);
    if (p.kernel == LN_TINY) {
        NGC_LAUNCH((layer_norm_tiny<T>), dim3(p.grid), dim3(256), 0, st, x, gamma, beta, y, mean, rstd, rows, cols, eps);
        return launch_result();
    }
    constexpr int most = 1 << 21;                        // a grid holds fewer than 2^32 threads
    for (int r0 = 0; r0 < rows; r0 += most) {
        const size_t at = (size_t)r0 * cols;
        NGC_LAUNCH((layer_norm_long<T>), dim3(rows - r0 < most ? rows - r0 : most), dim3(1024), 0, st, x + at, gamma, beta, y + at, mean ? mean + r0 : nullptr,
                   rstd ? rstd + r0 : nullptr, cols, eps);
        const hipError_t e = launch_result();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t launch_norm_bwd_t(int rows, int cols, const T *x, const float *gamma, const float *mean, const float *rstd, const T *dy, T *dx,
                                    float *dgamma, float *dbeta, float *ws, hipStream_t st)
{
    const int dtype = sizeof(T) == 2 ? NGC_BF16 : NGC_F32;
    const NormPlan p = norm_plan(dtype, rows, cols, true);
    const bool weights = dgamma || dbeta;
    int parts = norm_parts(dtype, rows, cols);
    hipError_t e = hipSuccess;
    if (p.kernel == LN_REG) {
        e = whole_vectors<T>(cols, x, dy, dx) ? launch_norm_bwd_reg<T, false>(p, rows, cols, x, gamma, mean, rstd, dy, dx, weights ? ws : nullptr, st)
                                              : launch_norm_bwd_reg<T, true>(p, rows, cols, x, gamma, mean, rstd, dy, dx, weights ? ws : nullptr, st);
    } else if (weights) {                                // before dx, which may be dy or x
        const int chunk = (rows - 1) / parts + 1;
        parts = (rows - 1) / chunk + 1;
        const int64_t tiles = ((int64_t)cols + 63) / 64;
        NGC_LAUNCH((layer_norm_bwd_cols<T>), dim3(parts, (unsigned)(tiles < 4096 ? tiles : 4096)), dim3(256), 0, st, x, mean, rstd, dy, ws, rows, cols, chunk);
        e = launch_result();
    }
    if (e != hipSuccess) return e;
    if (weights) {
        const int64_t tiles = ((int64_t)cols + 31) / 32;
        NGC_LAUNCH(layer_norm_bwd_join, dim3((unsigned)(tiles < 65536 ? tiles : 65536), 2), dim3(256), 0, st, ws, dgamma, dbeta, parts, cols);
        if ((e = launch_result()) != hipSuccess) return e;
    }
    if (p.kernel == LN_TINY) {
        NGC_LAUNCH((layer_norm_bwd_tiny<T>), dim3(p.grid), dim3(256), 0, st, x, gamma, mean, rstd, dy, dx, rows, cols);
        return launch_result();
    }
    constexpr int most = 1 << 21;
    for (int r0 = 0; p.kernel == LN_LONG && r0 < rows; r0 += most) {
        const size_t at = (size_t)r0 * cols;
        NGC_LAUNCH((layer_norm_bwd_long<T>), dim3(rows - r0 < most ? rows - r0 : most), dim3(1024), 0, st, x + at, gamma, mean + r0, rstd + r0, dy + at, dx + at, cols);
        if ((e = launch_result()) != hipSuccess) return e;
    }
    return e;
}

hipError_t launch_layer_norm(int dtype, int rows, int cols, float eps, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                             float *rstd, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_norm_t(rows, cols, eps, static_cast<const uint16_t *>(x), gamma, beta, static_cast<uint16_t *>(y), mean, rstd, st);
    return launch_norm_t(rows, cols, eps, static_cast<const float *>(x), gamma, beta, static_cast<float *>(y), mean, rstd, st);
}

hipError_t launch_layer_norm_bwd(int dtype, int rows, int cols, const void *x, const float *gamma, const float *mean, const float *rstd,
                                 const void *dy, void *dx, float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_norm_bwd_t(rows, cols, static_cast<const uint16_t *>(x), gamma, mean, rstd, static_cast<const uint16_t *>(dy),
                                 static_cast<uint16_t *>(dx), dgamma, dbeta, static_cast<float *>(ws), st);
    return launch_norm_bwd_t(rows, cols, static_cast<const float *>(x), gamma, mean, rstd, static_cast<const float *>(dy), static_cast<float *>(dx),
                             dgamma, dbeta, static_cast<float *>(ws), st);
}

}  // namespace ngc
