// Softmax cross entropy of a linear layer over a vocabulary, and the gradients of both operands (gfx950).
//
//   z = x w^T,  lse[n] = log sum_v exp z[n][v],  loss[n] = lse[n] - z[n][label[n]]   (0 where the label is outside the vocabulary)
//   g[n][v] = (exp(z[n][v] - lse[n]) - [v = label[n]]) dloss[n],  dx = g w,  dw = g^T x
//
// The logits are never kept: the forward pass leaves of every tile the maximum and the sum of each row; the backward pass forms g again
// for a piece of the vocabulary at a time.
#include "mm_bf16.h"
#include "rows.h"

namespace ngc {

static size_t r256(size_t b) { return (b + 255) & ~(size_t)255; }

// One 64 x 64 tile of c[m][n] = sum_k a(m, k) b(n, k) in fp32; thread (ty, tx) of 16 x 16 holds rows 4 ty .. and columns 4 tx ..
template <class A, class B>
__device__ __forceinline__ void tile64(int M, int N, int K, int m0, int n0, A a, B b, float (&acc)[4][4])
{
    __shared__ float sa[16][68], sb[16][68];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
    for (int k0 = 0; k0 < K; k0 += 16) {
        __syncthreads();
        for (int e = threadIdx.x; e < 1024; e += 256) {
            const int k = e & 15, r = e >> 4;
            sa[k][r] = m0 + r < M && k0 + k < K ? a(m0 + r, k0 + k) : 0.f;
            sb[k][r] = n0 + r < N && k0 + k < K ? b(n0 + r, k0 + k) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += sa[k][4 * ty + i] * sb[k][4 * tx + j];
    }
}

template <typename T>
__global__ __launch_bounds__(256) void xent_tiles(const T *__restrict__ x, const T *__restrict__ w, const int64_t *__restrict__ labels,
                                                  float2 *__restrict__ part, float *__restrict__ target, int rows, int width, int vocab)
{
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4];
    tile64(rows, vocab, width, m0, n0, [&](int m, int k) { return SmElem<T>::load(x + (size_t)m * width + k); },
           [&](int n, int k) { return SmElem<T>::load(w + (size_t)n * width + k); }, acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + 4 * ty + i;
        float top = -INFINITY, s = 0.f;
        for (int j = 0; j < 4; ++j)
            if (n0 + 4 * tx + j < vocab) top = fmaxf(top, acc[i][j]);
        top = group_max<16>(top);
        for (int j = 0; j < 4; ++j)
            if (n0 + 4 * tx + j < vocab) s += expf(acc[i][j] - top);
        s = group_sum<16>(s);
        if (m >= rows) continue;
        if (tx == 0) part[(size_t)blockIdx.x * rows + m] = make_float2(top, s);
        for (int j = 0; j < 4; ++j)
            if (labels[m] == n0 + 4 * tx + j && labels[m] < vocab) target[m] = acc[i][j];
    }
}

__global__ __launch_bounds__(256) void xent_join(const float2 *__restrict__ part, const float *__restrict__ target, const int64_t *__restrict__ labels,
                                                 float *__restrict__ loss, float *__restrict__ lse, int rows, int vocab, int tiles)
{
    const int m = blockIdx.x * 256 + threadIdx.x;
    if (m >= rows) return;
    float top = -INFINITY, s = 0.f;
    for (int t = 0; t < tiles; ++t) top = fmaxf(top, part[(size_t)t * rows + m].x);
    for (int t = 0; t < tiles; ++t) s += part[(size_t)t * rows + m].y * expf(part[(size_t)t * rows + m].x - top);
    const float l = top + logf(s);
    lse[m] = l;
    loss[m] = labels[m] >= 0 && labels[m] < vocab ? l - target[m] : 0.f;
}

// g of the piece of the vocabulary from v0 on: [rows][piece]
template <typename T>
__global__ __launch_bounds__(256) void xent_grad_tiles(const T *__restrict__ x, const T *__restrict__ w, const int64_t *__restrict__ labels,
                                                       const float *__restrict__ lse, const float *__restrict__ dloss, float *__restrict__ g, int rows,
                                                       int width, int vocab, int v0, int piece)
{
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4];
    tile64(rows, piece, width, m0, n0, [&](int m, int k) { return SmElem<T>::load(x + (size_t)m * width + k); },
           [&](int n, int k) { return SmElem<T>::load(w + (size_t)(v0 + n) * width + k); }, acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + 4 * ty + i;
        if (m >= rows) continue;
        const int64_t label = labels[m];
        const bool live = label >= 0 && label < vocab;
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + 4 * tx + j;
            if (n < piece) g[(size_t)m * piece + n] = live ? (expf(acc[i][j] - lse[m]) - (label == v0 + n ? 1.f : 0.f)) * dloss[m] : 0.f;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void xent_dx_tiles(const float *__restrict__ g, const T *__restrict__ w, float *__restrict__ dx, int rows, int width,
                                                     int v0, int piece)
{
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4];
    tile64(rows, width, piece, m0, n0, [&](int m, int k) { return g[(size_t)m * piece + k]; },
           [&](int n, int k) { return SmElem<T>::load(w + (size_t)(v0 + k) * width + n); }, acc);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 4 * ty + i, n = n0 + 4 * tx + j;
            if (m < rows && n < width) dx[(size_t)m * width + n] = acc[i][j] + (v0 ? dx[(size_t)m * width + n] : 0.f);
        }
}

template <typename T>
__global__ __launch_bounds__(256) void xent_dw_tiles(const float *__restrict__ g, const T *__restrict__ x, T *__restrict__ dw, int rows, int width,
                                                     int v0, int piece)
{
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4];
    tile64(piece, width, rows, m0, n0, [&](int m, int k) { return g[(size_t)k * piece + m]; },
           [&](int n, int k) { return SmElem<T>::load(x + (size_t)k * width + n); }, acc);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + 4 * ty + i, n = n0 + 4 * tx + j;
            if (m < piece && n < width) SmElem<T>::store(dw + (size_t)(v0 + m) * width + n, acc[i][j]);
        }
}

template <typename T>
__global__ __launch_bounds__(256) void xent_dx_store(const float *__restrict__ sum, T *__restrict__ dx, size_t n)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) SmElem<T>::store(dx + i, sum[i]);
}

constexpr int XENT_PIECE = 4096;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// ---- bf16: the products on the matrix cores -------------------------------------------------------------------------------

// What the backward pass needs of a row: lse in units of log 2, dloss over the largest |dloss| (0 for rows that do not count), the label (-1)
struct XentRow {
    float lse2, factor;
    int label, pad;
};

// One workgroup.  The gradient's rows are scaled by dloss / max |dloss| before they are rounded to bf16, and the results by max |dloss| in
// fp32: where all rows weigh the same (a mean), the weight's own rounding would otherwise be the same in every term of the sums.
__global__ __launch_bounds__(1024) void xent_rows(const int64_t *__restrict__ labels, const float *__restrict__ lse, const float *__restrict__ dloss,
                                                  XentRow *__restrict__ info, float *__restrict__ scale, int rows, int vocab)
{
    __shared__ float sm[16];
    float top = 0.f;
    for (int m = threadIdx.x; m < rows; m += 1024)
        if (labels[m] >= 0 && labels[m] < vocab) top = fmaxf(top, fabsf(dloss[m]));
    top = fmaxf(block_reduce<16>(top, true, sm), 0x1p-100f);             // all zero: any scale
    const float inv = 1.0f / top;
    for (int m = threadIdx.x; m < rows; m += 1024) {
        const bool live = labels[m] >= 0 && labels[m] < vocab;
        info[m] = XentRow{lse[m] * LOG2E, live ? dloss[m] * inv : 0.f, live ? (int)labels[m] : -1, 0};
    }
    if (threadIdx.x == 0) *scale = top;
}

enum XentEpilogue { XE_STATS, XE_GRAD, XE_SLAB, XE_OUT };

struct XentMm {
    MmParams mm;
    int v0, vocab;                       // STATS, GRAD: first class of the piece, classes in all
    const int64_t *labels;               // STATS
    float2 *part;                        // STATS: [tiles][rows], from this piece's first tile on
    float *target;                       // STATS
    const XentRow *info;                 // GRAD
    const float *scale;                  // OUT
    uint16_t *out;                       // GRAD: g, OUT: the result
    int64_t ldo;
    int store_n;                         // columns that are stored (GRAD: zeros past the piece)
    float *slab;                         // SLAB: [splits][M][ldo]
    int add;                             // SLAB: onto what is there
};

template <int BM, int BN, int WM, int WN, bool AT, bool BT, XentEpilogue E>
__global__ __launch_bounds__(64 * WM * WN) void xent_mm(const XentMm p)
{
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tiles = p.mm.mt * p.mm.nt, split = blockIdx.x / tiles;
    int tm, tn;
    mm_tile_of(blockIdx.x - split * tiles, tiles, p.mm.mt, p.mm.nt, tm, tn);
    const int k0 = split * p.mm.kper, k1 = p.mm.K - k0 < p.mm.kper ? p.mm.K : k0 + p.mm.kper;
    mm_f32x4 acc[FN][FM];
    mm_tile<BM, BN, WM, WN, AT, BT>(p.mm, smem, tm * BM, tn * BN, k0, k1, acc);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int wm = (wave % WM) * (BM / WM), wn = (wave / WM) * (BN / WN);
    const int m_ = tm * BM + wm + (lane & 15), n_ = tn * BN + wn + 4 * g;       // + 16 fm, + 16 fn + element
    if constexpr (E == XE_STATS) {
        // a row of the tile: its maximum and sum of exponentials over 4 FN values of a lane, 4 lanes, WN waves
        float2 *red = reinterpret_cast<float2 *>(smem);                          // [WN][BM]
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int m = m_ + 16 * j;
            float top = -INFINITY, s = 0.f;
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z = n_ + 16 * i + e < p.mm.N ? acc[i][j][e] * LOG2E : -INFINITY;
                    top = fmaxf(top, z);
                }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float t = top == -INFINITY ? 0.f : top;                        // a wave whose columns are all past the end: sum 0
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s += n_ + 16 * i + e < p.mm.N ? __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, -t)) : 0.f;
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            if (g == 0) red[(wave / WM) * BM + wm + 16 * j + lane] = make_float2(top, s);
            if (m < p.mm.M) {
                const int64_t label = p.labels[m] - p.v0;
                if (label >= tn * BN + wn && label < tn * BN + wn + BN / WN && label < p.mm.N) {
#pragma unroll
                    for (int i = 0; i < FN; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (label == n_ + 16 * i + e) p.target[m] = acc[i][j][e];
                }
            }
        }
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += 64 * WM * WN) {
            float2 v = red[r];
#pragma unroll
            for (int w = 1; w < WN; ++w) {
                const float2 o = red[w * BM + r];
                const float top = fmaxf(v.x, o.x);                               // the first wave always has columns
                v = make_float2(top, v.y * __builtin_amdgcn_exp2f(v.x - top) + o.y * __builtin_amdgcn_exp2f(o.x - top));
            }
            if (tm * BM + r < p.mm.M) p.part[(size_t)tn * p.mm.M + tm * BM + r] = v;
        }
        return;
    }
    float scale = 1.f;
    if constexpr (E == XE_OUT) scale = *p.scale;
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int m = m_ + 16 * j;
        if (m >= p.mm.M) continue;
        XentRow row;
        if constexpr (E == XE_GRAD) row = p.info[m];
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const int n = n_ + 16 * i;
            mm_f32x4 v = acc[i][j];
            if constexpr (E == XE_SLAB) {
                if (n >= p.store_n) continue;
                float *at = p.slab + ((size_t)split * p.mm.M + m) * p.ldo + n;  // ldo and store_n are multiples of 8
                if (p.add) v += *reinterpret_cast<const mm_f32x4 *>(at);
                *reinterpret_cast<mm_f32x4 *>(at) = v;
                continue;
            }
            if constexpr (E == XE_GRAD) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float prob = __builtin_amdgcn_exp2f(fmaf(v[e], LOG2E, -row.lse2));
                    v[e] = row.label >= 0 && n + e < p.mm.N ? (prob - (row.label == p.v0 + n + e ? 1.f : 0.f)) * row.factor : 0.f;
                }
            } else {
                v *= scale;
            }
            uint16_t *at = p.out + (size_t)m * p.ldo + n;
            const uint32_t lo = pack_bf16x2_hw(v[0], v[1]), hi = pack_bf16x2_hw(v[2], v[3]);
            if (n + 4 <= p.store_n && (p.ldo & 3) == 0) {
                *reinterpret_cast<uint2 *>(at) = make_uint2(lo, hi);
            } else {
                if (n < p.store_n) at[0] = (uint16_t)lo;
                if (n + 1 < p.store_n) at[1] = (uint16_t)(lo >> 16);
                if (n + 2 < p.store_n) at[2] = (uint16_t)hi;
                if (n + 3 < p.store_n) at[3] = (uint16_t)(hi >> 16);
            }
        }
    }
}

// lse and loss of 32 rows from the tiles' maxima and sums, eight parts of the tiles each
__global__ __launch_bounds__(256) void xent_join2(const float2 *__restrict__ part, const float *__restrict__ target, const int64_t *__restrict__ labels,
                                                  float *__restrict__ loss, float *__restrict__ lse, int rows, int vocab, int tiles)
{
    __shared__ float2 red[8][32];
    const int r = threadIdx.x & 31, q = threadIdx.x >> 5, m = blockIdx.x * 32 + r;
    float top = -INFINITY, s = 0.f;
    if (m < rows)
        for (int t = q; t < tiles; t += 8) {
            const float2 v = part[(size_t)t * rows + m];
            const float up = fmaxf(top, v.x);
            s = s * __builtin_amdgcn_exp2f(top - up) + v.y * __builtin_amdgcn_exp2f(v.x - up);
            top = up;
        }
    red[q][r] = make_float2(top, s);
    __syncthreads();
    if (q || m >= rows) return;
    for (int i = 1; i < 8; ++i) {
        const float2 v = red[i][r];
        if (v.x == -INFINITY) continue;                                          // fewer tiles than parts
        const float up = fmaxf(top, v.x);
        s = s * __builtin_amdgcn_exp2f(top - up) + v.y * __builtin_amdgcn_exp2f(v.x - up);
        top = up;
    }
    const float l = (top + log2f(s)) * LN2;
    lse[m] = l;
    loss[m] = labels[m] >= 0 && labels[m] < vocab ? l - target[m] : 0.f;
}

// rows of `width` elements to rows of `pitch` (zeros behind them)
__global__ __launch_bounds__(256) void xent_pad(const uint16_t *__restrict__ src, uint16_t *__restrict__ dst, int64_t rows, int width, int pitch)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int j = threadIdx.x; j < pitch; j += 256) dst[(size_t)r * pitch + j] = j < width ? src[(size_t)r * width + j] : (uint16_t)0;
}

// out[r][j] = scale * sum of the slabs
__global__ __launch_bounds__(256) void xent_sum(const float *__restrict__ slab, const float *__restrict__ scale, uint16_t *__restrict__ out, int rows,
                                                int width, int pitch, int splits)
{
    const int j = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (j >= width) return;
    const float s = *scale;
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        mm_f32x4 v = mm_f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < splits; ++q) v += *reinterpret_cast<const mm_f32x4 *>(slab + ((size_t)q * rows + r) * pitch + j);
        for (int e = 0; e < 4 && j + e < width; ++e) out[(size_t)r * width + j + e] = (uint16_t)(pack_bf16x2_hw(v[e] * s, 0.f) & 0xFFFFu);
    }
}

static int up(int v, int to) { return (v + to - 1) / to * to; }

// How a call goes through the vocabulary.  Pieces are as large as 512 MiB of g, and of a padded copy of w, allow.
struct XentPlan {
    bool pad;                    // rows of no multiple of 16 bytes, or tensors off that grid, are copied first
    int pitch, piece;            // elements of a row of x and w as the products read them; classes of a piece
    int dx_splits, dw_splits;
    size_t info, scale, xpad, wpad, g, dx_slab, dw_slab, total;         // offsets in the workspace
};

static int splits_for(int64_t tiles, int k)
{
    // parts of at least 512: fewer than half the compute units have a tile otherwise
    int s = 1;
    while (tiles * s * 2 <= 256 && k / (s * 2) >= 512) s *= 2;
    return s;
}
static int64_t tiles128(int64_t m, int64_t n) { return ((m + 127) / 128) * ((n + 127) / 128); }

static XentPlan xent_plan(int64_t rows, int width, int vocab, bool bwd, bool dx, bool dw)
{
    XentPlan p{};
    p.pitch = up(width, 8);
    p.pad = p.pitch != width;
    const int64_t most = (int64_t)512 << 20;
    int64_t piece = vocab;
    if (bwd) piece = piece < most / 2 / rows ? piece : most / 2 / rows;
    piece = piece < most / 2 / p.pitch ? piece : most / 2 / p.pitch;
    p.piece = (int)(piece < vocab ? (piece / 256 > 0 ? piece / 256 * 256 : 256) : vocab);
    p.dx_splits = dx ? splits_for(tiles128(rows, width), p.piece) : 1;
    p.dw_splits = dw ? splits_for(tiles128(p.piece, width), (int)rows) : 1;
    return p;
}

static size_t xent_lay_out(XentPlan &p, int64_t rows, int vocab, bool bwd)
{
    size_t at = 0;
    auto take = [&](size_t &where, size_t bytes) { where = at; at += r256(bytes); };
    if (!bwd) {
        take(p.info, (size_t)rows * 8 * ((size_t)(vocab + 63) / 64 + (vocab + p.piece - 1) / p.piece));      // part
        take(p.scale, (size_t)rows * 4);                                                                    // target
    } else {
        take(p.info, (size_t)rows * sizeof(XentRow));
        take(p.scale, 4);
        take(p.g, (size_t)rows * up(p.piece, 64) * 2);
        take(p.dx_slab, (size_t)rows * p.pitch * 4 * p.dx_splits);
        take(p.dw_slab, p.dw_splits > 1 ? (size_t)p.piece * p.pitch * 4 * p.dw_splits : 0);
    }
    take(p.xpad, (size_t)rows * p.pitch * 2);
    take(p.wpad, (size_t)p.piece * p.pitch * 2);
    p.total = at;
    return at;
}

template <int BM, int BN, int WM, int WN, bool AT, bool BT, XentEpilogue E>
static hipError_t launch_mm_tile(XentMm p, hipStream_t st)
{
    static LdsLimitOnce lds;
    const hipError_t e = lds.raise(reinterpret_cast<const void *>(&xent_mm<BM, BN, WM, WN, AT, BT, E>));
    if (e != hipSuccess) return e;
    p.mm.mt = (p.mm.M + BM - 1) / BM;
    p.mm.nt = (p.mm.N + BN - 1) / BN;
    p.mm.kper = up((p.mm.K + p.mm.splits - 1) / p.mm.splits, 32);
    NGC_LAUNCH((xent_mm<BM, BN, WM, WN, AT, BT, E>), dim3((unsigned)(p.mm.mt * p.mm.nt * p.mm.splits)), dim3(64 * WM * WN), (mm_lds_bytes<BM, BN>()), st, p);
    return launch_result();
}

// The largest tile that still gives most compute units one
static int mm_tile_size(int64_t m, int64_t n, int splits)
{
    if (((m + 255) / 256) * ((n + 255) / 256) * splits >= 192) return 256;
    if (tiles128(m, n) * splits >= 128) return 128;
    return 64;
}

template <bool AT, bool BT, XentEpilogue E>
static hipError_t launch_mm(const XentMm &p, int tile, hipStream_t st)
{
    if (tile == 256) return launch_mm_tile<256, 256, 2, 2, AT, BT, E>(p, st);
    if (tile == 128) return launch_mm_tile<128, 128, 2, 2, AT, BT, E>(p, st);
    return launch_mm_tile<64, 64, 2, 2, AT, BT, E>(p, st);
}

static hipError_t pad_rows(const uint16_t *src, uint16_t *dst, int64_t rows, int width, int pitch, hipStream_t st)
{
    NGC_LAUNCH(xent_pad, dim3((unsigned)(rows < 65536 ? rows : 65536)), dim3(256), 0, st, src, dst, rows, width, pitch);
    return launch_result();
}

static bool on_grid(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

static hipError_t launch_xent_bf16(int rows, int width, int vocab, const uint16_t *x, const uint16_t *w, const int64_t *labels, float *loss, float *lse,
                                   char *ws, hipStream_t st)
{
    XentPlan pl = xent_plan(rows, width, vocab, false, false, false);
    xent_lay_out(pl, rows, vocab, false);
    const bool pad_x = pl.pad || !on_grid(x), pad_w = pl.pad || !on_grid(w);
    hipError_t e;
    if (pad_x && (e = pad_rows(x, reinterpret_cast<uint16_t *>(ws + pl.xpad), rows, width, pl.pitch, st)) != hipSuccess) return e;
    int tiles = 0;
    for (int v0 = 0, piece; v0 < vocab; v0 += piece) {
        piece = pad_w ? (vocab - v0 < pl.piece ? vocab - v0 : pl.piece) : vocab;
        const uint16_t *wp = w + (size_t)v0 * width;
        if (pad_w) {
            if ((e = pad_rows(wp, reinterpret_cast<uint16_t *>(ws + pl.wpad), piece, width, pl.pitch, st)) != hipSuccess) return e;
            wp = reinterpret_cast<uint16_t *>(ws + pl.wpad);
        }
        XentMm p{};
        p.mm.a = pad_x ? reinterpret_cast<uint16_t *>(ws + pl.xpad) : x;
        p.mm.b = wp;
        p.mm.lda = p.mm.ldb = pl.pitch;
        p.mm.M = rows; p.mm.N = piece; p.mm.K = pl.pitch; p.mm.splits = 1;
        p.v0 = v0; p.vocab = vocab; p.labels = labels;
        p.part = reinterpret_cast<float2 *>(ws + pl.info) + (size_t)tiles * rows;
        p.target = reinterpret_cast<float *>(ws + pl.scale);
        const int tile = mm_tile_size(rows, piece, 1);
        if ((e = launch_mm<false, false, XE_STATS>(p, tile, st)) != hipSuccess) return e;
        tiles += (piece + tile - 1) / tile;
    }
    NGC_LAUNCH(xent_join2, dim3((rows + 31) / 32), dim3(256), 0, st, reinterpret_cast<float2 *>(ws + pl.info), reinterpret_cast<float *>(ws + pl.scale), labels,
               loss, lse, rows, vocab, tiles);
    return launch_result();
}

static hipError_t sum_slabs(const float *slab, const float *scale, uint16_t *out, int rows, int width, int pitch, int splits, hipStream_t st)
{
    NGC_LAUNCH(xent_sum, dim3((width + 1023) / 1024, rows < 32768 ? rows : 32768), dim3(256), 0, st, slab, scale, out, rows, width, pitch, splits);
    return launch_result();
}

static hipError_t launch_xent_bwd_bf16(int rows, int width, int vocab, const uint16_t *x, const uint16_t *w, const int64_t *labels, const float *lse,
                                       const float *dloss, uint16_t *dx, uint16_t *dw, char *ws, hipStream_t st)
{
    XentPlan pl = xent_plan(rows, width, vocab, true, true, true);
    xent_lay_out(pl, rows, vocab, true);
    XentRow *info = reinterpret_cast<XentRow *>(ws + pl.info);
    float *scale = reinterpret_cast<float *>(ws + pl.scale), *dx_slab = reinterpret_cast<float *>(ws + pl.dx_slab), *dw_slab = reinterpret_cast<float *>(ws + pl.dw_slab);
    uint16_t *g = reinterpret_cast<uint16_t *>(ws + pl.g);
    const bool pad_x = pl.pad || !on_grid(x), pad_w = pl.pad || !on_grid(w);
    hipError_t e;
    NGC_LAUNCH(xent_rows, dim3(1), dim3(1024), 0, st, labels, lse, dloss, info, scale, rows, vocab);
    if ((e = launch_result()) != hipSuccess) return e;
    if (pad_x && (e = pad_rows(x, reinterpret_cast<uint16_t *>(ws + pl.xpad), rows, width, pl.pitch, st)) != hipSuccess) return e;
    const uint16_t *xp = pad_x ? reinterpret_cast<uint16_t *>(ws + pl.xpad) : x;
    const bool one = pl.piece >= vocab && pl.dx_splits == 1;
    for (int v0 = 0; v0 < vocab; v0 += pl.piece) {
        const int piece = vocab - v0 < pl.piece ? vocab - v0 : pl.piece, gp = up(piece, 64);
        const uint16_t *wp = w + (size_t)v0 * width;
        if (pad_w) {
            if ((e = pad_rows(wp, reinterpret_cast<uint16_t *>(ws + pl.wpad), piece, width, pl.pitch, st)) != hipSuccess) return e;
            wp = reinterpret_cast<uint16_t *>(ws + pl.wpad);
        }
        XentMm p{};
        p.v0 = v0; p.vocab = vocab; p.info = info; p.scale = scale;
        p.mm.a = xp; p.mm.b = wp; p.mm.lda = p.mm.ldb = pl.pitch;
        p.mm.M = rows; p.mm.N = piece; p.mm.K = pl.pitch; p.mm.splits = 1;
        p.out = g; p.ldo = gp; p.store_n = gp;
        if ((e = launch_mm<false, false, XE_GRAD>(p, mm_tile_size(rows, piece, 1), st)) != hipSuccess) return e;
        if (dx) {
            XentMm q = p;
            q.mm.a = g; q.mm.lda = gp; q.mm.M = rows; q.mm.N = pl.pitch; q.mm.K = piece; q.mm.splits = pl.dx_splits;
            const int tile = mm_tile_size(rows, width, pl.dx_splits);
            if (one) {
                q.out = dx; q.ldo = width; q.store_n = width;
                e = launch_mm<false, true, XE_OUT>(q, tile, st);
            } else {
                q.slab = dx_slab; q.ldo = pl.pitch; q.store_n = pl.pitch; q.add = v0 > 0;
                e = launch_mm<false, true, XE_SLAB>(q, tile, st);
            }
            if (e != hipSuccess) return e;
        }
        if (dw) {
            XentMm q = p;
            q.mm.a = g; q.mm.lda = gp; q.mm.b = xp; q.mm.M = piece; q.mm.N = pl.pitch; q.mm.K = rows; q.mm.splits = pl.dw_splits;
            const int tile = mm_tile_size(piece, width, pl.dw_splits);
            uint16_t *out = dw + (size_t)v0 * width;
            if (pl.dw_splits == 1) {
                q.out = out; q.ldo = width; q.store_n = width;
                e = launch_mm<true, true, XE_OUT>(q, tile, st);
            } else {
                q.slab = dw_slab; q.ldo = pl.pitch; q.store_n = pl.pitch; q.add = 0;
                e = launch_mm<true, true, XE_SLAB>(q, tile, st);
                if (e == hipSuccess) e = sum_slabs(dw_slab, scale, out, piece, width, pl.pitch, pl.dw_splits, st);
            }
            if (e != hipSuccess) return e;
        }
    }
    return dx && !one ? sum_slabs(dx_slab, scale, dx, rows, width, pl.pitch, pl.dx_splits, st) : hipSuccess;
}

size_t linear_xent_workspace(int dtype, int64_t rows, int width, int vocab, bool bwd)
{
    if (dtype == NGC_BF16) {
        XentPlan p = xent_plan(rows, width, vocab, bwd, true, true);
        return xent_lay_out(p, rows, vocab, bwd);
    }
    const size_t tiles = ((size_t)vocab + 63) / 64, piece = vocab < XENT_PIECE ? vocab : XENT_PIECE;
    return bwd ? r256((size_t)rows * piece * 4) + r256((size_t)rows * width * 4) : r256((size_t)rows * tiles * 8) + r256((size_t)rows * 4);
}

template <typename T>
static hipError_t launch_xent_t(int rows, int width, int vocab, const T *x, const T *w, const int64_t *labels, float *loss, float *lse, void *ws,
                                hipStream_t st)
{
    const int tiles = (vocab + 63) / 64;
    float2 *part = static_cast<float2 *>(ws);
    float *target = reinterpret_cast<float *>(static_cast<char *>(ws) + r256((size_t)rows * tiles * 8));
    NGC_LAUNCH((xent_tiles<T>), dim3(tiles, (rows + 63) / 64), dim3(256), 0, st, x, w, labels, part, target, rows, width, vocab);
    const hipError_t e = launch_result();
    if (e != hipSuccess) return e;
    NGC_LAUNCH(xent_join, dim3((rows + 255) / 256), dim3(256), 0, st, part, target, labels, loss, lse, rows, vocab, tiles);
    return launch_result();
}

template <typename T>
static hipError_t launch_xent_bwd_t(int rows, int width, int vocab, const T *x, const T *w, const int64_t *labels, const float *lse,
                                    const float *dloss, T *dx, T *dw, void *ws, hipStream_t st)
{
    const int most = vocab < XENT_PIECE ? vocab : XENT_PIECE;
    float *g = static_cast<float *>(ws), *sum = reinterpret_cast<float *>(static_cast<char *>(ws) + r256((size_t)rows * most * 4));
    const unsigned mt = (rows + 63) / 64, dt = (width + 63) / 64;
    for (int v0 = 0; v0 < vocab; v0 += most) {
        const int piece = vocab - v0 < most ? vocab - v0 : most;
        NGC_LAUNCH((xent_grad_tiles<T>), dim3((piece + 63) / 64, mt), dim3(256), 0, st, x, w, labels, lse, dloss, g, rows, width, vocab, v0, piece);
        hipError_t e = launch_result();
        if (e != hipSuccess) return e;
        if (dx) NGC_LAUNCH((xent_dx_tiles<T>), dim3(dt, mt), dim3(256), 0, st, g, w, sum, rows, width, v0, piece);
        if ((e = launch_result()) != hipSuccess) return e;
        if (dw) NGC_LAUNCH((xent_dw_tiles<T>), dim3(dt, (piece + 63) / 64), dim3(256), 0, st, g, x, dw, rows, width, v0, piece);
        if ((e = launch_result()) != hipSuccess) return e;
    }
    const size_t n = (size_t)rows * width;
    if (dx) NGC_LAUNCH((xent_dx_store<T>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, sum, dx, n);
    return launch_result();
}

hipError_t launch_linear_xent(int dtype, int rows, int width, int vocab, const void *x, const void *w, const int64_t *labels, float *loss, float *lse,
                              void *ws, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_xent_bf16(rows, width, vocab, static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(w), labels, loss, lse, static_cast<char *>(ws), st);
    return launch_xent_t(rows, width, vocab, static_cast<const float *>(x), static_cast<const float *>(w), labels, loss, lse, ws, st);
}

hipError_t launch_linear_xent_bwd(int dtype, int rows, int width, int vocab, const void *x, const void *w, const int64_t *labels, const float *lse,
                                  const float *dloss, void *dx, void *dw, void *ws, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_xent_bwd_bf16(rows, width, vocab, static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(w), labels, lse, dloss,
                                    static_cast<uint16_t *>(dx), static_cast<uint16_t *>(dw), static_cast<char *>(ws), st);
    return launch_xent_bwd_t(rows, width, vocab, static_cast<const float *>(x), static_cast<const float *>(w), labels, lse, dloss,
                             static_cast<float *>(dx), static_cast<float *>(dw), ws, st);
}

}  // namespace ngc
