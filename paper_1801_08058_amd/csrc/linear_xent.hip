// Softmax cross entropy of a linear layer over a vocabulary, and the gradients of both operands (gfx950).
//
//   z = x w^T,  lse[n] = log sum_v exp z[n][v],  loss[n] = lse[n] - z[n][label[n]]   (0 where the label is outside the vocabulary)
//   g[n][v] = (exp(z[n][v] - lse[n]) - [v = label[n]]) dloss[n],  dx = g w,  dw = g^T x
//
// The logits are never kept: the forward pass leaves of every tile the maximum and the sum of each row; the backward pass forms g again
// for a piece of the vocabulary at a time.
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

size_t linear_xent_workspace(int, int64_t rows, int width, int vocab, bool bwd)
{
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
        return launch_xent_t(rows, width, vocab, static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(w), labels, loss, lse, ws, st);
    return launch_xent_t(rows, width, vocab, static_cast<const float *>(x), static_cast<const float *>(w), labels, loss, lse, ws, st);
}

hipError_t launch_linear_xent_bwd(int dtype, int rows, int width, int vocab, const void *x, const void *w, const int64_t *labels, const float *lse,
                                  const float *dloss, void *dx, void *dw, void *ws, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_xent_bwd_t(rows, width, vocab, static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(w), labels, lse, dloss,
                                 static_cast<uint16_t *>(dx), static_cast<uint16_t *>(dw), ws, st);
    return launch_xent_bwd_t(rows, width, vocab, static_cast<const float *>(x), static_cast<const float *>(w), labels, lse, dloss,
                             static_cast<float *>(dx), static_cast<float *>(dw), ws, st);
}

}  // namespace ngc
