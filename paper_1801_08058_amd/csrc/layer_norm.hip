// Layer norm over the last axis of a [rows, cols] tensor and its backprop (gfx950).
//
//   mean = sum_j x[j] / cols,  rstd = (sum_j (x[j] - mean)^2 / cols + eps)^(-1/2)
//   y[j] = (x[j] - mean) rstd gamma[j] + beta[j]
//   g = dy gamma, xh = (x - mean) rstd:  dx[j] = rstd (g[j] - sum_k g[k] / cols - xh[j] sum_k g[k] xh[k] / cols)
//   dgamma[j] = sum over the rows of dy[j] xh[j],  dbeta[j] = sum over the rows of dy[j]
#include "rows.h"

namespace ngc {

template <typename T>
__global__ __launch_bounds__(256) void layer_norm_rows(const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                       T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd, int cols, float eps)
{
    __shared__ float sm[4];
    const size_t base = (size_t)blockIdx.x * cols;
    float s = 0.f, q = 0.f;
    for (int j = threadIdx.x; j < cols; j += 256) s += SmElem<T>::load(x + base + j);
    const float mu = block_reduce<4>(s, false, sm) / (float)cols;
    for (int j = threadIdx.x; j < cols; j += 256) {
        const float d = SmElem<T>::load(x + base + j) - mu;
        q += d * d;
    }
    const float rs = 1.0f / sqrtf(block_reduce<4>(q, false, sm) / (float)cols + eps);
    for (int j = threadIdx.x; j < cols; j += 256)
        SmElem<T>::store(y + base + j, (SmElem<T>::load(x + base + j) - mu) * rs * (gamma ? gamma[j] : 1.f) + (beta ? beta[j] : 0.f));
    if (threadIdx.x == 0) {
        if (mean) mean[blockIdx.x] = mu;
        if (rstd) rstd[blockIdx.x] = rs;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void layer_norm_bwd_rows(const T *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ mean,
                                                           const float *__restrict__ rstd, const T *__restrict__ dy, T *__restrict__ dx, int cols)
{
    __shared__ float sm[4];
    const size_t base = (size_t)blockIdx.x * cols;
    const float mu = mean[blockIdx.x], rs = rstd[blockIdx.x];
    float a = 0.f, b = 0.f;
    for (int j = threadIdx.x; j < cols; j += 256) {
        const float g = SmElem<T>::load(dy + base + j) * (gamma ? gamma[j] : 1.f);
        a += g;
        b += g * (SmElem<T>::load(x + base + j) - mu) * rs;
    }
    a = block_reduce<4>(a, false, sm) / (float)cols;
    b = block_reduce<4>(b, false, sm) / (float)cols;
    for (int j = threadIdx.x; j < cols; j += 256) {
        const float g = SmElem<T>::load(dy + base + j) * (gamma ? gamma[j] : 1.f);
        SmElem<T>::store(dx + base + j, rs * (g - a - (SmElem<T>::load(x + base + j) - mu) * rs * b));
    }
}

// Column sums of a chunk of rows; part 0 .. nparts-1 of [nparts][2][cols].
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_bwd_cols(const T *__restrict__ x, const float *__restrict__ mean, const float *__restrict__ rstd,
                                                           const T *__restrict__ dy, float *__restrict__ part, int rows, int cols, int chunk)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= cols) return;
    const int r0 = blockIdx.y * chunk, r1 = rows - r0 < chunk ? rows : r0 + chunk;
    float dg = 0.f, db = 0.f;
    for (int r = r0; r < r1; ++r) {
        const float d = SmElem<T>::load(dy + (size_t)r * cols + j);
        dg += d * (SmElem<T>::load(x + (size_t)r * cols + j) - mean[r]) * rstd[r];
        db += d;
    }
    part[((size_t)blockIdx.y * 2) * cols + j] = dg;
    part[((size_t)blockIdx.y * 2 + 1) * cols + j] = db;
}

__global__ __launch_bounds__(256) void layer_norm_bwd_join(const float *__restrict__ part, float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                           int nparts, int cols)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= cols) return;
    float dg = 0.f, db = 0.f;
    for (int p = 0; p < nparts; ++p) {
        dg += part[((size_t)p * 2) * cols + j];
        db += part[((size_t)p * 2 + 1) * cols + j];
    }
    if (dgamma) dgamma[j] = dg;
    if (dbeta) dbeta[j] = db;
}

static int norm_parts(int rows) { return rows < 64 ? 1 : rows < 64 * 256 ? rows / 64 : 256; }

hipError_t launch_layer_norm(int dtype, int rows, int cols, float eps, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                             float *rstd, hipStream_t st)
{
    if (dtype == NGC_BF16)
        NGC_LAUNCH((layer_norm_rows<uint16_t>), dim3(rows), dim3(256), 0, st, static_cast<const uint16_t *>(x), gamma, beta, static_cast<uint16_t *>(y), mean, rstd, cols, eps);
    else
        NGC_LAUNCH((layer_norm_rows<float>), dim3(rows), dim3(256), 0, st, static_cast<const float *>(x), gamma, beta, static_cast<float *>(y), mean, rstd, cols, eps);
    return launch_result();
}

size_t layer_norm_bwd_workspace(int, int rows, int cols) { return (size_t)norm_parts(rows) * 2 * cols * sizeof(float); }

template <typename T>
static hipError_t launch_norm_bwd_t(int rows, int cols, const T *x, const float *gamma, const float *mean, const float *rstd, const T *dy, T *dx,
                                    float *dgamma, float *dbeta, float *ws, hipStream_t st)
{
    if (dgamma || dbeta) {                               // before dx, which may be dy
        const int n = norm_parts(rows), chunk = (rows + n - 1) / n, parts = (rows + chunk - 1) / chunk;
        NGC_LAUNCH((layer_norm_bwd_cols<T>), dim3((cols + 255) / 256, parts), dim3(256), 0, st, x, mean, rstd, dy, ws, rows, cols, chunk);
        const hipError_t e = launch_result();
        if (e != hipSuccess) return e;
        NGC_LAUNCH(layer_norm_bwd_join, dim3((cols + 255) / 256), dim3(256), 0, st, ws, dgamma, dbeta, parts, cols);
        const hipError_t e2 = launch_result();
        if (e2 != hipSuccess) return e2;
    }
    NGC_LAUNCH((layer_norm_bwd_rows<T>), dim3(rows), dim3(256), 0, st, x, gamma, mean, rstd, dy, dx, cols);
    return launch_result();
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
