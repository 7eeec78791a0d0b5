// Embedding lookup with scaling and its gradient (gfx950): the node that turns the tokens of a batch into rows.
//
//   y[t]      = scale * table[id[t]]                       for 0 <= id[t] < vocab, else +0
//   dtable[v] = scale * sum over t with id[t] = v of dy[t]  (ascending t, fp32)
#include "rows.h"

namespace ngc {

template <typename T>
__global__ __launch_bounds__(256) void embedding_rows(const T *__restrict__ table, const int64_t *__restrict__ ids, T *__restrict__ y,
                                                      int64_t tokens, int vocab, int width, float scale)
{
    for (int64_t t = blockIdx.x; t < tokens; t += gridDim.x) {
        const int64_t id = ids[t];
        const bool live = id >= 0 && id < vocab;
        const T *src = table + (size_t)(live ? id : 0) * width;
        for (int j = threadIdx.x; j < width; j += 256) SmElem<T>::store(y + (size_t)t * width + j, live ? SmElem<T>::load(src + j) * scale : 0.f);
    }
}

// A workgroup per row of the table: it looks through all tokens.
template <typename T>
__global__ __launch_bounds__(256) void embedding_bwd_scan(const T *__restrict__ dy, const int64_t *__restrict__ ids, float *__restrict__ dtable,
                                                          int64_t tokens, int width, float scale)
{
    __shared__ int64_t sid[1024];
    const int v = blockIdx.x;
    for (int j0 = 0; j0 < width; j0 += 256 * 4) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int64_t t0 = 0; t0 < tokens; t0 += 1024) {
            __syncthreads();
            for (int i = threadIdx.x; i < 1024; i += 256) sid[i] = t0 + i < tokens ? ids[t0 + i] : -1;
            __syncthreads();
            for (int i = 0; i < 1024; ++i) {
                if (sid[i] != v) continue;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int j = j0 + u * 256 + threadIdx.x;
                    if (j < width) acc[u] += SmElem<T>::load(dy + (size_t)(t0 + i) * width + j);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u * 256 + threadIdx.x;
            if (j < width) dtable[(size_t)v * width + j] = acc[u] * scale;
        }
    }
}

hipError_t launch_embedding(int dtype, int64_t tokens, int vocab, int width, float scale, const void *table, const int64_t *ids, void *y,
                            hipStream_t st)
{
    const dim3 grid((unsigned)(tokens < 65536 ? tokens : 65536));
    if (dtype == NGC_BF16)
        NGC_LAUNCH((embedding_rows<uint16_t>), grid, dim3(256), 0, st, static_cast<const uint16_t *>(table), ids, static_cast<uint16_t *>(y), tokens, vocab, width, scale);
    else
        NGC_LAUNCH((embedding_rows<float>), grid, dim3(256), 0, st, static_cast<const float *>(table), ids, static_cast<float *>(y), tokens, vocab, width, scale);
    return launch_result();
}

size_t embedding_bwd_workspace(int64_t, int, int) { return 0; }

hipError_t launch_embedding_bwd(int dtype, int64_t tokens, int vocab, int width, float scale, const void *dy, const int64_t *ids, float *dtable,
                                void *, hipStream_t st)
{
    if (dtype == NGC_BF16)
        NGC_LAUNCH((embedding_bwd_scan<uint16_t>), dim3(vocab), dim3(256), 0, st, static_cast<const uint16_t *>(dy), ids, dtable, tokens, width, scale);
    else
        NGC_LAUNCH((embedding_bwd_scan<float>), dim3(vocab), dim3(256), 0, st, static_cast<const float *>(dy), ids, dtable, tokens, width, scale);
    return launch_result();
}

}  // namespace ngc
