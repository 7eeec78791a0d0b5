// C entry points of the operators over tokens and a vocabulary: embedding lookup, layer norm, softmax cross entropy of a linear layer,
// and their gradients.  Validation and launches only.
#include "common.h"

#include <math.h>
#include <stdio.h>

using namespace ngc;

namespace {

int launch_status_tokens(hipError_t e)
{
    if (e == hipSuccess) return NGC_OK;
    fprintf(stderr, "ngconv: HIP launch failed: %s\n", hipGetErrorString(e));   // error path only
    return NGC_LAUNCH_FAILED;
}

bool known_type(int32_t dtype) { return dtype == NGC_F32 || dtype == NGC_BF16; }
uintptr_t elem_mask(int32_t dtype) { return dtype == NGC_BF16 ? 1 : 3; }
bool off(const void *p, uintptr_t mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

// a [rows, cols] tensor: fewer than 2^40 elements, as softmax takes
bool sizes_ok(int64_t rows, int64_t cols)
{
    return rows >= 1 && cols >= 1 && rows <= 0x7fffffffll && (unsigned long long)rows * (unsigned long long)cols < (1ull << 40);
}

constexpr int32_t EMBEDDING_BWD_VOCAB = 1 << 21;

// The operands and the logits of a linear layer: the tiles of their products stay within a grid, and offsets inside a tile below 2 GiB
bool xent_sizes_ok(int64_t rows, int32_t width, int32_t vocab)
{
    constexpr unsigned long long most = 1ull << 37;
    return sizes_ok(rows, width) && sizes_ok(vocab, width) && rows < (1 << 28) && vocab < (1 << 28) && width < (1 << 20) && (unsigned long long)rows * (unsigned)width < most &&
           (unsigned long long)(unsigned)vocab * (unsigned)width < most && (unsigned long long)rows * (unsigned)vocab < most;
}

}  // namespace

extern "C" {

int ngc_embedding(int32_t dtype, int64_t tokens, int32_t vocab, int32_t width, float scale, const void *table, const int64_t *ids, void *y,
                  void *hip_stream)
{
    if (!known_type(dtype)) return NGC_BAD_ARG;
    if (!sizes_ok(tokens, width) || !sizes_ok(vocab, width)) return NGC_BAD_SHAPE;
    if (!table || !ids || !y || off(table, elem_mask(dtype)) || off(y, elem_mask(dtype)) || off(ids, 7)) return NGC_BAD_ARG;
    return launch_status_tokens(launch_embedding(dtype, tokens, vocab, width, scale, table, ids, y, static_cast<hipStream_t>(hip_stream)));
}

size_t ngc_embedding_workspace_bytes(int64_t tokens, int32_t vocab, int32_t width)
{
    if (!sizes_ok(tokens, width) || !sizes_ok(vocab, width) || vocab > EMBEDDING_BWD_VOCAB) return 0;
    return embedding_bwd_workspace(tokens, vocab, width);
}

int ngc_embedding_bwd(int32_t dtype, int64_t tokens, int32_t vocab, int32_t width, float scale, const void *dy, const int64_t *ids, float *dtable,
                      void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!known_type(dtype)) return NGC_BAD_ARG;
    if (!sizes_ok(tokens, width) || !sizes_ok(vocab, width) || vocab > EMBEDDING_BWD_VOCAB) return NGC_BAD_SHAPE;
    if (!dy || !ids || !dtable || off(dy, elem_mask(dtype)) || off(dtable, 3) || off(ids, 7) || off(ws, 15)) return NGC_BAD_ARG;
    const size_t need = embedding_bwd_workspace(tokens, vocab, width);
    if (need && (!ws || ws_bytes < need)) return NGC_WORKSPACE_TOO_SMALL;
    return launch_status_tokens(launch_embedding_bwd(dtype, tokens, vocab, width, scale, dy, ids, dtable, ws, static_cast<hipStream_t>(hip_stream)));
}

int ngc_layer_norm(int32_t dtype, int64_t rows, int32_t cols, float eps, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                   float *rstd, void *hip_stream)
{
    if (!known_type(dtype) || !(eps >= 0.f) || isinf(eps)) return NGC_BAD_ARG;
    if (!sizes_ok(rows, cols)) return NGC_BAD_SHAPE;
    if (!x || !y || off(x, elem_mask(dtype)) || off(y, elem_mask(dtype)) || off(gamma, 3) || off(beta, 3) || off(mean, 3) || off(rstd, 3)) return NGC_BAD_ARG;
    return launch_status_tokens(launch_layer_norm(dtype, (int)rows, cols, eps, x, gamma, beta, y, mean, rstd, static_cast<hipStream_t>(hip_stream)));
}

size_t ngc_layer_norm_workspace_bytes(int32_t dtype, int64_t rows, int32_t cols)
{
    return known_type(dtype) && sizes_ok(rows, cols) ? layer_norm_bwd_workspace(dtype, (int)rows, cols) : 0;
}

int ngc_layer_norm_bwd(int32_t dtype, int64_t rows, int32_t cols, const void *x, const float *gamma, const float *mean, const float *rstd,
                       const void *dy, void *dx, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!known_type(dtype)) return NGC_BAD_ARG;
    if (!sizes_ok(rows, cols)) return NGC_BAD_SHAPE;
    if (!x || !mean || !rstd || !dy || !dx || off(x, elem_mask(dtype)) || off(dy, elem_mask(dtype)) || off(dx, elem_mask(dtype)) || off(gamma, 3) ||
        off(mean, 3) || off(rstd, 3) || off(dgamma, 3) || off(dbeta, 3) || off(ws, 15))
        return NGC_BAD_ARG;
    if ((dgamma || dbeta) && (!ws || ws_bytes < layer_norm_bwd_workspace(dtype, (int)rows, cols))) return NGC_WORKSPACE_TOO_SMALL;
    return launch_status_tokens(launch_layer_norm_bwd(dtype, (int)rows, cols, x, gamma, mean, rstd, dy, dx, dgamma, dbeta, ws,
                                                      static_cast<hipStream_t>(hip_stream)));
}

size_t ngc_linear_xent_workspace_bytes(int32_t dtype, int64_t rows, int32_t width, int32_t vocab, int32_t bwd)
{
    return known_type(dtype) && xent_sizes_ok(rows, width, vocab) ? linear_xent_workspace(dtype, rows, width, vocab, bwd != 0) : 0;
}

int ngc_linear_xent(int32_t dtype, int64_t rows, int32_t width, int32_t vocab, const void *x, const void *w, const int64_t *labels, float *loss,
                    float *lse, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!known_type(dtype)) return NGC_BAD_ARG;
    if (!xent_sizes_ok(rows, width, vocab)) return NGC_BAD_SHAPE;
    if (!x || !w || !labels || !loss || !lse || off(x, elem_mask(dtype)) || off(w, elem_mask(dtype)) || off(labels, 7) || off(loss, 3) || off(lse, 3) ||
        off(ws, 15))
        return NGC_BAD_ARG;
    if (!ws || ws_bytes < linear_xent_workspace(dtype, rows, width, vocab, false)) return NGC_WORKSPACE_TOO_SMALL;
    return launch_status_tokens(launch_linear_xent(dtype, (int)rows, width, vocab, x, w, labels, loss, lse, ws, static_cast<hipStream_t>(hip_stream)));
}

int ngc_linear_xent_bwd(int32_t dtype, int64_t rows, int32_t width, int32_t vocab, const void *x, const void *w, const int64_t *labels,
                        const float *lse, const float *dloss, void *dx, void *dw, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!known_type(dtype)) return NGC_BAD_ARG;
    if (!xent_sizes_ok(rows, width, vocab)) return NGC_BAD_SHAPE;
    if (!x || !w || !labels || !lse || !dloss || (!dx && !dw) || off(x, elem_mask(dtype)) || off(w, elem_mask(dtype)) || off(labels, 7) || off(lse, 3) ||
        off(dloss, 3) || off(dx, elem_mask(dtype)) || off(dw, elem_mask(dtype)) || off(ws, 15))
        return NGC_BAD_ARG;
    if (!ws || ws_bytes < linear_xent_workspace(dtype, rows, width, vocab, true)) return NGC_WORKSPACE_TOO_SMALL;
    return launch_status_tokens(launch_linear_xent_bwd(dtype, (int)rows, width, vocab, x, w, labels, lse, dloss, dx, dw, ws,
                                                       static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
