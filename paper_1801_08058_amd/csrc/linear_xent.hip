// Softmax cross entropy of a linear layer over a vocabulary, and the gradients of both operands (gfx950).
//
//   z = x w^T,  lse[n] = log sum_v exp z[n][v],  loss[n] = lse[n] - z[n][label[n]]   (0 where the label is outside the vocabulary)
//   g[n][v] = (exp(z[n][v] - lse[n]) - [v = label[n]]) dloss[n],  dx = g w,  dw = g^T x
//
// The logits are never kept: the forward pass leaves of every tile the maximum and the sum of each row; the backward pass forms g again
// for a piece of the vocabulary at a time.  All products run on the bf16 matrix cores (mm_bf16.h); fp32 tensors as three limbs of bf16, which
// six products of limbs multiply as exactly as fp32 arithmetic does, at a sixth of the bf16 rate: the fp32 matrix instructions have a sixteenth.
//
// Bound: matrix pipes; few rows HBM, the weight read once per product (loss of 1 x 4096 over 50257 classes bf16: 99 us, 4.2 TB/s); few rows and classes
// the chain of launches (128 x 2048 over 1000 classes: six of 4 to 9 us).  8192 x 4096 over 50257 classes bf16: loss 2.8 ms, with gradients 10.7 ms
// of which the logits, formed again, are 2.9.
#include "mm_bf16.h"
#include "rows.h"

#include <stdlib.h>

namespace ngc {

static size_t r256(size_t b) { return (b + 255) & ~(size_t)255; }

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// exp(z - top).  The difference comes first: a masked logit may be the lowest number of its type, which times log2 e leaves the range of fp32.  Where all
// of a part's logits are -inf (or it has none) there is no difference: top 0 makes their exponentials 0.
__device__ __forceinline__ float exp_below(float z, float top) { return __builtin_amdgcn_exp2f((z - (top == -INFINITY ? 0.f : top)) * LOG2E); }

// What the backward pass needs of a row: lse, dloss over the largest |dloss| (0 for rows that do not count), the label (-1)
struct XentRow {
    float lse, factor;
    int label, pad;
};

constexpr int XENT_ROWS = 8192, XENT_TOPS = 256;         // rows of a workgroup's step; workgroups at most

// What a workgroup of 1024 takes of XENT_ROWS rows from m0 on: eight rows a thread, whose loads are under way together
struct XentRows {
    static constexpr int B = XENT_ROWS / 1024;
    int64_t label[B];                                                    // -1: does not count
    float weight[B], l[B];
    __device__ __forceinline__ void load(const int64_t *labels, const float *dloss, const float *lse, int64_t m0, int rows, int vocab)
    {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const int64_t m = m0 + 1024 * b + threadIdx.x;
            label[b] = -1;
            if (m < rows) label[b] = labels[m], weight[b] = dloss[m], l[b] = lse ? lse[m] : 0.f;
            if (label[b] >= vocab) label[b] = -1;
        }
    }
    __device__ __forceinline__ float most(float top) const
    {
#pragma unroll
        for (int b = 0; b < B; ++b)
            if (label[b] >= 0) top = fmaxf(top, fabsf(weight[b]));
        return top;
    }
};

// Largest |dloss| of the rows that count, workgroup by workgroup: where one workgroup does not take all rows in a step
__global__ __launch_bounds__(1024) void xent_tops(const int64_t *__restrict__ labels, const float *__restrict__ dloss, float *__restrict__ tops, int rows, int vocab)
{
    __shared__ float sm[16];
    XentRows r;
    float top = 0.f;
    for (int64_t m0 = (int64_t)blockIdx.x * XENT_ROWS; m0 < rows; m0 += (int64_t)gridDim.x * XENT_ROWS) {
        r.load(labels, dloss, nullptr, m0, rows, vocab);
        top = r.most(top);
    }
    top = block_reduce<16>(top, true, sm);
    if (threadIdx.x == 0) tops[blockIdx.x] = top;
}

// The gradient's rows are scaled by dloss / max |dloss| before they are rounded to bf16, and the results by max |dloss| in fp32: where all rows
// weigh the same (a mean), the weight's own rounding would otherwise be the same in every term of the sums.  count: the workgroups that left tops;
// 0: the only workgroup sees all rows.  (65536 rows: 38 us by one workgroup, 11 us in two launches of eight.)
__global__ __launch_bounds__(1024) void xent_rows(const int64_t *__restrict__ labels, const float *__restrict__ lse, const float *__restrict__ dloss,
                                                  const float *__restrict__ tops, int count, XentRow *__restrict__ info, float *__restrict__ scale, int rows, int vocab)
{
    __shared__ float sm[16];
    XentRows r;
    r.load(labels, dloss, lse, (int64_t)blockIdx.x * XENT_ROWS, rows, vocab);
    float top = count ? ((int)threadIdx.x < count ? tops[threadIdx.x] : 0.f) : r.most(0.f);
    top = fmaxf(block_reduce<16>(top, true, sm), 0x1p-100f);             // all zero: any scale
    const float inv = 1.0f / top;
    for (int64_t m0 = (int64_t)blockIdx.x * XENT_ROWS; m0 < rows;) {
#pragma unroll
        for (int b = 0; b < XentRows::B; ++b) {
            const int64_t m = m0 + 1024 * b + threadIdx.x;
            if (m < rows) info[m] = XentRow{r.l[b], r.label[b] >= 0 ? r.weight[b] * inv : 0.f, r.label[b] >= 0 ? (int)r.label[b] : -1, 0};
        }
        m0 += (int64_t)gridDim.x * XENT_ROWS;
        if (m0 < rows) r.load(labels, dloss, lse, m0, rows, vocab);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *scale = top;
}

// The first limb of a finite value is finite: the numbers above the largest bf16, which would be rounded to infinity, leave up to 2^-8 of themselves to the second
__device__ __forceinline__ float within_bf16(float v)
{
    constexpr float most = 0x1.fep127f;
    return __builtin_amdgcn_fmed3f(v, -most, most);
}

// Eight values as L limbs: the value rounded to bf16, what that leaves, rounded, and what that leaves (one limb: values that bf16 holds)
template <int L>
__device__ __forceinline__ void split_limbs(const float (&f)[8], mm_bf16x8 (&out)[L])
{
    float r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = f[k];
#pragma unroll
    for (int q = 0; q < L; ++q) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = L > 1 && q == 0 ? pack_bf16x2_hw(within_bf16(r[2 * k]), within_bf16(r[2 * k + 1])) : pack_bf16x2_hw(r[2 * k], r[2 * k + 1]);
            r[2 * k] -= __uint_as_float(w[k] << 16);
            r[2 * k + 1] -= __uint_as_float(w[k] & 0xFFFF0000u);
        }
        __builtin_memcpy(&out[q], w, 16);
    }
}
// c + a b^T: of three limbs the six products that mm_bf16.h forms, of one and two both
template <int PA, int PB>
__device__ __forceinline__ mm_f32x4 limb_products(const mm_bf16x8 (&a)[PA], const mm_bf16x8 (&b)[PB], mm_f32x4 c)
{
    static_assert((PA == 1 && PB <= 2) || (PA == 3 && PB == 3), "limbs");
    if constexpr (PB == 2) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[1], c, 0, 0, 0);
    if constexpr (PA == 3) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[2], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[2], b[0], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1], b[1], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[1], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1], b[0], c, 0, 0, 0);
    }
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b[0], c, 0, 0, 0);
}

// g as an operand of dx and dw has the three limbs of fp32 tensors, and of bf16 tensors two (16 bits) up to XENT_FINE_ROWS rows or XENT_FINE_WORK multiply-adds
// of a product, one (rounded to bf16) in larger calls.  The rounding of the g at a label is the same in all elements of the row's dx that come from it, and
// in those of the label's dw: with one limb the distance from exact gradients is 0.0018 to 0.0022 of their norm, with two the 0.0017 that rounding the
// results leaves (1 to 2048 rows).  Two limbs are twice the matrix instructions.  In small calls and with few rows launches and memory bound dx and dw, above
// that those instructions do.  Loss and gradients with one limb and with two: 128 x 2048 over 1000 classes 28 -> 30 us, 1000 x 512 over 1000 29 -> 32,
// 1024 x 1024 over 2048 46 -> 53; 2048 wide over 32000 classes 111 -> 117 us for 8 rows, 152 -> 175 for 128, 207 -> 254 for 256, 0.95 -> 1.47 ms for 2048; 2048 x
// 2048 over 2048 91 -> 143 us; 8192 x 4096 over 50257 10.7 -> 18.3 ms.
constexpr int XENT_FINE_ROWS = 128;
constexpr double XENT_FINE_WORK = 2147483648.0;
static int xent_glimbs(int limbs, int64_t rows, int width, int vocab)
{
    const char *forced = env_switch(SW_XENT_LIMBS);
    if (forced && limbs == 1) return atoi(forced) == 2 ? 2 : 1;
    return limbs == 3 ? 3 : rows <= XENT_FINE_ROWS || (double)rows * (double)width * (double)vocab <= XENT_FINE_WORK ? 2 : 1;
}

// T: uint16_t (bf16) or float (in limbs)
enum XentEpilogue { XE_STATS, XE_GRAD, XE_SLAB, XE_OUT };

struct XentMm {
    MmParams mm;
    int v0;                              // STATS, GRAD: first class of the piece
    const int64_t *labels;               // STATS
    float2 *part;                        // STATS: [tiles][rows], from this piece's first tile on
    float *target;                       // STATS
    const XentRow *info;                 // GRAD
    const float *scale;                  // OUT
    void *out;                           // GRAD: g (its limbs, glimb elements apart), OUT: the result
    int64_t ldo, glimb;
    int store_m, store_n;                // rows and columns that are stored (GRAD: zeros past the rows and the piece)
    float *slab;                         // SLAB: [splits][M][ldo]
    int add;                             // SLAB: onto what is there; OUT: the slab ([M][N]) joins the result
};

// limbs of the operands: dx and dw (BT) take g, of G limbs, first
template <typename T, int G, bool BT> constexpr int xent_pa() { return BT ? G : sizeof(T) == 4 ? 3 : 1; }
template <typename T> constexpr int xent_pb() { return sizeof(T) == 4 ? 3 : 1; }

template <typename T, int G, int BM, int BN, bool AT, bool BT, XentEpilogue E>
__device__ __forceinline__ void xent_product(const XentMm &p, int block)
{
    constexpr int FM = BM / 32, FN = BN / 32;
    constexpr bool LIMBS = sizeof(T) == 4;
    extern __shared__ __align__(16) unsigned char smem[];
    const int tiles = p.mm.mt * p.mm.nt, split = block / tiles;
    int tm, tn;
    mm_tile_of(block - split * tiles, tiles, p.mm.mt, p.mm.nt, tm, tn);
    const int k0 = split * p.mm.kper, k1 = p.mm.K - k0 < p.mm.kper ? p.mm.K : k0 + p.mm.kper;
    mm_f32x4 acc[FN][FM];
    mm_tile<BM, BN, AT, BT, xent_pa<T, G, BT>(), xent_pb<T>()>(p.mm, smem, tm * BM, tn * BN, k0, k1, acc);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int wm = (wave % 2) * (BM / 2), wn = (wave / 2) * (BN / 2);
    const int m_ = tm * BM + wm + (lane & 15), n_ = tn * BN + wn + 4 * g;       // + 16 fm, + 16 fn + element
    if constexpr (E == XE_STATS) {
        // a row of the tile: its maximum and sum of exponentials over 4 FN values of a lane, 4 lanes, 2 waves
        float2 *red = reinterpret_cast<float2 *>(smem);                          // [2][BM]
        int label[FM];                                                           // class of the piece, or -1
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const uint64_t at = m_ + 16 * j < p.mm.M ? (uint64_t)p.labels[m_ + 16 * j] - (uint64_t)p.v0 : ~0ull;     // in front of the piece: huge
            label[j] = at < (uint64_t)p.mm.N ? (int)at : -1;
        }
        auto rows = [&](auto whole) {                                            // whole: no columns past the end, which count nothing
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                float top = -INFINITY, s = 0.f;
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, whole || n_ + 16 * i + e < p.mm.N ? acc[i][j][e] : -INFINITY);
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));                       // -inf: columns past the end (or logits that are -inf) only, sum 0
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = exp_below(acc[i][j][e], top);
                        s += whole || n_ + 16 * i + e < p.mm.N ? v : 0.f;
                    }
                s += __shfl_xor(s, 16, 64);
                s += __shfl_xor(s, 32, 64);
                if (g == 0) red[(wave / 2) * BM + wm + 16 * j + lane] = make_float2(top, s);
                if (label[j] >= tn * BN + wn && label[j] < tn * BN + wn + BN / 2) {      // in the same pass: 256 values are not kept for another
#pragma unroll
                    for (int i = 0; i < FN; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (label[j] == n_ + 16 * i + e) p.target[m_ + 16 * j] = acc[i][j][e];
                }
            }
        };
        if ((tn + 1) * BN <= p.mm.N) rows(std::true_type());
        else rows(std::false_type());
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += 64 * MM_WAVES) {
            float2 v = red[r];
            const float2 o = red[BM + r];
            const float top = fmaxf(v.x, o.x);
            v = make_float2(top, v.y * exp_below(v.x, top) + o.y * exp_below(o.x, top));
            if (tm * BM + r < p.mm.M) p.part[(size_t)tn * p.mm.M + tm * BM + r] = v;
        }
        return;
    }
    float scale = 1.f;
    if constexpr (E == XE_OUT) scale = *p.scale;
    const bool whole = (tn + 1) * BN <= p.store_n;
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int m = m_ + 16 * j;
        if constexpr (E == XE_SLAB) {
            if (m >= p.store_m) continue;
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const int n = n_ + 16 * i;
                if (n >= p.store_n) continue;
                float *at = p.slab + ((size_t)split * p.mm.M + m) * p.ldo + n;  // ldo and store_n are multiples of 8
                mm_f32x4 v = acc[i][j];
                if (p.add) v += *reinterpret_cast<const mm_f32x4 *>(at);
                *reinterpret_cast<mm_f32x4 *>(at) = v;
            }
            continue;
        }
        if constexpr (E == XE_GRAD) {
            XentRow row = {0.f, 0.f, -1, 0};
            if (m < p.mm.M) row = p.info[m];
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = exp_below(acc[i][j][e], row.lse) * row.factor;
            const int label = row.label - p.v0;                                  // few waves hold one
            if (__any(label >= tn * BN + wn && label < tn * BN + wn + BN / 2)) {
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] -= label == n_ + 16 * i + e ? row.factor : 0.f;
            }
            if ((tn + 1) * BN > p.mm.N || __any(row.label < 0)) {                // +0 past the piece and in rows that do not count
#pragma unroll
                for (int i = 0; i < FN; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row.label < 0 || n_ + 16 * i + e >= p.mm.N) acc[i][j][e] = 0.f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const int n = n_ + 16 * i;
                if (p.add && m < p.store_m && n < p.mm.N) acc[i][j] += *reinterpret_cast<const mm_f32x4 *>(p.slab + (size_t)m * p.mm.N + n);
                acc[i][j] *= scale;
            }
        }
        if constexpr (E == XE_OUT && LIMBS) {
            if (m >= p.store_m) continue;
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const int n = n_ + 16 * i;
                float *at = static_cast<float *>(p.out) + (size_t)m * p.ldo + n;
                if (whole || n + 4 <= p.store_n) {
                    __builtin_memcpy(at, &acc[i][j], 16);                        // any element address
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + e < p.store_n) at[e] = acc[i][j][e];
                }
            }
            continue;
        }
        // bf16: the four lanes of a row exchange quarters of two fragments, so that each has 8 neighbouring columns and a store covers 64 bytes of
        // the row.  Swapping the upper half wave of the first with the lower of the second gives lane g of fragment g / 2 the quarters g % 2 and
        // 2 + g % 2, swapping odd and even rows of 16 lanes then the quarters 2 (g % 2) and 2 (g % 2) + 1.
#pragma unroll
        for (int i = 0; i < FN; i += 2)
#pragma unroll
            for (int l = 0; l < (E == XE_GRAD ? G : 1); ++l) {
                uint32_t q[2][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    mm_f32x4 &v = acc[i + k][j];
                    q[k][0] = pack_bf16x2_hw(v[0], v[1]);
                    q[k][1] = pack_bf16x2_hw(v[2], v[3]);
                    if (E == XE_GRAD && G > 1)
                        v -= mm_f32x4{__uint_as_float(q[k][0] << 16), __uint_as_float(q[k][0] & 0xFFFF0000u), __uint_as_float(q[k][1] << 16), __uint_as_float(q[k][1] & 0xFFFF0000u)};
                }
                uint32_t o[4];
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const auto a = __builtin_amdgcn_permlane32_swap(q[0][w], q[1][w], false, false);
                    const auto b = __builtin_amdgcn_permlane16_swap(a[0], a[1], false, false);
                    o[w] = b[0];
                    o[2 + w] = b[1];
                }
                const int n = tn * BN + wn + 16 * i + 16 * (g >> 1) + 8 * (g & 1);
                uint16_t *at = static_cast<uint16_t *>(p.out) + (size_t)m * p.ldo + n + l * p.glimb;
                if (m >= p.store_m) continue;
                if (whole || n + 8 <= p.store_n) {
                    __builtin_memcpy(at, o, 16);                                 // any element address
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < p.store_n) at[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
                }
            }
    }
}

template <typename T, int G, int EDGE, bool AT, bool BT, XentEpilogue E>
__global__ __launch_bounds__(64 * MM_WAVES) void xent_mm(const XentMm p)
{
    xent_product<T, G, EDGE, EDGE, AT, BT, E>(p, blockIdx.x);
}

// dx and dw of one piece, which both read g: the workgroups of dx, then those of dw
template <typename T, int G, int EDGE, XentEpilogue EDX>
__global__ __launch_bounds__(64 * MM_WAVES) void xent_mm_both(const XentMm dx, const XentMm dw, int first)
{
    if ((int)blockIdx.x < first) xent_product<T, G, EDGE, EDGE, false, true, EDX>(dx, blockIdx.x);
    else xent_product<T, G, EDGE, EDGE, true, true, XE_OUT>(dw, blockIdx.x - first);
}

// Few tiles: the logits' product runs in parts (fp32 slabs, `stride` elements apart, rows of `ld`), and a workgroup per row adds them up.
__device__ __forceinline__ mm_f32x4 sum_parts(const float *at, int splits, size_t stride)
{
    constexpr int B = 8;                                                         // parts under way together, added in their order
    mm_f32x4 v = *reinterpret_cast<const mm_f32x4 *>(at);
    int q = 1;
    for (; q + B <= splits; q += B) {
        mm_f32x4 f[B];
#pragma unroll
        for (int b = 0; b < B; ++b) f[b] = *reinterpret_cast<const mm_f32x4 *>(at + (q + b) * stride);
#pragma unroll
        for (int b = 0; b < B; ++b) v += f[b];
    }
#pragma unroll 4
    for (; q < splits; ++q) v += *reinterpret_cast<const mm_f32x4 *>(at + q * stride);
    return v;
}

constexpr int XENT_BATCH = 4;                                            // groups of four classes of a thread under way together

template <int NW>
__global__ __launch_bounds__(64 * NW) void xent_row_loss(const float *__restrict__ slab, int splits, size_t stride, int ld, const int64_t *__restrict__ labels,
                                                         float *__restrict__ loss, float *__restrict__ lse, int vocab)
{
    __shared__ float sm[NW], target;
    const int m = blockIdx.x;
    const int64_t label = labels[m];
    const bool live = label >= 0 && label < vocab;
    float top = -INFINITY, s = 0.f;
    for (int w0 = 0; w0 < vocab; w0 += 256 * NW * XENT_BATCH) {
        const int v0 = w0 + threadIdx.x * 4;
        mm_f32x4 z[XENT_BATCH];
#pragma unroll
        for (int b = 0; b < XENT_BATCH; ++b) {
            if (w0 + 256 * NW * b >= vocab) break;
            const int v = v0 + 256 * NW * b;
            z[b] = sum_parts(slab + (size_t)m * ld + (v < vocab ? v : 0), splits, stride);
        }
        float up = top;
#pragma unroll
        for (int b = 0; b < XENT_BATCH; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = v0 + 256 * NW * b + e;
                if (v >= vocab) z[b][e] = -INFINITY;                             // groups that were not loaded among them
                up = fmaxf(up, z[b][e]);
                if (label == v && live) target = z[b][e];
            }
        s *= exp_below(top, up);                                                 // 0 the first time
        top = up;
#pragma unroll
        for (int b = 0; b < XENT_BATCH; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s += exp_below(z[b][e], top);
    }
    const float all = block_reduce<NW>(top, true, sm);
    s = block_reduce<NW>(s * exp_below(top, all), false, sm);
    if (threadIdx.x) return;
    const float l = all + log2f(s) * LN2;
    lse[m] = l;
    loss[m] = live ? l - target : 0.f;
}

// g of a row, as xent_rows and the epilogue of the product form it; rows from `rows` on are zeros.  Workgroup 0 leaves the scale.
template <int G, int NW>
__global__ __launch_bounds__(64 * NW) void xent_row_grad(const float *__restrict__ slab, int splits, size_t stride, int ld, const int64_t *__restrict__ labels,
                                                         const float *__restrict__ lse, const float *__restrict__ dloss, uint16_t *__restrict__ g,
                                                         int64_t glimb, int gp, float *__restrict__ scale, int rows, int vocab)
{
    __shared__ float sm[NW];
    const int m = blockIdx.x;
    float most = 0.f;
#pragma unroll 4
    for (int r = threadIdx.x; r < rows; r += 64 * NW) {
        const int64_t label = labels[r];
        const float weight = fabsf(dloss[r]);
        most = fmaxf(most, label >= 0 && label < vocab ? weight : 0.f);
    }
    most = fmaxf(block_reduce<NW>(most, true, sm), 0x1p-100f);
    if (m == 0 && threadIdx.x == 0) *scale = most;
    const int64_t label = m < rows ? labels[m] : -1;
    const bool live = label >= 0 && label < vocab;
    const float factor = live ? dloss[m] * (1.0f / most) : 0.f, below = live ? lse[m] : 0.f;
    const size_t row = (size_t)(live ? m : 0) * ld;
    for (int w0 = 0; w0 < gp; w0 += 256 * NW * XENT_BATCH) {
        const int v0 = w0 + threadIdx.x * 4;
        mm_f32x4 z[XENT_BATCH];
#pragma unroll
        for (int b = 0; b < XENT_BATCH; ++b) {
            if (w0 + 256 * NW * b >= gp) break;
            const int v = v0 + 256 * NW * b;
            z[b] = sum_parts(slab + row + (v < vocab ? v : 0), splits, stride);
        }
#pragma unroll
        for (int b = 0; b < XENT_BATCH; ++b) {
            const int v = v0 + 256 * NW * b;
            if (v >= gp) break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                z[b][e] = live && v + e < vocab ? exp_below(z[b][e], below) * factor - (label == v + e ? factor : 0.f) : 0.f;
#pragma unroll
            for (int l = 0; l < G; ++l) {
                const uint2 q = make_uint2(pack_bf16x2_hw(z[b][0], z[b][1]), pack_bf16x2_hw(z[b][2], z[b][3]));
                *reinterpret_cast<uint2 *>(g + l * glimb + (size_t)m * gp + v) = q;
                z[b] -= mm_f32x4{__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u)};
            }
        }
    }
}

// ---- few rows, and a weight that the products above would have to copy (fp32, rows of no multiple of 16 bytes) ----
//
// The weight goes straight from memory to registers, at any alignment, and becomes limbs there: it is read once per product, where a copy
// reads it, writes three bf16 values per element and reads those.  Bound: HBM (fp32, 33024 classes of 1024: 29 us for 8 rows, 4.7 TB/s, 48 for 64);
// bf16 rows of odd lengths the L1, which serves loads off the 4-byte grid in pieces (54005 classes of 2541, 18 rows: 109 us, fp32 150).

// The k of element e of lane group g within a step of 32: a lane's 16 bytes, and with them 64 bytes of a row in one load, lie together
template <typename T> __host__ __device__ constexpr int few_k(int g, int e) { return sizeof(T) == 4 ? 16 * (e / 4) + 4 * g + e % 4 : 8 * g + e; }

// A lane's eight elements of a step of a row, `left` elements of which are from the step on (those behind the row are zeros)
template <typename T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ void load(const T *step, int g, int left)
    {
        constexpr int E = 16 / sizeof(T);                                        // elements of a load
#pragma unroll
        for (int e = 0; e < 8; e += E) {
            const int k = few_k<T>(g, e);
            T v[E];
            if (k + E <= left) {
                __builtin_memcpy(v, step + k, 16);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = k + i < left ? step[k + i] : T(0);
            }
            __builtin_memcpy(w + e * sizeof(T) / 4, v, 16);
        }
    }
    template <int L> __device__ __forceinline__ void limbs(mm_bf16x8 (&out)[L]) const
    {
        if constexpr (L == 1) {
            __builtin_memcpy(&out[0], w, 16);
        } else {
            float f[8];
            __builtin_memcpy(f, w, 32);
            split_limbs(f, out);
        }
    }
};

template <typename T> constexpr int few_g() { return sizeof(T) == 4 ? 3 : 2; }          // limbs of g

// blocks of 16 classes of a workgroup: more rows of x, which every workgroup reads, more classes for them
constexpr int xent_few_blocks(int mt) { return mt == 1 ? 2 : 4; }

// x for xent_few_z: of every step, block of 16 rows and limb what the 64 lanes hold, 1 KB in their order: eight lines a load, where rows are sixteen
template <typename T>
__global__ __launch_bounds__(256) void xent_pack(const T *__restrict__ x, uint4 *__restrict__ dst, int rows, int width, int blocks)
{
    constexpr int L = sizeof(T) == 4 ? 3 : 1;
    const int lane = threadIdx.x & 63, g = lane >> 4, n = blockIdx.x;
    for (int j = threadIdx.x >> 6; j < blocks; j += 4) {
        const int m = 16 * j + (lane & 15);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = 32 * n + few_k<T>(g, e);
            f[e] = m < rows && k < width ? SmElem<T>::load(x + (size_t)m * width + k) : 0.f;
        }
        mm_bf16x8 limb[L];
        split_limbs(f, limb);
#pragma unroll
        for (int q = 0; q < L; ++q) dst[(((size_t)n * blocks + j) * L + q) * 64 + lane] = __builtin_bit_cast(uint4, limb[q]);
    }
}

// z[m][v] of 16 IB classes and MT blocks of 16 rows.  The four waves take every fourth step of 32 elements and are added up through LDS: what the
// workgroup has under way of a class lies together (fp32, 54005 classes of 2541, 18 rows: 205 us with 32 classes of its own for each wave, 143).
// One step ahead and as many waves as fit: four steps ahead in a wave take the registers of the others, and no less time.
template <typename T, int MT>
__global__ __launch_bounds__(256) void xent_few_z(const uint4 *__restrict__ x, const T *__restrict__ w, float *__restrict__ z, int ld, int rows, int width,
                                                  int vocab)
{
    constexpr int L = sizeof(T) == 4 ? 3 : 1, IB = xent_few_blocks(MT);
    __shared__ mm_f32x4 sums[3][IB * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4, v0 = blockIdx.x * 16 * IB, j0 = blockIdx.y * MT, blocks = gridDim.y * MT;
    const T *row[IB];
#pragma unroll
    for (int i = 0; i < IB; ++i) row[i] = w + (size_t)(v0 + 16 * i + l < vocab ? v0 + 16 * i + l : vocab - 1) * width;
    mm_f32x4 acc[IB][MT];
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = mm_f32x4{0.f, 0.f, 0.f, 0.f};
    // x is under way as far ahead as the weight: loads arrive in their order, and a step that asked for its x itself would wait for the next weights
    struct Step {
        Eight<T> w[IB];
        uint4 x[MT][L];
    };
    const int full = (width / 32 - wave + 3) / 4;                                // whole steps of this wave: wave, wave + 4, ..
    auto load = [&](Step &to, int n, int left) {
#pragma unroll
        for (int i = 0; i < IB; ++i) to.w[i].load(row[i] + 32 * n, g, left);
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int q = 0; q < L; ++q) to.x[j][q] = x[(((size_t)n * blocks + j0 + j) * L + q) * 64 + lane];
    };
    auto products = [&](const Step &from) {
        mm_bf16x8 a[IB][L], b[MT][L];
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int q = 0; q < L; ++q) b[j][q] = __builtin_bit_cast(mm_bf16x8, from.x[j][q]);
#pragma unroll
        for (int i = 0; i < IB; ++i) from.w[i].template limbs<L>(a[i]);
#pragma unroll
        for (int i = 0; i < IB; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = limb_products(a[i], b[j], acc[i][j]);
    };
    Step now, next;
    if (full > 0) load(next, wave, 32);
    for (int n = 0; n < full; ++n) {
        now = next;
        if (n + 1 < full) load(next, 4 * (n + 1) + wave, 32);
        products(now);
    }
    if (width % 32 && wave == (width / 32 & 3)) {
        load(now, width / 32, width % 32);
        products(now);
    }
    if (wave)
#pragma unroll
        for (int q = 0; q < IB * MT; ++q) sums[wave - 1][q][lane] = acc[q / MT][q % MT];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int q = 0; q < IB * MT; ++q) acc[q / MT][q % MT] += sums[s][q][lane];
#pragma unroll
    for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const int m = 16 * (j0 + j) + l, v = v0 + 16 * i + 4 * g;
            if (m < rows && v < ld) *reinterpret_cast<mm_f32x4 *>(z + (size_t)m * ld + v) = acc[i][j];
        }
}

// dx[m][d] = sum_v g[m][v] w[v][d] of 64 columns and MT blocks of 16 rows over the classes of part blockIdx.y: a slab.  The four waves take every
// fourth step of 32 classes and are added up through LDS.  Column 4 r + c is row r of fragment c, so that a lane loads four columns of a class.
template <typename T, int MT>
__global__ __launch_bounds__(256) void xent_few_dx(const uint16_t *__restrict__ gr, int64_t glimb, int gp, const T *__restrict__ w, float *__restrict__ slab,
                                                   int pitch, int rows, int width, int vocab, int per_part)
{
    constexpr int L = sizeof(T) == 4 ? 3 : 1, G = few_g<T>();
    __shared__ mm_f32x4 sums[3][4 * MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, g = lane >> 4;
    const int d = blockIdx.x * 64 + 4 * l, m0 = blockIdx.z * 16 * MT, end = per_part * (blockIdx.y + 1) < vocab ? per_part * (blockIdx.y + 1) : vocab;
    mm_f32x4 acc[4][MT];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[c][j] = mm_f32x4{0.f, 0.f, 0.f, 0.f};
    const uint16_t *xr[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) xr[j] = gr + (size_t)(m0 + 16 * j + l < rows ? m0 + 16 * j + l : rows - 1) * gp;
    // A step is 32 classes, of which a lane holds four columns of eight.  A lane whose four columns end behind the row loads the row's last four, of
    // which the products take what is theirs (shift).  fp32: one step ahead (a ring of two, unrolled, takes 216 registers instead of 160: 187 against
    // 131 us for 54005 classes of 2541); bf16 steps are half as long, three ahead and g with them (146 -> 80 us with one
    // limb of g, 84 with both).
    struct Step {
        uint32_t w[8][sizeof(T)];                                                // four elements
        uint4 g[L == 1 ? MT : 1][G];
    };
    const int from = d + 4 <= width ? d : width - 4, shift = d - from;
    auto load = [&](Step &to, int v0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int v = v0 + 8 * g + k < vocab ? v0 + 8 * g + k : vocab - 1;                          // g is zero past the classes
            const T *p = w + (size_t)v * width;
            if (width >= 4) {
                __builtin_memcpy(to.w[k], p + from, 4 * sizeof(T));
            } else {
                T e[4] = {p[0], width > 1 ? p[1] : T(0), width > 2 ? p[2] : T(0), T(0)};
                __builtin_memcpy(to.w[k], e, sizeof(e));
            }
        }
        if constexpr (L == 1)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int q = 0; q < G; ++q) to.g[j][q] = *reinterpret_cast<const uint4 *>(xr[j] + q * glimb + v0 + 8 * g);
    };
    const bool edge = width < 4 ? l != 0 : shift != 0, edges = __any(edge);
    auto products = [&](const Step &now, int v0) {
        float4 e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if constexpr (sizeof(T) == 4) __builtin_memcpy(&e[k], now.w[k], 16);
            else e[k] = make_float4(__uint_as_float(now.w[k][0] << 16), __uint_as_float(now.w[k][0] & 0xFFFF0000u), __uint_as_float(now.w[k][1] << 16), __uint_as_float(now.w[k][1] & 0xFFFF0000u));
        }
        if (edges)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 q = e[k];
                if (!edge) continue;
                e[k] = width < 4 || shift > 3 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                              : make_float4(shift == 1 ? q.y : shift == 2 ? q.z : q.w, shift == 1 ? q.z : shift == 2 ? q.w : 0.f, shift == 1 ? q.w : 0.f, 0.f);
            }
        mm_bf16x8 b[MT][G];
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int q = 0; q < G; ++q)
                if constexpr (L == 1) b[j][q] = __builtin_bit_cast(mm_bf16x8, now.g[j][q]);
                else b[j][q] = *reinterpret_cast<const mm_bf16x8 *>(xr[j] + q * glimb + v0 + 8 * g);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = c == 0 ? e[k].x : c == 1 ? e[k].y : c == 2 ? e[k].z : e[k].w;
            mm_bf16x8 a[L];
            split_limbs(f, a);
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[c][j] = limb_products(a, b[j], acc[c][j]);
        }
    };
    const int begin = per_part * blockIdx.y + 32 * wave;
    if constexpr (L == 3) {
        Step now, next;
        if (begin < end) load(next, begin);
        for (int v0 = begin; v0 < end; v0 += 128) {
            now = next;
            if (v0 + 128 < end) load(next, v0 + 128);
            products(now, v0);
        }
    } else {
        constexpr int NB = 4;
        const int steps = begin < end ? (end - begin + 127) / 128 : 0;
        Step step[NB];
#pragma unroll
        for (int u = 0; u < NB - 1; ++u)
            if (u < steps) load(step[u], begin + 128 * u);
        for (int n = 0; n < steps; n += NB)
#pragma unroll
            for (int u = 0; u < NB; ++u) {
                if (n + u >= steps) break;
                if (n + u + NB - 1 < steps) load(step[(u + NB - 1) % NB], begin + 128 * (n + u + NB - 1));
                products(step[u], begin + 128 * (n + u));
            }
    }
    if (wave)
#pragma unroll
        for (int q = 0; q < 4 * MT; ++q) sums[wave - 1][q][lane] = acc[q / MT][q % MT];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int s = 0; s < 3; ++s)
#pragma unroll
        for (int q = 0; q < 4 * MT; ++q) acc[q / MT][q % MT] += sums[s][q][lane];
    float *out = slab + (size_t)blockIdx.y * rows * pitch;
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = m0 + 16 * j + l, at = blockIdx.x * 64 + 16 * g + 4 * e;
            if (m < rows && at < pitch) *reinterpret_cast<mm_f32x4 *>(out + (size_t)m * pitch + at) = mm_f32x4{acc[0][j][e], acc[1][j][e], acc[2][j][e], acc[3][j][e]};
        }
}

// dw[v][d] = scale sum_m g[m][v] x[m][d] of at most R rows: a thread keeps four columns of x and stores them for class after class.  A workgroup
// takes 64 classes, their g in LDS, and 4 LPR columns; 256 / LPR classes at a time.  Bound: HBM for 16 rows, with 32 the vector instructions (fp32,
// 54005 x 2541: 190 us, the matrix cores' tile 208; bf16 184 and 121, so 16 at most).
template <typename T, int R, int LPR>
__global__ __launch_bounds__(256) void xent_few_dw(const uint16_t *__restrict__ gr, int64_t glimb, int gp, const T *__restrict__ x, const float *__restrict__ scale,
                                                   T *__restrict__ dw, int rows, int width, int vocab)
{
    constexpr int CLASSES = 64;
    __shared__ float gs[CLASSES][R];
    const int v0 = blockIdx.x * CLASSES, d = (blockIdx.y * LPR + (threadIdx.x & (LPR - 1))) * 4;
    const float sc = *scale;
    for (int i = threadIdx.x; i < CLASSES * R; i += 256) {
        const int v = i % CLASSES, m = i / CLASSES;
        float s = 0.f;
        if (m < rows)
#pragma unroll
            for (int q = few_g<T>() - 1; q >= 0; --q) s += bf16_bits_to_float(gr[q * glimb + (size_t)m * gp + v0 + v]);        // gp is a multiple of 64
        gs[v][m] = s * sc;
    }
    float4 f[R];
#pragma unroll
    for (int m = 0; m < R; ++m) {
        const T *p = x + (size_t)(m < rows ? m : 0) * width;
        auto at = [&](int c) { return m < rows && c < width ? SmElem<T>::load(p + c) : 0.f; };
        if (d + 4 <= width && m < rows) f[m] = load4_any(p + d);
        else f[m] = make_float4(at(d), at(d + 1), at(d + 2), at(d + 3));
    }
    __syncthreads();
    const int end = vocab - v0 < CLASSES ? vocab - v0 : CLASSES;
    if (d >= width) return;
    for (int v = threadIdx.x / LPR; v < end; v += 256 / LPR) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int m = 0; m < R; ++m) {
            const float g = gs[v][m];
            s.x = fmaf(g, f[m].x, s.x), s.y = fmaf(g, f[m].y, s.y), s.z = fmaf(g, f[m].z, s.z), s.w = fmaf(g, f[m].w, s.w);
        }
        T *at = dw + (size_t)(v0 + v) * width + d;
        if (d + 4 <= width) {
            if constexpr (sizeof(T) == 4) {
                store16_any(at, make_uint4(__float_as_uint(s.x), __float_as_uint(s.y), __float_as_uint(s.z), __float_as_uint(s.w)));
            } else {
                const uint2 b = make_uint2(pack_bf16x2_hw(s.x, s.y), pack_bf16x2_hw(s.z, s.w));
                __builtin_memcpy(at, &b, 8);
            }
        } else {
            SmElem<T>::store(at, s.x);
            if (d + 1 < width) SmElem<T>::store(at + 1, s.y);
            if (d + 2 < width) SmElem<T>::store(at + 2, s.z);
        }
    }
}

// lse and loss of 32 rows from the tiles' maxima and sums, eight parts of the tiles each
__global__ __launch_bounds__(256) void xent_join(const float2 *__restrict__ part, const float *__restrict__ target, const int64_t *__restrict__ labels,
                                                  float *__restrict__ loss, float *__restrict__ lse, int rows, int vocab, int tiles)
{
    __shared__ float2 red[8][32];
    const int r = threadIdx.x & 31, q = threadIdx.x >> 5, m = blockIdx.x * 32 + r;
    float top = -INFINITY, s = 0.f;
    if (m < rows)
        for (int t0 = q; t0 < tiles; t0 += 32) {
            float2 v[4];                                                         // four tiles at a time
#pragma unroll
            for (int b = 0; b < 4; ++b) v[b] = t0 + 8 * b < tiles ? part[(size_t)(t0 + 8 * b) * rows + m] : make_float2(-INFINITY, 0.f);
            float up = top;
#pragma unroll
            for (int b = 0; b < 4; ++b) up = fmaxf(up, v[b].x);
            s *= exp_below(top, up);
#pragma unroll
            for (int b = 0; b < 4; ++b) s += v[b].y * exp_below(v[b].x, up);
            top = up;
        }
    red[q][r] = make_float2(top, s);
    __syncthreads();
    if (q || m >= rows) return;
    for (int i = 1; i < 8; ++i) {
        const float2 v = red[i][r];
        const float up = fmaxf(top, v.x);
        s = s * exp_below(top, up) + v.y * exp_below(v.x, up);
        top = up;
    }
    const float l = top + log2f(s) * LN2;
    lse[m] = l;
    loss[m] = labels[m] >= 0 && labels[m] < vocab ? l - target[m] : 0.f;
}

// Rows of `width` elements as the products read them: of `pitch` elements, zeros behind them and in the rows from `rows` to `all`.  fp32 values
// become three limbs, `limb` elements apart: the value rounded to bf16, what that leaves, rounded, and what that leaves.
template <typename T>
__global__ __launch_bounds__(256) void xent_pad(const T *__restrict__ src, uint16_t *__restrict__ dst, int64_t rows, int64_t all, int width, int pitch,
                                                int64_t limb)
{
    for (int64_t r = blockIdx.x; r < all; r += gridDim.x)
        for (int j = threadIdx.x * 2; j < pitch; j += 512) {                                    // pitch is even
            float a = r < rows && j < width ? SmElem<T>::load(src + (size_t)r * width + j) : 0.f;
            float b = r < rows && j + 1 < width ? SmElem<T>::load(src + (size_t)r * width + j + 1) : 0.f;
#pragma unroll
            for (int l = 0; l < (sizeof(T) == 4 ? 3 : 1); ++l) {
                const uint32_t q = sizeof(T) == 4 && l == 0 ? pack_bf16x2_hw(within_bf16(a), within_bf16(b)) : pack_bf16x2_hw(a, b);
                *reinterpret_cast<uint32_t *>(dst + l * limb + (size_t)r * pitch + j) = q;
                a -= __uint_as_float(q << 16);
                b -= __uint_as_float(q & 0xFFFF0000u);
            }
        }
}

// out[r][j] = scale * sum of the slabs
template <typename T>
__global__ __launch_bounds__(256) void xent_sum(const float *__restrict__ slab, const float *__restrict__ scale, T *__restrict__ out, int rows, int width,
                                                int pitch, int splits)
{
    const int j = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (j >= width) return;
    const float s = *scale;
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        const mm_f32x4 v = sum_parts(slab + (size_t)r * pitch + j, splits, (size_t)rows * pitch);
        for (int e = 0; e < 4 && j + e < width; ++e) SmElem<T>::store(out + (size_t)r * width + j + e, v[e] * s);
    }
}

// Tile of a product (its edge), parts of its reduction, and the expected time, us
struct MmChoice {
    int edge, splits;
    float us;
};

// From the tiles of the fullest compute unit: a start and an end per tile and a time per stage of 32.  Two workgroups of a 128 tile and four of a
// 64 tile share a compute unit and hide each other's waits (three limbs: one and two).  Fitted to times with each tile forced.  limbs: of the first operand.
static float mm_expected(int edge, int limbs, int64_t m, int64_t n, int64_t stages, int splits)
{
    const int64_t tiles = ((m + edge - 1) / edge) * ((n + edge - 1) / edge) * splits, per_cu = (tiles + 255) / 256;
    const float s = (float)((stages + splits - 1) / splits), t = (float)per_cu;
    if (limbs == 3) return edge == 128 ? t * (5.f + 1.1f * s) : per_cu == 1 ? 3.f + 0.5f * s : t * (1.f + 0.38f * s);
    if (limbs == 2) return edge == 128 ? (float)(per_cu / 2) * (3.f + 1.1f * s) + (float)(per_cu % 2) * (2.5f + 0.78f * s) : per_cu == 1 ? 2.f + 0.25f * s : t * (0.6f + 0.18f * s);
    if (edge == 256) return t * (10.f + 0.85f * s);
    if (edge == 128) return (float)(per_cu / 2) * (3.f + 0.54f * s) + (float)(per_cu % 2) * (2.5f + 0.39f * s);
    return per_cu == 1 ? 2.f + 0.2f * s : t * (0.6f + 0.115f * s);
}

// pa, pb: limbs of the operands; most: parts at most; slab: also a single part is written and read again as fp32
static MmChoice mm_choose(int64_t m, int64_t n, int64_t k, int pa, int pb, int most, bool slab)
{
    static const int parts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const int64_t stages = (k + 31) / 32;
    // what memory takes for the operands: a small tile is no faster than a large one then
    const float bytes = ((float)m * (float)pa + (float)n * (float)pb) * (float)k * 2.f / 4.4e6f;
    MmChoice best = {64, 1, INFINITY};
    // a forced tile that slabs do not have is no choice of theirs; one that no form of these operands has is left alone
    const int largest = pa > 1 || slab ? 128 : 256;
    const char *forced = env_switch(SW_XENT_TILE);
    int only = forced ? atoi(forced) : 0;
    if (only > largest && slab) return best;
    if (only > largest) only = 0;
    for (int edge = largest; edge >= 64; edge /= 2)
        for (int p : parts) {
            if (p > most || (p > 1 && k / p < 128)) break;
            if (edge < 128 && ((m + edge - 1) / edge) * ((n + edge - 1) / edge) * p > (1 << 22)) break;      // a grid holds fewer than 2^32 threads
            const float run = mm_expected(edge, pa, m, n, stages, p), t = (run > bytes ? run : bytes) + (p > 1 || slab ? 3.f + (float)m * (float)n * 8.f * (float)p / 4e6f : 0.f);
            if (t < best.us && (!only || only == edge)) best = {edge, p, t};
        }
    return best;
}

// How a call goes through the vocabulary.  Pieces are as large as 512 MiB of g, and of a copy of w, allow.
struct XentPlan {
    bool copy;                   // x and w are copied first: fp32, or rows of no multiple of 16 bytes (tensors off that grid are as well)
    int limbs, glimbs, pitch, piece;     // limbs of an element and of g; elements of a row of x and w as the products read them; classes of a piece
    int64_t krows;               // rows as the products count them where they are the reduction
    MmChoice z, dx, dw;          // products of a whole piece
    bool by_rows;                // z in slabs, then a workgroup per row
    bool few;                    // by_rows with the weight straight from memory; dx as well, in dx.splits parts
    bool few_dw;                 // and dw without a copy of x
    size_t info, scale, tops, zslab, xpack, xcopy, wcopy, g, dx_slab, dw_slab, total; // offsets in the workspace
};

static int64_t up(int64_t v, int to) { return (v + to - 1) / to * to; }

// Rows that the kernels for few rows take, 16, 32 or (fp32) 64 a workgroup; fp32 in two groups, which read the weight again.  Loss and gradients over
// 33171 classes of 1921, with copies and without: bf16 321 -> 218 us for 1 row, 345 -> 296 for 30 (40: 317 -> 325 with one limb of g); fp32 716 -> 328 for 30,
// 796 -> 432 for 60, and 495 -> 384 for 100 rows over 33000 of 1000.  Fewer than 8192 classes are fewer than 256 waves, and their copy is short
// (128 x 2048 over 1000 classes fp32: 121 us without, 25 with copies).
constexpr int XENT_FEW_VOCAB = 8192;
static int few_rows(int limbs) { return limbs == 3 ? 128 : 32; }
static_assert(XENT_FINE_ROWS >= 32, "the kernels for few rows take two limbs of g");
static int few_tiles(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }       // blocks of 16 rows of a workgroup
static int few_groups(int64_t rows) { return (int)((rows + 63) / 64); }                  // workgroups for all rows

static XentPlan xent_plan(int dtype, int64_t rows, int width, int vocab, bool bwd)
{
    XentPlan p{};
    p.limbs = dtype == NGC_F32 ? 3 : 1;
    p.glimbs = xent_glimbs(p.limbs, rows, width, vocab);
    p.pitch = (int)up(width, p.limbs == 3 ? 32 : 8);
    p.copy = p.limbs == 3 || p.pitch != width;
    p.krows = p.limbs == 3 ? up(rows, 32) : rows;
    const int64_t most = ((int64_t)512 << 20) / 2;                       // bf16 values
    int64_t piece = vocab;
    if (bwd && piece > most / p.glimbs / p.krows) piece = most / p.glimbs / p.krows;
    if (piece > most / p.limbs / p.pitch) piece = most / p.limbs / p.pitch;
    if (piece > (1 << 21)) piece = 1 << 21;                              // offsets in a tile of g stay below 2 GiB
    const char *cap = env_switch(SW_XENT_PIECE);
    if (cap && piece > atoi(cap)) piece = atoi(cap);
    p.piece = (int)(piece >= vocab ? vocab : piece < 256 ? 256 : piece / 256 * 256);
    if (p.piece > vocab) p.piece = vocab;
    // only copies and gradients make pieces of the vocabulary (copies are also made of tensors off the 16-byte grid)
    p.z = mm_choose(rows, p.piece, p.pitch, p.limbs, p.limbs, 1, false);
    if (bwd) {
        p.dx = mm_choose(rows, p.pitch, p.piece, p.glimbs, p.limbs, 64, false);
        p.dw = mm_choose(p.piece, p.pitch, rows, p.glimbs, p.limbs, 64, false);
    }
    // One piece of few tiles: in parts, as long as these take no more than 32 MiB and (backprop: every row looks at all weights) the rows are few.
    // Two launches either way.
    if (p.piece == vocab && rows <= 1024) {
        const MmChoice parts = mm_choose(rows, vocab, p.pitch, p.limbs, p.limbs, 64, true);
        p.by_rows = parts.us < p.z.us && (int64_t)rows * up(vocab, 8) * 4 * parts.splits <= (32 << 20);
        if (p.by_rows) p.z = parts;
    }
    if (p.copy && rows <= few_rows(p.limbs) && vocab >= XENT_FEW_VOCAB && p.glimbs > 1 && !(cap && p.piece < vocab) && (int64_t)rows * up(vocab, 8) * 4 <= (64 << 20) && vocab <= (1 << 21)) {
        p.few = p.by_rows = true;
        p.few_dw = rows <= (p.limbs == 3 ? 32 : 16);
        p.piece = vocab;
        p.z = {64, 1, 0.f};
        // about two workgroups per compute unit, parts of at least 512 classes
        const int blocks = (int)((width + 63) / 64), most = (int)((vocab + 511) / 512);
        p.dx = {64, 512 / blocks < 1 ? 1 : 512 / blocks, 0.f};
        if (p.dx.splits > most) p.dx.splits = most;
        if (p.dx.splits > 64) p.dx.splits = 64;
        if (bwd) p.dw = mm_choose(vocab, p.pitch, rows, p.glimbs, p.limbs, 1, false);
    }
    size_t at = 0;
    auto take = [&](size_t &where, size_t bytes) { where = at; at += r256(bytes); };
    if (p.by_rows) take(p.zslab, (size_t)rows * up(vocab, 8) * 4 * p.z.splits);
    if (!bwd) {
        take(p.info, (size_t)rows * 8 * ((size_t)((int64_t)vocab + 63) / 64 + (vocab - 1) / p.piece + 1));       // part
        take(p.scale, (size_t)rows * 4);                                                                        // target
    } else {
        take(p.info, (size_t)rows * sizeof(XentRow));
        take(p.scale, 4);
        take(p.tops, rows > XENT_ROWS ? XENT_TOPS * 4 : 0);
        take(p.g, (size_t)p.krows * up(p.piece, 64) * 2 * p.glimbs);
        take(p.dx_slab, p.dx.splits > 1 || p.few || p.piece < vocab ? (size_t)rows * p.pitch * 4 * p.dx.splits : 0);
        take(p.dw_slab, p.dw.splits > 1 ? (size_t)p.piece * p.pitch * 4 * p.dw.splits : 0);
    }
    if (p.few) take(p.xpack, (size_t)up(width, 32) * 16 * few_tiles(rows) * few_groups(rows) * 2 * p.limbs);
    take(p.xcopy, p.few && (!bwd || p.few_dw) ? 0 : (size_t)p.krows * p.pitch * 2 * p.limbs);
    if (!p.few) take(p.wcopy, (size_t)up(p.piece, 32) * p.pitch * 2 * p.limbs);
    p.total = at;
    return p;
}

static unsigned mm_grid(MmParams &mm, int edge)
{
    mm.mt = (int)(((int64_t)mm.M + edge - 1) / edge);
    mm.nt = (int)(((int64_t)mm.N + edge - 1) / edge);
    mm.kper = (int)up(((int64_t)mm.K + mm.splits - 1) / mm.splits, 32);
    return (unsigned)mm.mt * (unsigned)mm.nt * (unsigned)mm.splits;
}

template <typename T, int G, int EDGE, bool AT, bool BT, XentEpilogue E>
static hipError_t launch_mm_tile(XentMm p, hipStream_t st)
{
    static LdsLimitOnce lds;
    const hipError_t e = lds.raise(reinterpret_cast<const void *>(&xent_mm<T, G, EDGE, AT, BT, E>));
    if (e != hipSuccess) return e;
    const unsigned grid = mm_grid(p.mm, EDGE);
    NGC_LAUNCH((xent_mm<T, G, EDGE, AT, BT, E>), dim3(grid), dim3(64 * MM_WAVES),
               (mm_lds_bytes<EDGE, EDGE, xent_pa<T, G, BT>(), xent_pb<T>()>()), st, p);
    return launch_result();
}

// G: limbs of g (of the products that neither form nor read it: any)
template <typename T, int G, bool AT, bool BT, XentEpilogue E>
static hipError_t launch_mm(const XentMm &p, int edge, hipStream_t st)
{
    if constexpr (sizeof(T) == 2 && !(E == XE_SLAB && !BT) && !(BT && G > 1))    // slabs of z and products of two limbs: 128 at most
        if (edge == 256) return launch_mm_tile<T, G, 256, AT, BT, E>(p, st);
    return edge == 128 ? launch_mm_tile<T, G, 128, AT, BT, E>(p, st) : launch_mm_tile<T, G, 64, AT, BT, E>(p, st);
}

template <typename T, int G, int EDGE, XentEpilogue EDX>
static hipError_t launch_both(XentMm dx, XentMm dw, hipStream_t st)
{
    static LdsLimitOnce lds;
    const hipError_t e = lds.raise(reinterpret_cast<const void *>(&xent_mm_both<T, G, EDGE, EDX>));
    if (e != hipSuccess) return e;
    const unsigned first = mm_grid(dx.mm, EDGE), grid = first + mm_grid(dw.mm, EDGE);
    NGC_LAUNCH((xent_mm_both<T, G, EDGE, EDX>), dim3(grid), dim3(64 * MM_WAVES), (mm_lds_bytes<EDGE, EDGE, G, xent_pb<T>()>()), st, dx, dw, (int)first);
    return launch_result();
}

// z of all classes into a slab
template <typename T>
static hipError_t launch_few_z(const T *x, char *packed, const T *w, float *z, int rows, int width, int vocab, hipStream_t st)
{
    const int ld = (int)up(vocab, 8), mt = few_tiles(rows), classes = 16 * xent_few_blocks(mt);
    uint4 *xp = reinterpret_cast<uint4 *>(packed);
    NGC_LAUNCH((xent_pack<T>), dim3((unsigned)((width + 31) / 32)), dim3(256), 0, st, x, xp, rows, width, mt * few_groups(rows));
    const hipError_t e = launch_result();
    if (e != hipSuccess) return e;
    auto kernel = mt == 1 ? xent_few_z<T, 1> : xent_few_z<T, 2>;
    if constexpr (sizeof(T) == 4)
        if (mt == 4) kernel = xent_few_z<T, 4>;
    NGC_LAUNCH(kernel, dim3((unsigned)((vocab + classes - 1) / classes), few_groups(rows)), dim3(256), 0, st, xp, w, z, ld, rows, width, vocab);
    return launch_result();
}

template <typename T>
static hipError_t launch_few_dx(const uint16_t *g, int64_t glimb, int gp, const T *w, float *slab, int pitch, int rows, int width, int vocab, int splits,
                                hipStream_t st)
{
    const dim3 grid((unsigned)((width + 63) / 64), (unsigned)splits, few_groups(rows));
    const int per = (int)up(((int64_t)vocab + splits - 1) / splits, 128), mt = few_tiles(rows);
    auto kernel = mt == 1 ? xent_few_dx<T, 1> : xent_few_dx<T, 2>;
    if constexpr (sizeof(T) == 4)
        if (mt == 4) kernel = xent_few_dx<T, 4>;
    NGC_LAUNCH(kernel, grid, dim3(256), 0, st, g, glimb, gp, w, slab, pitch, rows, width, vocab, per);
    return launch_result();
}

// x or rows of w as the products read them: where they are, or a copy.  all: rows of the copy
template <typename T>
static hipError_t operand(const XentPlan &pl, const T *src, char *copy, int64_t rows, int64_t all, int width, const uint16_t *&out, hipStream_t st)
{
    out = reinterpret_cast<const uint16_t *>(src);
    if (!pl.copy && (reinterpret_cast<uintptr_t>(src) & 15) == 0) return hipSuccess;
    out = reinterpret_cast<const uint16_t *>(copy);
    NGC_LAUNCH((xent_pad<T>), dim3((unsigned)(all < 65536 ? all : 65536)), dim3(256), 0, st, src, reinterpret_cast<uint16_t *>(copy), rows, all, width, pl.pitch,
               all * pl.pitch);
    return launch_result();
}

// rows of more classes than one batch of 256 threads take 1024
constexpr int XENT_WIDE = 1024 * XENT_BATCH;

static hipError_t row_loss(const float *z, int splits, int rows, int ld, const int64_t *labels, float *loss, float *lse, int vocab, hipStream_t st)
{
    const auto kernel = vocab > XENT_WIDE ? xent_row_loss<16> : xent_row_loss<4>;
    NGC_LAUNCH(kernel, dim3(rows), dim3(vocab > XENT_WIDE ? 1024 : 256), 0, st, z, splits, (size_t)rows * ld, ld, labels, loss, lse, vocab);
    return launch_result();
}

template <typename T>
static hipError_t launch_xent_t(int rows, int width, int vocab, const T *x, const T *w, const int64_t *labels, float *loss, float *lse, char *ws, hipStream_t st)
{
    const XentPlan pl = xent_plan(sizeof(T) == 4 ? NGC_F32 : NGC_BF16, rows, width, vocab, false);
    const bool copy_w = pl.copy || (reinterpret_cast<uintptr_t>(w) & 15) != 0;
    XentMm p{};
    hipError_t e = hipSuccess;
    if (!pl.few && (e = operand(pl, x, ws + pl.xcopy, rows, rows, width, p.mm.a, st)) != hipSuccess) return e;
    p.mm.lda = p.mm.ldb = pl.pitch;
    p.mm.M = rows; p.mm.K = pl.pitch; p.mm.splits = 1;
    p.mm.alimb = (int64_t)rows * pl.pitch;
    p.labels = labels;
    p.target = reinterpret_cast<float *>(ws + pl.scale);
    float2 *part = reinterpret_cast<float2 *>(ws + pl.info);
    if (pl.few) {
        float *z = reinterpret_cast<float *>(ws + pl.zslab);
        const int ld = (int)up(vocab, 8);
        if ((e = launch_few_z(x, ws + pl.xpack, w, z, rows, width, vocab, st)) != hipSuccess) return e;
        return row_loss(z, 1, rows, ld, labels, loss, lse, vocab, st);
    }
    int tiles = 0;
    for (int64_t v0 = 0; v0 < vocab; v0 += p.mm.N) {
        const int64_t left = vocab - v0;
        p.mm.N = (int)(!copy_w || left < pl.piece ? left : pl.piece);    // only copies make pieces
        if ((e = operand(pl, w + (size_t)v0 * width, ws + pl.wcopy, p.mm.N, p.mm.N, width, p.mm.b, st)) != hipSuccess) return e;
        p.mm.blimb = (int64_t)p.mm.N * pl.pitch;
        p.v0 = (int)v0;
        p.part = part + (size_t)tiles * rows;
        if (pl.by_rows) {                                                // one piece
            const int ld = (int)up(vocab, 8);
            p.slab = reinterpret_cast<float *>(ws + pl.zslab);
            p.ldo = p.store_n = ld; p.store_m = rows;
            p.mm.splits = pl.z.splits;
            if ((e = launch_mm<T, 1, false, false, XE_SLAB>(p, pl.z.edge, st)) != hipSuccess) return e;
            return row_loss(p.slab, pl.z.splits, rows, ld, labels, loss, lse, vocab, st);
        }
        const int edge = copy_w || pl.piece == vocab ? pl.z.edge : mm_choose(rows, vocab, pl.pitch, pl.limbs, pl.limbs, 1, false).edge;
        if ((e = launch_mm<T, 1, false, false, XE_STATS>(p, edge, st)) != hipSuccess) return e;
        tiles += (int)(((int64_t)p.mm.N + edge - 1) / edge);
    }
    NGC_LAUNCH(xent_join, dim3(((unsigned)rows + 31) / 32), dim3(256), 0, st, part, p.target, labels, loss, lse, rows, vocab, tiles);
    return launch_result();
}

template <typename T>
static hipError_t sum_slabs(const float *slab, const float *scale, T *out, int rows, int width, int pitch, int splits, hipStream_t st)
{
    NGC_LAUNCH((xent_sum<T>), dim3((unsigned)(((int64_t)width + 1023) / 1024), rows < 32768 ? rows : 32768), dim3(256), 0, st, slab, scale, out, rows, width,
               pitch, splits);
    return launch_result();
}

template <typename T, int G>
static hipError_t launch_xent_bwd_t(int rows, int width, int vocab, const T *x, const T *w, const int64_t *labels, const float *lse, const float *dloss,
                                    T *dx, T *dw, char *ws, hipStream_t st)
{
    const XentPlan pl = xent_plan(sizeof(T) == 4 ? NGC_F32 : NGC_BF16, rows, width, vocab, true);
    XentRow *info = reinterpret_cast<XentRow *>(ws + pl.info);
    float *scale = reinterpret_cast<float *>(ws + pl.scale), *dx_slab = reinterpret_cast<float *>(ws + pl.dx_slab), *dw_slab = reinterpret_cast<float *>(ws + pl.dw_slab);
    hipError_t e = hipSuccess;
    if (!pl.by_rows) {
        const int need = (rows - 1) / XENT_ROWS + 1, grid = need < XENT_TOPS ? need : XENT_TOPS;
        float *tops = reinterpret_cast<float *>(ws + pl.tops);
        if (grid > 1) {
            NGC_LAUNCH(xent_tops, dim3(grid), dim3(1024), 0, st, labels, dloss, tops, rows, vocab);
            if ((e = launch_result()) != hipSuccess) return e;
        }
        NGC_LAUNCH(xent_rows, dim3(grid), dim3(1024), 0, st, labels, lse, dloss, tops, grid > 1 ? grid : 0, info, scale, rows, vocab);
        if ((e = launch_result()) != hipSuccess) return e;
    }
    const uint16_t *xp = nullptr, *wp, *g = reinterpret_cast<const uint16_t *>(ws + pl.g);
    if ((!pl.few || (dw && !pl.few_dw)) && (e = operand(pl, x, ws + pl.xcopy, rows, pl.krows, width, xp, st)) != hipSuccess) return e;
    const bool one = pl.dx.splits == 1 && !pl.few;                       // dx leaves the products whole
    const bool together = dx && dw && !pl.few && pl.piece >= vocab && pl.dw.splits == 1 && pl.dx.edge == pl.dw.edge && pl.dw.edge < 256;
    for (int64_t v0 = 0; v0 < vocab; v0 += pl.piece) {
        const int piece = vocab - v0 < pl.piece ? (int)(vocab - v0) : pl.piece, gp = (int)up(piece, 64);
        const int kpiece = (int)(pl.limbs == 3 ? up(piece, 32) : piece);
        if (pl.few) wp = nullptr;                                        // w is read where it is
        else if ((e = operand(pl, w + (size_t)v0 * width, ws + pl.wcopy, piece, kpiece, width, wp, st)) != hipSuccess) return e;
        XentMm p{};
        p.v0 = (int)v0; p.info = info; p.scale = scale;
        p.mm.a = xp; p.mm.b = wp;
        p.mm.lda = p.mm.ldb = pl.pitch;
        p.mm.alimb = pl.krows * pl.pitch; p.mm.blimb = (int64_t)kpiece * pl.pitch;
        p.mm.M = rows; p.mm.N = piece; p.mm.K = pl.pitch; p.mm.splits = 1;
        p.out = ws + pl.g; p.ldo = gp; p.glimb = pl.krows * gp; p.store_m = (int)pl.krows; p.store_n = gp;
        if (pl.by_rows) {                                                // one piece
            const int ld = (int)up(vocab, 8);
            XentMm q = p;
            q.slab = reinterpret_cast<float *>(ws + pl.zslab);
            q.ldo = q.store_n = ld; q.store_m = rows;
            q.mm.splits = pl.z.splits;
            e = pl.few ? launch_few_z(x, ws + pl.xpack, w, q.slab, rows, width, vocab, st) : launch_mm<T, 1, false, false, XE_SLAB>(q, pl.z.edge, st);
            if (e != hipSuccess) return e;
            const auto kernel = vocab > XENT_WIDE ? xent_row_grad<G, 16> : xent_row_grad<G, 4>;
            NGC_LAUNCH(kernel, dim3((unsigned)pl.krows), dim3(vocab > XENT_WIDE ? 1024 : 256), 0, st, q.slab, pl.z.splits, (size_t)rows * ld, ld, labels, lse, dloss,
                       reinterpret_cast<uint16_t *>(ws + pl.g), p.glimb, gp, scale, rows, vocab);
            e = launch_result();
        } else {
            e = launch_mm<T, G, false, false, XE_GRAD>(p, pl.z.edge, st);
        }
        if (e != hipSuccess) return e;
        XentMm both{};                                                   // dx, while it waits to run together with dw
        if (dx && pl.few) {
            if ((e = launch_few_dx(g, p.glimb, gp, w, dx_slab, pl.pitch, rows, width, vocab, pl.dx.splits, st)) != hipSuccess) return e;
        } else if (dx) {
            XentMm q = p;
            q.mm.a = g; q.mm.lda = gp; q.mm.alimb = p.glimb;
            q.mm.M = rows; q.mm.N = pl.pitch; q.mm.K = kpiece; q.mm.splits = pl.dx.splits;
            q.store_m = rows;
            if (pl.dx.splits == 1 && v0 + piece >= vocab) {              // the last piece leaves the result
                q.out = dx; q.ldo = width; q.store_n = width;
                q.slab = dx_slab; q.add = v0 > 0;
                if (!together) e = launch_mm<T, G, false, true, XE_OUT>(q, pl.dx.edge, st);
            } else {
                q.slab = dx_slab; q.ldo = pl.pitch; q.store_n = pl.pitch; q.add = v0 > 0;
                if (!together) e = launch_mm<T, G, false, true, XE_SLAB>(q, pl.dx.edge, st);
            }
            if (e != hipSuccess) return e;
            both = q;
        }
        if (dw && pl.few_dw) {
            const int lanes = width <= 64 ? 16 : width <= 256 ? 64 : 256;
            auto kernel = lanes == 16 ? xent_few_dw<T, 16, 16> : lanes == 64 ? xent_few_dw<T, 16, 64> : xent_few_dw<T, 16, 256>;
            if constexpr (sizeof(T) == 4)
                if (rows > 16) kernel = lanes == 16 ? xent_few_dw<T, 32, 16> : lanes == 64 ? xent_few_dw<T, 32, 64> : xent_few_dw<T, 32, 256>;
            NGC_LAUNCH(kernel, dim3((unsigned)((vocab + 63) / 64), (unsigned)((width + 4 * lanes - 1) / (4 * lanes))), dim3(256), 0, st, g, p.glimb, gp, x, scale, dw,
                       rows, width, vocab);
            if ((e = launch_result()) != hipSuccess) return e;
        } else if (dw) {
            XentMm q = p;
            q.mm.a = g; q.mm.lda = gp; q.mm.alimb = p.glimb;
            q.mm.b = xp; q.mm.blimb = pl.krows * pl.pitch;
            q.mm.M = piece; q.mm.N = pl.pitch; q.mm.K = (int)pl.krows; q.mm.splits = pl.dw.splits;
            q.store_m = piece;
            T *out = dw + (size_t)v0 * width;
            if (pl.dw.splits == 1) {
                q.out = out; q.ldo = width; q.store_n = width;
                if (!together) e = launch_mm<T, G, true, true, XE_OUT>(q, pl.dw.edge, st);
                else if (pl.dw.edge == 128) e = one ? launch_both<T, G, 128, XE_OUT>(both, q, st) : launch_both<T, G, 128, XE_SLAB>(both, q, st);
                else e = one ? launch_both<T, G, 64, XE_OUT>(both, q, st) : launch_both<T, G, 64, XE_SLAB>(both, q, st);
            } else {
                q.slab = dw_slab; q.ldo = pl.pitch; q.store_n = pl.pitch; q.add = 0;
                e = launch_mm<T, G, true, true, XE_SLAB>(q, pl.dw.edge, st);
                if (e == hipSuccess) e = sum_slabs(dw_slab, scale, out, piece, width, pl.pitch, pl.dw.splits, st);
            }
            if (e != hipSuccess) return e;
        }
    }
    return dx && !one ? sum_slabs(dx_slab, scale, dx, rows, width, pl.pitch, pl.dx.splits, st) : hipSuccess;
}

size_t linear_xent_workspace(int dtype, int64_t rows, int width, int vocab, bool bwd) { return xent_plan(dtype, rows, width, vocab, bwd).total; }

hipError_t launch_linear_xent(int dtype, int rows, int width, int vocab, const void *x, const void *w, const int64_t *labels, float *loss, float *lse,
                              void *ws, hipStream_t st)
{
    if (dtype == NGC_BF16)
        return launch_xent_t(rows, width, vocab, static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(w), labels, loss, lse, static_cast<char *>(ws), st);
    return launch_xent_t(rows, width, vocab, static_cast<const float *>(x), static_cast<const float *>(w), labels, loss, lse, static_cast<char *>(ws), st);
}

hipError_t launch_linear_xent_bwd(int dtype, int rows, int width, int vocab, const void *x, const void *w, const int64_t *labels, const float *lse,
                                  const float *dloss, void *dx, void *dw, void *ws, hipStream_t st)
{
    const auto call = [&](auto type, auto g) {
        typedef decltype(type) T;
        return launch_xent_bwd_t<T, decltype(g)::value>(rows, width, vocab, static_cast<const T *>(x), static_cast<const T *>(w), labels, lse, dloss,
                                                        static_cast<T *>(dx), static_cast<T *>(dw), static_cast<char *>(ws), st);
    };
    if (dtype == NGC_F32) return call(float(), std::integral_constant<int, 3>());
    return xent_glimbs(1, rows, width, vocab) == 2 ? call(uint16_t(), std::integral_constant<int, 2>()) : call(uint16_t(), std::integral_constant<int, 1>());
}

}  // namespace ngc
