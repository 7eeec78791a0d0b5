// Matrix products of bf16 operands with fp32 sums for the linear cross entropy (gfx950), with the operands as they lie in memory:
//
//   c[m][n] = sum_k A(m, k) B(n, k)      A stored [M][K] or (AT) [K][M], B stored [N][K] or (BT) [K][N]
//
// A workgroup of four waves forms a BM x BN tile; a wave BM/2 x BN/2 of it from v_mfma_f32_16x16x32_bf16, whose first operand is B: an
// accumulator then holds four neighbouring n of one m.  The reduction runs in stages of 32 through a ring of NS stages in LDS, filled by direct
// global->LDS loads (16 bytes a lane, the scalar base moves along k).  While the products of a stage run, its successor goes from LDS to
// registers and the stage NS ahead is asked for: one barrier and one counted wait per stage.
//
// An operand is the sum of PA or PB bf16 limbs of 8 significant bits each.  3, 3: fp32 operands; of the nine products of limbs the six that reach
// 2^-24 of the result are formed.  2, 1: an fp32 operand that 16 bits hold well enough, with a bf16 one; both products.  A stage holds all limbs, so
// that a 128 x 128 tile of 3, 3 has 96 matrix instructions a wave for its 48 KB where one of 1, 1 has 16 for 16 KB.
//
// LDS of a stage, in units of 16 bytes so that 64 lanes fill 1 KB in lane order:
//   [R][K] operands   rows of 64 bytes; chunk c of row r sits at c ^ (0 or 3 for r / 8 % 2 = 0 or 1).  ds_read_b128 takes lanes 0-3, 12-15, 20-23
//                     and 24-27 in one cycle, 4-11, 16-19 and 28-31 in the next: rows and chunks that touch every bank once.  (With
//                     c ^ (r / 4 % 4), which 16 lanes in a row would need, half of the LDS cycles were bank conflicts.)
//   [K][R] operands   blocks of 8 k x 64 columns, rows of 128 bytes; the 32-byte piece b of a row k sits at b ^ (k / 2 % 2) ^ 2 (k / 8 % 2), and
//                     ds_read_b64_tr_b16 turns 4 k x 16 columns into four k of one column per lane: two lane groups touch every bank once
// Rows and k past the ends are read as zeros: lanes whose offset is past the range of the buffer descriptor.
//
// Bound: matrix pipes, at the clock that the power allows (about 2 GHz under this load).  8192 x 4096 x 50257 bf16, 256 x 256 tiles: 1.21 PFLOP/s as
// x w^T (1.17 with the epilogue of g), 1.31 as g w, 1.21 as g^T x, the pipes busy 0.60 to 0.68 of the cycles, no LDS bank conflicts (an 8192^3 library
// product: 1.38 and 1.20).  Three limbs, 128 x 128 tiles: 1.1 us a stage, 4096 x 4096 x 32768 at 205 TFLOP/s of fp32 (library: 150).
#pragma once
#include "common.h"

#include <type_traits>

namespace ngc {

typedef __bf16 mm_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mm_f32x4 __attribute__((ext_vector_type(4)));
typedef short mm_s16x4 __attribute__((ext_vector_type(4)));
typedef short mm_s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void mm_lds_void;
typedef __attribute__((address_space(3))) mm_s16x4 mm_lds_s16x4;

constexpr unsigned MM_OOB = 0x80000000u;

struct MmParams {
    const uint16_t *a, *b;
    int64_t lda, ldb;            // elements between rows as stored, multiples of 8; a, b on the 16-byte grid
    // K: rows of a [K][.] operand past it are not read.  Rows are read in whole groups of 8 elements: what a [.][K] operand holds behind K up to
    // there has to be zero, and a [K][.] operand has to hold something behind M or N.
    int M, N, K;
    int mt, nt, splits, kper;    // tiles; parts of the reduction and their length (a multiple of 32)
    int64_t alimb, blimb;        // elements between the limbs of an operand
};

constexpr int MM_WAVES = 4;

template <int R, bool T>
struct MmOperand {
    static constexpr int NW = MM_WAVES, LOADS = R / 16 / NW;             // 1 KB loads per wave, stage and limb
    static_assert(R % 64 == 0 && LOADS >= 1, "tile");
    uint64_t base;                                                       // of the tile's first row / column, first k of the part
    uint64_t step;                                                       // bytes per stage
    unsigned voff[LOADS];

    // column / row and k within the tile and stage of what a lane loads
    __device__ static __forceinline__ int rin(int i, int wave)
    {
        const int lane = threadIdx.x & 63, q = i * NW + wave;
        if constexpr (!T) return q * 16 + (lane >> 2);
        const int kg = q / (R / 64), nb = q % (R / 64), row = lane >> 3, c = lane & 7;
        return nb * 64 + (((c >> 1) ^ ((row >> 1) & 1) ^ (2 * (kg & 1))) << 4) + (c & 1) * 8;
    }
    __device__ static __forceinline__ int kin(int i, int wave)
    {
        const int lane = threadIdx.x & 63, q = i * NW + wave;
        return T ? 8 * (q / (R / 64)) + (lane >> 3) : 8 * ((lane & 3) ^ ((rin(i, wave) >> 3) & 1 ? 3 : 0));
    }
    __device__ __forceinline__ void init(const uint16_t *p, int64_t ld, int r0, int extent, int k0, int wave)
    {
        base = reinterpret_cast<uint64_t>(p) + 2 * (T ? (int64_t)k0 * ld + r0 : (int64_t)r0 * ld + k0);
        step = 2 * (T ? 32 * ld : 32);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = rin(i, wave), k = kin(i, wave);
            voff[i] = r0 + r < extent ? 2u * (unsigned)(T ? k * (int)ld + r : r * (int)ld + k) : MM_OOB;
        }
    }
    // Load i of limb l (`limb` elements from limb to limb) of the stage.  kleft: k that are left from this stage on; FULL: at least 32.  The load
    // goes straight to LDS and has no result register.  It is written out because the compiler waits for every such load that it knows of in front of
    // a transposing LDS read, whatever part of the ring that reads.  It is not said to write memory: LDS reads may move across it, as what they read
    // is not what it writes.  The order of a place in the ring is that of mm_tile's counted waits and barriers, which nothing moves across.
    template <bool FULL>
    __device__ __forceinline__ void load(int i, int l, int64_t limb, unsigned lds, int wave, int kleft) const
    {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        const uint64_t at = base + 2 * l * limb;
        const u32x4 rs = {(unsigned)at, (unsigned)(at >> 32) & 0xFFFFu, 0x7fffffffu, 0x00020000u};
        const unsigned v = FULL || kin(i, wave) < kleft ? voff[i] : MM_OOB;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds + (unsigned)((l * LOADS + i) * NW + wave) * 1024u), "v"(v), "s"(rs)
                     : "m0");
    }
    __device__ __forceinline__ void next() { base += step; }
};

// this lane's part of the operand of 16 rows / columns: k 8 (lane / 16) .. + 7
template <int R, bool T>
struct MmFragments {
    unsigned at[T ? 4 : 1];
    __device__ __forceinline__ void init(int r0, int lane)               // r0: first row / column of the wave, a multiple of 16
    {
        const int g = lane >> 4, l = lane & 15;
        if constexpr (T) {
            const int i = l >> 2, key = ((i >> 1) & 1) ^ (2 * (g & 1));
#pragma unroll
            for (int b = 0; b < 4; ++b)
                at[b] = (unsigned)(g * (R / 64) * 1024 + (r0 >> 6) * 1024 + i * 128 + (((((r0 >> 4) + b) & 3) ^ key) << 5) + (l & 3) * 8 +
                                   ((((r0 >> 4) & 3) + b) >> 2) * 1024);
        } else {
            at[0] = (unsigned)((r0 + l) * 64 + ((g ^ (l >> 3 ? 3 : 0)) << 4));
        }
    }
    __device__ __forceinline__ mm_bf16x8 read(const unsigned char *lds, int f) const
    {
        if constexpr (T) {
            const unsigned char *p = lds + at[f & 3] + (f >> 2) * 1024;
            const mm_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mm_lds_s16x4 *)p);
            const mm_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((mm_lds_s16x4 *)(p + 512));
            return __builtin_bit_cast(mm_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const mm_bf16x8 *>(lds + at[0] + f * 1024);
        }
    }
};

// 160 KB of a 256 x 256 tile, two workgroups of a 128 x 128 tile; with three limbs each 144 KB of one, two of a 64 x 64 tile; with two and one two
// workgroups of a 128 x 128 tile, four of a 64 x 64 tile
template <int PA> constexpr int mm_stages() { return PA == 1 ? 5 : 3; }
template <int BM, int BN, int PA, int PB> constexpr int mm_lds_bytes() { return mm_stages<PA>() * (PA * BM + PB * BN) * 64; }

// Two products, c0 += b a0^T and c1 += b a1^T.  Written out so that the accumulators stay where they are: 256 of them fill the accumulation
// registers, and the compiler moves them about instead of updating them in place.  The leading wait is the one a matrix instruction needs behind
// a vector instruction that wrote an operand; mm_settle is the one in front of the first read of a result.
__device__ __forceinline__ void mm_pair(mm_f32x4 &c0, mm_f32x4 &c1, const mm_bf16x8 &b, const mm_bf16x8 &a0, const mm_bf16x8 &a1)
{
    asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %2, %3, %0\n\tv_mfma_f32_16x16x32_bf16 %1, %2, %4, %1" : "+a"(c0), "+a"(c1) : "v"(b), "v"(a0), "v"(a1));
}
template <int FN, int FM>
__device__ __forceinline__ void mm_settle(mm_f32x4 (&acc)[FN][FM])
{
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) asm volatile("" : "+a"(acc[i][j]));         // no read of it moves in front of the wait
}

// Tile of a workgroup: ids go round-robin to the 8 XCDs (one L2 each); each XCD gets a run of tiles, in groups of 8 rows of tiles, so that
// the tiles that run together share operands in its L2.
__device__ __forceinline__ void mm_tile_of(int id, int total, int mt, int nt, int &tm, int &tn)
{
    const int xcd = id & 7, each = total >> 3, more = total & 7;
    const int lin = xcd * each + (xcd < more ? xcd : more) + (id >> 3);
    const int group = lin / (8 * nt), first = group * 8, rows = mt - first < 8 ? mt - first : 8, in = lin - group * 8 * nt;
    tm = first + in % rows;
    tn = in / rows;
}

// acc[fn][fm]: n = 16 fn + 4 (lane / 16) + element, m = 16 fm + lane % 16 of the wave's part
template <int BM, int BN, bool AT, bool BT, int PA, int PB>
__device__ __forceinline__ void mm_tile(const MmParams &p, unsigned char *smem, int m0, int n0, int k0, int k1, mm_f32x4 (&acc)[BN / 32][BM / 32])
{
    constexpr int FM = BM / 32, FN = BN / 32, STAGE = (PA * BM + PB * BN) * 64, NS = mm_stages<PA>();
    constexpr int LA = MmOperand<BM, AT>::LOADS * PA, LB = MmOperand<BN, BT>::LOADS * PB, LPS = LA + LB;
    static_assert((PA == 1 && PB == 1) || (PA == 2 && PB == 1) || (PA == 3 && PB == 3), "limbs");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    MmOperand<BM, AT> la;
    MmOperand<BN, BT> lb;
    la.init(p.a, p.lda, m0, p.M, k0, wave);
    lb.init(p.b, p.ldb, n0, p.N, k0, wave);
    MmFragments<BM, AT> ra;
    MmFragments<BN, BT> rb;
    ra.init((wave % 2) * (BM / 2), lane);
    rb.init((wave / 2) * (BN / 2), lane);
    const int steps = (k1 - k0 + 31) / 32, full = (k1 - k0) / 32;
    const unsigned ring = (unsigned)(uintptr_t)(mm_lds_void *)smem;          // LDS address
    auto load = [&](auto whole, int f, unsigned to, int kleft) {             // load f of a stage
        constexpr bool FULL = decltype(whole)::value;
        if (f < LA) la.template load<FULL>(f % (LA / PA), f / (LA / PA), p.alimb, to, wave, kleft);
        else lb.template load<FULL>((f - LA) % (LB / PB), (f - LA) / (LB / PB), p.blimb, to + PA * BM * 64, wave, kleft);
    };
    // the PAIRS products of limbs, and the GAPS between pairs of matrix instructions of a stage
    constexpr int PAIRS = PA == 3 ? 6 : PA, GAPS = PAIRS * FN * FM / 2, READS = PA * FM + PB * FN, ITEM_GAPS = GAPS * 3 / 4 > 0 ? GAPS * 3 / 4 : 1;
    mm_bf16x8 fa[2][PA][FM], fb[2][PB][FN];
    auto read = [&](int f, const unsigned char *st, int u) {                 // fragment f of a stage
        if (f < PA * FM) fa[u][f / FM][f % FM] = ra.read(st + f / FM * BM * 64, f % FM);
        else fb[u][(f - PA * FM) / FN][(f - PA * FM) % FN] = rb.read(st + PA * BM * 64 + (f - PA * FM) / FN * BN * 64, (f - PA * FM) % FN);
    };
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = mm_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < NS && s < steps; ++s) {
#pragma unroll
        for (int f = 0; f < LPS; ++f) load(std::false_type(), f, ring + s * STAGE, k1 - k0 - 32 * s);
        la.next();
        lb.next();
    }
    // the first stage has landed when at most the loads of the others are under way
    if (steps >= NS) wait_vmcnt63(LPS * (NS - 1));
    else wait_vmcnt63(0);
    wg_barrier_nofence();
#pragma unroll
    for (int f = 0; f < READS; ++f) read(f, smem, 0);
    int place = 0;                                                           // of stage t in the ring
    // Stage t: its products, between them the LDS reads of stage t + 1 and the loads of stage t + NS.  FULL: both exist, the latter whole.
    auto stage = [&](auto whole, int t, int u) {
        constexpr bool FULL = decltype(whole)::value;
        // stage t + 1 has landed, and this wave has stage t in registers: after the barrier its place in the ring is free
        if (FULL || t + NS - 1 < steps) wait_vmcnt63(LPS * (NS - 2));
        else wait_vmcnt63(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);                                  // lgkmcnt(0)
        wg_barrier_nofence();
        const unsigned to = ring + place;
        place = place == (NS - 1) * STAGE ? 0 : place + STAGE;
        const unsigned char *next = smem + place;                             // past the end: what is left in the ring, not used
        const int kleft = k1 - k0 - 32 * (t + NS);
        const bool more = FULL || t + NS < steps;
        // One or two other instructions between two pairs of products, which run for as long as those take to issue; none in the last gaps, so that
        // no LDS read is under way at the end of the stage, where all of them have to have arrived.
#pragma unroll
        for (int q = 0; q < GAPS; ++q) {
#pragma unroll
            for (int f = 0; f < READS; ++f)
                if (f * ITEM_GAPS / READS == q) read(f, next, u ^ 1);
            if (more)
#pragma unroll
                for (int f = 0; f < LPS; ++f)
                    if (f * ITEM_GAPS / LPS == q) load(whole, f, to, kleft);
            // products of limbs (2,0) (0,2) (1,1) (1,0) (0,1) (0,0), or (1,0) (0,0): the largest last, so that the first two limbs of the largest numbers,
            // which may be 2^128 together, meet behind the third
            const int pair = PAIRS - 1 - q / (FN * FM / 2), i = q % (FN * FM / 2) / (FM / 2), j = q % (FM / 2) * 2;
            const int l = PA == 2 ? pair : pair == 5 ? 2 : pair == 2 || pair == 3 ? 1 : 0, r = PA == 2 ? 0 : pair == 4 ? 2 : pair == 1 || pair == 3 ? 1 : 0;
            mm_pair(acc[i][j], acc[i][j + 1], fb[u][r][i], fa[u][l][j], fa[u][l][j + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        la.next();
        lb.next();
    };
    int s = 0;
    for (; s + NS + 1 < full; s += 2) {
        stage(std::true_type(), s, 0);
        stage(std::true_type(), s + 1, 1);
    }
    for (; s < steps; s += 2) {
        stage(std::false_type(), s, 0);
        if (s + 1 < steps) stage(std::false_type(), s + 1, 1);
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    mm_settle(acc);
    wg_barrier_nofence();                                                // the ring is free for the caller
}

}  // namespace ngc
