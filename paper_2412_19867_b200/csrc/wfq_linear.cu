// Linear layer on group-wise int8 operands:
//   z[r][k] = sum_g sx[g][r] sw[g][k] (sum_{c in g} xq[r][c] wq[k][c]) + bias[k]
//   y[r][k] = act(z[r][k]) + residual[r][k],   gated: y[r][j] = act(z[r][j]) z[r][K + j] + residual[r][j]
//
// linear_mma_kernel: persistent, warp-specialised, one CTA per SM.  A tile is 128 rows x BN columns of z; "rows" are the
// 128 TMEM lanes of the accumulator: rows of x, or with SWAP output channels (few rows of x, so that all lanes carry
// work).  With PAIR two CTAs share a tile of 256 rows (tcgen05.mma.cta_group::2): each loads its 128 rows and half of the
// columns' operand.  Gated weights are stored with gate and value channels alternating, so that a pair is two neighbours.
//   warp 0      TMA producer: 128 channels of both operands per stage (128-byte swizzle)
//   warp 1      allocates TMEM, issues tcgen05.mma kind::i8 (K = 32): a piece is a group, as far as this CTA has its
//               channels; pieces of a chunk (up to 128 channels where the group divides 128) lie side by side in one TMEM
//               slot
//   warp 2      scale loader: 128 row scales and BN column scales per piece
//   warps 4-11  epilogue: int32 sums to fp32, times the scales, into registers; then bias, activation, gate, residual
// With few tiles a cluster of up to eight CTAs shares one: each takes a range of the channels, the partial sums are
// added in rank order through distributed shared memory, each CTA for a share of the columns.
// What bounds it.  Short groups: the epilogue's arithmetic, a conversion and two products per group sum.  2048 x 8192 ->
// 2048 in groups of 128 on pairs (one tile per pair of CTAs): 60 us, 1.1 POPS; a piece of 128 x 256 sums takes the eight
// epilogue warps 1200 cycles, of which the conversions are 300, one product 250, the loads 160, against 512 of its MMAs.
// Long groups: the MMAs at the clock that the power limit leaves; 8192 x 4096 -> 8192 with one scale per row 178 us,
// 3.1 POPS of the 4.6 that MMAs without loads reach.  Few rows: the weights' bytes; 24 x 4096 -> 32768 31 us, 4.4 TB/s,
// where 256 tiles on 148 SMs leave the second round half empty.
// Every wait is bounded; on expiry the CTA records where, stops, drains and frees TMEM.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <new>
#include <type_traits>

#include "wfq_output_store.cuh"
#include "wfq_ptx.cuh"
#include "wfq_rows.h"
#include "wfq_weight_order.h"

struct wfq_linear {
    int C = 0, K = 0, gs = 0, gated = 0;
    int Cp = 0, G = 0, Kz = 0, Kp = 0;         // Kz: columns of z (2K if gated); Kp: Kz rounded up to 256
    wfq_dtype_t in_dtype = WFQ_F16, out_dtype = WFQ_F16;
    const float *bias = nullptr;
    int act = 0;
    int device = -1, sm_count = 0;
    int clusters[4] = {0, 0, 0, 0};            // of 1, 2, 4 and 8 CTAs that run at once
    int8_t *Wq = nullptr;                      // [Kz][Cp]
    CUtensorMap tmap_w[2];                     // Wq in boxes of 64 and of 128 rows x 128 channels
    bool tmap_w_ok[2] = {false, false};
    float *sW = nullptr;                       // [G][Kp], zero behind Kz
    int *status = nullptr;                     // int32[4]
    bool prepared = false;
    wfq::WeightOrder order;                    // may a product fetch weights early?
    int8_t *xq = nullptr;                      // workspace: codes of up to max_rows rows
    float *sx = nullptr;
    int max_rows = 0;
    long long wait_cycles = 2000000000LL;
    int debug_skip_stage = -1;
    int debug_shape = 0;
    int shape_rows = -1, shape_orient = 0, shape_bn = 0, shape_split = 0;   // what choose() said last, and for which rows
};

namespace wfq {

namespace {

constexpr int BM = 128;
constexpr int BK = 128;
constexpr int UK = 32;
constexpr int TMEM_COLS = 512;
constexpr int MAX_SLOTS = 16;
constexpr int A_BYTES = BM * BK;
constexpr int EPI_WARPS = 8;
constexpr int FIRST_EPI_WARP = 4;
constexpr int PATCH_PITCH = 40;                                  // floats; 32 columns of z on their way out
constexpr int RESIDUAL_BYTES = 8 * 32 * 16;                      // a warp's residual on its way in: eight 16-byte pieces a lane
constexpr int THREADS = 32 * (FIRST_EPI_WARP + EPI_WARPS);

struct Shared {
    uint64_t full[16], empty[16];
    uint64_t acc_full[MAX_SLOTS], slot_free[MAX_SLOTS];
    uint64_t scale_free[MAX_SLOTS];  // PAIR: this CTA's epilogue is done with a slot (slot_free counts both CTAs')
    uint64_t mma_done;
    uint32_t tmem_base;
    volatile int abort;
};

template <int BN, bool SWAP, bool PAIR>
struct Cfg {
    static_assert(!(SWAP && PAIR), "pairs: rows of x on the lanes");
    static constexpr int B_ROWS = PAIR ? BN / 2 : BN;             // of the columns' operand in this CTA
    static constexpr int STAGE_BYTES = A_BYTES + B_ROWS * BK;
    static constexpr int STAGES = STAGE_BYTES > 24 * 1024 ? 4 : STAGE_BYTES > 20 * 1024 ? (SWAP ? 8 : 5) : 9;
    static constexpr int PATCH_BYTES = SWAP ? 0 : 32 * PATCH_PITCH * 4 + RESIDUAL_BYTES;      // of one epilogue warp
    // Pieces in tensor memory at a time, with their scales: chunks of one (of up to CG_MAX short groups) in as many slots
    // as that gives.  The scales of a slot are asked for when it is free; with two slots whatever the number of columns
    // that took longer than a stage of weights (24 rows, 4096 -> 16384 gated: 0.6 us per 128 channels).
    static constexpr int PIECES = 512 / BN < 16 ? 512 / BN : 16;
    static constexpr int CG_MAX = PIECES / 2 < 4 ? PIECES / 2 : 4;
    static constexpr int GROUP_SCALE_FLOATS = BM + BN;
    static constexpr size_t SMEM_BYTES = 1024 + (size_t)STAGES * STAGE_BYTES + EPI_WARPS * PATCH_BYTES +
                                         (size_t)PIECES * GROUP_SCALE_FLOATS * 4 + sizeof(Shared);
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
    static_assert(PAIR || (size_t)BN * (BM + 1) * 4 <= (size_t)STAGES * STAGE_BYTES, "partial sums fit the stages");
    // Registers behind setmaxnreg: the epilogue holds BN / 2 sums and two blocks of loads.
    // 128 * 56 + 256 * 216 <= 384 * 168, what the block is launched with.
    static constexpr bool MOVE_REGS = PAIR && BN == 256;
};

template <typename C>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const WaitCtx &ctx, int where)
{
    if constexpr (C::MOVE_REGS) return wait_warp_inline(bar, parity, ctx, where);
    else return wait_warp(bar, parity, ctx, where);
}

struct OutArgs {
    const float *bias;
    const void *residual;
    void *y;
    long long ldr, ldy;
    int K, Kz;                 // columns of y and of z
    int R;                     // rows of x
    int act, gated, dtype;     // dtype: wfq_dtype_t of residual and y
    int vec;                   // rows of y and the residual start on 16-byte boundaries
};

struct MmaArgs {
    const float *row_scale, *col_scale;
    long long row_pitch, col_pitch;
    int rows, cols;            // (R, Kz), with SWAP (Kz, R)
    int tiles, MT;             // tiles, blocks of 128 (PAIR: 256) rows
    int split;                 // CTAs that share the channels of a tile (cluster size; 1 with PAIR)
    int steps, gsteps, cg;     // MMA steps of 32 channels in all, per group; pieces per chunk (as in issue())
    int slots;                 // chunks in tensor memory
    int *status;
    long long wait_cycles;
    int debug_skip_stage;
    OutArgs out;
};

// The channels of this CTA: stages, steps and the pieces (groups, or parts of them) that they fall into.
struct Range { int kb0, kb1, s0, s1, g0, np; };
__device__ __forceinline__ Range range_of(const MmaArgs &a, int rank)
{
    Range r;
    const int KB = (a.steps + 3) / 4;
    r.kb0 = (int)((long long)KB * rank / a.split);
    r.kb1 = (int)((long long)KB * (rank + 1) / a.split);
    r.s0 = 4 * r.kb0;
    r.s1 = min(a.steps, 4 * r.kb1);
    r.g0 = r.s0 / a.gsteps;
    r.np = (r.s1 - 1) / a.gsteps - r.g0 + 1;
    return r;
}

// NaN stays NaN (fmaxf would make it 0): what comes of a group with an infinity or a NaN in it is NaN.
__device__ __forceinline__ float relu(float t)
{
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(t));
    return r;
}
// t Phi(t).  Phi(-a) = exp(-a^2 / 2) R(a), R = erfcx(a / sqrt(2)) / 2 smooth: s P(s), s = 1 / (1 + 0.3 a), with the polynomial
// fitted to R on [0, 13.5], where the exponential ends, for the least relative error, 1.3e-7.  The tail keeps its relative
// accuracy: 12 + 0.75 t^2 units in the last place, the last part from the exponent's rounding; 0 below t = -13.2.  The sum
// 1 + erf(t / sqrt(2)) cancels there (5 % off at t = -5, 0 below -5.6), and erfcf costs more: 4096 x 640 -> 2 x 2560 fp16
// 67.9 us, with erfcf 80.2.
__device__ __forceinline__ float gelu(float t)
{
    const float a = fabsf(t);
    float s, e;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(fmaf(a, 0.3f, 1.f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a * a * -0.721347520f));
    float p = 0.0359317362f;
    p = fmaf(p, s, -0.158276007f);
    p = fmaf(p, s, 0.208206624f);
    p = fmaf(p, s, -0.055393856f);
    p = fmaf(p, s, 0.129469201f);
    p = fmaf(p, s, 0.0996374935f);
    p = fmaf(p, s, 0.120798357f);
    p = fmaf(p, s, 0.119626388f);
    const float q = e * s * p;
    return t * (t < 0.f ? q : 1.f - q);
}
__device__ __forceinline__ float activate(float t, int act)
{
    switch (act) {
        case WFQ_ACT_RELU: return relu(t);
        case WFQ_ACT_SILU: return silu(t);
        case WFQ_ACT_GELU: return gelu(t);
        default: return t;
    }
}

__device__ __forceinline__ float out_load(const void *p, long long i, int dtype)
{
    if (dtype == WFQ_F32) return static_cast<const float *>(p)[i];
    if (dtype == WFQ_F16) return __half2float(static_cast<const __half *>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}
__device__ __forceinline__ void out_store(void *p, long long i, float v, int dtype)
{
    if (dtype == WFQ_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == WFQ_F16) static_cast<__half *>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// Columns k and k + 1 (k even) of row r of z.
__device__ __forceinline__ void finish_pair(const OutArgs &o, int r, int k, float v0, float v1)
{
    if (r >= o.R || k >= o.Kz) return;
    if (o.gated) {
        const int j = k >> 1;
        if (o.bias) { v0 += __ldg(o.bias + j); v1 += __ldg(o.bias + o.K + j); }
        float y = activate(v0, o.act) * v1;
        if (o.residual) y += out_load(o.residual, r * o.ldr + j, o.dtype);
        out_store(o.y, r * o.ldy + j, y, o.dtype);
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float y = i ? v1 : v0;
        if (k + i >= o.Kz) return;
        if (o.bias) y += __ldg(o.bias + k + i);
        y = activate(y, o.act);
        if (o.residual) y += out_load(o.residual, r * o.ldr + k + i, o.dtype);
        out_store(o.y, r * o.ldy + k + i, y, o.dtype);
    }
}

// y += n (4 or 8) values of the residual from 16-byte pieces in shared memory, `next` floats apart.
template <int N>
__device__ __forceinline__ void add_residual(float *y, const float *piece, int next, int dtype)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(piece);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if (dtype == WFQ_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += __uint_as_float(w[i]);
        if constexpr (N == 8) {
            const float4 v = *reinterpret_cast<const float4 *>(piece + next);
            y[4] += v.x; y[5] += v.y; y[6] += v.z; y[7] += v.w;
        }
    } else if (dtype == WFQ_F16) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            y[2 * i] += f.x; y[2 * i + 1] += f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            y[2 * i] += __uint_as_float(w[i] << 16);
            y[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
// N (4 or 8) consecutive values of y, aligned to their size up to 16 bytes.
template <int N>
__device__ __forceinline__ void store_packed(char *p, const float *y, int dtype)
{
    if (dtype == WFQ_F32) {
        float4 *q = reinterpret_cast<float4 *>(p);
#pragma unroll
        for (int e = 0; e < N / 4; ++e) q[e] = make_float4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
        return;
    }
    uint32_t w[N / 2];
    if (dtype == WFQ_F16) {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) *reinterpret_cast<__half2 *>(&w[e]) = __floats2half2_rn(y[2 * e], y[2 * e + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < N / 2; ++e)
            *reinterpret_cast<__nv_bfloat162 *>(&w[e]) = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
    }
    if constexpr (N == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}

template <int N>
__device__ __forceinline__ void activate_all(float (&z)[N], int act)
{
    if (act == WFQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = relu(z[i]);
    } else if (act == WFQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = silu(z[i]);
    } else if (act == WFQ_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = gelu(z[i]);
    }
}

// The sums of an epilogue warp, 32 rows of TMEM lanes x CW columns.  Where there are many columns (!SWAP) a thread has four
// rows, lane / 4 + 8 q, and every fourth pair of columns, 8 j + 2 (lane % 4): a column scale is then read from shared
// memory by eight lanes instead of by all 32.  With a row per thread the reads return CW floats to
// every lane, 1024 cycles of the SM's 128 bytes a clock for a piece of 128 x 256, which then takes 1700 cycles instead of
// 1300 with its wait.  Sums that start from the bit pattern of 1.5 * 2^23, so that they need no conversion, cost more in
// writing the pattern back (2000 to 2500 cycles); sixteen epilogue warps with half the columns each are 10 % slower.  With
// SWAP (few columns) a thread has one row.
template <int CW, bool SWAP> struct Sums;
template <int CW> struct Sums<CW, false> {
    float2 v[4][CW / 8];         // [q][j]
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int j = 0; j < CW / 8; ++j) v[q][j] = make_float2(0.f, 0.f);
    }
};
template <int CW> struct Sums<CW, true> {
    float2 v[CW / 2];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int j = 0; j < CW / 2; ++j) v[j] = make_float2(0.f, 0.f);
    }
};

// One piece: int32 sums to fp32, times the row scale, times the column scale, added.  Up to 64 columns at a time, 16 lanes
// after the other, with the next load on its way.  `rs`: scales of the thread's rows; `cs`: the warp's column scales, from
// the thread's first column on.
template <int CW>
__device__ __forceinline__ void promote(uint32_t taddr, const float (&rs)[4], const float *cs, Sums<CW, false> &sums)
{
    constexpr int LC = CW < 64 ? CW : 64;        // columns of a load
    uint32_t rr[2][LC / 2];
    float2 c[LC / 8];
    auto fetch = [&](int b) {                    // block b: columns LC (b / 2) on, lanes 16 (b % 2) on
        ptx::tmem_ld_16x256b(taddr + (uint32_t)(b / 2 * LC) + ((uint32_t)(b % 2 * 16) << 16), rr[b & 1]);
    };
    fetch(0);
#pragma unroll
    for (int b = 0; b < 2 * CW / LC; ++b) {
        uint32_t (&r)[LC / 2] = rr[b & 1];
        if (b % 2 == 0) {
#pragma unroll
            for (int j = 0; j < LC / 8; ++j) c[j] = *reinterpret_cast<const float2 *>(cs + b / 2 * LC + 8 * j);
        }
        ptx::tmem_ld_wait(r);
        if (b + 1 < 2 * CW / LC) fetch(b + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int q = b % 2 * 2 + h;
            const float2 rs2 = make_float2(rs[q], rs[q]);
#pragma unroll
            for (int j = 0; j < LC / 8; ++j) {
                const float2 f = make_float2(__int2float_rn((int)r[4 * j + 2 * h]), __int2float_rn((int)r[4 * j + 2 * h + 1]));
                float2 &s = sums.v[q][b / 2 * (LC / 8) + j];
                s = __ffma2_rn(__fmul2_rn(f, rs2), c[j], s);
            }
        }
    }
}
template <int CW>
__device__ __forceinline__ void promote(uint32_t taddr, float rs, const float *cs, Sums<CW, true> &sums)
{
    constexpr int LD = CW < 16 ? CW : 16;
    const float2 rs2 = make_float2(rs, rs);
    uint32_t rr[2][LD];
    auto fetch = [&](int h) {
        if constexpr (LD == 16) ptx::tmem_ld_x16(taddr + (uint32_t)(LD * h), rr[h & 1]);
        else ptx::tmem_ld_x8(taddr + (uint32_t)(LD * h), rr[h & 1]);
    };
    fetch(0);
#pragma unroll
    for (int h = 0; h < CW / LD; ++h) {
        uint32_t (&r)[LD] = rr[h & 1];
        ptx::tmem_ld_wait(r);
        if (h + 1 < CW / LD) fetch(h + 1);
#pragma unroll
        for (int i = 0; i < LD; i += 4) {
            const float4 c4 = *reinterpret_cast<const float4 *>(cs + LD * h + i);
            const int k = (LD * h + i) / 2;
            const float2 f0 = make_float2(__int2float_rn((int)r[i]), __int2float_rn((int)r[i + 1]));
            const float2 f1 = make_float2(__int2float_rn((int)r[i + 2]), __int2float_rn((int)r[i + 3]));
            sums.v[k] = __ffma2_rn(__fmul2_rn(f0, rs2), make_float2(c4.x, c4.y), sums.v[k]);
            sums.v[k + 1] = __ffma2_rn(__fmul2_rn(f1, rs2), make_float2(c4.z, c4.w), sums.v[k + 1]);
        }
    }
}

// The code of an epilogue runs once per tile and streams through the instruction cache: what is unrolled over the columns
// of a thread is kept to moving registers (a first version, unrolled as a whole, took 15 us for 128 columns).
//
// A warp's 32 rows from row0 on, CW columns of z from column k0 on: 32 at a time through the warp's
// patch of shared memory, so that lanes write neighbouring pieces of a row.  The pitch of 40 floats keeps the 8-byte writes
// of sixteen lanes on different banks; reads of eight lanes are 16 bytes of two rows, of which one takes its upper half first.
//
// The residual comes in by asynchronous copies, each lane's own pieces (16 or 8 bytes; two of 16 for eight fp32 values) of
// 32 columns at a time: the first 32 columns are asked for before the sums are formed, with 16-bit types the second, too.
// Loaded where it is added it cost a memory latency per step, 16 us of 44 for 4096 x 128 -> 4096 bf16; held in registers
// meanwhile it costs the promotion spills.
template <int CW>
__device__ __forceinline__ void ask_residual(const OutArgs &o, uint32_t buffer, int lane, int row0, int k0, int h)
{
    const int k = k0 + h + 8 * (lane % 4), j = o.gated ? k / 2 : k, elem = o.dtype == WFQ_F32 ? 4 : 2;
    const int bytes = (o.gated ? 4 : 8) * elem;
    if (o.vec && h < CW && k + 8 <= o.Kz) {
        // 16-bit types: the other half of the buffer for every other 32 columns; fp32: all of it
        const uint32_t dst = buffer + (elem == 2 && h % 64 ? 4u * 512u : 0u) + 16u * lane;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const long long r = row0 + 8 * q + lane / 4;
            if (r >= o.R) break;
            const char *src = static_cast<const char *>(o.residual) + (r * o.ldr + j) * elem;
            if (bytes == 8) {
                ptx::copy_async8(dst + 512u * q, src);
            } else {
                ptx::copy_async16(dst + 512u * q, src);
                if (bytes == 32) ptx::copy_async16(dst + 512u * (4 + q), src + 16);
            }
        }
    }
    ptx::copy_async_commit();
}
template <int CW>
__device__ __forceinline__ void finish_rows(const OutArgs &o, float *patch, int lane, int row0, int k0,
                                            const Sums<CW, false> &sums)
{
    constexpr int COLS = 32, PITCH = PATCH_PITCH, PIECES = COLS / 8;      // pieces of eight columns
    constexpr int ROWS = 32 / PIECES;                             // rows per step
    const int piece = lane % PIECES, r_in = lane / PIECES;
    float *residual = patch + 32 * PATCH_PITCH;
    const bool wide = o.dtype == WFQ_F32;
    const int elem = wide ? 4 : 2;
#pragma unroll 1
    for (int h = 0; h < CW; h += COLS) {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < CW; c += COLS)
            if (h == c) {
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float2 *>(patch + (lane / 4 + 8 * q) * PITCH + 8 * j + 2 * (lane % 4)) =
                            sums.v[q][c / 8 + j];
            }
        __syncwarp();
        const int k = k0 + h + 8 * piece;                         // first column of this lane's piece
        if (o.residual) {
            if (wide) ptx::copy_async_wait<0>();
            else ptx::copy_async_wait<1>();                       // the next 32 columns may still be on their way
        }
        if (o.vec && k + 8 <= o.Kz) {
            const int j = o.gated ? k / 2 : k;
            const float *res = residual + (!wide && h % 64 ? 512 : 0) + 4 * lane;
            float b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                b[i] = !o.bias ? 0.f : o.gated ? __ldg(o.bias + (i & 1 ? o.K : 0) + j + i / 2) : __ldg(o.bias + j + i);
            const int odd = r_in & 1;
            const float4 *src = reinterpret_cast<const float4 *>(patch + r_in * PITCH + 8 * piece);
            const int live = o.R - row0 - r_in;                   // steps q < live have a row
            const long long first = (row0 + r_in) * o.ldy + j, step = ROWS * o.ldy;
            char *to = static_cast<char *>(o.y) + first * elem;
            // two steps at a time: their chains of instructions overlap (one at a time: 4096 x 640 -> 5120 31.6 us, here
            // 29.6; all four: 30.8)
            auto rows_out = [&](auto gated) {
#pragma unroll 1
                for (int q = 0; q < 32 && q < live; q += 2 * ROWS, to += 2 * step * elem) {
                    float z[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 8) {
                        const float4 s0 = src[odd], s1 = src[odd ^ 1];
                        const float4 lo = odd ? s1 : s0, hi = odd ? s0 : s1;
                        src += ROWS * PITCH / 4;
                        z[i] = lo.x + b[0]; z[i + 1] = lo.y + b[1]; z[i + 2] = lo.z + b[2]; z[i + 3] = lo.w + b[3];
                        z[i + 4] = hi.x + b[4]; z[i + 5] = hi.y + b[5]; z[i + 6] = hi.z + b[6]; z[i + 7] = hi.w + b[7];
                    }
                    constexpr int N = decltype(gated)::value ? 4 : 8;     // values of y per row
                    float y[2 * N];
                    if constexpr (N == 4) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = z[2 * i];
                        activate_all(y, o.act);
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] *= z[2 * i + 1];
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = z[i];
                        activate_all(y, o.act);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (q + i * ROWS < live) {
                            if (o.residual) add_residual<N>(y + i * N, res + (q / ROWS + i) * 128, 512, o.dtype);
                            store_packed<N>(to + i * step * elem, y + i * N, o.dtype);
                        }
                }
            };
            if (o.gated) rows_out(std::true_type{});
            else rows_out(std::false_type{});
        } else {
#pragma unroll 1
            for (int q = 0; q < 32; q += ROWS)
#pragma unroll 1
                for (int i = 0; i < 8; i += 2) {
                    const float *src = patch + (q + r_in) * PITCH + 8 * piece + i;
                    finish_pair(o, row0 + q + r_in, k + i, src[0], src[1]);
                }
        }
        if (o.residual) ask_residual<CW>(o, ptx::smem_u32(residual), lane, row0, k0, h + (wide ? 32 : 64));
    }
}

// With SWAP a lane has one column k of z for CW rows from r0 on; neighbouring lanes neighbouring columns.
template <int CW>
__device__ __forceinline__ void finish_columns(const OutArgs &o, int r0, int k, const Sums<CW, true> &sums)
{
    const int half = k & 1, j = o.gated ? k >> 1 : k;
    const bool live = k < o.Kz, mine = live && !(o.gated && half);
    const float bias = o.bias && live ? __ldg(o.bias + (o.gated && half ? o.K + j : j)) : 0.f;
#pragma unroll 1
    for (int h = 0; h < CW; h += 8) {
        float y[8], res[8];
#pragma unroll
        for (int c = 0; c < CW; c += 8)
            if (h == c) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (e & 1 ? sums.v[(c + e) / 2].y : sums.v[(c + e) / 2].x) + bias;
            }
        const int r = r0 + h;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            res[e] = o.residual && mine && r + e < o.R ? out_load(o.residual, (r + e) * o.ldr + j, o.dtype) : 0.f;
        if (o.gated) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __shfl_down_sync(0xffffffffu, y[e], 1);
            activate_all(y, o.act);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= v[e];
        } else {
            activate_all(y, o.act);
        }
        if (o.residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] += res[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (mine && r + e < o.R) out_store(o.y, (r + e) * o.ldy + j, y[e], o.dtype);
    }
}

// What an epilogue warp keeps through the kernel.
struct EpiCtx {
    uint32_t tmem;               // its lanes and first column in tensor memory
    const float *scales;
    float *patch, *partial;
    uint32_t free_bar;           // slot_free[0]: this CTA's, or with PAIR the leader's
    int c0, quarter, lane;       // first column of the tile that is this warp's
};

template <int BN, bool SWAP, bool PAIR>
__device__ __forceinline__ bool epilogue_tile(Shared *sh, const MmaArgs &a, const WaitCtx &ctx, const EpiCtx &ec, int row0,
                                              int col0, const Range &rg, int &slot, uint32_t &sphase)
{
    using C = Cfg<BN, SWAP, PAIR>;
    constexpr int CW = BN / 2;                    // columns of a warp
    const int quarter = ec.quarter, lane = ec.lane;
    // warp-uniform: does this warp have rows and columns of z?
    const bool active = row0 + quarter * 32 < a.rows && col0 + ec.c0 < a.cols;
    Sums<CW, SWAP> sums;
    sums.zero();
    if constexpr (!SWAP) {
        if (a.out.residual && active && a.split == 1) {
            const uint32_t buffer = ptx::smem_u32(ec.patch + 32 * PATCH_PITCH);
            ask_residual<CW>(a.out, buffer, lane, row0 + quarter * 32, col0 + ec.c0, 0);
            if (a.out.dtype != WFQ_F32) ask_residual<CW>(a.out, buffer, lane, row0 + quarter * 32, col0 + ec.c0, 32);
        }
    }
    bool ready = false;              // the slot was seen to be full ahead of its turn
    for (int q0 = 0; q0 < rg.np; q0 += a.cg) {
        const int n = min(a.cg, rg.np - q0);
        if (!__all_sync(0xffffffffu, ready) &&
            !wait<C>(ptx::smem_u32(&sh->acc_full[slot]), sphase, ctx, kWaitTmemFull))
            return false;
        if (active) {
            ptx::tc_fence_after();
            const float *sc = ec.scales + (size_t)slot * a.cg * C::GROUP_SCALE_FLOATS;
            for (int j = 0; j < n; ++j) {
                const uint32_t taddr = ec.tmem + (uint32_t)((slot * a.cg + j) * BN);
                const float *rows = sc + j * C::GROUP_SCALE_FLOATS + quarter * 32;
                const float *cs = sc + j * C::GROUP_SCALE_FLOATS + BM + ec.c0;
                if constexpr (SWAP) {
                    promote<CW>(taddr, rows[lane], cs, sums);
                } else {
                    float rs[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) rs[q] = rows[lane / 4 + 8 * q];
                    promote<CW>(taddr, rs, cs + 2 * (lane % 4), sums);
                }
            }
            ptx::tc_fence_before();
        }
        if constexpr (BN >= 128) {       // wide tiles: a wait on a full slot is 10 % of a piece (2000 x 8192 -> 2048, groups of
                                         // 128: 64.8 -> 61.3 us; with 64 columns 2 % slower)
            const int after = slot + 1 == a.slots ? 0 : slot + 1;
            ready = ptx::mbar_test_wait(ptx::smem_u32(&sh->acc_full[after]), after ? sphase : sphase ^ 1u);
        }
        __syncwarp();
        if (ptx::elect_one()) {
            if constexpr (PAIR) {
                ptx::mbar_arrive(ptx::smem_u32(&sh->scale_free[slot]));
                ptx::mbar_arrive_cluster(ec.free_bar + 8u * slot);
            } else {
                ptx::mbar_arrive(ec.free_bar + 8u * slot);
            }
        }
        __syncwarp();
        if (++slot == a.slots) { slot = 0; sphase ^= 1u; }
    }
    if constexpr (!PAIR) {
        if (a.split > 1) {           // [column][lane of TMEM], one float of padding per column
            float *to = ec.partial + ec.c0 * (BM + 1) + quarter * 32;
            if constexpr (SWAP) {
#pragma unroll
                for (int j = 0; j < CW; ++j) to[j * (BM + 1) + lane] = j & 1 ? sums.v[j / 2].y : sums.v[j / 2].x;
            } else {
                to += 2 * (lane % 4) * (BM + 1) + lane / 4;
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < CW / 8; ++j) {
                        to[8 * j * (BM + 1) + 8 * q] = sums.v[q][j].x;
                        to[(8 * j + 1) * (BM + 1) + 8 * q] = sums.v[q][j].y;
                    }
            }
            return true;
        }
    }
    if (active) {
        if constexpr (SWAP) finish_columns<CW>(a.out, col0 + ec.c0, row0 + quarter * 32 + lane, sums);
        else finish_rows<CW>(a.out, ec.patch, lane, row0 + quarter * 32, col0 + ec.c0, sums);
    }
    return true;
}

// The MMA issuer's loop.  GST: steps of 32 channels per group, 4 standing for any multiple of four (groups begin and end
// with a stage), 0 for every other number.  Its instructions form one dependent chain: with the place of a step in its
// group decided at run time a stage of four MMAs took 1270 cycles.
template <int BN, bool SWAP, bool PAIR, int GST>
__device__ __forceinline__ void issue(Shared *sh, uint32_t tiles_lo, uint32_t tmem_base, const MmaArgs &a, const Range &rg,
                                      const WaitCtx &ctx, int first, int stride)
{
    using C = Cfg<BN, SWAP, PAIR>;
    constexpr uint32_t dhi = ptx::smem_desc_sw128_hi();
    constexpr uint32_t idesc = ptx::idesc_i8(PAIR ? 2 * BM : BM, BN);
    constexpr int PER = GST == 1 || GST == 2 ? 4 / GST : 1;              // groups per stage
    constexpr int CG = PER < C::CG_MAX ? PER : C::CG_MAX;                // pieces per chunk
    const uint32_t full0 = ptx::smem_u32(&sh->full[0]), empty0 = ptx::smem_u32(&sh->empty[0]);
    const uint32_t acc0 = ptx::smem_u32(&sh->acc_full[0]), free0 = ptx::smem_u32(&sh->slot_free[0]);
    auto mma = [&](uint32_t d, uint32_t al, uint32_t bl, bool first_step) {
        if constexpr (PAIR) ptx::umma_i8_pair(d, al, bl, dhi, idesc, !first_step);
        else ptx::umma_i8_lo(d, al, bl, dhi, idesc, !first_step);
    };
    auto commit = [&](uint32_t bar) {
        if constexpr (PAIR) ptx::umma_commit_pair(bar);
        else ptx::umma_commit(bar);
    };
    int stage = 0, slot = 0;
    uint32_t phase = 0, sphase = 0;
    for (int t = first; t < a.tiles; t += stride) {
        int in_group = rg.s0 % a.gsteps;                                 // GST 4 and 0: steps into the current group
        bool begins = true;                                              // the next step is the first of its piece
        for (int kb = rg.kb0; kb < rg.kb1; ++kb) {
            const int n = min(4, rg.s1 - 4 * kb);
            if (!wait<C>(full0 + 8u * stage, phase, ctx, kWaitSmemFull)) return;
            const uint32_t a_lo = tiles_lo + (uint32_t)(stage * (C::STAGE_BYTES >> 4));
            const uint32_t b_lo = a_lo + (uint32_t)(A_BYTES >> 4);
            if constexpr (GST == 4) {
                if (begins && !wait<C>(free0 + 8u * slot, sphase ^ 1u, ctx, kWaitTmemEmpty)) return;
                in_group += n;
                const bool ends = in_group == a.gsteps || 4 * kb + n == rg.s1;
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
                    const uint32_t d = tmem_base + (uint32_t)(slot * CG * BN);
                    mma(d, a_lo, b_lo, begins);
                    if (n > 1) mma(d, a_lo + 2, b_lo + 2, false);
                    if (n > 2) mma(d, a_lo + 4, b_lo + 4, false);
                    if (n > 3) mma(d, a_lo + 6, b_lo + 6, false);
                    commit(empty0 + 8u * stage);
                    if (ends) commit(acc0 + 8u * slot);
                }
                __syncwarp();
                begins = ends;
                if (in_group == a.gsteps) in_group = 0;
                if (ends) {
                    if (++slot == a.slots) { slot = 0; sphase ^= 1u; }
                }
            } else if constexpr (GST > 0) {
#pragma unroll
                for (int c = 0; c < 4; c += CG * GST) {                  // chunks of the stage
                    if (c < n) {
                        if (!wait<C>(free0 + 8u * slot, sphase ^ 1u, ctx, kWaitTmemEmpty)) return;
                        ptx::tc_fence_after();
                        if (ptx::elect_one()) {
                            const uint32_t d = tmem_base + (uint32_t)(slot * CG * BN);
#pragma unroll
                            for (int s = c; s < c + CG * GST; ++s)
                                if (s < n) {
                                    const uint32_t dj = d + (uint32_t)((s - c) / GST * BN), off = 2u * s;
                                    mma(dj, a_lo + off, b_lo + off, s % GST == 0);
                                }
                            commit(acc0 + 8u * slot);
                        }
                        __syncwarp();
                        if (++slot == a.slots) { slot = 0; sphase ^= 1u; }
                    }
                }
                if (ptx::elect_one()) commit(empty0 + 8u * stage);
                __syncwarp();
            } else {
                ptx::tc_fence_after();
                for (int s = 0; s < n; ++s) {
                    if (begins) {
                        if (!wait<C>(free0 + 8u * slot, sphase ^ 1u, ctx, kWaitTmemEmpty)) return;
                        ptx::tc_fence_after();
                    }
                    const bool ends = ++in_group == a.gsteps || 4 * kb + s + 1 == rg.s1;
                    if (ptx::elect_one()) {
                        const uint32_t d = tmem_base + (uint32_t)(slot * CG * BN);
                        mma(d, a_lo + 2 * s, b_lo + 2 * s, begins);
                        if (ends) commit(acc0 + 8u * slot);
                    }
                    __syncwarp();
                    begins = ends;
                    if (in_group == a.gsteps) in_group = 0;
                    if (ends) {
                        if (++slot == a.slots) { slot = 0; sphase ^= 1u; }
                    }
                }
                if (ptx::elect_one()) commit(empty0 + 8u * stage);
                __syncwarp();
            }
            if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
        }
    }
}

template <int BN, bool SWAP, bool PAIR>
__global__ void __launch_bounds__(THREADS, 1)
linear_mma_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, MmaArgs a)
{
    using C = Cfg<BN, SWAP, PAIR>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *tiles = ptx::align_smem<1024>(smem_raw);
    float *patches = reinterpret_cast<float *>(tiles + (size_t)C::STAGES * C::STAGE_BYTES);
    float *scales = patches + EPI_WARPS * (C::PATCH_BYTES / 4);
    Shared *sh = reinterpret_cast<Shared *>(scales + (size_t)C::PIECES * C::GROUP_SCALE_FLOATS);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ctas = PAIR ? 2 : a.split;                                   // of a cluster
    const int rank = (int)blockIdx.x % ctas, first = (int)blockIdx.x / ctas, stride = (int)gridDim.x / ctas;
    const Range rg = range_of(a, PAIR ? 0 : rank);
    const int row_block = PAIR ? 2 * BM : BM, row_off = PAIR ? rank * BM : 0;
    const WaitCtx ctx{&sh->abort, a.status, a.wait_cycles};

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh->full[s]), 1);
            ptx::mbar_init(ptx::smem_u32(&sh->empty[s]), 1);
        }
        for (int s = 0; s < MAX_SLOTS; ++s) {
            ptx::mbar_init(ptx::smem_u32(&sh->acc_full[s]), 2);       // MMAs, scales
            ptx::mbar_init(ptx::smem_u32(&sh->slot_free[s]), (PAIR ? 2 : 1) * EPI_WARPS);
            ptx::mbar_init(ptx::smem_u32(&sh->scale_free[s]), EPI_WARPS);
        }
        ptx::mbar_init(ptx::smem_u32(&sh->mma_done), 1);
        sh->abort = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            ptx::tmem_alloc_pair(ptx::smem_u32(&sh->tmem_base), TMEM_COLS);
            ptx::tmem_relinquish_pair();
        } else {
            ptx::tmem_alloc(ptx::smem_u32(&sh->tmem_base), TMEM_COLS);
            ptx::tmem_relinquish();
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) ptx::cluster_sync();          // the other CTA's barriers are initialised, its tensor memory is allocated
    ptx::tc_fence_after();
    const uint32_t tmem_base = sh->tmem_base;
    const bool rank_issues = !PAIR || rank == 0;
    if (warp == 0 && ptx::elect_one()) {
        ptx::prefetch_tmap(&tmA);
        ptx::prefetch_tmap(&tmB);
    }
    if (warp == 0) __syncwarp();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    if (warp < FIRST_EPI_WARP) {
        if constexpr (C::MOVE_REGS) ptx::fewer_registers<56>();
        if (warp == 0) {
            // ---------------- TMA producer ----------------
            int stage = 0;
            uint32_t phase = 0;
            long long issued = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += stride) {
                const int a_row = t % a.MT * row_block + row_off, b_row = t / a.MT * BN + (PAIR ? rank * C::B_ROWS : 0);
                for (int kb = rg.kb0; kb < rg.kb1; ++kb) {
                    ok = wait<C>(ptx::smem_u32(&sh->empty[stage]), phase ^ 1u, ctx, kWaitSmemEmpty);
                    if (!ok) break;
                    if (ptx::elect_one() && !(blockIdx.x == 0 && issued == a.debug_skip_stage)) {
                        const uint32_t bar = ptx::smem_u32(&sh->full[stage]);
                        const uint32_t dst = ptx::smem_u32(tiles + (size_t)stage * C::STAGE_BYTES);
                        if constexpr (PAIR) {      // the leader's barrier counts both CTAs' bytes
                            const uint32_t lead = ptx::map_rank(bar, 0);
                            if (rank == 0) ptx::mbar_arrive_expect_tx(bar, 2 * C::STAGE_BYTES);
                            ptx::tma_load_2d_pair(dst, &tmA, lead, kb * BK, a_row);
                            ptx::tma_load_2d_pair(dst + A_BYTES, &tmB, lead, kb * BK, b_row);
                        } else {
                            ptx::mbar_arrive_expect_tx(bar, C::STAGE_BYTES);
                            ptx::tma_load_2d(dst, &tmA, bar, kb * BK, a_row);
                            ptx::tma_load_2d(dst + A_BYTES, &tmB, bar, kb * BK, b_row);
                        }
                    }
                    __syncwarp();
                    ++issued;
                    if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok || sh->abort) {      // give copies in flight a bounded time to land
                int s = stage;
                uint32_t ph = phase;
                const long long n = issued < C::STAGES ? issued : C::STAGES;
                for (long long i = 0; i < n; ++i) {
                    if (--s < 0) { s = C::STAGES - 1; ph ^= 1u; }
                    drain(ptx::smem_u32(&sh->full[s]), ph);
                }
            }
        } else if (warp == 1 && rank_issues) {
            // ---------------- MMA issuer ----------------
            const uint32_t tiles_lo = ptx::smem_desc_sw128_lo(ptx::smem_u32(tiles));
            if (a.gsteps % 4 == 0 || a.gsteps >= a.steps) issue<BN, SWAP, PAIR, 4>(sh, tiles_lo, tmem_base, a, rg, ctx, first, stride);
            else if (a.gsteps == 2) issue<BN, SWAP, PAIR, 2>(sh, tiles_lo, tmem_base, a, rg, ctx, first, stride);
            else if (a.gsteps == 1) issue<BN, SWAP, PAIR, 1>(sh, tiles_lo, tmem_base, a, rg, ctx, first, stride);
            else issue<BN, SWAP, PAIR, 0>(sh, tiles_lo, tmem_base, a, rg, ctx, first, stride);
        } else if (warp == 2) {
            // ---------------- scale loader ----------------
            const uint32_t scale_bar = ptx::smem_u32(PAIR ? &sh->scale_free[0] : &sh->slot_free[0]);
            int slot = 0;
            uint32_t sphase = 0;
            long long issued = 0;
            bool ok = true;
            for (int t = first; t < a.tiles && ok; t += stride) {
                const int mt = t % a.MT, nt = t / a.MT;
                // the second CTA of a pair may have no rows: it then reads scales that it does not use
                const long long row0 = min((long long)mt * row_block + row_off, a.row_pitch - BM);
                for (int q0 = 0; q0 < rg.np; q0 += a.cg) {
                    const int n = min(a.cg, rg.np - q0);
                    ok = wait<C>(scale_bar + 8u * slot, sphase ^ 1u, ctx, kWaitScaleEmpty);
                    if (!ok) break;
                    const uint32_t bar = ptx::smem_u32(&sh->acc_full[slot]);
                    const uint32_t dst = ptx::smem_u32(scales + (size_t)slot * a.cg * C::GROUP_SCALE_FLOATS);
                    if (ptx::elect_one()) ptx::mbar_arrive_expect_tx(bar, (uint32_t)(n * C::GROUP_SCALE_FLOATS * 4));
                    __syncwarp();
                    if (lane < 8 && (lane & 3) < n) {      // lane j: row scales of piece j, lane 4 + j: column scales
                        const int j = lane & 3;
                        const long long g = rg.g0 + q0 + j;
                        const uint32_t d = dst + (uint32_t)(j * C::GROUP_SCALE_FLOATS * 4);
                        if (lane < 4) ptx::bulk_load(d, a.row_scale + g * a.row_pitch + row0, BM * 4, bar);
                        else ptx::bulk_load(d + BM * 4, a.col_scale + g * a.col_pitch + nt * BN, BN * 4, bar);
                    }
                    __syncwarp();
                    ++issued;
                    if (++slot == a.slots) { slot = 0; sphase ^= 1u; }
                }
            }
            if (!ok || sh->abort) {
                int s = slot;
                uint32_t ph = sphase;
                const long long n = issued < a.slots ? issued : a.slots;
                for (long long i = 0; i < n; ++i) {
                    if (--s < 0) { s = a.slots - 1; ph ^= 1u; }
                    drain(ptx::smem_u32(&sh->acc_full[s]), ph);
                }
            }
        }
    } else {
        // ---------------- epilogue ----------------
        if constexpr (C::MOVE_REGS) ptx::more_registers<216>();
        const int e = warp - FIRST_EPI_WARP, quarter = warp & 3;
        int slot = 0;
        uint32_t sphase = 0;
        EpiCtx ec;
        ec.c0 = (e >> 2) * (BN / 2);
        ec.tmem = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)ec.c0;
        ec.scales = scales;
        ec.patch = patches + e * (C::PATCH_BYTES / 4);
        ec.partial = reinterpret_cast<float *>(tiles);
        ec.free_bar = ptx::smem_u32(&sh->slot_free[0]);
        if constexpr (PAIR) ec.free_bar = ptx::map_rank(ec.free_bar, 0);
        ec.quarter = quarter;
        ec.lane = lane;
        for (int t = first; t < a.tiles; t += stride) {
            const int mt = t % a.MT, nt = t / a.MT;
            if (!epilogue_tile<BN, SWAP, PAIR>(sh, a, ctx, ec, mt * row_block + row_off, nt * BN, rg, slot, sphase)) break;
        }
        if constexpr (!SWAP) ptx::copy_async_wait<0>();      // where a wait ran out, residuals may still be on their way
    }

    __syncwarp();
    if (!PAIR && a.split > 1) {
        // one tile per cluster: the partial sums are complete, each CTA adds up its share of the columns in rank order
        ptx::cluster_sync();
        const int share = BN / a.split;             // even: at least 2
        const int mt = first % a.MT, nt = first / a.MT, col0 = rank * share;
        const uint32_t mine = ptx::smem_u32(tiles);
        if (first < a.tiles) {
            for (int i = threadIdx.x; i < BM * share / 2; i += THREADS) {
                int r0, c0, r1, c1;                 // the pair's places in the tile
                if constexpr (SWAP) { r0 = 2 * (i % (BM / 2)); r1 = r0 + 1; c0 = c1 = col0 + i / (BM / 2); }
                else { r0 = r1 = i / (share / 2); c0 = col0 + 2 * (i % (share / 2)); c1 = c0 + 1; }
                float w0[8], w1[8], v0 = 0.f, v1 = 0.f;
#pragma unroll
                for (int p = 0; p < 8; ++p)         // all loads on their way before the first addition
                    if (p < a.split) {
                        const uint32_t base = ptx::map_rank(mine, (uint32_t)p);
                        w0[p] = ptx::ld_cluster(base + (uint32_t)((c0 * (BM + 1) + r0) * 4));
                        w1[p] = ptx::ld_cluster(base + (uint32_t)((c1 * (BM + 1) + r1) * 4));
                    }
#pragma unroll
                for (int p = 0; p < 8; ++p)
                    if (p < a.split) { v0 += w0[p]; v1 += w1[p]; }
                if constexpr (SWAP) finish_pair(a.out, nt * BN + c0, mt * BM + r0, v0, v1);
                else finish_pair(a.out, mt * BM + r0, nt * BN + c0, v0, v1);
            }
        }
        ptx::cluster_sync();                        // nobody leaves while others read its sums
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 1 && sh->abort) {       // MMAs may still be in flight; with PAIR the other CTA's copies and MMAs too
        if (rank_issues && ptx::elect_one()) {
            if constexpr (PAIR) ptx::umma_commit_pair(ptx::smem_u32(&sh->mma_done));
            else ptx::umma_commit(ptx::smem_u32(&sh->mma_done));
        }
        __syncwarp();
        drain(ptx::smem_u32(&sh->mma_done), 0);
    }
    if constexpr (PAIR) ptx::cluster_sync();        // nobody leaves while the pair's MMAs read or write its memory
    if (warp == 1) {
        ptx::tc_fence_after();
        if constexpr (PAIR) ptx::tmem_dealloc_pair(tmem_base, TMEM_COLS);
        else ptx::tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// Up to eight rows: linear_dot_kernel, dot products by the integer units (dp4a), bound by the weights' bytes.  A warp has
// four columns of z and a part of the channels; a lane reads 16 channels of each column at a time, which lie in one group,
// so their int32 sum is scaled at once and one fp32 sum per row and column is left to add over the lanes.  The rows' codes
// are in shared memory; rows that come as values are quantized there by every CTA, which saves a launch.  The first
// weights are asked for ahead of that, and ahead of the previous kernel's end where they are known to be in place.
constexpr int DOT_THREADS = 256, DOT_WARPS = DOT_THREADS / 32, DOT_COLS = 4, DOT_AHEAD = 2;
constexpr int DOT_MAX_ROWS = 8;
constexpr int DOT_SMEM_MAX = 96 * 1024;
// Values that a CTA quantizes for itself: what its registers keep without taking them from the products.  With twice as many
// 2 x 4096 -> 4096 takes 10.6 us and 1 x 4096 8.4 us, against 8.5 and 7.9 us (the first through the row quantizer); one row of
// 5120 -> 5120 11.5 against 10.4 us, 8192 -> 8192 16.0 against 14.2, 8192 -> 1024 5.3 against 5.6 (all replayed from a
// graph); every CTA reading 4 rows of 8192 twice takes 46 us.  Where the host is the bound the quantizer's launch costs 2 us.
constexpr int DOT_KEEP = 2;
constexpr int DOT_QUANTIZE_MAX = 8 * DOT_THREADS * DOT_KEEP;

struct DotArgs {
    const void *x;               // values [rows][C], or null:
    const int8_t *xq;            // codes and scales
    const float *sx;
    long long ldx, sx_pitch;
    const int8_t *Wq;
    const float *sW;
    int C, Cp, G, rows, Kp;
    int parts;                   // warps that share a column's channels: 1, 2, 4 or 8
    int units;                   // blocks of DOT_COLS columns times parts
    int early;                   // the weights are complete whatever the previous kernel does
    FastDiv by_gs, by_vectors;   // channels of a group; 8-channel vectors of a row
    OutArgs out;
};

int dot_smem(int rows, int Cp, int G)
{
    const int r = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8;
    return r * Cp + 2 * 4 * r * G + DOT_WARPS * r * DOT_COLS * 4;
}

template <typename T> __device__ __forceinline__ float value_of(T v) { return (float)v; }

template <int R, typename T>       // T: type of x, int8_t for codes
__global__ void __launch_bounds__(DOT_THREADS) linear_dot_kernel(DotArgs a)
{
    extern __shared__ __align__(16) unsigned char smem_dot[];
    int8_t *codes = reinterpret_cast<int8_t *>(smem_dot);                 // [R][Cp]
    float *sx = reinterpret_cast<float *>(codes + R * a.Cp);              // [R][G]
    int *gmax = reinterpret_cast<int *>(sx + R * a.G);                    // [R][G]
    float *part = reinterpret_cast<float *>(gmax + R * a.G);              // [warp][R][DOT_COLS]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // One unit per warp where warps share a column; else a warp goes on to further units, their weights in one stream
    int unit = (int)blockIdx.x * DOT_WARPS + warp;
    const int seg = unit % a.parts, units = a.units, stride = a.parts > 1 ? units : (int)gridDim.x * DOT_WARPS;
    const int nv = a.Cp / 16, v0 = (int)((long long)nv * seg / a.parts), v1 = (int)((long long)nv * (seg + 1) / a.parts);

    uint4 now[DOT_AHEAD][DOT_COLS], next[DOT_AHEAD][DOT_COLS];
    auto fetch = [&](uint4 (&to)[DOT_AHEAD][DOT_COLS], int of, int v) {
        if (of >= units) return;
        const int k = of / a.parts * DOT_COLS;
        const uint4 *w = reinterpret_cast<const uint4 *>(a.Wq + (size_t)k * a.Cp) + v;
        const int cols = a.out.Kz - k;
#pragma unroll
        for (int u = 0; u < DOT_AHEAD; ++u)
#pragma unroll
            for (int j = 0; j < DOT_COLS; ++j)
                if (j < cols && v + 32 * u < v1) to[u][j] = __ldg(w + (size_t)j * nv + 32 * u);
    };
    if (!a.early) ptx::grid_dependency_wait();
    fetch(now, unit, v0 + lane);
    if (a.early) ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    // ---- the rows' codes and scales ----
    if constexpr (std::is_same<T, int8_t>::value) {
        const int n = a.Cp / 16;
        for (int i = threadIdx.x; i < R * n; i += DOT_THREADS)
            reinterpret_cast<uint4 *>(codes)[i] =
                i < a.rows * n ? reinterpret_cast<const uint4 *>(a.xq)[i] : make_uint4(0, 0, 0, 0);
        for (int i = threadIdx.x; i < R * a.G; i += DOT_THREADS) {
            const int r = i / a.G, g = i - r * a.G;
            sx[i] = r < a.rows ? a.sx[(size_t)g * a.sx_pitch + r] : 0.f;
        }
    } else {
        for (int i = threadIdx.x; i < R * a.G; i += DOT_THREADS) gmax[i] = 0;
        __syncthreads();
        const int vec = a.Cp / 8, total = a.rows * vec;                   // vectors of eight channels, four to 32
        const bool wide = a.C % 8 == 0 && a.ldx * sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0;
        float u[DOT_KEEP][8];
        auto load = [&](int i, float (&to)[8]) {
            const int r = i / a.by_vectors, c = (i - r * vec) * 8;
            const T *p = static_cast<const T *>(a.x) + r * a.ldx + c;
            if (wide) {
                if (c >= a.C) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[e] = 0.f;
                } else if constexpr (sizeof(T) == 4) {
                    const float4 lo = reinterpret_cast<const float4 *>(p)[0], hi = reinterpret_cast<const float4 *>(p)[1];
                    to[0] = lo.x; to[1] = lo.y; to[2] = lo.z; to[3] = lo.w;
                    to[4] = hi.x; to[5] = hi.y; to[6] = hi.z; to[7] = hi.w;
                } else {
                    const uint4 q = *reinterpret_cast<const uint4 *>(p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[e] = value_of(reinterpret_cast<const T *>(&q)[e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) to[e] = c + e < a.C ? value_of(p[e]) : 0.f;
            }
        };
        auto group_at = [&](int i) {          // index of the group of vector i, row by row
            const int r = i / a.by_vectors;
            return r * a.G + (i - r * vec) * 8 / a.by_gs;
        };
#pragma unroll
        for (int k = 0; k < DOT_KEEP; ++k) {
            const int i = k * DOT_THREADS + threadIdx.x;
            if (i < total) load(i, u[k]);
        }
#pragma unroll
        for (int k = 0; k < DOT_KEEP; ++k) {
            const int i = k * DOT_THREADS + threadIdx.x;
            int m = 0;
            if (i < total) {
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, __float_as_int(u[k][e]) & 0x7fffffff);
            }
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));      // the four lanes of 32 channels
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            if (i < total && (lane & 3) == 0) atomicMax(&gmax[group_at(i)], m);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.rows * a.G; i += DOT_THREADS) {
            float inv;
            quantizer_scale(__int_as_float(gmax[i]), sx[i], inv);
        }
#pragma unroll
        for (int k = 0; k < DOT_KEEP; ++k) {
            const int i = k * DOT_THREADS + threadIdx.x;
            if (i < total) {
                float scale, inv;
                quantizer_scale(__int_as_float(gmax[group_at(i)]), scale, inv);
                uint32_t q[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = inv > 0.f ? code_bits(u[k][e], inv) : 0u;
                const uint32_t lo = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
                const uint32_t hi = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
                reinterpret_cast<uint2 *>(codes)[i] = make_uint2(lo, hi);
            }
        }
        for (int i = total + threadIdx.x; i < R * vec; i += DOT_THREADS) reinterpret_cast<uint2 *>(codes)[i] = make_uint2(0, 0);
        for (int i = a.rows * a.G + threadIdx.x; i < R * a.G; i += DOT_THREADS) sx[i] = 0.f;
    }
    __syncthreads();

    // ---- dot products ----
    for (; unit < units; unit += stride) {
        const int k0 = unit / a.parts * DOT_COLS;
        float acc[R][DOT_COLS];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < DOT_COLS; ++j) acc[r][j] = 0.f;
        for (int v = v0 + lane; v < v1 + lane; v += 32 * DOT_AHEAD) {    // the same number of turns for all lanes
            const bool more = v + 32 * DOT_AHEAD < v1 + lane;
            fetch(next, more ? unit : unit + stride, more ? v + 32 * DOT_AHEAD : v0 + lane);
#pragma unroll
            for (int u = 0; u < DOT_AHEAD; ++u) {
                const int vu = v + 32 * u;
                if (vu < v1) {
                    const int g = vu * 16 / a.by_gs;
                    const float4 sw = __ldg(reinterpret_cast<const float4 *>(a.sW + (size_t)g * a.Kp + k0));
                    const float s[DOT_COLS] = {sw.x, sw.y, sw.z, sw.w};
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const uint4 q = *reinterpret_cast<const uint4 *>(codes + r * a.Cp + vu * 16);
                        const float sr = sx[r * a.G + g];
#pragma unroll
                        for (int j = 0; j < DOT_COLS; ++j) {
                            int d = __dp4a((int)q.x, (int)now[u][j].x, 0);
                            d = __dp4a((int)q.y, (int)now[u][j].y, d);
                            d = __dp4a((int)q.z, (int)now[u][j].z, d);
                            d = __dp4a((int)q.w, (int)now[u][j].w, d);
                            acc[r][j] = fmaf((float)d * sr, s[j], acc[r][j]);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < DOT_COLS; ++j) now[u][j] = next[u][j];
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < DOT_COLS; ++j)
#pragma unroll
                for (int o = 16; o; o >>= 1) acc[r][j] += __shfl_xor_sync(0xffffffffu, acc[r][j], o);
        // lane 2 r + p finishes columns 2 p and 2 p + 1 of row r
        float f0 = 0.f, f1 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int p = 0; p < DOT_COLS / 2; ++p)
                if (lane == 2 * r + p) { f0 = acc[r][2 * p]; f1 = acc[r][2 * p + 1]; }
        if (a.parts == 1) {
            if (lane < 2 * R) finish_pair(a.out, lane / 2, k0 + 2 * (lane & 1), f0, f1);
        } else if (lane < 2 * R) {
            float *mine = part + warp * R * DOT_COLS;
            mine[2 * lane] = f0;
            mine[2 * lane + 1] = f1;
        }
    }
    if (a.parts > 1) {
        __syncthreads();
        const int k0 = ((int)blockIdx.x * DOT_WARPS + warp) / a.parts * DOT_COLS;
        if (seg == 0 && lane < 2 * R && k0 < a.out.Kz) {
            float f0 = 0.f, f1 = 0.f;
            for (int p = 0; p < a.parts; ++p) {       // in order
                f0 += part[(warp + p) * R * DOT_COLS + 2 * lane];
                f1 += part[(warp + p) * R * DOT_COLS + 2 * lane + 1];
            }
            finish_pair(a.out, lane / 2, k0 + 2 * (lane & 1), f0, f1);
        }
    }
}

// How a call is laid out: orientation (1: rows of x on the lanes, 2: outputs, 3: pairs of CTAs with rows of x, 4: dot
// products), columns per tile, CTAs that share a tile's channels.
struct Shape { int orient, bn, split; };

bool known_shape(const Shape &s)
{
    if (s.orient == 1) return s.bn == 64 || s.bn == 128;
    if (s.orient == 2) return s.bn == 16 || s.bn == 32 || s.bn == 64;
    if (s.orient == 4) return s.bn == 4 && s.split == 1;
    return s.orient == 3 && s.split == 1 && (s.bn == 128 || s.bn == 256);
}

// Microseconds of a tile: a stage of 128 channels takes its copies and MMAs or the promotion of its chunks, whichever is
// longer; then the results' way out, or, where CTAs share the channels, the sum of their parts (kSharedOut whatever the
// shape).  Fitted to the times of every shape on 170 random sizes (32 to 8192 rows, 32 to 8192 channels, 128 to 32768
// columns of z, groups of 32 to whole rows, all types); on 148 others the chosen shape takes 4 % longer than the best of
// them in the mean, 13 % or less on nine out of ten and 39 % at worst.
struct TileTime { double stage, chunk, piece, out; };
constexpr double kSharedOut = 3.9;
TileTime tile_time(const Shape &s)
{
    if (s.orient == 2) return s.bn == 16 ? TileTime{.31, .09, .02, 2.} : s.bn == 32 ? TileTime{.25, .18, .03, 6.2} : TileTime{.16, .23, .11, 7.2};
    if (s.orient == 3) return s.bn == 128 ? TileTime{.26, .34, .32, 4.3} : TileTime{.4, .33, .71, 8.7};
    return s.bn == 64 ? TileTime{.21, .2, .15, 2.2} : TileTime{.35, .25, .45, 3.5};
}

Shape choose(const wfq_linear &l, int rows)
{
    const bool dot = rows <= DOT_MAX_ROWS && dot_smem(rows, l.Cp, l.G) <= DOT_SMEM_MAX;
    if (l.debug_shape && (dot || l.debug_shape / 1000 % 10 != 4))
        return Shape{l.debug_shape / 1000 % 10, l.debug_shape % 1000, l.debug_shape / 10000};
    const int KB = (l.Cp / 32 + 3) / 4;
    Shape best{1, 64, 1};
    double best_cost = 1e300;
    if (dot) {       // bytes at a rate that falls with the rows' arithmetic (4096 -> 4096: 1 row 6.3 us, 4 rows 8.1; shared
                     // tensor-core tiles 6.9 and 7.1)
        best = Shape{4, 4, 1};
        best_cost = (double)l.Kz * l.Cp / (rows <= 2 ? 4.2e6 : rows <= 4 ? 2.8e6 : 2.0e6) + .7;
    }
    for (int orient = 1; orient <= 3; ++orient)
        for (int bn : {256, 128, 64, 32, 16})
            for (int split : {1, 2, 4, 8}) {
                const Shape sp{orient, bn, split};
                if (!known_shape(sp)) continue;
                const int lanes = orient == 3 ? 2 * BM : BM, per_tile = orient == 3 ? 2 : split;
                const int r = orient == 2 ? l.Kz : rows, c = orient == 2 ? rows : l.Kz;
                const double tiles = (double)((r + lanes - 1) / lanes) * ((c + bn - 1) / bn);
                // Clusters beyond those that run at once would take a second round: 16 of 8 CTAs do not fit the processor
                // clusters of 148 SMs, 8192 -> 2048 12.9 us instead of 7.2 us for the 14 of 8192 -> 1792.
                const int log2_split = split == 8 ? 3 : split / 2;
                if (split > 1 && (tiles > l.clusters[log2_split] || KB < 2 * split)) continue;
                const TileTime t = tile_time(sp);
                const int pieces = 512 / bn < 16 ? 512 / bn : 16, cg_max = pieces / 2 < 4 ? pieces / 2 : 4;
                const int cg = BK % l.gs != 0 || l.G == 1 ? 1 : BK / l.gs < cg_max ? BK / l.gs : cg_max;
                double stage = 128.0 / l.gs / cg * (t.chunk + t.piece * cg);
                if (stage < t.stage) stage = t.stage;
                const int at_once = l.sm_count / per_tile;
                const double waves = (double)(long long)((tiles + at_once - 1) / at_once);
                const double cost = waves * ((KB + split - 1) / split * stage + (split > 1 ? kSharedOut : t.out));
                if (cost < best_cost) { best_cost = cost; best = sp; }
            }
    return best;
}

bool encode_codes(CUtensorMap *map, const int8_t *codes, int Cp, int rows, int box_rows)
{
    const unsigned long long dims[2] = {(unsigned long long)Cp, (unsigned long long)rows};
    const unsigned long long strides[1] = {(unsigned long long)Cp};
    const unsigned box[2] = {128u, (unsigned)box_rows};
    return encode_tmap(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int BN, bool SWAP, bool PAIR>
cudaError_t setup_variant()
{
    return cudaFuncSetAttribute(linear_mma_kernel<BN, SWAP, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)Cfg<BN, SWAP, PAIR>::SMEM_BYTES);
}

template <int BN, bool SWAP, bool PAIR>
cudaError_t launch_variant(wfq_linear &l, MmaArgs &a, int grid, const int8_t *xq, int rows, cudaStream_t stream)
{
    a.cg = 1;                    // also where one group is all there is, however short: the MMA loop takes it as whole stages
    if (BK % l.gs == 0 && l.G > 1) a.cg = BK / l.gs < Cfg<BN, SWAP, PAIR>::CG_MAX ? BK / l.gs : Cfg<BN, SWAP, PAIR>::CG_MAX;
    a.slots = Cfg<BN, SWAP, PAIR>::PIECES / a.cg;
    constexpr int w_rows = SWAP ? BM : Cfg<BN, SWAP, PAIR>::B_ROWS;
    constexpr int w_map = w_rows == 128 ? 1 : 0;
    static_assert(w_rows == 128 || w_rows == 64, "rows of a box of weights");
    CUtensorMap tx;
    if (!l.tmap_w_ok[w_map]) l.tmap_w_ok[w_map] = encode_codes(&l.tmap_w[w_map], l.Wq, l.Cp, l.Kz, w_rows);
    if (!l.tmap_w_ok[w_map] || !encode_codes(&tx, xq, l.Cp, rows, SWAP ? BN : BM)) return cudaErrorInvalidValue;
    const CUtensorMap &tw = l.tmap_w[w_map];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Cfg<BN, SWAP, PAIR>::SMEM_BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
    if (PAIR || a.split > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = PAIR ? 2u : (unsigned)a.split;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, linear_mma_kernel<BN, SWAP, PAIR>, SWAP ? tw : tx, SWAP ? tx : tw, a);
}

template <int R, typename T>
cudaError_t launch_dot_kernel(const DotArgs &a, int grid, int smem, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(DOT_THREADS);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_dot_kernel<R, T>, a);
}
template <typename T>
cudaError_t launch_dot_rows(const DotArgs &a, int grid, int smem, cudaStream_t stream)
{
    if (a.rows <= 1) return launch_dot_kernel<1, T>(a, grid, smem, stream);
    if (a.rows <= 2) return launch_dot_kernel<2, T>(a, grid, smem, stream);
    if (a.rows <= 4) return launch_dot_kernel<4, T>(a, grid, smem, stream);
    return launch_dot_kernel<8, T>(a, grid, smem, stream);
}
template <typename T>
cudaError_t setup_dot()
{
    cudaError_t e = cudaSuccess;
    auto set = [&](auto kernel) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DOT_SMEM_MAX);
    };
    set(linear_dot_kernel<1, T>);
    set(linear_dot_kernel<2, T>);
    set(linear_dot_kernel<4, T>);
    set(linear_dot_kernel<8, T>);
    return e;
}

// x: values in the layer's input type, or null with codes and scales.
cudaError_t launch_dot(const wfq_linear &l, const void *x, long long ldx, const int8_t *xq, const float *sx, int rows,
                       const OutArgs &out, cudaStream_t stream, bool early)
{
    DotArgs a;
    a.x = x; a.ldx = ldx;
    a.xq = xq; a.sx = sx; a.sx_pitch = (rows + 127LL) / 128 * 128;
    a.Wq = l.Wq; a.sW = l.sW;
    a.C = l.C; a.Cp = l.Cp; a.G = l.G; a.rows = rows; a.Kp = l.Kp;
    a.by_gs = FastDiv(l.gs);
    a.by_vectors = FastDiv(l.Cp / 8);
    a.early = early;
    a.out = out;
    // as many warps to a column as give every SM two CTAs, but a lane two vectors at least
    const int quads = (l.Kz + DOT_COLS - 1) / DOT_COLS;
    a.parts = 1;
    while (a.parts < 8 && (long long)quads * a.parts < 16LL * l.sm_count && l.Cp / 16 / (2 * a.parts) >= 64) a.parts *= 2;
    a.units = quads * a.parts;
    const int smem = dot_smem(rows, l.Cp, l.G), ctas = (a.units + DOT_WARPS - 1) / DOT_WARPS;
    const int grid = a.parts > 1 || ctas < 2 * l.sm_count ? ctas : 2 * l.sm_count;
    if (!x) return launch_dot_rows<int8_t>(a, grid, smem, stream);
    if (l.in_dtype == WFQ_F32) return launch_dot_rows<float>(a, grid, smem, stream);
    if (l.in_dtype == WFQ_F16) return launch_dot_rows<__half>(a, grid, smem, stream);
    return launch_dot_rows<__nv_bfloat16>(a, grid, smem, stream);
}

Shape shape_for(wfq_linear &l, int rows)
{
    if (l.shape_rows != rows) {
        const Shape s = choose(l, rows);
        l.shape_rows = rows; l.shape_orient = s.orient; l.shape_bn = s.bn; l.shape_split = s.split;
    }
    return Shape{l.shape_orient, l.shape_bn, l.shape_split};
}

cudaError_t launch_product(wfq_linear &l, const int8_t *xq, const float *sx, int rows, const OutArgs &out,
                           cudaStream_t stream)
{
    const Shape sp = shape_for(l, rows);
    MmaArgs a;
    const long long sx_pitch = (rows + 127LL) / 128 * 128;
    const bool swap = sp.orient == 2, pair = sp.orient == 3;
    a.row_scale = swap ? l.sW : sx;
    a.col_scale = swap ? sx : l.sW;
    a.row_pitch = swap ? l.Kp : sx_pitch;
    a.col_pitch = swap ? sx_pitch : l.Kp;
    a.rows = swap ? l.Kz : rows;
    a.cols = swap ? rows : l.Kz;
    a.MT = (int)((a.rows + (pair ? 2LL : 1LL) * BM - 1) / (pair ? 2 * BM : BM));
    a.tiles = a.MT * ((a.cols + sp.bn - 1) / sp.bn);
    a.split = sp.split;
    a.steps = l.Cp / UK;
    a.gsteps = l.gs / UK;
    a.status = l.status;
    a.wait_cycles = l.wait_cycles;
    a.debug_skip_stage = l.debug_skip_stage;
    a.out = out;
    const int at_once = pair ? l.sm_count / 2 : l.sm_count;
    const int grid = sp.split > 1 ? a.tiles * sp.split : (a.tiles < at_once ? a.tiles : at_once) * (pair ? 2 : 1);
    if (swap) {
        if (sp.bn == 16) return launch_variant<16, true, false>(l, a, grid, xq, rows, stream);
        if (sp.bn == 32) return launch_variant<32, true, false>(l, a, grid, xq, rows, stream);
        return launch_variant<64, true, false>(l, a, grid, xq, rows, stream);
    }
    if (pair) {
        if (sp.bn == 128) return launch_variant<128, false, true>(l, a, grid, xq, rows, stream);
        return launch_variant<256, false, true>(l, a, grid, xq, rows, stream);
    }
    if (sp.bn == 64) return launch_variant<64, false, false>(l, a, grid, xq, rows, stream);
    return launch_variant<128, false, false>(l, a, grid, xq, rows, stream);
}

bool known(wfq_dtype_t t) { return t == WFQ_F32 || t == WFQ_F16 || t == WFQ_BF16; }
size_t elem_bytes(wfq_dtype_t t) { return t == WFQ_F32 ? 4 : 2; }
bool misaligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
size_t up1024(size_t v) { return (v + 1023) / 1024 * 1024; }
wfq_status_t to_status(cudaError_t e)
{
    return e == cudaSuccess ? WFQ_OK : e == cudaErrorMemoryAllocation ? WFQ_ERR_ALLOC : WFQ_ERR_CUDA;
}

// How many clusters of 1 << i CTAs of the tensor-core kernels (one CTA per SM, whatever the shape) run at once.
cudaError_t count_clusters(int (&clusters)[4])
{
    for (int i = 1; i < 4; ++i) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1u << i);
        cfg.blockDim = dim3(THREADS);
        cfg.dynamicSmemBytes = Cfg<16, true, false>::SMEM_BYTES;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 1u << i;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters[i], linear_mma_kernel<16, true, false>, &cfg);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// Binds the layer to the current device the first time, refuses another one later.
wfq_status_t bind(wfq_linear *l)
{
    int dev = -1, sms = 0;
    const wfq_status_t s = current_device(&dev, &sms);
    if (s != WFQ_OK) return s;
    if (l->device == dev) return WFQ_OK;
    if (l->device >= 0) return WFQ_ERR_INVALID_ARG;
    cudaError_t e = setup_variant<16, true, false>();
    if (e == cudaSuccess) e = setup_variant<32, true, false>();
    if (e == cudaSuccess) e = setup_variant<64, true, false>();
    if (e == cudaSuccess) e = setup_variant<64, false, false>();
    if (e == cudaSuccess) e = setup_variant<128, false, false>();
    if (e == cudaSuccess) e = setup_variant<128, false, true>();
    if (e == cudaSuccess) e = setup_variant<256, false, true>();
    if (e == cudaSuccess) e = setup_dot<int8_t>();
    if (e == cudaSuccess) e = setup_dot<float>();
    if (e == cudaSuccess) e = setup_dot<__half>();
    if (e == cudaSuccess) e = setup_dot<__nv_bfloat16>();
    if (e == cudaSuccess) e = count_clusters(l->clusters);
    if (e != cudaSuccess) return WFQ_ERR_CUDA;
    l->device = dev;
    l->sm_count = sms;
    return WFQ_OK;
}

wfq_status_t check_io(const wfq_linear *l, int rows, const void *in, const void *residual, long long ldr, const void *y,
                      long long ldy)
{
    const size_t e = elem_bytes(l->out_dtype);
    if (!y || ldy < l->K || misaligned(y, e)) return WFQ_ERR_INVALID_ARG;
    if (residual && (ldr < l->K || misaligned(residual, e))) return WFQ_ERR_INVALID_ARG;
    // Outputs leave while other CTAs still read inputs; a residual is read where its output goes, if it lies there.
    if (y == in || (y == residual && rows > 1 && ldy != ldr)) return WFQ_ERR_INVALID_ARG;
    if (rows > 0x7fffff00) return WFQ_ERR_UNSUPPORTED;
    if (((rows + 127LL) / 128) * ((l->Kz + 63LL) / 64) > 0x7fffffffLL) return WFQ_ERR_UNSUPPORTED;
    return WFQ_OK;
}

// The layer on codes, or on values `x` (then xq and sx are the workspace).
wfq_status_t run(wfq_linear *l, const void *x, long long ldx, int8_t *xq, float *sx, int rows, const void *residual,
                 long long ldr, void *y, long long ldy, cudaStream_t st)
{
    OutArgs o;
    o.bias = l->bias; o.residual = residual; o.y = y;
    o.ldr = ldr; o.ldy = ldy;
    o.K = l->K; o.Kz = l->Kz; o.R = rows;
    o.act = l->act; o.gated = l->gated; o.dtype = (int)l->out_dtype;
    const size_t elem = elem_bytes(l->out_dtype);
    o.vec = !misaligned(y, 16) && ldy * elem % 16 == 0 && (!residual || (!misaligned(residual, 16) && ldr * elem % 16 == 0));

    const bool dot = shape_for(*l, rows).orient == 4;
    const bool quantize = x && !(dot && (long long)rows * l->Cp <= DOT_QUANTIZE_MAX);
    if (quantize) {
        RowsArgs a;
        a.x = x; a.ldx = ldx;
        a.codes = xq; a.scales = sx;
        a.rows = rows; a.C = l->C; a.Cp = l->Cp;
        a.gs = l->gs; a.G = l->G;
        a.scale_pitch = (rows + 127LL) / 128 * 128;
        if (launch_rows(a, l->in_dtype, st, true) != cudaSuccess) return WFQ_ERR_CUDA;
    }
    // The product's launch may begin before the kernel in front of it has ended, and may fetch weights then if that cannot
    // be the one that writes them: the row quantizer lets it begin only after its own wait for what was in front of it, and
    // otherwise wfq_weight_order.h says.
    const bool settled = l->order.settled(st), first = l->order.pending() && !settled;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    if (first && cudaStreamIsCapturing(st, &cap) != cudaSuccess) return WFQ_ERR_CUDA;
    const cudaError_t e = dot ? launch_dot(*l, quantize ? nullptr : x, ldx, xq, sx, rows, o, st, quantize || settled)
                              : launch_product(*l, xq, sx, rows, o, st);
    if (e == cudaSuccess && first) l->order.waited(st, cap != cudaStreamCaptureStatusNone);
    return to_status(e);
}

}  // namespace

}  // namespace wfq

using namespace wfq;

extern "C" {

wfq_status_t wfq_linear_create(wfq_linear_t **out, int C, int K, int group_size, int gated)
{
    if (!out) return WFQ_ERR_INVALID_ARG;
    *out = nullptr;
    if (C < 1 || K < 1 || group_size < 0 || (gated != 0 && gated != 1)) return WFQ_ERR_INVALID_ARG;
    if (group_size % 32 != 0 || C > kMaxRowChannels || K > (1 << 22)) return WFQ_ERR_UNSUPPORTED;
    wfq_linear *l = new (std::nothrow) wfq_linear();
    if (!l) return WFQ_ERR_ALLOC;
    l->C = C; l->K = K; l->gated = gated;
    l->Cp = row_pitch_codes(C);
    l->G = row_groups(C, group_size);
    l->gs = l->G == 1 ? l->Cp : group_size;
    l->Kz = gated ? 2 * K : K;
    l->Kp = (l->Kz + 255) / 256 * 256;
    *out = l;
    return WFQ_OK;
}

wfq_status_t wfq_linear_set_input_dtype(wfq_linear_t *l, wfq_dtype_t dtype)
{
    if (!l || !known(dtype)) return WFQ_ERR_INVALID_ARG;
    l->in_dtype = dtype;
    return WFQ_OK;
}

wfq_status_t wfq_linear_set_output_dtype(wfq_linear_t *l, wfq_dtype_t dtype)
{
    if (!l || !known(dtype)) return WFQ_ERR_INVALID_ARG;
    l->out_dtype = dtype;
    return WFQ_OK;
}

wfq_status_t wfq_linear_set_epilogue(wfq_linear_t *l, const float *bias_dev, wfq_activation_t act)
{
    if (!l || (act != WFQ_ACT_NONE && act != WFQ_ACT_RELU && act != WFQ_ACT_SILU && act != WFQ_ACT_GELU))
        return WFQ_ERR_INVALID_ARG;
    if (misaligned(bias_dev, 4)) return WFQ_ERR_INVALID_ARG;
    l->bias = bias_dev;
    l->act = (int)act;
    return WFQ_OK;
}

size_t wfq_linear_workspace_bytes(const wfq_linear_t *l, int rows)
{
    if (!l || rows < 1 || rows > 0x7fffff00) return 0;
    return up1024((size_t)rows * l->Cp) + up1024((size_t)l->G * ((rows + 127LL) / 128 * 128) * sizeof(float));
}

wfq_status_t wfq_linear_set_workspace(wfq_linear_t *l, void *dev_ptr, size_t bytes, int rows)
{
    if (!l || !dev_ptr || rows < 1 || rows > 0x7fffff00) return WFQ_ERR_INVALID_ARG;
    if (bytes < wfq_linear_workspace_bytes(l, rows) || misaligned(dev_ptr, 1024)) return WFQ_ERR_INVALID_ARG;
    const wfq_status_t s = bind(l);
    if (s != WFQ_OK) return s;
    l->xq = static_cast<int8_t *>(dev_ptr);
    l->sx = reinterpret_cast<float *>(static_cast<char *>(dev_ptr) + up1024((size_t)rows * l->Cp));
    l->max_rows = rows;
    return WFQ_OK;
}

wfq_status_t wfq_linear_prepare_weights(wfq_linear_t *l, const void *w_dev, long long ldw, wfq_dtype_t dtype, void *stream)
{
    if (!l || !w_dev || !known(dtype) || ldw < l->C || misaligned(w_dev, elem_bytes(dtype))) return WFQ_ERR_INVALID_ARG;
    const wfq_status_t s = bind(l);
    if (s != WFQ_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &cap) != cudaSuccess) return WFQ_ERR_CUDA;
    if (cap != cudaStreamCaptureStatusNone && !l->status) return WFQ_ERR_INVALID_ARG;       // cudaMalloc ends a capture
    cudaError_t e;
    if (!l->Wq && (e = cudaMalloc(&l->Wq, (size_t)l->Kz * l->Cp)) != cudaSuccess) return to_status(e);
    if (!l->sW) {
        const size_t n = (size_t)l->G * l->Kp * sizeof(float);
        float *p = nullptr;
        if ((e = cudaMalloc(&p, n)) != cudaSuccess) return to_status(e);
        if (cudaMemsetAsync(p, 0, n, st) != cudaSuccess) { cudaFree(p); return WFQ_ERR_CUDA; }
        l->sW = p;
    }
    if (!l->status) {
        int *p = nullptr;
        if ((e = cudaMalloc(&p, 4 * sizeof(int))) != cudaSuccess) return to_status(e);
        if (cudaMemsetAsync(p, 0, 4 * sizeof(int), st) != cudaSuccess) { cudaFree(p); return WFQ_ERR_CUDA; }
        l->status = p;
    }
    RowsArgs a;
    a.x = w_dev; a.ldx = ldw;
    a.codes = l->Wq; a.scales = l->sW;
    a.rows = l->Kz; a.C = l->C; a.Cp = l->Cp;
    a.gs = l->gs; a.G = l->G;
    a.scale_pitch = l->Kp;
    a.half = l->gated ? l->K : 0;
    l->order.written(st, cap != cudaStreamCaptureStatusNone);
    if (launch_rows(a, dtype, st, false) != cudaSuccess) { l->prepared = false; return WFQ_ERR_CUDA; }
    l->prepared = true;
    return WFQ_OK;
}

wfq_status_t wfq_linear_forward_codes(wfq_linear_t *l, const int8_t *codes_dev, const float *scales_dev, int rows,
                                      const void *residual_dev, long long ldr, void *y_dev, long long ldy, void *stream)
{
    if (!l || rows < 0) return WFQ_ERR_INVALID_ARG;
    if (!l->prepared) return WFQ_ERR_NOT_PREPARED;
    if (rows == 0) return WFQ_OK;
    wfq_status_t s = check_io(l, rows, codes_dev, residual_dev, ldr, y_dev, ldy);
    if (s != WFQ_OK) return s;
    if (!codes_dev || !scales_dev || misaligned(codes_dev, 32) || misaligned(scales_dev, 16)) return WFQ_ERR_INVALID_ARG;
    if ((s = bind(l)) != WFQ_OK) return s;
    return run(l, nullptr, 0, const_cast<int8_t *>(codes_dev), const_cast<float *>(scales_dev), rows, residual_dev, ldr,
               y_dev, ldy, reinterpret_cast<cudaStream_t>(stream));
}

wfq_status_t wfq_linear_forward(wfq_linear_t *l, const void *x_dev, long long ldx, int rows, const void *residual_dev,
                                long long ldr, void *y_dev, long long ldy, void *stream)
{
    if (!l || rows < 0) return WFQ_ERR_INVALID_ARG;
    if (!l->prepared || !l->xq) return WFQ_ERR_NOT_PREPARED;
    if (rows == 0) return WFQ_OK;
    wfq_status_t s = check_io(l, rows, x_dev, residual_dev, ldr, y_dev, ldy);
    if (s != WFQ_OK) return s;
    if (!x_dev || ldx < l->C || misaligned(x_dev, elem_bytes(l->in_dtype)) || rows > l->max_rows)
        return WFQ_ERR_INVALID_ARG;
    if ((s = bind(l)) != WFQ_OK) return s;
    return run(l, x_dev, ldx, l->xq, l->sx, rows, residual_dev, ldr, y_dev, ldy, reinterpret_cast<cudaStream_t>(stream));
}

wfq_status_t wfq_linear_set_debug_option(wfq_linear_t *l, wfq_debug_option_t option, long long value)
{
    if (!l) return WFQ_ERR_INVALID_ARG;
    switch (option) {
        case WFQ_DEBUG_WAIT_CYCLES:
            if (value < 1000) return WFQ_ERR_INVALID_ARG;
            l->wait_cycles = value;
            return WFQ_OK;
        case WFQ_DEBUG_SKIP_GEMM_STAGE:
            if (value < -1 || value > 0x7fffffff) return WFQ_ERR_INVALID_ARG;
            l->debug_skip_stage = (int)value;
            return WFQ_OK;
        case WFQ_DEBUG_GEMM_SHAPE: {
            const Shape sp{(int)(value / 1000 % 10), (int)(value % 1000), (int)(value / 10000)};
            const bool parts = sp.split == 1 || sp.split == 2 || sp.split == 4 || sp.split == 8;
            // every CTA of a tile needs at least 128 channels
            if (value != 0 && (value < 0 || value > 99999 || !parts || !known_shape(sp) || (l->Cp + 127) / 128 < sp.split))
                return WFQ_ERR_INVALID_ARG;
            l->debug_shape = (int)value;
            l->shape_rows = -1;
            return WFQ_OK;
        }
        default: return WFQ_ERR_INVALID_ARG;
    }
}

wfq_status_t wfq_linear_check_status(wfq_linear_t *l, void *stream, int *where)
{
    if (!l) return WFQ_ERR_INVALID_ARG;
    if (!l->status) return WFQ_ERR_NOT_PREPARED;
    int host[4] = {0, 0, 0, 0};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(host, l->status, sizeof(host), cudaMemcpyDeviceToHost, st) != cudaSuccess) return WFQ_ERR_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return WFQ_ERR_CUDA;
    if (where) *where = host[1];
    return host[0] == 0 ? WFQ_OK : WFQ_ERR_TIMEOUT;
}

wfq_status_t wfq_linear_debug_get(wfq_linear_t *l, wfq_buffer_t which, void **dev_ptr, size_t *bytes)
{
    if (!l || !dev_ptr || !bytes) return WFQ_ERR_INVALID_ARG;
    *dev_ptr = nullptr;
    *bytes = 0;
    switch (which) {
        case WFQ_BUF_WQ:
            if (!l->prepared) return WFQ_ERR_NOT_PREPARED;
            *dev_ptr = l->Wq; *bytes = (size_t)l->Kz * l->Cp; return WFQ_OK;
        case WFQ_BUF_SW:
            if (!l->prepared) return WFQ_ERR_NOT_PREPARED;
            *dev_ptr = l->sW; *bytes = (size_t)l->G * l->Kp * sizeof(float); return WFQ_OK;
        default: return WFQ_ERR_INVALID_ARG;
    }
}

wfq_status_t wfq_linear_destroy(wfq_linear_t *l)
{
    if (!l) return WFQ_OK;
    if (l->Wq) cudaFree(l->Wq);
    if (l->sW) cudaFree(l->sW);
    if (l->status) cudaFree(l->status);
    delete l;
    return WFQ_OK;
}

}  // extern "C"
