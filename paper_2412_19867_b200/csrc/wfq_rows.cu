// Rows of values to int8 codes with one fp32 scale per group of consecutive channels (the quantizer of wfq.h), with the
// root-mean-square norm and the residual's addition in front of it where asked, and back.
//
//   h = round(x + residual),  u = fl32(h * gain),  rstd = 1 / sqrt(mean(h^2) + eps)
//   scale[g] = fl32(max_g |u| / 127) * rstd,       code = rint(fl32(u * fl32(127 / max_g |u|)))
//
// The row's factor rstd is the same for a whole group and cancels in its codes, so these do not wait for the sum of
// squares and do not depend on its rounding: for 16-bit h and any gain u is one rounding of an exact product, and every
// implementation of the definition gives the same codes.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "wfq_ptx.cuh"
#include "wfq_rows.h"

namespace wfq {

namespace {

template <typename T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};

// N (8 or 4) consecutive elements, aligned to their size up to 16 bytes.
template <int N, typename T> __device__ __forceinline__ void store_wide(T *p, const float (&v)[N])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
        typename std::conditional<N == 8, uint4, uint2>::type a;
        T *e = reinterpret_cast<T *>(&a);
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = Elem<T>::put(v[i]);
        *reinterpret_cast<decltype(a) *>(p) = a;
    }
}

// The larger magnitude; NaN where one of the two is.
__device__ __forceinline__ float larger(float m, float u)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(u)));
    return r;
}
// Magnitudes as integers are ordered as the numbers are, with infinity and NaN above them.
__device__ __forceinline__ int magnitude_bits(float u) { return __float_as_int(u) & 0x7fffffff; }

__device__ __forceinline__ int target_row(const RowsArgs &a, int row)
{
    return a.half > 0 ? 2 * (row % a.half) + row / a.half : row;
}
__device__ __forceinline__ float rstd_of(float sum, const RowsArgs &a)
{
    return rsqrtf(fmaf(sum, a.per_C, a.eps));      // two units in the last place, and the rounding of 1 / C
}

// Rows of more channels than 1024 threads take.  One CTA per row, two passes over it; the second
// reads the first one's h where it was stored (h may be x or residual itself).
template <typename T, bool NORM>
__global__ void __launch_bounds__(256) rows_any_kernel(RowsArgs a)
{
    extern __shared__ int group_max[];        // [G]
    __shared__ float warp_sum[8];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ldr : nullptr;
        T *h = a.h ? static_cast<T *>(a.h) + row * a.ldh : nullptr;
        for (int g = threadIdx.x; g < a.G; g += 256) group_max[g] = 0;
        __syncthreads();
        auto value = [&](int c, bool again) {
            if (again && h) return Elem<T>::get(h[c]);
            const float v = Elem<T>::get(x[c]);
            return r ? Elem<T>::get(Elem<T>::put(__fadd_rn(v, Elem<T>::get(r[c])))) : v;
        };
        float sum = 0.f;
        for (int c0 = warp * 32; c0 < a.C; c0 += 256) {
            const int c = c0 + lane;
            float u = 0.f;
            if (c < a.C) {
                u = value(c, false);
                if (NORM) {
                    sum = fmaf(u, u, sum);
                    if (h) h[c] = Elem<T>::put(u);
                    u = __fmul_rn(u, a.gain[c]);
                }
            }
            const int m = __reduce_max_sync(0xffffffffu, magnitude_bits(u));
            if (lane == 0) atomicMax(&group_max[c0 / a.gs], m);
        }
        if (NORM) {
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) warp_sum[warp] = sum;
        }
        __syncthreads();
        float rstd = 1.f;
        if (NORM) {
            float s = 0.f;
            for (int w = 0; w < 8; ++w) s += warp_sum[w];
            rstd = rstd_of(s, a);
        }
        const int to = target_row(a, row);
        for (int g = threadIdx.x; g < a.G; g += 256) {
            float scale, inv;
            quantizer_scale(__int_as_float(group_max[g]), scale, inv);
            a.scales[(size_t)g * a.scale_pitch + to] = NORM ? __fmul_rn(scale, rstd) : scale;
        }
        for (int c0 = warp * 32; c0 < a.Cp; c0 += 256) {
            const int c = c0 + lane;
            float scale, inv;
            quantizer_scale(__int_as_float(group_max[c0 / a.gs]), scale, inv);
            uint32_t code = 0;
            if (c < a.C && inv > 0.f) {
                float u = value(c, true);
                if (NORM) u = __fmul_rn(u, a.gain[c]);
                code = code_bits(u, inv);
            }
            a.codes[(size_t)to * a.Cp + c] = (int8_t)code;
        }
        __syncthreads();
    }
}

// a += b for N elements, each sum rounded once.  A 16-bit sum rounded from 32 bits is the same: where 32 bits do not
// hold it exactly the smaller term is less than a quarter of a step of the larger.
template <int N> __device__ __forceinline__ void add_words(float *a, const float *b)
{
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = __fadd_rn(a[i], b[i]);
}
template <int N> __device__ __forceinline__ void add_words(__half *a, const __half *b)
{
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
        reinterpret_cast<__half2 *>(a)[i] = __hadd2(reinterpret_cast<__half2 *>(a)[i], reinterpret_cast<const __half2 *>(b)[i]);
}
template <int N> __device__ __forceinline__ void add_words(__nv_bfloat16 *a, const __nv_bfloat16 *b)
{
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
        reinterpret_cast<__nv_bfloat162 *>(a)[i] =
            __hadd2(reinterpret_cast<__nv_bfloat162 *>(a)[i], reinterpret_cast<const __nv_bfloat162 *>(b)[i]);
}

// VEC (8 or 4) consecutive elements as they lie in memory, aligned to their size up to 16 bytes.
template <typename T, int VEC> struct Raw {
    using Word = typename std::conditional<sizeof(T) * VEC == 8, uint2, uint4>::type;
    static constexpr int N = (int)(sizeof(T) * VEC / sizeof(Word));
    Word q[N];
    __device__ __forceinline__ void load(const T *p)
    {
        const Word *src = reinterpret_cast<const Word *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = src[i];
    }
    __device__ __forceinline__ void put(T *p) const
    {
        Word *dst = reinterpret_cast<Word *>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) dst[i] = q[i];
    }
    __device__ __forceinline__ float get(int e) const { return Elem<T>::get(reinterpret_cast<const T *>(q)[e]); }
    __device__ __forceinline__ void add(const Raw &o)
    {
        add_words<VEC>(reinterpret_cast<T *>(q), reinterpret_cast<const T *>(o.q));
    }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void put(T *p) const { *p = v; }
    __device__ __forceinline__ float get(int) const { return Elem<T>::get(v); }
    __device__ __forceinline__ void add(const Raw &o)
    {
        if constexpr (sizeof(T) == 4) v = __fadd_rn(v, o.v);
        else v = __hadd(v, o.v);
    }
};
template <int VEC, typename T> __device__ __forceinline__ void store(T *p, const float (&v)[VEC])
{
    if constexpr (VEC > 1) store_wide<VEC>(p, v);
    else *p = Elem<T>::put(v[0]);
}

// Rows of up to 32768 channels: one pass.  They are held in registers up to 4096 channels (8192 in fp32 and in calls of few
// rows) but for a few words that single elements spill; beyond, 1024 threads have 64 registers each and spill 0 to 284 bytes
// a thread up to 16384 channels and 116 (quantized) to 972 (fp32 norm with a residual) up to 32768, where two passes by
// rows_any_kernel take longer all the same: 2000 x 32768 fp32 with a residual 431 against 597 us, bf16 218 against 606,
// quantized alone 45 against 410.  `tpr` threads (whole warps) have a row, thread t the
// vectors t, t + tpr, ... of VEC elements; a CTA has several short rows.  A group of gs = VEC * lanes channels (lanes a
// power of two up to 32) lies in neighbouring lanes; other groups are joined in shared memory (`direct` 0).
// Bound by memory and by issue slots (a dozen instructions per value) alike: CTAs walk over the rows and ask for the next
// one's values before they work on this one's, so that loads are on their way throughout; the gain stays in registers.
// 16384 x 4096 bf16 with a residual 86 us, 5.5 TB/s (with 80 registers, three CTAs of 256 threads per SM, 100 us; without a
// residual three are better, 16384 x 1280 23 against 34 us); 8192 x 4096 bf16 quantized alone 24 us, 4.2 TB/s.
template <typename T, bool NORM, bool RES, int VEC, int NV, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 && NV * VEC <= 16 ? (RES && VEC > 1 ? 2 : 3) : 1)
rows_kernel(RowsArgs a, int tpr, int lanes, int direct)
{
    extern __shared__ int group_max[];        // [2][rows of the CTA][G] where groups are joined, alternately
    __shared__ float warp_sum[2][32];
    const int local = (int)threadIdx.x / tpr, t = (int)threadIdx.x - local * tpr, per_cta = (int)blockDim.x / tpr;
    const int lane = threadIdx.x & 31;
    const int n = a.C / VEC;                  // vectors of a row
    const long long step = (long long)gridDim.x * per_cta;
    const long long rounds = (a.rows + step - 1) / step;      // the same for all threads: they meet at barriers
    if (!direct) {
        for (int i = threadIdx.x; i < 2 * per_cta * a.G; i += blockDim.x) group_max[i] = 0;
        __syncthreads();
    }
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    Raw<T, VEC> x[NV], r[RES ? NV : 1];
    float gain[NORM ? NV : 1][VEC];
    auto ask = [&](long long row) {
        if (row >= a.rows) return;
        const T *px = static_cast<const T *>(a.x) + row * a.ldx;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * tpr + t < n) x[i].load(px + (i * tpr + t) * VEC);
        if constexpr (RES) {
            const T *pr = static_cast<const T *>(a.residual) + row * a.ldr;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * tpr + t < n) r[i].load(pr + (i * tpr + t) * VEC);
        }
    };
    long long row = (long long)blockIdx.x * per_cta + local;
    ask(row);
    // what a thread's vectors are to every row: their group, and whether they begin it
    int group[NV];
    float *to_scale[VEC == 1 ? 1 : NV];
    if constexpr (VEC == 1) {                 // of step `lane`
        const int c = lane * tpr + (t & ~31);
        to_scale[0] = lane < NV && c < a.C && c % a.gs == 0 ? a.scales + (size_t)(c / a.gs) * a.scale_pitch : nullptr;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * tpr + t) * VEC;
        group[i] = c / a.gs;
        if constexpr (VEC > 1) to_scale[i] = c < a.C && c == group[i] * a.gs ? a.scales + (size_t)group[i] * a.scale_pitch : nullptr;
        if constexpr (NORM) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) gain[i][e] = c < a.C ? __ldg(a.gain + c + e) : 0.f;
        }
    }
    for (long long k = 0; k < rounds; ++k, row += step) {
        const bool live = row < a.rows;
        const int odd = (int)(k & 1);
        int *gmax = group_max + (odd * per_cta + local) * a.G;
        float u[NV][VEC];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool has = live && i * tpr + t < n;
#pragma unroll
            for (int e = 0; e < VEC; ++e) u[i][e] = 0.f;
            if (has) {
                if constexpr (RES) {
                    x[i].add(r[i]);
                    if (a.h) x[i].put(static_cast<T *>(a.h) + row * a.ldh + (i * tpr + t) * VEC);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) u[i][e] = x[i].get(e);
            }
        }
        ask(row + step);
        int amax[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (NORM) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum = fmaf(u[i][e], u[i][e], sum);
#pragma unroll
                for (int e = 0; e < VEC; ++e) u[i][e] = __fmul_rn(u[i][e], gain[i][e]);
            }
            float m = fabsf(u[i][0]);
#pragma unroll
            for (int e = 1; e < VEC; ++e) m = larger(m, u[i][e]);
            amax[i] = magnitude_bits(m);
        }
        if constexpr (VEC == 1) {          // groups are multiples of 32: a warp's elements of a step are in one
#pragma unroll
            for (int i = 0; i < NV; ++i) amax[i] = __reduce_max_sync(0xffffffffu, amax[i]);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
            if (VEC > 1 && o < lanes) {
#pragma unroll
                for (int i = 0; i < NV; ++i) amax[i] = max(amax[i], __shfl_xor_sync(0xffffffffu, amax[i], o));
            }
        if (!direct && (lane & (lanes - 1)) == 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * tpr + t < n) atomicMax(&gmax[group[i]], amax[i]);
        }
        if constexpr (NORM) {
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (tpr > 32 && lane == 0) warp_sum[odd][threadIdx.x >> 5] = sum;
        }
        if (!direct) {
            __syncthreads();
            // the other half is free: everybody is past last round's reads of it
            int *other = group_max + ((odd ^ 1) * per_cta + local) * a.G;
            for (int g = t; g < a.G; g += tpr) other[g] = 0;
        }
        const int to = live ? target_row(a, (int)row) : 0;
        int8_t *codes = a.codes + (size_t)to * a.Cp;
        float scale[VEC == 1 ? 1 : NV];
        if constexpr (VEC == 1) {
            // one group per step and warp: lane i works out step i's scale for all
            int m = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!direct && i * tpr + (t & ~31) < n) amax[i] = gmax[group[i]];      // the warp's, also of lanes behind the row
                if (lane == i) m = amax[i];
            }
            float inv;
            quantizer_scale(__int_as_float(m), scale[0], inv);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float iv = __shfl_sync(0xffffffffu, inv, i);
                const int v = i * tpr + t;
                if (live && v < a.Cp) codes[v] = iv > 0.f ? (int8_t)code_bits(u[i][0], iv) : (int8_t)0;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int v = i * tpr + t;
                float inv;
                quantizer_scale(__int_as_float(direct || v >= n ? amax[i] : gmax[group[i]]), scale[i], inv);
                if (live && v < a.Cp / VEC) {
                    uint32_t w[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) w[e] = code_bits(u[i][e], inv);
                    uint32_t lo = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
                    if (!(inv > 0.f)) lo = 0;
                    if constexpr (VEC == 8) {
                        uint32_t hi = __byte_perm(__byte_perm(w[4], w[5], 0x0040), __byte_perm(w[6], w[7], 0x0040), 0x5410);
                        if (!(inv > 0.f)) hi = 0;
                        *reinterpret_cast<uint2 *>(codes + v * 8) = make_uint2(lo, hi);
                    } else {
                        *reinterpret_cast<uint32_t *>(codes + v * 4) = lo;
                    }
                }
            }
        }
        float rstd = 1.f;             // the scales alone wait for the row's sum
        if constexpr (NORM) {
            if (tpr > 32) {
                if (direct) __syncthreads();
                const float *part = warp_sum[odd] + local * (tpr >> 5);
                sum = 0.f;
#pragma unroll 4
                for (int w = 0; w < tpr >> 5; ++w) sum += part[w];
            }
            rstd = rstd_of(sum, a);
        }
        if (live) {
#pragma unroll
            for (int i = 0; i < (VEC == 1 ? 1 : NV); ++i)
                if (to_scale[i]) to_scale[i][to] = NORM ? __fmul_rn(scale[i], rstd) : scale[i];
        }
        if (!direct) __syncthreads();     // the zeros are in place before the next round's maxima
    }
}

// Codes back to values, VEC of them at a time, four such pieces of a row on their way per thread.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) dequantize_kernel(const int8_t *__restrict__ codes, const float *__restrict__ scales,
                                                         int rows, int C, int Cp, FastDiv by_gs, long long scale_pitch,
                                                         T *__restrict__ v, long long ldv, int tpr)
{
    constexpr int N = 4;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int local = (int)threadIdx.x / tpr, per_cta = 256 / tpr, t = (int)threadIdx.x - local * tpr;
    if (local >= per_cta) return;
    for (long long row = (long long)blockIdx.x * per_cta + local; row < rows; row += (long long)gridDim.x * per_cta)
        for (int c0 = t * VEC; c0 < C; c0 += N * tpr * VEC) {
            uint2 q[N];
            float s[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = c0 + i * tpr * VEC;
                if (c < C) {
                    if constexpr (VEC == 8) q[i] = __ldg(reinterpret_cast<const uint2 *>(codes + row * Cp + c));
                    else if constexpr (VEC == 4) q[i].x = __ldg(reinterpret_cast<const uint32_t *>(codes + row * Cp + c));
                    else q[i].x = (uint32_t)(uint8_t)__ldg(codes + row * Cp + c);
                    s[i] = __ldg(scales + (size_t)(c / by_gs) * scale_pitch + row);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = c0 + i * tpr * VEC;
                if (c < C) {
                    float out[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) out[e] = (float)(int8_t)((e < 4 ? q[i].x : q[i].y) >> (8 * (e & 3))) * s[i];
                    store<VEC>(v + row * ldv + c, out);
                }
            }
        }
}

template <typename K, typename... A>
cudaError_t launch(K kernel, dim3 grid, int threads, size_t smem, cudaStream_t stream, bool pdl, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// CTAs that fit an SM, from the registers a thread.
int resident_ctas(int regs, int threads, size_t smem)
{
    const int per_warp = (regs * 32 + 255) / 256 * 256;
    int n = 65536 / (per_warp * (threads / 32));
    const int by_smem = (int)(200 * 1024 / (smem + 1280));
    if (by_smem < n) n = by_smem;
    if (2048 / threads < n) n = 2048 / threads;
    return n < 1 ? 1 : n;
}

template <typename T, bool NORM, bool RES, int VEC, int NV, int THREADS>
cudaError_t launch_rows_kernel(const RowsArgs &a, int tpr, cudaStream_t stream, bool pdl)
{
    // lanes of the largest power of two of channels that no group's border cuts
    int lanes = 1, sms = 0;
    while (lanes < 32 && a.gs % (2 * lanes * VEC) == 0) lanes *= 2;
    const int direct = a.gs == lanes * VEC;
    if (current_device(nullptr, &sms) != WFQ_OK) return cudaErrorInvalidDevice;
    // short rows share a CTA of four warps where there are enough of them to go round
    int per_cta = tpr >= 128 || a.rows < 8 * sms ? 1 : 128 / tpr;
    const size_t row_smem = direct ? 0 : 2 * (size_t)a.G * sizeof(int);
    while (per_cta > 1 && per_cta * row_smem > 40 * 1024) --per_cta;
    const int ctas = (int)((a.rows + (long long)per_cta - 1) / per_cta), threads = tpr * per_cta;
    auto kernel = rows_kernel<T, NORM, RES, VEC, NV, THREADS>;
    static std::atomic<int> regs{0};       // of this kernel, looked up once
    int r = regs.load(std::memory_order_relaxed);
    if (r == 0) {
        cudaFuncAttributes fa;
        const cudaError_t err = cudaFuncGetAttributes(&fa, kernel);
        if (err != cudaSuccess) return err;
        r = fa.numRegs;
        regs.store(r, std::memory_order_relaxed);
    }
    const int resident = resident_ctas(r, threads, per_cta * row_smem) * sms;      // as many as run at once
    return launch(kernel, dim3((unsigned)(ctas < resident ? ctas : resident)), threads,
                  per_cta * row_smem, stream, pdl, a, tpr, lanes, direct);
}

template <typename T, int VEC, int NV, int THREADS>
cudaError_t launch_rows_mode(const RowsArgs &a, int tpr, cudaStream_t stream, bool pdl)
{
    if (!a.gain) return launch_rows_kernel<T, false, false, VEC, NV, THREADS>(a, tpr, stream, pdl);
    if (!a.residual) return launch_rows_kernel<T, true, false, VEC, NV, THREADS>(a, tpr, stream, pdl);
    return launch_rows_kernel<T, true, true, VEC, NV, THREADS>(a, tpr, stream, pdl);
}
template <typename T, int VEC, int NV>
cudaError_t launch_rows_size(const RowsArgs &a, int tpr, cudaStream_t stream, bool pdl)
{
    // what launch_rows_t gives rows of so few threads
    constexpr bool narrow = VEC * NV == 8 || (VEC * NV == 16 && sizeof(T) == 2);
    if constexpr (narrow) {
        if (tpr <= 256) return launch_rows_mode<T, VEC, NV, 256>(a, tpr, stream, pdl);
    }
    return launch_rows_mode<T, VEC, NV, 1024>(a, tpr, stream, pdl);
}

bool aligned(const void *p, long long ld, size_t elem, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (size_t)ld * elem % bytes == 0;
}

template <typename T>
cudaError_t launch_rows_t(const RowsArgs &a, cudaStream_t stream, bool pdl)
{
    const size_t e = sizeof(T);
    auto pieces = [&](int n) {       // do all rows consist of pieces of n elements, aligned to their size up to 16 bytes?
        const size_t bytes = n * e < 16 ? n * e : 16;
        return a.C % n == 0 && aligned(a.x, a.ldx, e, bytes) && (!a.residual || aligned(a.residual, a.ldr, e, bytes)) &&
               (!a.h || aligned(a.h, a.ldh, e, bytes));
    };
    // pieces of four: 9424 x 1500 fp16 norm with residual 25.6 us, element by element 57; 2000 x 4100 fp32 36 against 95
    const int vec = pieces(8) ? 8 : pieces(4) ? 4 : 1;
    // Elements per thread: 8 where there are few rows (latency) or the elements are single or 32-bit loads, else 16; 32 for
    // rows that would not fit a CTA otherwise.
    const int want = vec == 1 || e == 4 || a.rows < 592 ? 8 : 16;
    for (int per : {8, 16, 32}) {
        const int tpr = ((a.Cp + per - 1) / per + 31) / 32 * 32;
        if (tpr > 1024 || per < want || a.G > 2048) continue;
        if (vec == 8)
            return per == 8 ? launch_rows_size<T, 8, 1>(a, tpr, stream, pdl)
                            : per == 16 ? launch_rows_size<T, 8, 2>(a, tpr, stream, pdl)
                                        : launch_rows_size<T, 8, 4>(a, tpr, stream, pdl);
        if (vec == 4 && per <= 16)
            return per == 8 ? launch_rows_size<T, 4, 2>(a, tpr, stream, pdl) : launch_rows_size<T, 4, 4>(a, tpr, stream, pdl);
        if (vec == 1 && per == 8) return launch_rows_size<T, 1, 8>(a, tpr, stream, pdl);
    }
    const int grid = a.rows < (1 << 20) ? a.rows : 1 << 20;
    const size_t smem = (size_t)a.G * sizeof(int);
    return a.gain ? launch(rows_any_kernel<T, true>, dim3((unsigned)grid), 256, smem, stream, pdl, a)
                  : launch(rows_any_kernel<T, false>, dim3((unsigned)grid), 256, smem, stream, pdl, a);
}

template <typename T>
cudaError_t launch_dequantize(const int8_t *codes, const float *scales, int rows, int C, int gs, void *v, long long ldv,
                              cudaStream_t stream)
{
    constexpr size_t e = sizeof(T);
    const int vec = C % 8 == 0 && aligned(v, ldv, e, 16) ? 8 : C % 4 == 0 && aligned(v, ldv, e, 4 * e) ? 4 : 1;
    const int n = C / vec, tpr = n >= 256 ? 256 : (n + 31) / 32 * 32, per_cta = 256 / tpr;
    const long long ctas = (rows + (long long)per_cta - 1) / per_cta, pitch = (rows + 127LL) / 128 * 128;
    const dim3 grid((unsigned)(ctas < (1 << 20) ? ctas : 1 << 20));
    auto kernel = vec == 8 ? dequantize_kernel<T, 8> : vec == 4 ? dequantize_kernel<T, 4> : dequantize_kernel<T, 1>;
    return launch(kernel, grid, 256, 0, stream, true, codes, scales, rows, C, row_pitch_codes(C), FastDiv(gs), pitch,
                  static_cast<T *>(v), ldv, tpr);
}

bool known(wfq_dtype_t t) { return t == WFQ_F32 || t == WFQ_F16 || t == WFQ_BF16; }
size_t elem_bytes(wfq_dtype_t t) { return t == WFQ_F32 ? 4 : 2; }
bool misaligned(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

wfq_status_t check_rows(int rows, int C, int group_size)
{
    if (rows < 0 || C < 1 || group_size < 0) return WFQ_ERR_INVALID_ARG;
    if (group_size % 32 != 0 || C > kMaxRowChannels || rows > 0x7fffff00) return WFQ_ERR_UNSUPPORTED;
    return WFQ_OK;
}

wfq_status_t to_status(cudaError_t e) { return e == cudaSuccess ? WFQ_OK : WFQ_ERR_CUDA; }

}  // namespace

cudaError_t launch_rows(const RowsArgs &a, wfq_dtype_t dtype, cudaStream_t stream, bool pdl)
{
    if (dtype == WFQ_F32) return launch_rows_t<float>(a, stream, pdl);
    if (dtype == WFQ_F16) return launch_rows_t<__half>(a, stream, pdl);
    return launch_rows_t<__nv_bfloat16>(a, stream, pdl);
}

wfq_status_t current_device(int *device, int *sm_count)
{
    constexpr int kMax = 64;
    static std::atomic<int> sms[kMax];       // 0: not looked up yet
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return WFQ_ERR_CUDA;
    if (dev < 0 || dev >= kMax) return WFQ_ERR_UNSUPPORTED;
    int n = sms[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        int major = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
            return WFQ_ERR_CUDA;
        if (major != 10) return WFQ_ERR_UNSUPPORTED;
        sms[dev].store(n, std::memory_order_relaxed);
    }
    if (device) *device = dev;
    if (sm_count) *sm_count = n;
    return WFQ_OK;
}

}  // namespace wfq

using namespace wfq;

extern "C" {

wfq_status_t wfq_rms_norm_quantize(const void *x_dev, long long ldx, const void *residual_dev, long long ldr,
                                   const float *gain_dev, float eps, wfq_dtype_t dtype, int rows, int C, int group_size,
                                   void *h_dev, long long ldh, int8_t *codes_dev, float *scales_dev, void *stream)
{
    wfq_status_t s = check_rows(rows, C, group_size);
    if (s != WFQ_OK) return s;
    if (!known(dtype) || !(eps >= 0.f) || eps > 3e38f) return WFQ_ERR_INVALID_ARG;
    if (rows == 0) return WFQ_OK;
    const size_t e = elem_bytes(dtype);
    if (!x_dev || !gain_dev || !codes_dev || !scales_dev || (h_dev && !residual_dev)) return WFQ_ERR_INVALID_ARG;
    if (ldx < C || (residual_dev && ldr < C) || (h_dev && ldh < C)) return WFQ_ERR_INVALID_ARG;
    // in place only row onto row: a row that lands elsewhere may be another one's input
    if (h_dev && rows > 1 && ((h_dev == x_dev && ldh != ldx) || (h_dev == residual_dev && ldh != ldr))) return WFQ_ERR_INVALID_ARG;
    if (misaligned(x_dev, e) || misaligned(residual_dev, e) || misaligned(h_dev, e) || misaligned(gain_dev, 4) ||
        misaligned(codes_dev, 32) || misaligned(scales_dev, 16))
        return WFQ_ERR_INVALID_ARG;
    if ((s = current_device(nullptr, nullptr)) != WFQ_OK) return s;
    RowsArgs a;
    a.x = x_dev; a.residual = residual_dev; a.gain = gain_dev; a.h = h_dev;
    a.ldx = ldx; a.ldr = ldr; a.ldh = ldh;
    a.codes = codes_dev; a.scales = scales_dev;
    a.rows = rows; a.C = C; a.Cp = row_pitch_codes(C);
    a.G = row_groups(C, group_size);
    a.gs = a.G == 1 ? a.Cp : group_size;
    a.scale_pitch = (rows + 127LL) / 128 * 128;
    a.eps = eps;
    a.per_C = 1.f / (float)C;
    return to_status(launch_rows(a, dtype, reinterpret_cast<cudaStream_t>(stream), true));
}

wfq_status_t wfq_quantize_rows(const void *x_dev, long long ldx, wfq_dtype_t dtype, int rows, int C, int group_size,
                               int8_t *codes_dev, float *scales_dev, void *stream)
{
    wfq_status_t s = check_rows(rows, C, group_size);
    if (s != WFQ_OK) return s;
    if (!known(dtype)) return WFQ_ERR_INVALID_ARG;
    if (rows == 0) return WFQ_OK;
    if (!x_dev || !codes_dev || !scales_dev || ldx < C) return WFQ_ERR_INVALID_ARG;
    if (misaligned(x_dev, elem_bytes(dtype)) || misaligned(codes_dev, 32) || misaligned(scales_dev, 16))
        return WFQ_ERR_INVALID_ARG;
    if ((s = current_device(nullptr, nullptr)) != WFQ_OK) return s;
    RowsArgs a;
    a.x = x_dev; a.ldx = ldx;
    a.codes = codes_dev; a.scales = scales_dev;
    a.rows = rows; a.C = C; a.Cp = row_pitch_codes(C);
    a.G = row_groups(C, group_size);
    a.gs = a.G == 1 ? a.Cp : group_size;
    a.scale_pitch = (rows + 127LL) / 128 * 128;
    return to_status(launch_rows(a, dtype, reinterpret_cast<cudaStream_t>(stream), true));
}

wfq_status_t wfq_dequantize_rows(const int8_t *codes_dev, const float *scales_dev, int rows, int C, int group_size,
                                 wfq_dtype_t dtype, void *v_dev, long long ldv, void *stream)
{
    wfq_status_t s = check_rows(rows, C, group_size);
    if (s != WFQ_OK) return s;
    if (!known(dtype)) return WFQ_ERR_INVALID_ARG;
    if (rows == 0) return WFQ_OK;
    if (!codes_dev || !scales_dev || !v_dev || ldv < C) return WFQ_ERR_INVALID_ARG;
    if (misaligned(v_dev, elem_bytes(dtype)) || misaligned(codes_dev, 32) || misaligned(scales_dev, 16))
        return WFQ_ERR_INVALID_ARG;
    if ((s = current_device(nullptr, nullptr)) != WFQ_OK) return s;
    const int gs = row_groups(C, group_size) == 1 ? row_pitch_codes(C) : group_size;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == WFQ_F32) return to_status(launch_dequantize<float>(codes_dev, scales_dev, rows, C, gs, v_dev, ldv, st));
    if (dtype == WFQ_F16) return to_status(launch_dequantize<__half>(codes_dev, scales_dev, rows, C, gs, v_dev, ldv, st));
    return to_status(launch_dequantize<__nv_bfloat16>(codes_dev, scales_dev, rows, C, gs, v_dev, ldv, st));
}

}  // extern "C"
