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

#include "wfq_ptx.cuh"
#include "wfq_rows.h"

namespace wfq {

namespace {

constexpr int kNonFinite = 0x7f800000;    // bit patterns of |v| from here on are infinities and NaN

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

// Eight consecutive elements, 16-byte aligned.
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const T *e = reinterpret_cast<const T *>(&a);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = Elem<T>::get(e[i]);
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint4 a;
        T *e = reinterpret_cast<T *>(&a);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = Elem<T>::put(v[i]);
        *reinterpret_cast<uint4 *>(p) = a;
    }
}

// Scale and reciprocal of a group from the bit pattern of its largest magnitude.  A group that holds an infinity or a
// NaN has the scale NaN and codes 0, so that what is computed from it is NaN.
__device__ __forceinline__ void scale_of(int amax_bits, float &scale, float &inv)
{
    const float amax = __int_as_float(amax_bits);
    const bool some = amax_bits < kNonFinite && amax >= 1e-30f;
    scale = some ? __fdiv_rn(amax, 127.f) : amax_bits >= kNonFinite ? __int_as_float(0x7fc00000) : 0.f;
    inv = some ? __fdiv_rn(127.f, amax) : 0.f;
}
__device__ __forceinline__ uint32_t code_bits(float u, float inv)
{
    // product and sum rounded separately, as the quantizer is defined; the low byte of the sum is the code
    return __float_as_uint(__fadd_rn(__fmul_rn(u, inv), 12582912.f));
}
__device__ __forceinline__ int magnitude_bits(float u) { return __float_as_int(u) & 0x7fffffff; }

__device__ __forceinline__ int target_row(const RowsArgs &a, int row)
{
    return a.half > 0 ? 2 * (row % a.half) + row / a.half : row;
}
__device__ __forceinline__ float rstd_of(float sum, const RowsArgs &a)
{
    return __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)a.C), a.eps)));
}

// Any row: widths and strides without alignment, any group size.  One CTA per row, two passes over it; the second
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
            scale_of(group_max[g], scale, inv);
            a.scales[(size_t)g * a.scale_pitch + to] = NORM ? __fmul_rn(scale, rstd) : scale;
        }
        for (int c0 = warp * 32; c0 < a.Cp; c0 += 256) {
            const int c = c0 + lane;
            float scale, inv;
            scale_of(group_max[c0 / a.gs], scale, inv);
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

template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const int8_t *codes, const float *scales, int rows, int C, int Cp,
                                                         int gs, long long scale_pitch, T *v, long long ldv)
{
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    for (long long row = blockIdx.y; row < rows; row += gridDim.y)
        for (int c = blockIdx.x * 256 + threadIdx.x; c < C; c += gridDim.x * 256) {
            const float s = scales[(size_t)(c / gs) * scale_pitch + row];
            v[row * ldv + c] = Elem<T>::put((float)codes[row * Cp + c] * s);
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

template <typename T>
cudaError_t launch_rows_t(const RowsArgs &a, cudaStream_t stream, bool pdl)
{
    const int grid = a.rows < (1 << 20) ? a.rows : 1 << 20;
    const size_t smem = (size_t)a.G * sizeof(int);
    return a.gain ? launch(rows_any_kernel<T, true>, dim3((unsigned)grid), 256, smem, stream, pdl, a)
                  : launch(rows_any_kernel<T, false>, dim3((unsigned)grid), 256, smem, stream, pdl, a);
}

template <typename T>
cudaError_t launch_dequantize(const int8_t *codes, const float *scales, int rows, int C, int gs, void *v, long long ldv,
                              cudaStream_t stream)
{
    const unsigned gx = (unsigned)((C + 255) / 256), gy = (unsigned)(rows < 65535 ? rows : 65535);
    const long long pitch = (rows + 127LL) / 128 * 128;
    return launch(dequantize_kernel<T>, dim3(gx, gy), 256, 0, stream, true, codes, scales, rows, C, row_pitch_codes(C), gs,
                  pitch, static_cast<T *>(v), ldv);
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
