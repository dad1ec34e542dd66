// Declarations shared by the row operators (wfq_rows.cu) and the linear layer (wfq_linear.cu).
#pragma once

#include "wfq_internal.h"

namespace wfq {

constexpr int kMaxRowChannels = 131072;   // 127 * 127 * 131072 < 2^31: one group's products fit 32 bits

inline int row_pitch_codes(int C) { return (C + 31) / 32 * 32; }
inline int row_groups(int C, int gs) { return gs == 0 || gs >= C ? 1 : (C + gs - 1) / gs; }

// One launch of the row quantizer: rows of C values (optionally x + residual, optionally times a gain, see
// wfq_rms_norm_quantize) to codes [rows][Cp] and scales [G][scale_pitch].
struct RowsArgs {
    const void *x = nullptr, *residual = nullptr;
    const float *gain = nullptr;      // not null: the norm
    void *h = nullptr;                // x + residual in x's type, or null
    long long ldx = 0, ldr = 0, ldh = 0;
    int8_t *codes = nullptr;
    float *scales = nullptr;
    int rows = 0, C = 0, Cp = 0;
    int gs = 0, G = 0;                // gs: a multiple of 32; one group: gs >= C
    long long scale_pitch = 0;
    int half = 0;                     // > 0: input row r goes to row 2 (r % half) + r / half (gated weights)
    float eps = 0.f, per_C = 0.f;     // per_C: 1 / C
};
cudaError_t launch_rows(const RowsArgs &a, wfq_dtype_t dtype, cudaStream_t stream, bool pdl);

// Compute capability and SM count of the current device, looked up once per device.
wfq_status_t current_device(int *device, int *sm_count);

#ifdef __CUDACC__
// Scale amax / 127 and reciprocal 127 / amax of a group, both correctly rounded: a quotient from an approximate reciprocal
// is corrected by its remainder (Markstein's method), which gives the bits of __fdiv_rn for every float from 1e-30 to the
// largest in a fraction of the instructions.  A group that holds an infinity or a NaN has the scale NaN and codes 0, so that
// what is computed from it is NaN; inv is 0 where the codes are.
__device__ __forceinline__ void quantizer_scale(float amax, float &scale, float &inv)
{
    constexpr float r127 = 1.f / 127.f;
    float q = __fmul_rn(amax, r127);
    scale = fmaf(fmaf(-127.f, q, amax), r127, q);
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(amax));
    r = fmaf(r, fmaf(-amax, r, 1.f), r);
    q = __fmul_rn(127.f, r);
    inv = fmaf(fmaf(-amax, q, 127.f), r, q);
    if (!(amax >= 1e-30f)) scale = inv = 0.f;
    if (!(amax < __int_as_float(0x7f800000))) { scale = __int_as_float(0x7fc00000); inv = 0.f; }
}
__device__ __forceinline__ uint32_t code_bits(float u, float inv)
{
    // product and sum rounded separately, as the quantizer is defined; the low byte of the sum is the code
    return __float_as_uint(__fadd_rn(__fmul_rn(u, inv), 12582912.f));
}
#endif

}  // namespace wfq
