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

}  // namespace wfq
