// Entry points of the operators of a layer's projections in 8 bits: checks, then the launches.
#include <hip/hip_runtime.h>

#include "hr_block8.h"
#include "hr_block_mm.h"
#include "hr_kernels.h"

#define HR_OP_HIP(expr)                            \
    do {                                           \
        const hipError_t e__ = (expr);             \
        if (e__ != hipSuccess) {                   \
            hr::note_hip_error(e__, #expr);        \
            return HR_ERR_DEVICE;                  \
        }                                          \
    } while (0)

extern "C" {

int hr_rms_norm(const hr_norm_args* args, void* stream) {
    const int rc = hr::norm_check(args);
    if (rc != HR_OK || args->tokens == 0) return rc;
    HR_OP_HIP(hr::launch_rms_norm(*args, (hipStream_t)stream));
    return HR_OK;
}

int hr_block_quantize(int dtype, const void* x, int64_t x_stride, const hr_block8* out, void* stream) {
    const int rc = hr::quantize_check(dtype, x, x_stride, out);
    if (rc != HR_OK || out->rows == 0) return rc;
    HR_OP_HIP(hr::launch_block_quantize(dtype, x, x_stride, *out, (hipStream_t)stream));
    return HR_OK;
}

int hr_block_matmul(const hr_block8* a, const hr_block8* w, const hr_matmul_args* args, void* stream) {
    const int rc = hr::matmul_check(a, w, args);
    if (rc != HR_OK || a->rows == 0 || w->rows == 0) return rc;
    hr::MatmulArgs m = hr::matmul_args(*a, *w, *args);
    const hr::MatmulPlan plan = hr::matmul_plan(m);
    auto launch = [&](const hr::MatmulArgs& part, int shape) {
        if (shape <= hr::MM_FEW_32) return hr::launch_block_matmul_few(part, args->dtype, shape, (hipStream_t)stream);
        if (part.codes) return (part.eight ? hr::launch_block_matmul_codes_fast : hr::launch_block_matmul_codes)(part, shape, (hipStream_t)stream);
        if (args->dtype == HR_BF16) return (part.eight ? hr::launch_block_matmul_bf16_fast : hr::launch_block_matmul_bf16)(part, shape, (hipStream_t)stream);
        return (part.eight ? hr::launch_block_matmul_f32_fast : hr::launch_block_matmul_f32)(part, shape, (hipStream_t)stream);
    };
    if (plan.rows < m.M) {
        HR_OP_HIP(launch(hr::matmul_rows(m, args->dtype, 0, plan.rows), plan.shape));
        HR_OP_HIP(launch(hr::matmul_rows(m, args->dtype, plan.rows, m.M - plan.rows), plan.rest));
    } else {
        HR_OP_HIP(launch(m, plan.shape));
    }
    return HR_OK;
}

}  // extern "C"
