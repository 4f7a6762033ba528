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
    const hr::MatmulArgs m = hr::matmul_args(*a, *w, *args);
    const hr::MatmulTile t = hr::matmul_tile(m.M, m.N, m.K, args->dtype, m.gate, m.codes != nullptr);
    HR_OP_HIP((t.few ? hr::launch_block_matmul_few : hr::launch_block_matmul_tiles)(m, args->dtype, t, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
