// Entry points of the operators for models whose layers the caller runs: checks, then the launches.
#include <hip/hip_runtime.h>

#include "hr_kernels.h"
#include "hr_pair.h"

#define HR_OP_HIP(expr)                            \
    do {                                           \
        const hipError_t e__ = (expr);             \
        if (e__ != hipSuccess) {                   \
            hr::note_hip_error(e__, #expr);        \
            return HR_ERR_DEVICE;                  \
        }                                          \
    } while (0)

extern "C" {

int hr_rope_apply(const hr_rope_cfg* cfg, const double* freqs, int dtype, int64_t n_tokens, const int32_t* positions_dev,
                  int32_t first_position, int32_t period, const hr_rope_tensor* tensors, int32_t n_tensors, int inverse, void* stream) {
    const int rc = hr::rope_apply_check(cfg, freqs, dtype, n_tokens, positions_dev, first_position, period, tensors, n_tensors);
    if (rc != HR_OK || n_tokens == 0) return rc;
    HR_OP_HIP(hr::launch_rope_apply(*cfg, freqs, dtype, n_tokens, positions_dev, first_position, period, tensors, n_tensors, inverse != 0,
                                    (hipStream_t)stream));
    return HR_OK;
}

int hr_pair_tables_build(const hr_pool* pool, const hr_doc_list* docs, const int32_t* pair_doc_dev, const int32_t* query_lens_dev,
                         const hr_pair_tables* out, void* stream) {
    const int rc = hr::tables_build_check(pool, docs, pair_doc_dev, query_lens_dev, out);
    if (rc != HR_OK || out->n_pairs == 0) return rc;
    HR_OP_HIP(hr::launch_pair_tables(pool, docs, pair_doc_dev, query_lens_dev, out, (hipStream_t)stream));
    return HR_OK;
}

int hr_pair_attention(const hr_pool* pool, const hr_pair_tables* tables, const hr_attention_args* args, void* workspace_dev,
                      size_t workspace_bytes, void* stream) {
    int rc = hr::attention_check(pool, tables, args);
    if (rc != HR_OK || tables->n_pairs == 0 || tables->max_tokens == 0) return rc;
    const size_t need = hr_pair_attention_workspace_bytes(pool, tables);
    if (need > 0 && (!workspace_dev || (uintptr_t)workspace_dev % hr::kAlign != 0)) return HR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return HR_ERR_WORKSPACE_SMALL;
    rc = hr::attention_outputs_check(args);
    if (rc != HR_OK) return rc;
    HR_OP_HIP(hr::launch_pair_attention(pool, tables, args, workspace_dev, (hipStream_t)stream));
    return HR_OK;
}

}  // extern "C"
