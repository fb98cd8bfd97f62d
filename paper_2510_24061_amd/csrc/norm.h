// Norms of a block (norm.hip): arguments as include/falqon.h describes them.
#pragma once
#include "falqon_internal.h"

namespace falqon {

constexpr int64_t kNormMaxWidth = 16384;
constexpr int64_t kNormGroups = 512;      // most workgroups of the backward pass, each of which leaves two partial sums

struct NormFwd {
    const void *x, *b, *w, *w_post, *gate;
    float scale, eps;
    int64_t T, d, ld_x, ld_b;
    void *s, *h;
    float *rstd, *rstd_b;
    uint8_t *sq, *s_exp, *bq, *b_exp;
};
int64_t norm_fwd_threads(int64_t T, int64_t d, bool f32);   // of its launch
hipError_t launch_norm_fwd(const NormFwd& a, bool f32, hipStream_t stream);

struct NormBwd {
    const void *dh, *ds;
    int64_t ld_dh, ld_ds;
    const void* s; int64_t ld_s; const uint8_t* s_exp; const float* rstd;
    const void* b; int64_t ld_b; const uint8_t* b_exp; const float* rstd_b;
    const void *w, *w_post, *gate;
    float scale;
    int64_t T, d;
    void *dx, *db;
    float *dw, *dw_post, *dgate;
};
hipError_t launch_norm_bwd(const NormBwd& a, bool f32, float* partial, hipStream_t stream);

}  // namespace falqon
