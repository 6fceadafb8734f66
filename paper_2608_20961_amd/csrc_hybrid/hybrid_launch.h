// Kernel launchers behind the C ABI of treewy_hybrid.h.  Arguments are already
// validated by the caller; each returns the HIP error of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "treewy_hybrid.h"

namespace treewy {

struct AppendArgs {
    const void *k, *v;
    treewy_strides ks, vs;                               // elements
    void *k_pages, *v_pages;
    const int32_t *table, *len, *path, *count;
    const float *cos, *sin;
    int32_t *new_len, *err;
    int n_pages, max_pages, log2_page;
    int positions, rot;
    int L, N, B, H;
};

hipError_t launch_cache_append(const AppendArgs &a, int d, bool f32, hipStream_t stream);

struct AttendArgs {
    const void *q, *k, *v;
    treewy_strides qs, ks, vs, os;                       // elements
    const int32_t *parent;                               // null: a chain
    const void *k_pages, *v_pages;
    const int32_t *table, *len;
    const float *cos, *sin;
    void *o;
    int32_t *err;
    int n_pages, max_pages, log2_page;
    int positions, rot;
    int shared;                                          // cached tokens read once for the batch
    int N, B, H_q, H_kv;
    float scale;
};

size_t tree_attention_workspace(int shared, int N, int B, int H_q, int H_kv, int d, bool f32);
hipError_t launch_tree_attention(AttendArgs a, int d, bool f32, void *workspace, hipStream_t stream);

struct SampleArgs {
    const void *logits;
    int64_t row_stride;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int R, V;
    int32_t *token, *err;
    float *logprob;
};

hipError_t launch_sample(const SampleArgs &a, bool f32, hipStream_t stream);

}  // namespace treewy
