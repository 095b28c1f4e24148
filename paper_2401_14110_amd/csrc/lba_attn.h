// lba_attn.h -- parameters of the attention kernels
#ifndef LBA_ATTN_H_
#define LBA_ATTN_H_

#include "lba_attn_device.h"

namespace lba {

struct AttnParams {
    const void *Q, *K, *V;
    void* O;
    float* lse;
    CodeFmt fmt;
    // backward
    const void* G;
    void *dQ, *dK, *dV;
    float* delta;            // [T, H]: rowsum(G * O)
    const int32_t *starts, *starts_k;
    lba_strides q, k, v, dq, dk, dv;
    int32_t T, Tk, count, H, KV, group, D;
    int32_t causal, clear;
    float scale;
};

int attn_params(const lba_attn& a, AttnParams* p);       // checks and copies the description

}  // namespace lba
#endif
