// What the scan's host side hands to its kernels.
#pragma once
#include "icv_sequence.h"

namespace icv {

struct ScanArgs {
    const void *x, *dt, *B, *C, *z;
    const float *A, *D, *dtb;
    float* state;
    void* out;
    int64_t xs, dts, bs, cs, zs, os, slot_stride;
    int32_t channels, states, per_group, group_tiles, softplus;
    int32_t by_length;        // longest sequences first
    int32_t chunk, units;     // rows per piece of a sequence (0: sequences are not cut), pieces there is room for
    float *ws_state, *ws_sum; // of every piece: [channels][states] and [channels]
    SeqArgs seq;
};

// How a call is cut: lanes per channel, states per lane, rows per piece of a sequence (0: sequences stay whole).
struct ScanPlan {
    int S, NS;
    int32_t rows;
};

int launch_scan_f32(const ScanArgs& a, const ScanPlan& plan, bool step, hipStream_t s);
int launch_scan_bf16(const ScanArgs& a, const ScanPlan& plan, bool step, hipStream_t s);

}  // namespace icv
