// Short causal convolution along sequences (icv_causal_conv1d).
//
// Memory bound: 2 * taps operations per element read and written.  A thread owns VEC neighbouring channels (8 bytes of a
// row) over a run of consecutive rows, keeps the last taps - 1 rows in registers as floats, and so reads every row
// once, plus taps - 1 rows in front of its run; AHEAD rows are on their way at once.  Runs are counted over all rows of the call,
// whatever sequences they belong to, so that ragged batches load the chip evenly; a thread walks the sequences that its run meets.
//
// 24 sequences, 12347 rows, 4096 channels, 4 taps, bfloat16: 50 us, 4.0 TB/s (a copy: 39 us, 5.2 TB/s); 24576 rows, 2048 channels, 2 taps,
// float: 79 us, 5.1 TB/s.  Registers decide, not the width of a load: with 16 bytes a thread 68 and 90 us, with 4 bytes 51 and 77;
// 8 rows ahead 52 and 81.
//
// The state may be read and written in the same slot, so one thread does both: the run that holds a sequence's first
// row computes the sequence's first taps - 1 rows (all rows that the old state reaches), also where they pass the run's
// end, and writes the new state; the runs behind it leave those rows out.
#include "icv_sequence.h"

namespace icv {

struct ConvArgs {
    const void* in;
    const void* filt;
    const float* bias;
    void* state;
    void* out;
    int32_t channels, vecs, run, silu;
    int32_t per_xcd;
    int64_t in_stride, out_stride, slot_stride;
    SeqArgs seq;
};

template <typename T, int W, int VEC, int AHEAD, int ENDS>
__global__ __launch_bounds__(256) void k_causal_conv(ConvArgs a)
{
    constexpr bool ODD = ENDS != FULL;
    using Row = Raw<T, VEC, ENDS == ONE_BY_ONE>;
    // workgroups go to the 8 XCDs in turn: each gets neighbouring runs, so that the rows in front of a run are in its L2
    const int64_t id = ((int64_t)(blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3)) * 256 + threadIdx.x;
    const int32_t runs = (a.seq.tokens - 1) / a.run + 1;
    const int64_t r = id / a.vecs;
    if (r >= runs) return;
    const int32_t c0 = (int32_t)(id - r * a.vecs) * VEC;
    const int32_t nv = a.channels - c0 < VEC ? a.channels - c0 : VEC;
    const int shift = ENDS == PART ? VEC - nv : 0;
    const auto take = [&](Row& q, const T* p, int n) { q.load((const uint8_t*)(p - shift), 0, n); };
    const auto align = [&](auto& rows) {
        if constexpr (ENDS == PART)
            for (auto& q : rows) q.align(shift);
    };
    const T* in = (const T*)a.in + c0;
    T* out = (T*)a.out + c0;
    T* state = (T*)a.state + c0;
    const int32_t r0 = (int32_t)r * a.run, r1 = a.seq.tokens - r0 < a.run ? a.seq.tokens : r0 + a.run;

    float w[W][VEC], bias[VEC];
    {
        // the filter's rows of these channels lie side by side
        const T* f = (const T*)a.filt + (int64_t)c0 * W;
        T q[VEC * W];
        if (!ODD) {
            __builtin_memcpy(q, f, sizeof(q));
        } else {
#pragma unroll
            for (int j = 0; j < VEC * W; j++) q[j] = f[j < nv * W ? j : 0];
        }
#pragma unroll
        for (int j = 0; j < VEC; j++) {
            bias[j] = a.bias ? a.bias[c0 + (!ODD || j < nv ? j : 0)] : 0.0f;
#pragma unroll
            for (int k = 0; k < W; k++) w[k][j] = (float)q[j * W + k];
        }
    }

    // the last sequence that begins at or before the run's first row, else the first one
    int32_t i = 0;
    if (a.seq.start) {
        // begin(lo) <= r0 < begin(hi), if any begins there; seven places at a time, since each round waits for memory once
        int32_t lo = 0, hi = a.seq.count;
        while (hi - lo > 1) {
            const int32_t step = ((hi - lo - 1) >> 3) + 1;
            int32_t at[7], n = 0;
#pragma unroll
            for (int k = 0; k < 7; k++) at[k] = a.seq.start[lo + (k + 1) * step < hi ? lo + (k + 1) * step : lo];
#pragma unroll
            for (int k = 0; k < 7; k++) n += lo + (k + 1) * step < hi && clamp_row(at[k], a.seq.tokens) <= r0;
            lo += n * step;
            hi = lo + step < hi ? lo + step : hi;
        }
        i = lo;
    } else {
        i = r0 / a.seq.each;
    }
    for (; i < a.seq.count; i++) {
        const int32_t b = seq_begin(a.seq, i);
        if (b >= r1) break;
        const int32_t e = seq_end(a.seq, i, b);
        if (e == b) continue;
        const bool owner = b >= r0;                     // the run that holds the sequence's first row
        const int32_t own_end = e - b < W - 1 ? e : b + W - 1;
        int32_t lo = owner ? b : (r0 > own_end ? r0 : own_end);
        int32_t hi = e < r1 ? e : r1;
        if (owner && hi < own_end) hi = own_end;
        if (lo >= hi) continue;

        // everything that is read first is on its way together: the rows before the first one, AHEAD rows, the rows of the new state
        float win[W > 1 ? W - 1 : 1][VEC];
        Row before[W > 1 ? W - 1 : 1], q[AHEAD], last[W > 1 ? W - 1 : 1];
        const int32_t from = owner && a.state ? seq_slot(a.seq, a.seq.from, i) : -1, slot = owner && a.state ? seq_slot(a.seq, a.seq.to, i) : -1;
        const auto fetch = [&](int32_t t0) {            // past the end the last one again
#pragma unroll
            for (int u = 0; u < AHEAD; u++) take(q[u], in + (int64_t)(t0 + u < hi ? t0 + u : hi - 1) * a.in_stride, nv);
        };
        fetch(lo);
        if (from >= 0) {
#pragma unroll
            for (int k = 0; k < W - 1; k++) take(before[k], state + from * a.slot_stride + (int64_t)k * a.channels, nv);
        } else if (!owner) {
#pragma unroll
            for (int k = 0; k < W - 1; k++) take(before[k], in + (int64_t)(lo - (W - 1) + k) * a.in_stride, nv);
        }
        if (slot >= 0) {
#pragma unroll
            for (int k = 0; k < W - 1; k++) {
                const int32_t at = e - b - (W - 1) + k;  // the sequence's row that becomes state row k; below 0 an old one
                take(last[k], at < 0 && from >= 0 ? state + from * a.slot_stride + (int64_t)(W - 1 + at) * a.channels
                                                  : in + (int64_t)(b + (at > 0 ? at : 0)) * a.in_stride, nv);
            }
        }
        align(before);
#pragma unroll
        for (int k = 0; k < W - 1; k++)
#pragma unroll
            for (int j = 0; j < VEC; j++) win[k][j] = owner && from < 0 ? 0.0f : before[k].get(j);
        for (int32_t t0 = lo; t0 < hi; t0 += AHEAD) {
            if (t0 > lo) fetch(t0);
            align(q);
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                if (t0 + u >= hi) break;
                float x[VEC], y[VEC];
#pragma unroll
                for (int j = 0; j < VEC; j++) x[j] = q[u].get(j);
#pragma unroll
                for (int j = 0; j < VEC; j++) {
                    float s = bias[j];
#pragma unroll
                    for (int k = 0; k < W - 1; k++) s = fmaf(w[k][j], win[k][j], s);
                    y[j] = fmaf(w[W - 1][j], x[j], s);
                }
                if (a.silu)
#pragma unroll
                    for (int j = 0; j < VEC; j++) y[j] = silu(y[j]);
                store_row<VEC>(out + (int64_t)(t0 + u) * a.out_stride, ODD ? nv : VEC, y);
                if constexpr (W > 1) {
#pragma unroll
                    for (int k = 0; k + 1 < W - 1; k++)
#pragma unroll
                        for (int j = 0; j < VEC; j++) win[k][j] = win[k + 1][j];
#pragma unroll
                    for (int j = 0; j < VEC; j++) win[W - 2][j] = x[j];
                }
            }
        }
        if (slot >= 0) {
            align(last);
#pragma unroll
            for (int k = 0; k < W - 1; k++) {
                float v[VEC];
#pragma unroll
                for (int j = 0; j < VEC; j++) v[j] = e - b - (W - 1) + k < 0 && from < 0 ? 0.0f : last[k].get(j);
                store_row<VEC>(state + slot * a.slot_stride + (int64_t)k * a.channels, ODD ? nv : VEC, v);
            }
        }
    }
}

template <typename T, int W, int VEC, int ENDS>
static void launch_ahead(const ConvArgs& a, bool single, hipStream_t s)
{
    if (single) k_causal_conv<T, W, VEC, 1, ENDS><<<8 * a.per_xcd, 256, 0, s>>>(a);
    else k_causal_conv<T, W, VEC, 4, ENDS><<<8 * a.per_xcd, 256, 0, s>>>(a);
}

// Rows per run: 32, and fewer until there are 2048 wavefronts (two for every SIMD): a run reads taps - 1 rows more
// than it computes (12347 rows, 4096 channels: 50.4 us with 32, 52.5 with 16; 32 alone would leave 64 rows of 2048 channels to 16
// wavefronts).  Under 4 that costs more than half as much again and 1024 wavefronts are enough (33 sequences of 2707 rows, 768 channels: 6.7
// us with 4, 7.8 with 2; 20 of 3000 rows, 3 channels: 8.9 with 4, 6.0 with 1), except where sequences are short, which a thread goes
// through one after another (214 of 299 rows, 2048 channels: 9.6 with 4, 7.8 with 2, 6.1 with 1).
static int32_t rows_per_run(const ConvArgs& a, bool single)
{
    const bool short_ones = a.seq.tokens / a.seq.count < 16;
    for (int32_t run = single ? 1 : 32;; run /= 2) {
        const int64_t threads = (int64_t)a.vecs * (((int64_t)a.seq.tokens + run - 1) / run);
        if (run == 1 || threads >= (run > 4 || short_ones ? 2048 : 1024) * 64) return run;
    }
}

// a.run on the way in: a test hook, bits 8-13 of icv_causal_conv_params::silu (icv.h says they must be 0; the library's own tests set
// them to have runs of several rows and sequences in calls small enough for a reference): the rows per run, 0: the rule's.
template <typename T, int W>
static int launch(ConvArgs a, hipStream_t s)
{
    constexpr int VEC = 8 / sizeof(T);
    a.vecs = (a.channels + VEC - 1) / VEC;
    const bool single = !a.seq.start && a.seq.each == 1;
    if (!a.run) a.run = rows_per_run(a, single);
    const int64_t threads = (int64_t)a.vecs * (((int64_t)a.seq.tokens + a.run - 1) / a.run);
    const int64_t blocks = (threads + 255) / 256;
    if (too_many(blocks + 7, 256)) return ICV_ERR_UNSUPPORTED;
    a.per_xcd = (int32_t)((blocks + 7) / 8);
    if (a.channels % VEC == 0) launch_ahead<T, W, VEC, FULL>(a, single, s);
    else if (a.channels >= VEC) launch_ahead<T, W, VEC, PART>(a, single, s);
    else launch_ahead<T, W, VEC, ONE_BY_ONE>(a, single, s);
    ICV_HIP_CHECK(hipGetLastError());
    return ICV_OK;
}

template <typename T>
static int launch_taps(const ConvArgs& a, int taps, hipStream_t s)
{
    switch (taps) {
        case 1: return launch<T, 1>(a, s);
        case 2: return launch<T, 2>(a, s);
        case 3: return launch<T, 3>(a, s);
        case 4: return launch<T, 4>(a, s);
        case 5: return launch<T, 5>(a, s);
        case 6: return launch<T, 6>(a, s);
        case 7: return launch<T, 7>(a, s);
        default: return launch<T, 8>(a, s);
    }
}

}  // namespace icv

extern "C" int icv_causal_conv1d(const icv_causal_conv_params* p, const icv_sequences* seq, const void* input,
                                 const void* filter, const float* bias, void* state, void* output, void* stream)
{
    using namespace icv;
    if (!p || p->channels < 1 || p->taps < 1 || p->taps > 8 || p->silu < 0 || (p->silu & 255) > 1) return ICV_ERR_INVALID_ARG;
    if (p->silu >> 8 > 32) return ICV_ERR_UNSUPPORTED;
    if (p->dtype == ICV_U8I8) return ICV_ERR_UNSUPPORTED;
    if (p->dtype != ICV_F32 && p->dtype != ICV_BF16) return ICV_ERR_INVALID_ARG;
    if ((p->in_row_stride && p->in_row_stride < p->channels) || (p->out_row_stride && p->out_row_stride < p->channels))
        return ICV_ERR_INVALID_ARG;
    const int64_t slot = (int64_t)(p->taps - 1) * p->channels;
    if (p->state_slots < 0 || (p->state_slot_stride && p->state_slot_stride < slot)) return ICV_ERR_INVALID_ARG;
    ConvArgs a;
    const int st = make_seq_args(seq, p->state_slots, &a.seq);
    if (st != ICV_OK) return st;
    if (seq->count == 0 || seq->tokens == 0) return ICV_OK;
    const uintptr_t size = p->dtype == ICV_F32 ? 4 : 2;
    if (!input || !filter || !output || input == output) return ICV_ERR_INVALID_ARG;
    if (misaligned(input, size) || misaligned(filter, size) || misaligned(output, size) || misaligned(state, size) ||
        misaligned(bias, 4))
        return ICV_ERR_INVALID_ARG;
    a.in = input; a.filt = filter; a.bias = bias; a.state = state; a.out = output;
    a.channels = p->channels; a.silu = p->silu & 255; a.run = p->silu >> 8;
    a.in_stride = p->in_row_stride ? p->in_row_stride : p->channels;
    a.out_stride = p->out_row_stride ? p->out_row_stride : p->channels;
    a.slot_stride = p->state_slot_stride ? p->state_slot_stride : slot;
    hipStream_t s = (hipStream_t)stream;
    return p->dtype == ICV_F32 ? launch_taps<float>(a, p->taps, s) : launch_taps<__bf16>(a, p->taps, s);
}
