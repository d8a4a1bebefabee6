// Selective state space scan (icv_selective_scan): how a call is cut, and the entry points.  The kernels are
// icv_selective_scan_kernel.h's, instantiated per type in icv_selective_scan_f32.hip and icv_selective_scan_bf16.hip.
#include "icv_selective_scan_args.h"
#include <cmath>

namespace icv {

// Lanes per channel, NS states each.
static int lanes_per_channel(int states, int NS)
{
    int s = 1;
    while (NS * s < states) s *= 2;
    return s;
}

static bool is_step(const icv_sequences* seq) { return !seq->start && seq->tokens == seq->count; }

// Test hooks in icv_scan_params::softplus above its public value (icv.h says they must be 0; the library's own tests set them to run every
// cut on calls small enough for a reference): bits 8-9 1: four states per lane, 2: two, 3: one; bits 10-15 rows per piece in 64s
// (0: whole sequences).
static int hook_states_per_lane(int hook) { return 8 >> (hook & 3); }
// Fewer than four states per lane: where all have enough, and a group has two channels (a thread stages them in pairs).
static bool fewer_fit(int NS, int states, int per_group) { return states > 4 && states <= 16 * NS && per_group > 1; }

static bool hook_fits(int hook, int states, int per_group)
{
    const int NS = hook_states_per_lane(hook);
    return (hook & 3) != 0 && hook < 256 && (NS == 4 || fewer_fit(NS, states, per_group));
}

// Fewer states per lane shorten the steps that follow one another, for some more instructions in all; pieces let the rows of a
// sequence be worked on side by side, for a second pass over most of them that makes no outputs. Both sides are modelled, in
// us, and the fastest cut is taken: `chain`, a row's steps in a wavefront by itself, against `work`, all rows' instructions on
// a chip that is full; whichever is longer, and something of the other when they are close. A tile's inputs are staged whole,
// so that sequences shorter than one pay for all of it. The lengths in a ragged batch are in device memory: they are taken for
// widely varied ones, whose longest has 1 + 1.2 log(count) times the mean (at 0.75, fitted to milder ones, 24 sequences of
// 12347 rows, 3 to 8 times the mean the longest, took 4 states per lane and 292 us instead of 253 on the average). Constants
// fitted to 100 calls of 1 to 256 sequences, 30 to 32768 rows, 64 to 8192 channels, 8 to 64 states, each cut in 1 to 15 ways
// (MI355X): the cut taken took 1.015 times as long as the fastest. 16384 rows of 2048 channels: 1743 us whole with 4 states per
// lane, 733 with one, 258 in pieces of 512; 8 x 2048 rows: 221, 182 (two states), 210, in pieces 220; 24 ragged ones of 12347
// rows, 4096 channels: 234, 222, 292, in pieces 298; 2 x 512 rows, 512 channels: 58, 36, 26, in pieces 17; one of 1065 rows,
// 1048 channels: 127, 76, 54, in pieces of 128 27, of 64 23.
static ScanPlan plan_scan(const icv_scan_params* p, const icv_sequences* seq)
{
    ScanPlan best = {lanes_per_channel(p->states, 4), 4, 0};
    if (is_step(seq)) return best;
    if (const int hook = p->softplus >> 8) {
        const int NS = hook_states_per_lane(hook), S = lanes_per_channel(p->states, NS), tt = 8 * S < 64 ? 8 * S : 64;
        return {S, NS, ((hook >> 2) * 64 + tt - 1) / tt * tt};
    }
    const int32_t per_group = p->channels / p->groups;
    const bool equal = seq->count == 1 || (!seq->start && !seq->length);
    const double tokens = seq->tokens, mean = tokens / seq->count;
    const double longest = equal ? mean : fmin(tokens, mean * (1 + 1.2 * log((double)seq->count)));
    double least = 1e30;
    for (int NS = 4; NS >= 1; NS /= 2) {
        if (NS < 4 && !fewer_fit(NS, p->states, per_group)) continue;
        const int S = lanes_per_channel(p->states, NS), cw = 256 / S, tt = 8 * S < 64 ? 8 * S : 64;
        const bool odd = p->states != S * NS || per_group % 2 != 0;
        const double channels = (double)p->groups * ((per_group + cw - 1) / cw) * cw;
        const double staged = seq->count * (equal ? ceil(mean / tt) * tt : tt / (1 - exp(-tt / mean)));       // rows of whole tiles
        const double work = channels * (1.92 * staged + tokens * (0.171 * S * NS + 0.106 * S)) * 1e-6 * (odd ? 1.15 : 1.0);
        const double chain = (0.0209 + 0.0134 * NS + 0.0454 / S) * (odd ? 1.15 : 1.0);
        const auto both = [](double a, double b) {
            const double more = fmax(a, b), less = fmin(a, b);
            return more + 0.25 * less * (less / more) * (less / more);
        };
        for (int32_t rows = 0; rows <= 1024; rows = rows ? 2 * rows : 64) {
            if (rows >= (equal ? mean : tokens)) break;
            double us = 5.1 + both(longest * chain, work);
            if (rows) {
                const int32_t r = (rows + tt - 1) / tt * tt;
                const double whole = seq->count / (tokens / r + 0.5 * seq->count);      // pieces that end a sequence: no first pass
                const double steps = fmin(longest, r) * chain;
                us = 11 + both(0.7 * steps, 0.2 * work * fmax(0.0, 1 - whole)) + 1.2 * both(steps, work) + longest / r / 8;
            }
            if (us < least) {
                least = us;
                best = {S, NS, (rows + tt - 1) / tt * tt};
            }
        }
    }
    return best;
}

static int64_t piece_count(const icv_sequences* seq, int32_t rows) { return (int64_t)seq->tokens / rows + seq->count; }

// A tile's offsets (64 rows at most) are kept in 32 bits.
constexpr int32_t kMostStride = 1 << 24;

static int check_scan(const icv_scan_params* p, const icv_sequences* seq, SeqArgs* sa)
{
    if (!p || p->channels < 1 || p->states < 1 || p->groups < 1 || p->channels % p->groups != 0) return ICV_ERR_INVALID_ARG;
    if (p->states > 64) return ICV_ERR_UNSUPPORTED;
    if (p->softplus < 0 || (p->softplus & 255) > 1) return ICV_ERR_INVALID_ARG;
    if (p->softplus >> 8 && !hook_fits(p->softplus >> 8, p->states, p->channels / p->groups)) return ICV_ERR_UNSUPPORTED;
    if (p->dtype == ICV_U8I8) return ICV_ERR_UNSUPPORTED;
    if (p->dtype != ICV_F32 && p->dtype != ICV_BF16) return ICV_ERR_INVALID_ARG;
    for (int32_t r : {p->x_row_stride, p->dt_row_stride, p->z_row_stride, p->out_row_stride})
        if (r && r < p->channels) return ICV_ERR_INVALID_ARG;
    for (int32_t r : {p->x_row_stride, p->dt_row_stride, p->z_row_stride, p->out_row_stride, p->b_row_stride, p->c_row_stride})
        if (r >= kMostStride) return ICV_ERR_UNSUPPORTED;
    if (p->channels >= kMostStride || (int64_t)p->groups * p->states >= kMostStride) return ICV_ERR_UNSUPPORTED;
    for (int32_t r : {p->b_row_stride, p->c_row_stride})
        if (r && r < (int64_t)p->groups * p->states) return ICV_ERR_INVALID_ARG;
    if (p->state_slots < 0 || (p->state_slot_stride && p->state_slot_stride < (int64_t)p->channels * p->states))
        return ICV_ERR_INVALID_ARG;
    return make_seq_args(seq, p->state_slots, sa);
}

}  // namespace icv

extern "C" size_t icv_selective_scan_workspace_bytes(const icv_scan_params* p, const icv_sequences* seq)
{
    using namespace icv;
    SeqArgs sa;
    if (check_scan(p, seq, &sa) != ICV_OK || seq->count == 0 || seq->tokens == 0) return 0;
    const int32_t rows = plan_scan(p, seq).rows;
    if (!rows) return 0;
    return (size_t)piece_count(seq, rows) * p->channels * (p->states + 1) * sizeof(float);
}

extern "C" int icv_selective_scan(const icv_scan_params* p, const icv_sequences* seq, const icv_scan_tensors* t,
                                  void* workspace, void* stream)
{
    using namespace icv;
    ScanArgs a;
    const int st = check_scan(p, seq, &a.seq);
    if (st != ICV_OK) return st;
    if (!t) return ICV_ERR_INVALID_ARG;
    if (seq->count == 0 || seq->tokens == 0) return ICV_OK;
    if (!t->x || !t->dt || !t->A || !t->B || !t->C || !t->out) return ICV_ERR_INVALID_ARG;
    const uintptr_t size = p->dtype == ICV_F32 ? 4 : 2;
    for (const void* q : {t->x, t->dt, t->B, t->C, t->z, (const void*)t->out})
        if (misaligned(q, size)) return ICV_ERR_INVALID_ARG;
    for (const void* q : {(const void*)t->A, (const void*)t->D, (const void*)t->dt_bias, (const void*)t->state})
        if (misaligned(q, 4)) return ICV_ERR_INVALID_ARG;
    const auto stride = [](int32_t s, int64_t dense) { return s ? (int64_t)s : dense; };
    a.x = t->x; a.dt = t->dt; a.B = t->B; a.C = t->C; a.z = t->z;
    a.A = t->A; a.D = t->D; a.dtb = t->dt_bias; a.state = t->state; a.out = t->out;
    a.xs = stride(p->x_row_stride, p->channels);
    a.dts = stride(p->dt_row_stride, p->channels);
    a.zs = stride(p->z_row_stride, p->channels);
    a.os = stride(p->out_row_stride, p->channels);
    a.bs = stride(p->b_row_stride, (int64_t)p->groups * p->states);
    a.cs = stride(p->c_row_stride, (int64_t)p->groups * p->states);
    // an output over an input: an element is read before it is written, by the same thread, if both lie at the same place
    if ((a.out == a.x && a.os != a.xs) || (a.out == a.dt && a.os != a.dts) || (a.out == a.z && a.os != a.zs) ||
        a.out == a.B || a.out == a.C)
        return ICV_ERR_INVALID_ARG;
    a.slot_stride = p->state_slot_stride ? p->state_slot_stride : (int64_t)p->channels * p->states;
    a.channels = p->channels; a.states = p->states; a.per_group = p->channels / p->groups; a.softplus = p->softplus & 255;
    const ScanPlan plan = plan_scan(p, seq);
    const int cw = 256 / plan.S;
    a.group_tiles = (a.per_group + cw - 1) / cw;
    // Finding the order costs every workgroup a few instructions per sequence: done where workgroups have to wait for others and
    // there are rows enough to pay for it (20 sequences of 2000 rows, 4096 channels: 54 us as they came, 40 by length; 64 of 1000
    // rows: 35 and 47).
    a.by_length = (seq->start || seq->length) && seq->count > 1 && seq->count <= 64 && seq->tokens / seq->count >= 32 &&
                  (int64_t)a.group_tiles * p->groups * seq->count > 256;
    a.chunk = plan.rows;
    const int64_t pieces = a.chunk ? piece_count(seq, a.chunk) : 0;
    if (a.chunk && (!workspace || misaligned(workspace, 16))) return ICV_ERR_INVALID_ARG;
    a.units = (int32_t)pieces;
    a.ws_state = (float*)workspace;
    a.ws_sum = a.ws_state + pieces * a.channels * a.states;
    hipStream_t s = (hipStream_t)stream;
    return p->dtype == ICV_F32 ? launch_scan_f32(a, plan, is_step(seq), s) : launch_scan_bf16(a, plan, is_step(seq), s);
}
