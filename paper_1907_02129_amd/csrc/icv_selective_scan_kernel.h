// Selective state space scan (icv_selective_scan).
//
// Per row, channel and state: one exponential (the decay), two products and two multiply-adds.  Vector-ALU bound: 24 issue
// cycles for 64 of them (8 for the exponential, 4 for each of the others), and about 40 instructions per row and channel around
// them (softplus, gate, conversions), against 2 to 8 bytes of memory per row and channel.  24 sequences of 12347 rows, 4096
// channels, 16 states, bfloat16 with gate: 223 to 265 us, 1.8 TB/s, about what the instructions alone take; 310 where one sequence has a
// third of the rows, whose steps follow one another (525 us at first: what was in the way were waits for the next tile's loads
// inside conversions and branches, 64-bit address products, bank conflicts, and the longest sequence).
//
// A lane keeps NS (4, 2 or 1) states of a channel in registers, S lanes (1..16) a channel: the rows' delta and delta * x are then
// read from LDS once for NS states, and a channel's states take few enough registers for several workgroups on a compute
// unit, whose wavefronts hide each other's latencies.  A workgroup of 256 lanes owns 256 / S channels of one group
// (they share B and C) and walks a sequence in tiles of TT rows: the next tile's inputs are on their way from memory
// while this one's rows are stepped through from LDS; softplus and the products with x are computed once per row and
// channel when a tile is staged, and D * x and the gate once when it is stored.  The sums over a channel's lanes are
// taken for four rows at a time, by exchanges inside quads that leave each lane with one row's sum.
#pragma once
#include "icv_selective_scan_args.h"

namespace icv {

enum { SCAN_WHOLE = 0, SCAN_PIECE_STATE = 1, SCAN_PIECE_OUT = 2 };

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|).  With u = 1 + e rounded, log(1 + e) = log(u) + log(1 + (e - (u - 1)) / u): the
// second term is the rounding error of u, at most 2^-24, and what counts of it is there where e is small and u is 1, so
// that the quotient may be left out: exact to a few ulp for every v.
__device__ inline float softplus(float v)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(v) * -kLog2e), u = 1.0f + e;
    return fmaxf(v, 0.0f) + fmaf(__builtin_amdgcn_logf(u), kLn2, e - (u - 1.0f));
}

// A coefficient as a power of two's, kept finite, so that a step of 0 times it is 0: such a step keeps the state, and the
// rows past a sequence's end step by 0.  NaN stays NaN.
__device__ inline float decay_rate(float a)
{
    a *= kLog2e;
    return a < -3.0e38f ? -3.0e38f : (a > 3.0e38f ? 3.0e38f : a);
}

// h * 2^(2 e) + w.  Over a piece's rows 2^(2 e) may be past float's range, up or down, though no state ever is: taken as two
// factors, and never infinite, so that a state of 0 stays 0 (states below 2^-126 may grow too little past 2^254).  What is lost of
// a NaN in e, w has: its step or its coefficient made all of the piece NaN.  16384 rows of 2048 channels, whose pieces begin with up to
// 31 of these for every state: 237.6 us, with one factor 234.8.
__device__ inline float grow(float h, float e, float w)
{
    const float f = __builtin_amdgcn_exp2f(__builtin_amdgcn_fmed3f(e, -126.0f, 127.0f));
    return fmaf(h * f, f, w);
}

// lane -> its place among the S lanes of a channel, and the channel among the wavefront's.  The four lowest states of a
// channel sit in one quad; with 8 lanes the second quad is 8 lanes away, with 16 all of a row of 16 is one channel's,
// so that the sums over quads are rotations within a row.
template <int S>
__device__ inline void lane_place(int lane, int* s, int* ch)
{
    if constexpr (S == 8) { *s = (lane & 3) | ((lane >> 1) & 4); *ch = ((lane >> 4) << 1) | ((lane >> 2) & 1); }
    else { *s = lane & (S - 1); *ch = lane / S; }
}

template <int CTRL>
__device__ inline float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kRotate4 = 0x124, kRotate8 = 0x128;

// Sums over the S lanes of a channel of four rows' partial sums.  S >= 4: lane s returns row s & 3's; S = 2: lane s returns
// rows s and s + 2; S = 1: all four.
template <int S>
__device__ inline void reduce_rows(const float (&p)[4], int s, float (&y)[4])
{
    if constexpr (S == 1) {
#pragma unroll
        for (int u = 0; u < 4; u++) y[u] = p[u];
        return;
    }
    const bool odd = s & 1, high = s & 2;
    const float q0 = (odd ? p[1] : p[0]) + dpp<kXor1>(odd ? p[0] : p[1]);
    const float q1 = (odd ? p[3] : p[2]) + dpp<kXor1>(odd ? p[2] : p[3]);
    y[0] = q0; y[1] = q1;
    if constexpr (S >= 4) {
        float r = (high ? q1 : q0) + dpp<kXor2>(high ? q0 : q1);
        if constexpr (S == 16) r += dpp<kRotate4>(r);
        if constexpr (S >= 8) r += dpp<kRotate8>(r);
        y[0] = r;
    }
}

// The n-th of at most 64 sequences by length, longest first; the same for all lanes.  Workgroups start in the order of their
// numbers, and a long sequence that starts last keeps a few compute units busy alone: 24 sequences of 12347 rows and 4096 channels
// take 309 to 346 us as they come, 237 to 239 by length.
__device__ inline int32_t nth_longest(const SeqArgs& q, int32_t n, int lane)
{
    int32_t length = -1;
    if (lane < q.count) {
        const int32_t b = seq_begin(q, lane);
        length = seq_end(q, lane, b) - b;
    }
    int32_t rank = 0;
    for (int k = 0; k < q.count; k++) {
        const int32_t other = __builtin_amdgcn_readlane(length, k);
        rank += other > length || (other == length && k < lane);
    }
    return __builtin_ctzll(__ballot(lane < q.count && rank == n));
}

// R rows' values of a lane's channel and NS states.
template <int NS, int R>
struct Rows {
    float2 v[R];
    float b[R][NS], c[R][NS];
};

template <typename T, int S, int NS, int ENDS, int MODE>
__global__ __launch_bounds__(256) void k_scan(ScanArgs a)
{
    constexpr int CW = 256 / S, TT = 8 * S < 64 ? 8 * S : 64, PAIRS = CW / 2, RPT = TT * PAIRS / 256, ROWS = TT / RPT;
    constexpr bool ODD = ENDS != FULL, ONE = ENDS == ONE_BY_ONE;
    constexpr int NP = S * NS, VS = NP / 4;        // states with those that are not there, in vectors of 4
    constexpr int BCV = (TT * VS + 255) / 256;     // vectors of B (and C) a thread stages
    __shared__ __align__(16) float2 dtx[TT][CW];    // delta and delta * x; the row's output takes delta's place
    __shared__ __align__(16) float sB[TT][NP], sC[MODE == SCAN_PIECE_STATE ? 1 : TT][NP];

    const int tid = threadIdx.x, lane = tid & 63;
    const int32_t tiles = a.group_tiles * (a.channels / a.per_group);
    const int32_t tile = (int32_t)(blockIdx.x % tiles);
    int32_t unit = (int32_t)(blockIdx.x / tiles), piece = 0, pieces = 1, i = unit;
    int32_t begin, end;
    if (MODE == SCAN_WHOLE) {
        if (a.by_length) i = nth_longest(a.seq, unit, lane);
        begin = seq_begin(a.seq, i);
        end = seq_end(a.seq, i, begin);
        if (begin == end) return;
    } else {
        // the sequence that piece `unit` belongs to, counting every sequence's pieces: 64 sequences at a time, one to a lane
        int32_t left = unit, i0 = 0;
        for (;; i0 += 64) {
            if (i0 >= a.seq.count) return;
            int32_t mine = 0;
            if (i0 + lane < a.seq.count) {
                const int32_t b = seq_begin(a.seq, i0 + lane);
                mine = (seq_end(a.seq, i0 + lane, b) - b + a.chunk - 1) / a.chunk;
            }
            int32_t upto = mine;                      // pieces of the lanes up to this one
#pragma unroll
            for (int step = 1; step < 64; step *= 2) {
                const int32_t before = __shfl_up(upto, step);
                if (lane >= step) upto += before;
            }
            const int32_t all = __builtin_amdgcn_readlane(upto, 63);
            if (left < all) {
                const int at = __builtin_ctzll(__ballot(upto > left));
                i = i0 + at;
                pieces = __builtin_amdgcn_readlane(mine, at);
                piece = left - (__builtin_amdgcn_readlane(upto, at) - pieces);
                break;
            }
            left -= all;
        }
        begin = seq_begin(a.seq, i);
        end = seq_end(a.seq, i, begin);
        if (MODE == SCAN_PIECE_STATE && piece == pieces - 1) return;
    }
    const int32_t first_unit = unit - piece;
    if (MODE != SCAN_WHOLE && first_unit + pieces > a.units) return;      // sequences that overlap: more pieces than there is room for
    const int32_t row0 = begin + piece * a.chunk;
    const int32_t row1 = MODE == SCAN_WHOLE || piece == pieces - 1 ? end : row0 + a.chunk;

    const int32_t group = tile / a.group_tiles, tile_c = (tile - group * a.group_tiles) * CW;
    const int32_t c0 = group * a.per_group + tile_c;                  // the tile's first channel
    const int32_t cn = a.per_group - tile_c < CW ? a.per_group - tile_c : CW;

    int s, wch;
    lane_place<S>(lane, &s, &wch);
    const int ch = (tid >> 6) * (64 / S) + wch;
    const int32_t d = c0 + (ch < cn ? ch : 0);
    const int nv = a.states - NS * s < 0 ? 0 : (a.states - NS * s < NS ? a.states - NS * s : NS);

    float A[NS], h[NS];
    load_row<NS>(a.A + (int64_t)d * a.states + NS * s, nv, A);
#pragma unroll
    for (int j = 0; j < NS; j++) A[j] = decay_rate(A[j]);

    const int64_t state_at = (int64_t)d * a.states + NS * s;
    const int64_t plane = (int64_t)a.channels * a.states;
#pragma unroll
    for (int j = 0; j < NS; j++) h[j] = 0.0f;
    if (piece == 0 && !(MODE == SCAN_PIECE_OUT && pieces > 1)) {
        const int32_t slot = a.state ? seq_slot(a.seq, a.seq.from, i) : -1;
        if (slot >= 0) load_row<NS>(a.state + slot * a.slot_stride + state_at, nv, h);
        // the slot may be written while the pieces' outputs are computed: those read the copy in the last piece's place
        if (MODE == SCAN_PIECE_STATE && ch < cn) store_row<NS>(a.ws_state + (first_unit + pieces - 1) * plane + state_at, nv, h);
    } else if (MODE == SCAN_PIECE_OUT) {
        load_row<NS>(a.ws_state + (piece == 0 ? first_unit + pieces - 1 : first_unit) * plane + state_at, nv, h);
        for (int32_t q0 = 1; q0 < piece; q0 += 8) {
            float sum[8], w[8][NS];
#pragma unroll
            for (int u = 0; u < 8; u++) {              // past the last: the first again, not used
                const int32_t q = first_unit + (q0 + u < piece ? q0 + u : q0);
                sum[u] = a.ws_sum[(int64_t)q * a.channels + d];
                load_row<NS>(a.ws_state + q * plane + state_at, nv, w[u]);
            }
#pragma unroll
            for (int u = 0; u < 8; u++)
                if (q0 + u < piece)
#pragma unroll
                    for (int j = 0; j < NS; j++) h[j] = grow(h[j], sum[u] * (0.5f * A[j]), w[u][j]);
        }
    }

    // staging: a thread takes two neighbouring channels of RPT of the tile's rows (lanes side by side read a row's channels
    // side by side, and meet no bank conflicts in LDS), and vectors of B and C
    const int vrow = tid / PAIRS, vch = 2 * (tid % PAIRS);
    const int vn = cn - vch < 0 ? 0 : (cn - vch < 2 ? cn - vch : 2);
    float dtb[2], Dx[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
        dtb[j] = a.dtb && j < vn ? a.dtb[c0 + vch + j] : 0.0f;
        Dx[j] = a.D && j < vn ? a.D[c0 + vch + j] : 0.0f;
    }
    // Offsets inside a tile are 32-bit and the same for every tile, what moves is a scalar base: with 64-bit products for every
    // row a third of all vector instructions were address arithmetic.
    constexpr uint32_t SZ = sizeof(T);
    const uint32_t vc = c0 + (vn ? vch : 0);
    const int vshift = ENDS == PART ? 2 - vn : 0;      // 2: a pair of the group's first channels, not used
    const uint32_t vl = vshift == 2 ? group * a.per_group : vc - vshift;       // channel loaded from
    const uint32_t xo = (vrow * (uint32_t)a.xs + vl) * SZ, dto = (vrow * (uint32_t)a.dts + vl) * SZ, zo = (vrow * (uint32_t)a.zs + vl) * SZ,
                   oo = vrow * (uint32_t)a.os + vc;
    const auto row_of = [](const void* p, int64_t row, int64_t stride) { return (const uint8_t*)p + row * stride * SZ; };      // scalar
    // Rows past the end repeat the last one (and are made to change nothing when they are staged): loads without branches
    constexpr int BCT = TT * VS < 256 ? TT * VS : 256;              // threads with B and C of their own; the others repeat them
    const int bct = tid % BCT, n4 = 4 * (bct % VS), bcrow = bct / VS;
    const int bcn = a.states - n4 < 0 ? 0 : (a.states - n4 < 4 ? a.states - n4 : 4);
    const int bcshift = ENDS == PART && bcn ? 4 - bcn : 0;
    const uint32_t bc0 = (uint32_t)group * a.states + (bcn ? n4 - bcshift : 0);
    Raw<T, 2, ONE> nx[RPT], nd[RPT], nz[RPT];
    Raw<T, 4, ONE> nB[BCV], nC[BCV];
    auto fetch_tile = [&](int32_t r, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int32_t most = row1 - 1 - r;
        const auto pairs = [&](Raw<T, 2, ONE> (&q)[RPT], const void* p, int64_t stride, uint32_t at) {
#pragma unroll
            for (int k = 0; k < RPT; k++) {
                if constexpr (WHOLE) {
                    q[k].load(row_of(p, r + k * ROWS, stride), at, vn);
                } else {
                    const int32_t row = vrow + k * ROWS;
                    q[k].load(row_of(p, r, stride), ((uint32_t)(row < most ? row : most) * (uint32_t)stride + vl) * SZ, vn);
                }
            }
        };
        pairs(nx, a.x, a.xs, xo);
        pairs(nd, a.dt, a.dts, dto);
        if (MODE != SCAN_PIECE_STATE && a.z) pairs(nz, a.z, a.zs, zo);
        const auto fours = [&](Raw<T, 4, ONE> (&q)[BCV], const void* p, int64_t stride) {
            const uint8_t* base = row_of(p, r, stride);
#pragma unroll
            for (int k = 0; k < BCV; k++) {
                int32_t row = bcrow + k * (256 / VS);
                if (!WHOLE && row > most) row = most;
                q[k].load(base, ((uint32_t)row * (uint32_t)stride + bc0) * SZ, bcn);
            }
        };
        fours(nB, a.B, a.bs);
        if (MODE != SCAN_PIECE_STATE) fours(nC, a.C, a.cs);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    auto fetch = [&](int32_t r) {
        if (r + TT <= row1) fetch_tile(r, yes);
        else fetch_tile(r, no);
    };

    float total = 0.0f;                       // sum of delta over the piece
    fetch(row0);
    for (int32_t r = row0; r < row1; r += TT) {
        Raw<T, 2, ONE> cx[RPT], cz[RPT];
        const bool tail = r + TT > row1;
#pragma unroll
        for (int k = 0; k < RPT; k++) {
            cx[k] = nx[k];
            cz[k] = nz[k];
            if constexpr (ENDS == PART) {
                cx[k].align(vshift & 1);
                cz[k].align(vshift & 1);
                nd[k].align(vshift & 1);
            }
            float v[2] = {nd[k].get(0) + dtb[0], nd[k].get(1) + dtb[1]};
            if (a.softplus) { v[0] = softplus(v[0]); v[1] = softplus(v[1]); }
            float4 q = make_float4(v[0], v[0] * cx[k].get(0), v[1], v[1] * cx[k].get(1));
            if (tail && r + vrow + k * ROWS >= row1) q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);      // decay 1, nothing added
            *(float4*)&dtx[vrow + k * ROWS][vch] = q;
        }
#pragma unroll
        for (int k = 0; k < BCV; k++) {
            const int row = bcrow + k * (256 / VS);
            const bool out = tail && r + row >= row1;
            const auto values = [&](Raw<T, 4, ONE> q) {
                if constexpr (ENDS == PART) q.align(bcshift);
                float4 v = make_float4(q.get(0), q.get(1), q.get(2), q.get(3));
                if (ODD) v = make_float4(bcn > 0 ? v.x : 0.0f, bcn > 1 ? v.y : 0.0f, bcn > 2 ? v.z : 0.0f, bcn > 3 ? v.w : 0.0f);
                return out ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : v;
            };
            *(float4*)&sB[row][n4] = values(nB[k]);
            if (MODE != SCAN_PIECE_STATE) *(float4*)&sC[row][n4] = values(nC[k]);
        }
        __syncthreads();
        if (r + TT < row1) fetch(r + TT);

        // Four rows at a time, the next AHEAD always on their way from LDS, which takes longer than two rows of one or two states (16384
        // rows in one wavefront's steps: 843 -> 733 us with one, 1147 -> 1013 with two; with four states there are no registers for it, and
        // two rows take long enough); the sums over the lanes are then taken while the next four are stepped through.  Rows past
        // the end change nothing.
        constexpr int AHEAD = NS == 4 ? 2 : 4;
        const int rows = row1 - r < TT ? row1 - r : TT;
        Rows<NS, AHEAD> even, odd;
        auto read = [&](Rows<NS, AHEAD>& q, int t) {
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                q.v[u] = dtx[t + u][ch];
                __builtin_memcpy(q.b[u], __builtin_assume_aligned(&sB[t + u][NS * s], 4 * NS), 4 * NS);
                if (MODE != SCAN_PIECE_STATE) __builtin_memcpy(q.c[u], __builtin_assume_aligned(&sC[t + u][NS * s], 4 * NS), 4 * NS);
            }
        };
        auto step = [&](const Rows<NS, AHEAD>& q, float* p) {
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const float2 v = q.v[u];
                if (MODE == SCAN_PIECE_STATE) total += v.x;
#pragma unroll
                for (int j = 0; j < NS; j++) {
                    h[j] = fmaf(__builtin_amdgcn_exp2f(v.x * A[j]), h[j], v.y * q.b[u][j]);
                    if (ODD) h[j] = j < nv ? h[j] : 0.0f;    // an infinite input must not reach a state that is not there
                }
                if (MODE != SCAN_PIECE_STATE) {
                    p[u] = q.c[u][0] * h[0];
#pragma unroll
                    for (int j = 1; j < NS; j++) p[u] = fmaf(q.c[u][j], h[j], p[u]);
                }
            }
        };
        auto finish = [&](const float (&p)[4], int t) {
            if (MODE == SCAN_PIECE_STATE) return;
            float y[4];
            reduce_rows<S>(p, s, y);
            if constexpr (S >= 4) {
                if (s < 4) dtx[t + s][ch].x = y[0];
            } else if constexpr (S == 2) {
                dtx[t + s][ch].x = y[0];
                dtx[t + 2 + s][ch].x = y[1];
            } else {
#pragma unroll
                for (int u = 0; u < 4; u++) dtx[t + u][ch].x = y[u];
            }
        };
        read(even, 0);
        float p[4], was[4];
        if constexpr (AHEAD == 4) {
            for (int t = 0; t < rows; t += 8) {
                read(odd, t + 4);
                __builtin_amdgcn_sched_barrier(0);
                step(even, p);
                if (t > 0) finish(was, t - 4);
                read(even, t + 8 < TT ? t + 8 : 0);
                __builtin_amdgcn_sched_barrier(0);
                step(odd, was);
                finish(p, t);
            }
            finish(was, (rows - 1) / 8 * 8 + 4);
        } else {
            for (int t = 0; t < rows; t += 4) {
                read(odd, t + 2);
                __builtin_amdgcn_sched_barrier(0);
                step(even, p);
                read(even, t + 4 < TT ? t + 4 : 0);
                __builtin_amdgcn_sched_barrier(0);
                step(odd, p + 2);
                finish(p, t);
            }
        }
        __syncthreads();
        auto store_tile = [&](auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
            for (int k = 0; k < RPT; k++) {
                const float4 v = *(const float4*)&dtx[vrow + k * ROWS][vch];
                float y[2] = {v.x, v.z};
                if (a.D) {
                    y[0] = fmaf(Dx[0], cx[k].get(0), y[0]);
                    y[1] = fmaf(Dx[1], cx[k].get(1), y[1]);
                }
                if (a.z) {
                    y[0] *= silu(cz[k].get(0));
                    y[1] *= silu(cz[k].get(1));
                }
                if (WHOLE || r + vrow + k * ROWS < row1) store_row<2>((T*)a.out + (int64_t)(r + k * ROWS) * a.os + oo, !ODD && WHOLE ? 2 : vn, y);
            }
        };
        if (MODE != SCAN_PIECE_STATE) {
            if (r + TT <= row1 && cn == CW) store_tile(yes);
            else store_tile(no);
        }
        // the places a thread reads here are the ones it writes for the next tile, and B and C are done with
    }
    if (ch >= cn) return;
    if (MODE == SCAN_PIECE_STATE) {
        store_row<NS>(a.ws_state + unit * plane + state_at, nv, h);
        if (s == 0) a.ws_sum[(int64_t)unit * a.channels + d] = total;
    } else if (piece == pieces - 1) {
        const int32_t slot = a.state ? seq_slot(a.seq, a.seq.to, i) : -1;
        if (slot >= 0) store_row<NS>(a.state + slot * a.slot_stride + state_at, nv, h);
    }
}

// One row per sequence: the state is read and written once, which is what bounds it.  A workgroup takes its channels of Q
// sequences: a wavefront alone waits for the slot number, then for the state, then ends; with Q states on their way together
// the compute units' wavefronts cover that: 128 sequences, 4096 channels, 16 states, bfloat16 15.8 us, 4.5 TB/s, with two; 16.8 with
// one, 16.1 with four.  Loads have no branches around them (a sequence that continues no slot reads slot 0 and
// drops it; 18.5 us with branches).  89 sequences, 2560 channels, 40 states: 21 us; element by element 40.
template <typename T, int S, int ENDS, int Q>
__global__ __launch_bounds__(256) void k_scan_step(ScanArgs a)
{
    constexpr bool ODD = ENDS != FULL, ONE = ENDS == ONE_BY_ONE;
    constexpr int CW = 256 / S;
    const int tid = threadIdx.x, lane = tid & 63;
    const int32_t tiles = (a.channels + CW - 1) / CW;
    const int32_t tile = (int32_t)(blockIdx.x % tiles), i0 = (int32_t)(blockIdx.x / tiles) * Q;
    int s, wch;
    lane_place<S>(lane, &s, &wch);
    const int32_t d = tile * CW + (tid >> 6) * (64 / S) + wch;
    if (d >= a.channels) return;                      // whole channels, so whole exchange partners
    const int nv = a.states - 4 * s < 0 ? 0 : (a.states - 4 * s < 4 ? a.states - 4 * s : 4);
    const int shift = ENDS == PART && nv ? 4 - nv : 0;
    const uint32_t n4 = nv ? 4 * s : 0;
    const int64_t state_at = (int64_t)d * a.states + n4, first_at = state_at - shift, bc = (int64_t)(d / a.per_group) * a.states + n4 - shift;
    const bool slots = a.state && a.seq.slots > 0;

    int32_t seq[Q], src[Q], dst[Q];
    bool on[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        seq[q] = i0 + q < a.seq.count ? i0 + q : i0;
        on[q] = i0 + q < a.seq.count && seq_end(a.seq, seq[q], seq[q]) != seq[q];
        src[q] = slots ? seq_slot(a.seq, a.seq.from, seq[q]) : -1;
        dst[q] = slots && on[q] ? seq_slot(a.seq, a.seq.to, seq[q]) : -1;
    }
    Raw<float, 4, ONE> hr[Q], Ar;
    Raw<T, 4, ONE> br[Q], cr[Q];
    Raw<T, 1, false> xr[Q], dr[Q], zr[Q];
    const auto at = [](const void* p, int64_t element, size_t size) { return (const uint8_t*)p + element * (int64_t)size; };
    Ar.load(at(a.A, first_at, 4), 0, nv);
#pragma unroll
    for (int q = 0; q < Q; q++) {
        if (slots) hr[q].load(at(a.state, (src[q] >= 0 ? src[q] : 0) * a.slot_stride + first_at, 4), 0, nv);
        br[q].load(at(a.B, seq[q] * a.bs + bc, sizeof(T)), 0, nv);
        cr[q].load(at(a.C, seq[q] * a.cs + bc, sizeof(T)), 0, nv);
        xr[q].load(at(a.x, seq[q] * a.xs + d, sizeof(T)), 0, 1);
        dr[q].load(at(a.dt, seq[q] * a.dts + d, sizeof(T)), 0, 1);
        if (a.z) zr[q].load(at(a.z, seq[q] * a.zs + d, sizeof(T)), 0, 1);
    }
    const float dtb = a.dtb ? a.dtb[d] : 0.0f, D = a.D ? a.D[d] : 0.0f;
    if constexpr (ENDS == PART) Ar.align(shift);
    float A[4];
#pragma unroll
    for (int j = 0; j < 4; j++) A[j] = decay_rate(Ar.get(j));
#pragma unroll
    for (int q = 0; q < Q; q++) {
        if constexpr (ENDS == PART) {
            hr[q].align(shift);
            br[q].align(shift);
            cr[q].align(shift);
        }
        float dt = dr[q].get(0) + dtb, y = 0.0f, h[4];
        const float x = xr[q].get(0);
        if (a.softplus) dt = softplus(dt);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float old = src[q] >= 0 ? hr[q].get(j) : 0.0f;
            h[j] = fmaf(__builtin_amdgcn_exp2f(dt * A[j]), old, dt * x * br[q].get(j));
            if (!ODD || j < nv) y = fmaf(cr[q].get(j), h[j], y);
        }
        if (dst[q] >= 0) store_row<4>(a.state + dst[q] * a.slot_stride + state_at, nv, h);
        if (S >= 2) y += dpp<kXor1>(y);
        if (S >= 4) y += dpp<kXor2>(y);
        if (S == 16) y += dpp<kRotate4>(y);
        if (S >= 8) y += dpp<kRotate8>(y);
        if (a.D) y = fmaf(D, x, y);
        if (a.z) y *= silu(zr[q].get(0));
        if (s == 0 && on[q]) ((T*)a.out)[seq[q] * a.os + d] = (T)y;
    }
}

template <typename T, int S>
int launch_step(const ScanArgs& a, hipStream_t s)
{
    constexpr int CW = 256 / S;
    const int64_t tiles = (a.channels + CW - 1) / CW, wgs = tiles * a.seq.count;
    const bool two = wgs >= 2048 && a.states >= 4;      // more than the chip holds at once
    const int64_t n = two ? tiles * (((int64_t)a.seq.count + 1) / 2) : wgs;
    if (too_many(n, 256)) return ICV_ERR_UNSUPPORTED;
    if (a.states != 4 * S) {
        if constexpr (S == 1) k_scan_step<T, S, ONE_BY_ONE, 1><<<(uint32_t)n, 256, 0, s>>>(a);
        else if (two) k_scan_step<T, S, PART, 2><<<(uint32_t)n, 256, 0, s>>>(a);
        else k_scan_step<T, S, PART, 1><<<(uint32_t)n, 256, 0, s>>>(a);
    } else if (two) k_scan_step<T, S, FULL, 2><<<(uint32_t)n, 256, 0, s>>>(a);
    else k_scan_step<T, S, FULL, 1><<<(uint32_t)n, 256, 0, s>>>(a);
    ICV_HIP_CHECK(hipGetLastError());
    return ICV_OK;
}

template <typename T, int S, int NS, int ENDS>
void launch_modes(const ScanArgs& a, uint32_t n, hipStream_t s)
{
    if (!a.chunk) {
        k_scan<T, S, NS, ENDS, SCAN_WHOLE><<<n, 256, 0, s>>>(a);
        return;
    }
    k_scan<T, S, NS, ENDS, SCAN_PIECE_STATE><<<n, 256, 0, s>>>(a);
    k_scan<T, S, NS, ENDS, SCAN_PIECE_OUT><<<n, 256, 0, s>>>(a);
}

template <typename T, int S, int NS>
int launch(const ScanArgs& a, hipStream_t s)
{
    const bool full = a.states == NS * S && a.per_group % 2 == 0;
    const int64_t n = (int64_t)a.group_tiles * (a.channels / a.per_group) * (a.chunk ? a.units : a.seq.count);
    if (too_many(n, 256)) return ICV_ERR_UNSUPPORTED;
    const bool one = a.states < 4 || a.per_group == 1;
    if (full) launch_modes<T, S, NS, FULL>(a, (uint32_t)n, s);
    else if (NS == 4 && one) launch_modes<T, S, 4, ONE_BY_ONE>(a, (uint32_t)n, s);       // and never with fewer states per lane
    else launch_modes<T, S, NS, PART>(a, (uint32_t)n, s);
    ICV_HIP_CHECK(hipGetLastError());
    return ICV_OK;
}

template <typename T>
int launch_scan(const ScanArgs& a, const ScanPlan& plan, bool step, hipStream_t s)
{
    if (step) {
        switch (plan.S) {
            case 1: return launch_step<T, 1>(a, s);
            case 2: return launch_step<T, 2>(a, s);
            case 4: return launch_step<T, 4>(a, s);
            case 8: return launch_step<T, 8>(a, s);
            default: return launch_step<T, 16>(a, s);
        }
    }
    switch (plan.NS * 32 + plan.S) {
        case 4 * 32 + 1: return launch<T, 1, 4>(a, s);
        case 4 * 32 + 2: return launch<T, 2, 4>(a, s);
        case 4 * 32 + 4: return launch<T, 4, 4>(a, s);
        case 4 * 32 + 8: return launch<T, 8, 4>(a, s);
        case 2 * 32 + 4: return launch<T, 4, 2>(a, s);
        case 2 * 32 + 8: return launch<T, 8, 2>(a, s);
        case 2 * 32 + 16: return launch<T, 16, 2>(a, s);
        case 1 * 32 + 8: return launch<T, 8, 1>(a, s);
        case 1 * 32 + 16: return launch<T, 16, 1>(a, s);
        default: return launch<T, 16, 4>(a, s);
    }
}

}  // namespace icv
