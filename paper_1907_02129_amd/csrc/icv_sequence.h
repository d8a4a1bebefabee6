// What the operators on sequences share: which rows belong to a sequence (icv_sequences), rows of any alignment, the
// activations.
#pragma once
#include "icv_internal.h"

namespace icv {

// icv_sequences as the kernels see it; `each` is the rows per sequence without a start array.
struct SeqArgs {
    int32_t count, tokens, each;
    const int32_t* start;
    const int32_t* length;
    const int32_t* from;
    const int32_t* to;
    int32_t slots;
};

inline int make_seq_args(const icv_sequences* s, int32_t slots, SeqArgs* a)
{
    if (!s || s->count < 0 || s->tokens < 0) return ICV_ERR_INVALID_ARG;
    if (s->tokens > INT32_MAX - 65536) return ICV_ERR_UNSUPPORTED;      // row numbers past a tile's end stay in 32 bits
    if (!s->start && s->count > 0 && s->tokens % s->count != 0) return ICV_ERR_INVALID_ARG;
    for (const int32_t* q : {s->start, s->length, s->from, s->to})
        if ((uintptr_t)q & 3u) return ICV_ERR_INVALID_ARG;
    *a = {s->count, s->tokens, s->count > 0 ? s->tokens / s->count : 0, s->start, s->length, s->from, s->to, slots};
    return ICV_OK;
}

// A launch's threads are counted in 32 bits.
inline bool too_many(int64_t workgroups, int threads) { return workgroups > (int64_t)UINT32_MAX / threads; }

inline bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

__device__ inline int32_t clamp_row(int32_t v, int32_t tokens) { return v < 0 ? 0 : (v > tokens ? tokens : v); }

// Row of the first of sequence i's rows; i = count gives the end of the last one's.
__device__ inline int32_t seq_begin(const SeqArgs& s, int32_t i)
{
    return s.start ? clamp_row(s.start[i], s.tokens) : i * s.each;
}

// One past sequence i's last row: its length's worth of the rows up to the next sequence, never before `begin`.
__device__ inline int32_t seq_end(const SeqArgs& s, int32_t i, int32_t begin)
{
    int32_t n = seq_begin(s, i + 1) - begin;
    if (s.length && s.length[i] < n) n = s.length[i];
    return begin + (n > 0 ? n : 0);
}

// The slot a sequence continues or leaves its state in; -1: none.
__device__ inline int32_t seq_slot(const SeqArgs& s, const int32_t* which, int32_t i)
{
    const int32_t v = which ? which[i] : i;
    return v >= 0 && v < s.slots ? v : -1;
}

// N elements from any address of the element's own alignment (one wide load: global memory takes any address),
// `n` < N of them where a row ends; the rest read as zero.
template <int N, typename T>
__device__ inline void load_row(const T* p, int n, float (&v)[N])
{
    if (n >= N) {
        T r[N];
        __builtin_memcpy(r, p, sizeof(r));
#pragma unroll
        for (int j = 0; j < N; j++) v[j] = (float)r[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; j++) v[j] = j < n ? (float)p[j] : 0.0f;
    }
}

template <int N, typename T>
__device__ inline void store_row(T* p, int n, const float (&v)[N])
{
    if (n >= N) {
        T r[N];
#pragma unroll
        for (int j = 0; j < N; j++) r[j] = (T)v[j];
        __builtin_memcpy(p, r, sizeof(r));
    } else {
#pragma unroll
        for (int j = 0; j < N; j++)
            if (j < n) p[j] = (T)v[j];
    }
}

// How a row's ends are read.  FULL: vectors of channels or states are all there.  PART: where the last one is not, as many elements from
// further left in the row, shifted into place once they have come.  ONE_BY_ONE: rows too short to have them.  Scans of 24
// sequences of 12000 rows, bfloat16, 4096 channels: 246 us, 4095 channels 282, element by element 339; 15 sequences of 968 rows,
// 4800 channels, 42 states: 93, element by element 121.
enum { FULL = 0, PART = 1, ONE_BY_ONE = 2 };

// N neighbouring elements on their way to registers, held as loaded: taken apart where they are loaded, they would be waited
// for there, and a branch around a load makes them wait behind it.  ODD: some may not be there (an odd width), so each is loaded by itself,
// one that is not from the first one's place, which must be there.
template <typename T, int N, bool ODD>
struct Raw {
    static constexpr bool WORDS = !ODD && N * sizeof(T) >= 4;
    uint32_t w[WORDS ? N * sizeof(T) / 4 : N];
    __device__ float get(int j) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[j]);
        else if constexpr (!WORDS) return __builtin_bit_cast(float, w[j] << 16);
        else return __builtin_bit_cast(float, j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
    __device__ void load(const uint8_t* base, uint32_t at, int n)       // n of them are there, or none
    {
        if constexpr (WORDS) {
            __builtin_memcpy(w, base + at, sizeof(w));
        } else {
#pragma unroll
            for (int j = 0; j < N; j++) {
                const uint8_t* p = base + at + (j < n ? j : 0) * sizeof(T);
                if constexpr (sizeof(T) == 4) w[j] = *(const uint32_t*)p;
                else w[j] = *(const uint16_t*)p;
            }
        }
    }
    // Loaded whole from `shift` elements before: the first N - shift are put in their places.
    __device__ void align(int shift)
    {
        static_assert(WORDS, "");
        constexpr int WN = sizeof(w) / 4, PER = 4 / sizeof(T);
        if constexpr (PER == 2 && N == 4) {
            const uint64_t v = (w[0] | (uint64_t)w[1] << 32) >> (16 * shift);
            w[0] = (uint32_t)v;
            w[1] = (uint32_t)(v >> 32);
            return;
        }
        if (PER == 2 && shift & 1)
#pragma unroll
            for (int j = 0; j < WN; j++) w[j] = w[j] >> 16 | (j + 1 < WN ? w[j + 1] << 16 : 0);
#pragma unroll
        for (int by = 1; by < WN; by *= 2)
            if (shift & by * PER)
#pragma unroll
                for (int j = 0; j + by < WN; j++) w[j] = w[j + by];
    }
};

// v / (1 + exp(-v)).  The reciprocal is the hardware's, within 1 ulp, next to an output rounding of at least that; it has no
// denormals, so below -87.3, where the quotient is under 2^-119 in size, it is -0, as where exp(-v) overflows.
__device__ inline float silu(float v) { return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504088896341f)); }

}  // namespace icv
