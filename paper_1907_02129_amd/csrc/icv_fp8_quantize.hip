// Quantisation into e4m3 with a scale per block of 128 columns and 1 or 128 rows (icv_quantize_fp8).
//
// Memory bound: every element is read once and leaves as one byte. Sixteen lanes take a row's block of 128, 8 elements each, so
// the maximum of a row's block is four exchanges within a row of 16 lanes, and a wavefront covers four neighbouring blocks of a
// row. 12288 x 4096 with a scale a row from bfloat16 27 us, 5.6 TB/s, from float 37, 6.8 TB/s, both partly from cache (with
// other data in between 31 and 4.8 TB/s; a copy: 5.2 TB/s); 4100 deep, where rows begin anywhere, 30 and 40.
#include "icv_sequence.h"

namespace icv {

struct QuantArgs {
    const void* in;
    uint8_t* codes;
    float* scales;
    int32_t rows, depth, blocks;      // blocks of 128 columns
    int64_t in_stride, code_stride;
};

// fmaxf leaves NaN out.  Maximum over the 16 lanes of a row.
__device__ inline float row16_max(float v)
{
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x121, 0xF, 0xF, true)));
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x122, 0xF, 0xF, true)));
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x124, 0xF, 0xF, true)));
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xF, 0xF, true)));
    return v;
}

// The block's scale.  The floor keeps the quotients of a block of denormals in range.
__device__ inline float scale_of(float most)
{
    if (!(most > 0.0f)) return 1.0f;
    const float s = most / 448.0f;
    return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}

// Quotients by a scale, rounded correctly as the definition says.  For scales far from the ends of float's range:
// with r the rounded reciprocal, q = v * r and one correction by the exact remainder, q + (v - q * scale) * r, is the rounded
// quotient (Markstein's theorem), in three operations; the division that takes every case has eleven (12288 x 4096 bfloat16, four rows a wavefront: 43.4 us, 35.6 with
// this).  The step from the hardware's reciprocal to r rounds correctly for every significand but one of all ones (24 bits).
// There r is right if the hardware's value is, which a test shows; otherwise a power of two over such a scale, next to a
// tie between two codes, would be rounded to the wrong side.
struct Divider {
    float scale, r;
    bool plain;
    __device__ explicit Divider(float s) : scale(s), r(__builtin_amdgcn_rcpf(s)), plain(s > 0x1p-100f && s < 0x1p100f)
    {
        r = fmaf(fmaf(-s, r, 1.0f), r, r);
    }
    __device__ float operator()(float v) const
    {
        const float q = v * r;
        return fmaf(fmaf(-q, scale, v), r, q);
    }
};

// Eight quotients as e4m3; |v / scale| passes 448 by a rounding at most.
__device__ inline uint2 encode8(const float (&v)[8], const Divider& by)
{
    float q[8];
    if (by.plain) {
#pragma unroll
        for (int j = 0; j < 8; j++) q[j] = by(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) q[j] = v[j] / by.scale;
    }
#pragma unroll
    for (int j = 0; j < 8; j++) q[j] = q[j] > 448.0f ? 448.0f : (q[j] < -448.0f ? -448.0f : q[j]);
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// A wavefront takes R rows of four neighbouring blocks of columns.
template <typename T, int R, int ENDS>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantArgs a)
{
    const int lane = threadIdx.x & 63;
    const int32_t quads = (a.blocks + 3) / 4;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t strip = wave / quads;
    const int32_t block = (int32_t)(wave - strip * quads) * 4 + (lane >> 4);
    if (strip * R >= a.rows || block >= a.blocks) return;        // whole rows of 16 lanes
    const int32_t r0 = (int32_t)(strip * R), c = block * 128 + (lane & 15) * 8;
    const int n = a.depth - c < 0 ? 0 : (a.depth - c < 8 ? a.depth - c : 8);
    const int shift = ENDS == PART && n ? 8 - n : 0;
    float scale[R];
    Raw<T, 8, ENDS == ONE_BY_ONE> raw[R];
#pragma unroll
    for (int r = 0; r < R; r++)
        raw[r].load((const uint8_t*)((const T*)a.in + (int64_t)(r0 + r < a.rows ? r0 + r : r0) * a.in_stride + (n ? c - shift : 0)), 0, n);
#pragma unroll
    for (int r = 0; r < R; r++) {
        float v[8], m = 0.0f;
        if constexpr (ENDS == PART) raw[r].align(shift);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            v[j] = (ENDS != FULL ? j < n : n > 0) ? raw[r].get(j) : 0.0f;
            m = fmaxf(m, fabsf(v[j]));
        }
        scale[r] = scale_of(row16_max(m));
        const uint2 q = encode8(v, Divider(scale[r]));
        if (r0 + r < a.rows) *(uint2*)(a.codes + (int64_t)(r0 + r) * a.code_stride + c) = q;
    }
#pragma unroll
    for (int r = 0; r < R; r++)
        if ((lane & 15) == r && r0 + r < a.rows) a.scales[(int64_t)block * a.rows + r0 + r] = scale[r];
}

// A workgroup takes a block of 128 x 128: 16 rows at a time, 8 elements a lane, all held until the maximum is known.
template <typename T, int ENDS>
__global__ __launch_bounds__(256) void k_quantize_blocks(QuantArgs a)
{
    __shared__ float part[4];
    const int tid = threadIdx.x;
    const int32_t block = (int32_t)(blockIdx.x % a.blocks), strip = (int32_t)(blockIdx.x / a.blocks);
    const int32_t c = block * 128 + (tid & 15) * 8, row_blocks = (a.rows - 1) / 128 + 1;
    const int n = a.depth - c < 0 ? 0 : (a.depth - c < 8 ? a.depth - c : 8);
    const int shift = ENDS == PART && n ? 8 - n : 0;
    Raw<T, 8, ENDS == ONE_BY_ONE> raw[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int64_t r = (int64_t)strip * 128 + i * 16 + (tid >> 4);
        raw[i].load((const uint8_t*)((const T*)a.in + (r < a.rows ? r : a.rows - 1) * a.in_stride + (n ? c - shift : 0)), 0, n);
    }
    float m = 0.0f;
    const auto value = [&](int i, int j) { return (ENDS != FULL ? j < n : n > 0) ? raw[i].get(j) : 0.0f; };      // rows past the end: the last again
    if constexpr (ENDS == PART)
#pragma unroll
        for (int i = 0; i < 8; i++) raw[i].align(shift);
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) m = fmaxf(m, fabsf(value(i, j)));
    m = row16_max(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
    const float scale = scale_of(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    const Divider by(scale);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int64_t r = (int64_t)strip * 128 + i * 16 + (tid >> 4);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = value(i, j);
        if (r < a.rows) *(uint2*)(a.codes + r * a.code_stride + c) = encode8(v, by);
    }
    if (tid == 0) a.scales[(int64_t)block * row_blocks + strip] = scale;
}

template <typename T>
static int launch(const QuantArgs& a, int block_rows, hipStream_t s)
{
    if (block_rows == 1) {
        constexpr int R = 2;       // 12288 x 4096 bfloat16: 31.7 us; 33.6 with one row, 31.4 with four, which leaves short batches fewer wavefronts
        const int64_t waves = (int64_t)((a.blocks + 3) / 4) * ((a.rows - 1) / R + 1), n = (waves + 3) / 4;
        if (too_many(n, 256)) return ICV_ERR_UNSUPPORTED;
        if (a.depth % 8 == 0) k_quantize_rows<T, R, FULL><<<(uint32_t)n, 256, 0, s>>>(a);
        else if (a.depth >= 8) k_quantize_rows<T, R, PART><<<(uint32_t)n, 256, 0, s>>>(a);
        else k_quantize_rows<T, R, ONE_BY_ONE><<<(uint32_t)n, 256, 0, s>>>(a);
    } else {
        const int64_t n = (int64_t)a.blocks * ((a.rows - 1) / 128 + 1);
        if (too_many(n, 256)) return ICV_ERR_UNSUPPORTED;
        if (a.depth % 8 == 0) k_quantize_blocks<T, FULL><<<(uint32_t)n, 256, 0, s>>>(a);
        else if (a.depth >= 8) k_quantize_blocks<T, PART><<<(uint32_t)n, 256, 0, s>>>(a);
        else k_quantize_blocks<T, ONE_BY_ONE><<<(uint32_t)n, 256, 0, s>>>(a);
    }
    ICV_HIP_CHECK(hipGetLastError());
    return ICV_OK;
}

}  // namespace icv

extern "C" int icv_quantize_fp8(const icv_quantize_params* p, const void* input, void* codes, float* scales, void* stream)
{
    using namespace icv;
    if (!p || p->rows < 0 || p->depth < 1 || p->depth > INT32_MAX - 127 || (p->block_rows != 1 && p->block_rows != 128))
        return ICV_ERR_INVALID_ARG;
    if (p->dtype == ICV_U8I8) return ICV_ERR_UNSUPPORTED;
    if (p->dtype != ICV_F32 && p->dtype != ICV_BF16) return ICV_ERR_INVALID_ARG;
    const int32_t blocks = (p->depth + 127) / 128;
    if (p->in_row_stride && p->in_row_stride < p->depth) return ICV_ERR_INVALID_ARG;
    if (p->code_row_stride && (p->code_row_stride % 16 != 0 || p->code_row_stride < (int64_t)blocks * 128)) return ICV_ERR_INVALID_ARG;
    if (p->rows == 0) return ICV_OK;
    if (!input || !codes || !scales || misaligned(input, p->dtype == ICV_F32 ? 4 : 2) || misaligned(codes, 16) || misaligned(scales, 4) ||
        input == codes)
        return ICV_ERR_INVALID_ARG;
    QuantArgs a = {input, (uint8_t*)codes, scales, p->rows, p->depth, blocks,
                   p->in_row_stride ? p->in_row_stride : p->depth, p->code_row_stride ? p->code_row_stride : (int64_t)blocks * 128};
    hipStream_t s = (hipStream_t)stream;
    return p->dtype == ICV_F32 ? launch<float>(a, p->block_rows, s) : launch<__bf16>(a, p->block_rows, s);
}
