// Product of e4m3 matrices with a scale per block of 128 (icv_matmul_fp8).
//
// out[m][n] = sum over blocks k of sa[k][m] * sb[k][n / 128] * (a[m] . b[n] over the block's 128 columns).  The inner
// products run on the tensor cores, one 16 x 16 x 128 instruction per block; a block's sum is scaled and added to the
// float accumulator on the vector ALU, one multiply-add per output and block (the two scales' product is the same for
// the 4 outputs that a lane holds, which are neighbouring columns of one row).
#include "icv_internal.h"

namespace icv {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct MatmulArgs {
    const uint8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    int32_t rows, cols, blocks, col_blocks;
    int64_t as, bs, os;
};

// Eight codes as bfloat16.
__device__ inline bf16x8_t widen(int lo, int hi)
{
    const bf16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true)};
    return bf16x8_t{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

// One block's product of 16 rows of b (the instruction's rows) and 16 rows of a (its columns).  A lane holds 32 of a row's 128
// codes; which 32 does not matter as long as both operands agree.  Result: lane l, register r: column 4 * (l / 16) + r of
// the output, row l % 16.
//
// The e4m3 instruction adds 8 products at a time, each cut to 13 bits below the largest one's leading bit (measured:
// 2^16 + 15 gives 2^16 + 8, in the same 8 only); the eights are added in float.  Over random operands that is 1.5e-5 of the
// result, far below a bfloat16 output's rounding (2^-9) but not below a float's.  EXACT, for float outputs, widens the codes to bfloat16
// (no rounding) and uses that type's instruction, whose products and sums are float's, at half the rate.
template <bool EXACT>
__device__ inline f32x4_t block_product(i32x8_t b, i32x8_t a)
{
    const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (!EXACT) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, zero, 0, 0, 0, 0, 0, 0);
    } else {
        f32x4_t c = zero;
#pragma unroll
        for (int i = 0; i < 4; i++)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(b[2 * i], b[2 * i + 1]), widen(a[2 * i], a[2 * i + 1]), c, 0, 0, 0);
        return c;
    }
}

// 32 of the 128 codes at `row`: 16 from each half, so that the 4 lanes of a row read 64 bytes side by side.
__device__ inline i32x8_t load_codes(const uint8_t* row, int quarter)
{
    const int4 lo = *(const int4*)(row + 16 * quarter), hi = *(const int4*)(row + 64 + 16 * quarter);
    return i32x8_t{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
}

template <typename OUT>
__device__ inline void store_out(const MatmulArgs& g, int64_t m, int32_t n, f32x4_t v)
{
    OUT* o = (OUT*)g.out + m * g.os + n;
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (n + j < g.cols) o[j] = (OUT)(v[j] + (g.bias ? g.bias[n + j] : 0.0f));
}

// 16 columns x 16 * MB rows per workgroup, the blocks of the reduction dealt to its wavefronts, whose sums meet in LDS.
template <typename OUT, int MB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_matmul_split(MatmulArgs g)
{
    __shared__ f32x4_t part[WAVES][MB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, quarter = lane >> 4;
    const int32_t col_tiles = (g.cols + 15) / 16;
    const int32_t n0 = (int32_t)(blockIdx.x % col_tiles) * 16;
    const int64_t m0 = (int64_t)(blockIdx.x / col_tiles) * (16 * MB);
    const uint8_t* bp = g.b + (int64_t)(n0 + row < g.cols ? n0 + row : g.cols - 1) * g.bs;
    const uint8_t* ap[MB];
    int64_t m[MB];
#pragma unroll
    for (int i = 0; i < MB; i++) {
        m[i] = m0 + 16 * i + row < g.rows ? m0 + 16 * i + row : g.rows - 1;      // rows past the end repeat the last
        ap[i] = g.a + m[i] * g.as;
    }
    f32x4_t acc[MB];
#pragma unroll
    for (int i = 0; i < MB; i++) acc[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int32_t k = wave; k < g.blocks; k += WAVES) {
        const i32x8_t b = load_codes(bp + (int64_t)k * 128, quarter);
        const float sb = g.sb[(int64_t)k * g.col_blocks + n0 / 128];
#pragma unroll
        for (int i = 0; i < MB; i++) {
            const f32x4_t p = block_product<std::is_same<OUT, float>::value>(b, load_codes(ap[i] + (int64_t)k * 128, quarter));
            const float scale = sb * g.sa[(int64_t)k * g.rows + m[i]];
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = fmaf(p[j], scale, acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < MB; i++) part[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MB; i += WAVES) {
        f32x4_t v = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < WAVES; w++) v += part[w][i][lane];
        if (m0 + 16 * i + row < g.rows) store_out<OUT>(g, m0 + 16 * i + row, n0 + 4 * quarter, v);
    }
}

template <typename OUT>
static int launch(const MatmulArgs& g, hipStream_t s)
{
    constexpr int MB = 4, WAVES = 4;
    const int64_t n = (int64_t)((g.cols + 15) / 16) * (((int64_t)g.rows + 16 * MB - 1) / (16 * MB));
    if (n > INT32_MAX) return ICV_ERR_INVALID_ARG;
    k_matmul_split<OUT, MB, WAVES><<<(uint32_t)n, 64 * WAVES, 0, s>>>(g);
    ICV_HIP_CHECK(hipGetLastError());
    return ICV_OK;
}

}  // namespace icv

extern "C" int icv_matmul_fp8(const icv_matmul_params* p, const void* a, const float* a_scales, const void* b,
                              const float* b_scales, const float* bias, void* out, void* stream)
{
    using namespace icv;
    if (!p || p->rows < 0 || p->cols < 1 || p->depth < 1 || p->depth > INT32_MAX - 127 || p->cols > INT32_MAX - 255) return ICV_ERR_INVALID_ARG;
    if (p->out_type != ICV_OUT_ACC && p->out_type != ICV_OUT_BF16) return ICV_ERR_INVALID_ARG;
    const int32_t blocks = (p->depth + 127) / 128;
    for (int32_t r : {p->a_row_stride, p->b_row_stride})
        if (r && (r % 16 != 0 || r < (int64_t)blocks * 128)) return ICV_ERR_INVALID_ARG;
    if (p->out_row_stride && p->out_row_stride < p->cols) return ICV_ERR_INVALID_ARG;
    if (p->rows == 0) return ICV_OK;
    if (!a || !a_scales || !b || !b_scales || !out) return ICV_ERR_INVALID_ARG;
    const auto off = [](const void* q, uintptr_t bytes) { return ((uintptr_t)q & (bytes - 1)) != 0; };
    if (off(a, 16) || off(b, 16) || off(a_scales, 4) || off(b_scales, 4) || off(bias, 4) || off(out, p->out_type == ICV_OUT_ACC ? 4 : 2))
        return ICV_ERR_INVALID_ARG;
    MatmulArgs g = {(const uint8_t*)a, (const uint8_t*)b, a_scales, b_scales, bias, out, p->rows, p->cols, blocks, (p->cols + 127) / 128,
                    p->a_row_stride ? p->a_row_stride : (int64_t)blocks * 128, p->b_row_stride ? p->b_row_stride : (int64_t)blocks * 128,
                    p->out_row_stride ? p->out_row_stride : p->cols};
    return p->out_type == ICV_OUT_ACC ? launch<float>(g, (hipStream_t)stream) : launch<__bf16>(g, (hipStream_t)stream);
}
