"""e4m3 operators where a rounding or a lost product shows: quotients next to ties, products of whole numbers, the size of
all outputs' errors together."""
import pytest
import torch

import sequence_reference as ref
from paper_1907_02129_amd import binding as icv
from test_gpu_fp8 import KERNELS, TYPE, gen, operands, quantized, same_codes

pytestmark = pytest.mark.gpu


def test_quotients_by_scales_just_under_a_power_of_two():
    """A scale whose 24 bits are all set, (2 - 2^-23) 2^k: its reciprocal lies next to the middle of two floats, and 2^(k - 9)
    over it next to a tie between two codes."""
    largest = torch.tensor(0x445FFFFF, dtype=torch.int32).view(torch.float32)             # 448 (2 - 2^-23), rounded
    assert (largest / 448.0).view(torch.int32) == 0x3FFFFFFF
    x = torch.zeros(40, 384)
    for i in range(40):
        x[i, 0], x[i, 128], x[i, 256] = largest, -largest, largest
        x[i, 1:100] = torch.arange(1, 100) * 2.0 ** -9
        x[i, 129:200] = -torch.exp2(-torch.arange(1, 72) / 4).to(torch.bfloat16)
        x[i, 257:380] = torch.exp2(torch.arange(123) % 24 - 16.0)
        x[i] *= 2.0 ** (i - 20)
    for block_rows in (1, 128):
        for rows in (x, x[20:21]):
            codes, scales = quantized(rows, block_rows, "f32")
            want, want_scales = ref.quantize(rows, block_rows)
            assert torch.equal(scales.cpu(), want_scales)
            same_codes(codes, want)


def product(a, sa, b, sb, out, kernel):
    M, N = a.shape[0], b.shape[0]
    p = icv.make_matmul_params(M, N, a.shape[1], out)
    p.out_type |= kernel << 8
    y = torch.empty(M, N, dtype=TYPE[out], device="cuda")
    icv.matmul_fp8(p, a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, y)
    torch.cuda.synchronize()
    return y.cpu()


ALL = [(k, o) for k in ("auto", *KERNELS) for o in ("bf16", "f32") if (k, o) != ("256", "f32")]


@pytest.mark.parametrize("kernel,out", ALL)
def test_products_of_whole_numbers_are_exact(kernel, out):
    """Operands of 0 to 3 in size: a product is at most 9 and at least 1, so that none of eight loses a bit (13 below the
    largest's first), a block's sum at most 1152; times scales of 1/4 to 2 and of 1/2 to 4 all sums are multiples of 1/8 below 2^20
    (1152 * 8 * 60 blocks): every addition is exact, in any order, and the output has to be the whole sum rounded once."""
    hook = KERNELS.get(kernel, 0)
    for M, N, K in ((37, 150, 60 * 128), (1, 17, 128), (300, 270, 5 * 128), (130, 257, 1100)):
        g = gen(M + K)
        kb = -(-K // 128)

        def codes(rows):
            v = torch.zeros(rows, kb * 128)
            v[:, :K] = torch.randint(-3, 4, (rows, K), generator=g).float()
            return v.to(torch.float8_e4m3fn)

        a, b = codes(M), codes(N)
        sa, sb = (torch.exp2(torch.randint(-1, 3, (kb, n), generator=g).float()) / 2 ** (i == 0) for i, n in ((0, M), (1, -(-N // 128))))
        A = a.double() * sa.double().t().repeat_interleave(128, 1)
        B = b.double() * sb.double().t().repeat_interleave(128, 1).repeat_interleave(128, 0)[:N]
        want = A @ B.t()
        assert want.abs().max() < 2 ** 20 and torch.equal(want * 8, (want * 8).round())
        assert torch.equal(product(a, sa, b, sb, out, hook), want.to(TYPE[out]))


@pytest.mark.parametrize("kernel", ["auto", *KERNELS])
@pytest.mark.parametrize("M,N,K", [(40, 500, 8000), (160, 260, 1500)])
def test_error_of_all_outputs_together(kernel, M, N, K):
    """Root mean square of a bfloat16 product's errors: the output's own rounding (which is computed) and, independent of it, what
    the e4m3 instruction cuts.  Of every 8 products it cuts 7, each by less than 2^-13 of the largest one's leading bit, towards zero, so with
    the product's sign, which is as often one as the other here: the mean square is at most 7 * 2^-26 times the sum over all
    eights of their largest product squared.  The cross terms' sum over n outputs has a standard deviation of at most 2 sqrt(n) times
    both parts, so 1/sqrt(n) of the sum of the squares; five of these are allowed.  The sums in float add at most 2^-23 of the sizes' sum for each
    of the 16 eights of a block and, as the sums over blocks grow to the output with random signs, 2^-23 of the output twice per
    block (a multiply-add, and an addition between wavefronts).  A product left out in every output is at least three times the bound."""
    a, sa, b, sb, _ = operands(M, N, K, M + K)
    got = product(a, sa, b, sb, "bf16", KERNELS.get(kernel, 0)).double()
    A = a.double() * sa.double().t().repeat_interleave(128, 1)
    B = b.double() * sb.double().t().repeat_interleave(128, 1).repeat_interleave(128, 0)[:N]
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    cut = torch.zeros(M, N, dtype=torch.float64)
    for k in range(0, A.shape[1], 8):
        cut += (A[:, None, k:k + 8] * B[None, :, k:k + 8]).abs().amax(2) ** 2
    ms = lambda v: (v * v).mean()  # noqa: E731
    rounding, cuts = ms(want.to(torch.bfloat16).double() - want), 7 * 2.0 ** -26 * cut.mean()
    sums = 2.0 ** -23 * (16 * ms(size).sqrt() + 2 * sa.shape[0] * ms(want).sqrt())
    bound = ((rounding + cuts) * (1 + 5 / (M * N) ** 0.5)).sqrt() + sums
    assert ((A[:, :1] * B[None, :, 0]) ** 2).mean().sqrt() > 3 * bound
    off = ms(got - want).sqrt()
    print("%s %dx%dx%d: %.3g of the outputs' size, bound %.3g" % (kernel, M, N, K, off / ms(want).sqrt(), bound / ms(want).sqrt()))
    assert off <= bound
