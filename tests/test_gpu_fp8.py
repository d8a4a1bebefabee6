"""Quantisation into e4m3 and the product of e4m3 matrices on the GPU, against their definitions (sequence_reference)."""
import pytest
import torch

import sequence_reference as ref
from paper_1907_02129_amd import binding as icv

pytestmark = pytest.mark.gpu
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def same_codes(got, want):
    """Equal codes; a NaN of either sign counts as one."""
    a, b = got.cpu().view(torch.float8_e4m3fn), want
    nan = b.float().isnan()
    assert torch.equal(a.float().isnan(), nan)
    assert torch.equal(a.view(torch.uint8)[~nan], b.view(torch.uint8)[~nan])


def quantized(x, block_rows, dtype, pad=0, code_pad=0):
    M, K = x.shape
    kb = -(-K // 128)
    wide = torch.full((M, K + pad), float("nan"), dtype=TYPE[dtype])
    wide[:, pad:] = x
    room = torch.full((M, 128 * kb + code_pad), 77, dtype=torch.uint8, device="cuda")
    codes, scales = room[:, :128 * kb], torch.full((kb, -(-M // block_rows)), -1.0, device="cuda")
    p = icv.make_quantize_params(M, K, dtype, block_rows, K + pad, 128 * kb + code_pad)
    icv.quantize_fp8(p, wide.cuda()[:, pad:], codes, scales)
    torch.cuda.synchronize()
    assert (room[:, 128 * kb:] == 77).all()
    return codes, scales


@pytest.mark.parametrize("rows", [1, 2, 5, 127, 128, 129, 300])
@pytest.mark.parametrize("depth", [1, 7, 8, 9, 12, 13, 14, 15, 128, 129, 250, 515, 1024])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_sizes(rows, depth, block_rows):
    for dtype in ("bf16", "f32"):
        x = (torch.randn(rows, depth, generator=gen(rows + depth)) * torch.randn(rows, 1, generator=gen(depth)).exp()).to(TYPE[dtype])
        codes, scales = quantized(x, block_rows, dtype, pad=(rows + depth) % 3, code_pad=16 * (rows % 2))
        want, want_scales = ref.quantize(x, block_rows)
        assert torch.equal(scales.cpu(), want_scales)
        same_codes(codes.contiguous(), want)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_every_range(block_rows):
    """Blocks of zeros, of denormals, of the largest values, ties, and NaN and infinite elements."""
    g = gen(3)
    x = torch.randn(256, 512, generator=g)
    x[0] = 0
    x[1, :128] = 0
    x[2] *= 1e-39
    x[3] *= 1e-44
    x[4] *= 1e37
    x[5] = 0
    x[5, 3] = 1e-45
    x[6, :128] = torch.arange(128) / 8            # exact quotients and ties
    x[6, 0] = 448
    if block_rows == 1:
        x[7, 5], x[7, 200], x[7, 300], x[7, 301] = float("nan"), float("inf"), -float("inf"), float("nan")
        x[8, :] = float("nan")
    else:
        x[:128], x[128, 5], x[200, 130] = 0, float("nan"), -float("inf")
    codes, scales = quantized(x, block_rows, "f32")
    want, want_scales = ref.quantize(x, block_rows)
    assert torch.equal(scales.cpu(), want_scales)
    same_codes(codes, want)


def operands(M, N, K, seed, far=False):
    g = gen(seed)
    kb = -(-K // 128)

    def codes(rows):
        v = torch.zeros(rows, 128 * kb)
        v[:, :K] = (torch.randn(rows, K, generator=g) * 100).clamp(-448, 448)
        return v.to(torch.float8_e4m3fn)

    def scales(n):
        e = torch.rand(kb, n, generator=g) * 2 + 0.5
        return e * torch.exp2(torch.randint(-20, 20, (kb, n), generator=g).float()) if far else e

    return codes(M), scales(M), codes(N), scales(-(-N // 128)), torch.randn(N, generator=g)


def wide_codes(c, pad):
    full = torch.full((c.shape[0], c.shape[1] + pad), 0x7F, dtype=torch.uint8)      # NaN beside the matrix
    full[:, :c.shape[1]] = c.view(torch.uint8)
    return full.cuda()[:, :c.shape[1]]


KERNELS = {"256": 1, "128": 2, "128x64": 3, "64": 4, "32x64": 5, "split": 6}      # test hooks


def matmul_case(M, N, K, out, bias, seed, pad=0, far=False, kernel=0):
    a, sa, b, sb, bs = operands(M, N, K, seed, far)
    kb = a.shape[1]
    t = TYPE[out]
    room = torch.full((M + 2, N + pad), 3.0, dtype=t, device="cuda")
    y = room[1:M + 1, :N]
    p = icv.make_matmul_params(M, N, K, out, kb + 16 * pad, kb + 32 * pad, N + pad)
    p.out_type |= kernel << 8
    icv.matmul_fp8(p, wide_codes(a, 16 * pad), sa.cuda(), wide_codes(b, 32 * pad), sb.cuda(), bs.cuda() if bias else None, y)
    torch.cuda.synchronize()
    want, bound = ref.matmul(a, sa, b, sb, bs if bias else None, t)
    ref.check("out", y, want, bound)
    assert (room[0] == 3).all() and (room[M + 1] == 3).all() and (room[:, N:] == 3).all()


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 65, 127, 200, 300])
@pytest.mark.parametrize("N,K", [(1, 1), (15, 128), (17, 129), (128, 256), (130, 700), (257, 1024)])
def test_matmul_sizes(M, N, K):
    for out, bias in (("bf16", True), ("f32", False)):
        matmul_case(M, N, K, out, bias, M + N + K, pad=(M + N) % 3)


@pytest.mark.parametrize("M,N,K", [(5, 1000, 4000), (129, 640, 2048), (513, 1100, 1500), (1024, 1024, 512), (1030, 2050, 384), (2048, 512, 128)])
def test_matmul_larger(M, N, K):
    matmul_case(M, N, K, "f32", True, M + N, pad=1)
    matmul_case(M, N, K, "bf16", False, M + K)


@pytest.mark.parametrize("kernel,out", [(k, o) for k in KERNELS for o in ("bf16", "f32") if (k, o) != ("256", "f32")])
def test_matmul_every_kernel(kernel, out):
    """Every kernel on sizes that are no multiple of its tile, with reductions of one block, of a few and of many."""
    for M, N, K in ((1, 1, 5), (300, 270, 128), (70, 300, 256), (257, 130, 1100), (129, 600, 700), (31, 65, 3000), (520, 513, 384)):
        matmul_case(M, N, K, out, True, M + N + K, pad=M % 2, kernel=KERNELS[kernel])


@pytest.mark.parametrize("M,N,K,out", [(3000, 5000, 128, "bf16"), (2900, 3100, 1100, "bf16"), (2900, 3100, 1100, "f32"),
                                       (1100, 2050, 700, "bf16"), (500, 2050, 384, "bf16"), (100, 2050, 3000, "bf16"), (13, 1000, 8000, "bf16")])
def test_matmul_the_kernels_own_sizes(M, N, K, out):
    matmul_case(M, N, K, out, True, M + N + K, pad=M % 2)


def test_matmul_scales_of_very_different_size():
    matmul_case(70, 300, 1024, "f32", True, 5, far=True)
    matmul_case(600, 520, 1024, "f32", False, 6, far=True)


def test_matmul_nan_codes_and_infinite_scales_stay_in_their_rows():
    for M, N, K in ((40, 200, 300), (700, 520, 600)):
        a, sa, b, sb, _ = operands(M, N, K, 7)
        a.view(torch.uint8)[7, 3] = 0x7F
        b.view(torch.uint8)[150, 140] = 0xFF
        sa[1, 20] = float("inf")
        y = torch.empty(M, N, device="cuda")
        icv.matmul_fp8(icv.make_matmul_params(M, N, K, "f32"), a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, y)
        got = y.cpu()
        keep = torch.ones(M, N, dtype=torch.bool)
        keep[7], keep[20], keep[:, 150] = False, False, False
        assert got[7].isnan().all() and got[:, 150].isnan().all() and not got[20].isfinite().any() and got[keep].isfinite().all()


def test_matmul_past_32_bit_offsets():
    M, N, K, stride = 4200, 40, 256, 1 << 20
    a, sa, b, sb, _ = operands(M, N, K, 8)
    room = torch.empty(M * stride, dtype=torch.uint8, device="cuda")
    ad = torch.as_strided(room, (M, K), (stride, 1))
    ad.copy_(a.view(torch.uint8))
    out = torch.as_strided(room.view(torch.float32), (M, N), (stride // 4, 1), 1024)
    icv.matmul_fp8(icv.make_matmul_params(M, N, K, "f32", a_row_stride=stride, out_row_stride=stride // 4), ad, sa.cuda(), b.cuda(), sb.cuda(),
                   None, out)
    want, bound = ref.matmul(a, sa, b, sb, None, torch.float32)
    ref.check("out", out, want, bound)


@pytest.mark.parametrize("M", [3, 200])
def test_quantize_and_product_in_a_replayed_graph(M):
    """The path of a projection: activations quantised and multiplied, captured and replayed with new activations."""
    N, K = 300, 500
    g = gen(9)
    w = torch.randn(N, K, generator=g)
    wq, ws = quantized(w, 128, "f32")
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.zeros(M, 512, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(4, M, device="cuda")
    y = torch.zeros(M, N, device="cuda")
    pq, pm = icv.make_quantize_params(M, K), icv.make_matmul_params(M, N, K, "f32")

    def go():
        icv.quantize_fp8(pq, x, codes, scales)
        icv.matmul_fp8(pm, codes, scales, wq, ws, None, y)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        go()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    wc, wsc = ref.quantize(w, 128)
    for _ in range(4):
        xn = torch.randn(M, K, generator=g).bfloat16()
        x.copy_(xn)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        ac, sc = ref.quantize(xn, 1)
        want, bound = ref.matmul(ac, sc, wc, wsc, None, torch.float32)
        ref.check("out", got, want, bound)
        go()
        assert torch.equal(y, got)


def test_a_layer_of_them_together():
    """Projection, convolution, scan with gate, projection, as a state space layer runs them on a packed batch: every
    stage against the definition on the stage's own inputs, views of the stage before taken as they lie."""
    tokens, width, ch, N = 150, 200, 136, 16
    g = gen(10)
    start = [0, 90, 91, 150]
    rows = ref.spans(3, tokens, start)
    seq = icv.make_sequences(3, tokens, torch.tensor(start, dtype=torch.int32, device="cuda"))
    x = torch.randn(tokens, width, generator=g).bfloat16()
    w_in, w_out = torch.randn(2 * ch, width, generator=g) / 14, torch.randn(width, ch, generator=g) / 12

    def project(v, w, wq, ws, wr, cols):
        K = v.shape[1]
        kb = -(-K // 128)
        codes, scales = torch.empty(tokens, 128 * kb, dtype=torch.uint8, device="cuda"), torch.empty(kb, tokens, device="cuda")
        icv.quantize_fp8(icv.make_quantize_params(tokens, K, in_row_stride=v.stride(0)), v, codes, scales)
        y = torch.empty(tokens, cols, dtype=torch.bfloat16, device="cuda")
        icv.matmul_fp8(icv.make_matmul_params(tokens, cols, K), codes, scales, wq, ws, None, y)
        ac, sc = ref.quantize(v.cpu(), 1)
        want, bound = ref.matmul(ac, sc, *wr, None, torch.bfloat16)
        ref.check("projection", y, want, bound)
        return y

    xz = project(x.cuda(), w_in, *quantized(w_in, 128, "f32"), ref.quantize(w_in, 128), 2 * ch)
    filt, cb = torch.randn(ch, 4, generator=g).bfloat16(), torch.randn(ch, generator=g)
    cs, ss = torch.zeros(3, 3, ch, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, ch, N, device="cuda")
    u = torch.empty(tokens, ch, dtype=torch.bfloat16, device="cuda")
    icv.causal_conv1d(icv.make_causal_conv_params(ch, 4, in_row_stride=2 * ch, state_slots=3), seq, xz[:, :ch], filt.cuda(), cb.cuda(), cs, u)
    slots = [0, 1, 2]
    want, bound, st = ref.causal_conv(xz[:, :ch].cpu(), filt, cb, torch.zeros(3, 3, ch), rows, slots, slots, True, torch.zeros(tokens, ch), torch.bfloat16)
    ref.check("convolution", u, want, bound)
    assert torch.equal(cs.cpu().double(), st)
    dt, B, C = (torch.randn(tokens, w, generator=g).bfloat16() for w in (ch, N, N))
    A, D = -torch.rand(ch, N, generator=g) * 16, torch.randn(ch, generator=g)
    y = torch.empty_like(u)
    p = icv.make_scan_params(ch, N, z_row_stride=2 * ch, state_slots=3)
    icv.selective_scan(p, seq, u, dt.cuda(), A.cuda(), B.cuda(), C.cuda(), D.cuda(), xz[:, ch:], None, ss, y)
    want, bound, st, sb = ref.selective_scan(u.cpu(), dt, A, B, C, D, xz[:, ch:].cpu(), None, torch.zeros(3, ch, N), rows, slots, slots, 1, True,
                                             torch.zeros(tokens, ch), torch.bfloat16)
    ref.check("scan", y, want, bound)
    ref.check("state", ss, st, sb)
    project(y, w_out, *quantized(w_out, 128, "f32"), ref.quantize(w_out, 128), width)
