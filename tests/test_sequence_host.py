"""What the operators on sequences and in 8-bit floating point refuse, and their sizes: host logic only, no GPU."""
import ctypes
import os
import re

import pytest
import torch

from paper_1907_02129_amd import binding as icv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ADDRESS = 1 << 20          # never read: every call here is refused or has nothing to do
BAD, UNSUPPORTED, OK = icv.ICV_ERR_INVALID_ARG, icv.ICV_ERR_UNSUPPORTED, icv.ICV_OK


@pytest.fixture(scope="module")
def lib():
    return icv.load_library()


@pytest.mark.parametrize("name", ["icv_sequences", "icv_causal_conv_params", "icv_scan_params", "icv_scan_tensors",
                                  "icv_quantize_params", "icv_matmul_params"])
def test_structs_match_the_header(name):
    header = open(os.path.join(ROOT, "include", "icv.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), header, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    size = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64}
    want = []
    for decl in body.split(";"):
        decl = decl.replace("const ", "").strip()
        if decl:
            kind, rest = decl.split(None, 1)
            want += [(n.strip(), ctypes.c_void_p if "*" in kind else size[kind]) for n in rest.split(",")]
    fields = getattr(icv, name)._fields_
    assert [(n.rstrip("_"), t) for n, t in fields] == want


def seq(count=2, tokens=8, **kw):
    s = icv.icv_sequences(count, tokens)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def conv(lib, s=None, pointers=None, **kw):
    p = icv.make_causal_conv_params(16, 4)
    for k, v in kw.items():
        setattr(p, k, v)
    at = {"input": ADDRESS, "filter": ADDRESS + 4096, "bias": ADDRESS + 8192, "state": ADDRESS + 12288, "output": ADDRESS + 16384}
    at.update(pointers or {})
    return lib.icv_causal_conv1d(p, seq() if s is None else s, *at.values(), None)


def scan(lib, s=None, pointers=None, workspace=ADDRESS, **kw):
    p = icv.make_scan_params(16, 16)
    for k, v in kw.items():
        setattr(p, k, v)
    t = icv.icv_scan_tensors(*(ADDRESS + 65536 * (i + 1) for i in range(10)))
    for k, v in (pointers or {}).items():
        setattr(t, k, v)
    return lib.icv_selective_scan(p, seq() if s is None else s, t, workspace, None)


@pytest.mark.parametrize("call", [conv, scan])
def test_sequences_that_make_no_sense_are_refused(lib, call):
    for s in (seq(-1, 8), seq(2, -1), seq(3, 8), seq(2, 8, start=ADDRESS + 2), seq(2, 8, length=ADDRESS + 1),
              seq(2, 8, from_=ADDRESS + 3), seq(2, 8, to=ADDRESS + 2)):
        assert call(lib, s) == BAD
    for s in (seq(0, 8), seq(2, 0), seq(0, 0)):
        assert call(lib, s) == OK
    assert call(lib, seq(1, 2 ** 31 - 1)) == UNSUPPORTED
    p = icv.make_causal_conv_params(16, 4)
    assert lib.icv_causal_conv1d(p, None, ADDRESS, ADDRESS, None, None, ADDRESS + 64, None) == BAD


@pytest.mark.parametrize("kw", [dict(channels=0), dict(channels=-3), dict(taps=0), dict(taps=9), dict(silu=2), dict(dtype=7),
                                dict(in_row_stride=15), dict(out_row_stride=15), dict(in_row_stride=-16), dict(state_slots=-1),
                                dict(state_slot_stride=47), dict(state_slot_stride=-48)])
def test_convolutions_that_make_no_sense_are_refused(lib, kw):
    assert conv(lib, **kw) == BAD


def test_convolution_pointers_are_checked(lib):
    for name in ("input", "filter", "output"):
        assert conv(lib, pointers={name: None}) == BAD
    for name in ("input", "filter", "state", "output"):
        assert conv(lib, pointers={name: ADDRESS + 1}) == BAD
        assert conv(lib, pointers={name: ADDRESS + 2}, dtype=icv.ICV_F32) == BAD
    assert conv(lib, pointers={"bias": ADDRESS + 2}) == BAD
    assert conv(lib, pointers={"output": ADDRESS}) == BAD
    assert conv(lib, dtype=icv.ICV_U8I8) == UNSUPPORTED
    assert lib.icv_causal_conv1d(None, seq(), ADDRESS, ADDRESS, None, None, ADDRESS, None) == BAD


@pytest.mark.parametrize("kw", [dict(channels=0), dict(states=0), dict(groups=0), dict(groups=3), dict(softplus=2), dict(softplus=-1),
                                dict(dtype=-1), dict(x_row_stride=15), dict(dt_row_stride=1), dict(b_row_stride=15), dict(c_row_stride=8),
                                dict(z_row_stride=-1), dict(out_row_stride=3), dict(state_slots=-2), dict(state_slot_stride=255)])
def test_scans_that_make_no_sense_are_refused(lib, kw):
    assert scan(lib, **kw) == BAD


def test_scan_pointers_are_checked(lib):
    for name in ("x", "dt", "A", "B", "C", "out"):
        assert scan(lib, pointers={name: None}) == BAD
    for name in ("x", "dt", "B", "C", "z", "out"):
        assert scan(lib, pointers={name: ADDRESS + 1}) == BAD
    for name in ("A", "D", "dt_bias", "state"):
        assert scan(lib, pointers={name: ADDRESS + 2}) == BAD
    at = ADDRESS + 65536
    assert scan(lib, pointers={"x": at, "out": at}, x_row_stride=32) == BAD            # over x at another stride
    assert scan(lib, pointers={"B": at * 4, "out": at * 4}) == BAD
    assert scan(lib, states=65) == UNSUPPORTED and scan(lib, dtype=icv.ICV_U8I8) == UNSUPPORTED
    for name in ("x", "dt", "b", "c", "z", "out"):
        assert scan(lib, **{name + "_row_stride": 1 << 24}) == UNSUPPORTED
    for hook, states in ((4, 16), (2, 4), (2, 33), (3, 17), (256 + 1, 16)):              # test hooks that no kernel answers to
        assert scan(lib, softplus=hook << 8, states=states) == UNSUPPORTED
    p = icv.make_scan_params(16, 16)
    assert lib.icv_selective_scan(p, seq(), None, None, None) == BAD
    assert lib.icv_selective_scan(None, seq(), icv.icv_scan_tensors(), None, None) == BAD


def test_scan_workspace(lib):
    p = icv.make_scan_params(64, 16)
    size = lambda s, q=p: lib.icv_selective_scan_workspace_bytes(q, s)  # noqa: E731
    assert size(seq(4, 4)) == 0 and size(seq(0, 8)) == 0 and size(seq(8, 64)) == 0
    assert size(seq(3, 8)) == 0 and size(None) == 0 and size(seq(1, 1 << 20), None) == 0
    long = seq(1, 1 << 15)
    need = size(long)
    assert need > 0 and need % 4 == 0
    for bad in (None, ADDRESS + 4):
        assert scan(lib, long, workspace=bad, channels=64) == BAD
    # whatever cuts the sequences, there is room for a state and a step sum of every piece
    assert need % (4 * 64 * 17) == 0
    many = icv.make_scan_params(1 << 16, 16)
    assert size(seq(64, 64 * 4096), many) == 0


def quantize(lib, pointers=None, **kw):
    p = icv.make_quantize_params(4, 300)
    for k, v in kw.items():
        setattr(p, k, v)
    at = {"input": ADDRESS, "codes": ADDRESS + 4096, "scales": ADDRESS + 8192}
    at.update(pointers or {})
    return lib.icv_quantize_fp8(p, *at.values(), None)


def matmul(lib, pointers=None, **kw):
    p = icv.make_matmul_params(4, 20, 300)
    for k, v in kw.items():
        setattr(p, k, v)
    at = {n: ADDRESS + 4096 * i for i, n in enumerate(("a", "a_scales", "b", "b_scales", "bias", "out"))}
    at.update(pointers or {})
    return lib.icv_matmul_fp8(p, *at.values(), None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(depth=0), dict(depth=2 ** 31 - 1), dict(block_rows=0), dict(block_rows=64), dict(dtype=5),
                                dict(in_row_stride=299), dict(code_row_stride=256), dict(code_row_stride=392), dict(code_row_stride=-384)])
def test_quantisations_that_make_no_sense_are_refused(lib, kw):
    assert quantize(lib, **kw) == BAD


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(cols=0), dict(depth=0), dict(depth=2 ** 31 - 1), dict(a_row_stride=368), dict(a_row_stride=392),
                                dict(b_row_stride=383), dict(out_row_stride=19), dict(out_type=icv.ICV_OUT_U8), dict(out_type=9),
                                dict(out_type=-1)])
def test_products_that_make_no_sense_are_refused(lib, kw):
    assert matmul(lib, **kw) == BAD


def test_pointers_of_the_8_bit_operators_are_checked(lib):
    for name, odd in (("input", 1), ("codes", 8), ("scales", 2)):
        assert quantize(lib, {name: None}) == BAD and quantize(lib, {name: ADDRESS + odd}) == BAD
    assert quantize(lib, dtype=icv.ICV_U8I8) == UNSUPPORTED and quantize(lib, rows=0) == OK
    for name, odd in (("a", 8), ("a_scales", 2), ("b", 4), ("b_scales", 1), ("out", 1)):
        assert matmul(lib, {name: None}) == BAD and matmul(lib, {name: ADDRESS + odd}) == BAD
    assert quantize(lib, {"codes": ADDRESS}) == BAD                                     # over their inputs
    assert matmul(lib, {"out": ADDRESS}) == BAD and matmul(lib, {"out": ADDRESS + 8192}) == BAD
    for hook in (7, 15, 1 << 10):                                                       # test hooks that no kernel answers to
        assert matmul(lib, out_type=icv.ICV_OUT_BF16 | hook << 8) == UNSUPPORTED
    assert matmul(lib, out_type=icv.ICV_OUT_ACC | 1 << 8) == UNSUPPORTED
    assert matmul(lib, {"bias": ADDRESS + 1}) == BAD and matmul(lib, rows=0) == OK
    assert matmul(lib, {"out": ADDRESS + 2}, out_type=icv.ICV_OUT_ACC) == BAD
    assert lib.icv_quantize_fp8(None, ADDRESS, ADDRESS, ADDRESS, None) == BAD
    assert lib.icv_matmul_fp8(None, ADDRESS, ADDRESS, ADDRESS, ADDRESS, None, ADDRESS, None) == BAD


def test_calls_of_too_many_threads_are_refused(lib):
    many = 1 << 30
    assert conv(lib, seq(many, many), channels=1 << 20) == UNSUPPORTED
    assert conv(lib, seq(1, many), channels=1 << 24, dtype=icv.ICV_F32) == UNSUPPORTED
    assert scan(lib, seq(many, many), channels=4096) == UNSUPPORTED                        # single tokens
    assert scan(lib, seq(many // 2, many), channels=4096) == UNSUPPORTED
    assert quantize(lib, rows=2 ** 31 - 1, depth=1 << 20) == UNSUPPORTED
    assert quantize(lib, rows=2 ** 31 - 1, depth=1 << 24, block_rows=128) == UNSUPPORTED
    for out in (icv.ICV_OUT_ACC, icv.ICV_OUT_BF16):
        assert matmul(lib, rows=2 ** 31 - 1, cols=1 << 30, out_type=out) == UNSUPPORTED


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        icv.causal_conv1d(icv.make_causal_conv_params(16, 4), seq(1, 4), x, x, None, None, x)
    with pytest.raises(TypeError, match="a tensor expected"):
        icv.causal_conv1d(icv.make_causal_conv_params(16, 4), seq(1, 4), [1.0], x, None, None, x)
    with pytest.raises(ValueError):
        icv.make_sequences(1, 4, start=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        icv.quantize_fp8(icv.make_quantize_params(4, 16), x, x, x)


def test_the_checks_name_what_is_wrong():
    """The native checks themselves, on host tensors, which they refuse for that at the latest: nothing is launched."""
    native = icv._load_native()
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    p, s = icv.make_causal_conv_params(16, 4), seq(1, 4)
    with pytest.raises(ValueError, match="input: a BFloat16 matrix of at least 4 x 16, strides .16, 1., on GPU 0 expected"):
        native.causal_conv1d(0, 0, p, s, x, x, None, None, x)
    with pytest.raises(TypeError, match="input: a tensor expected"):
        native.causal_conv1d(0, 0, p, s, [1], x, None, None, x)
    with pytest.raises(TypeError, match="icv_causal_conv_params"):
        native.causal_conv1d(0, 0, s, s, x, x, None, None, x)
    with pytest.raises(TypeError, match="icv_sequences"):
        native.causal_conv1d(0, 0, p, p, x, x, None, None, x)
    with pytest.raises(TypeError, match="9 arguments"):
        native.causal_conv1d(0, 0, p, s, x)
    with pytest.raises(ValueError, match="input: a BFloat16 matrix of at least 4 x 16"):
        native.quantize_fp8(0, 0, icv.make_quantize_params(4, 16), x, x, x)
    with pytest.raises(ValueError, match="a: a Byte matrix of at least 4 x 128"):
        native.matmul_fp8(0, 0, icv.make_matmul_params(4, 16, 16), x, x, x, x, None, x)
    with pytest.raises(ValueError, match="x: a Float matrix"):
        native.selective_scan(0, 0, icv.make_scan_params(16, 16, "f32"), s, *[x] * 10, None)
    other = seq(1, 4)
    other.device = 1
    with pytest.raises(ValueError, match="one device"):
        native.causal_conv1d(0, 0, p, other, x, x, None, None, x)


def test_rows_per_run_that_no_convolution_has(lib):
    for hook in (33, 64, 1 << 20):                                                      # test hooks
        assert conv(lib, silu=1 | hook << 8) == UNSUPPORTED
    assert conv(lib, silu=-1) == BAD and conv(lib, silu=4 << 8 | 2) == BAD


@pytest.mark.parametrize("name", ["start", "length", "from_slot", "to_slot"])
def test_sequences_of_something_else_than_tensors_are_a_type_error(name):
    for wrong in ([0, 4], 0, "0"):
        with pytest.raises(TypeError, match=name + ": a tensor expected"):
            icv.make_sequences(1, 4, **{name: wrong})
    with pytest.raises(ValueError, match="device tensors"):
        icv.make_sequences(1, 4, start=[0, 4], length=torch.zeros(1, dtype=torch.int32))
