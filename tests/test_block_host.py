"""Host-side checks of the feed-forward sub-block's C ABI: exports, structures, refusals.  No compute calls."""
import ctypes
import os
import re

import pytest

from paper_1802_06905_b200 import binding, block

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "cconv_block.h")


@pytest.fixture(scope="module")
def lib():
    from paper_1802_06905_b200 import build
    build.build()
    return binding.load_library()


def header():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_every_declared_symbol_is_exported(lib):
    declared = set(re.findall(r"\b(cconv_[a-z_0-9]+)\s*\(", header()))
    assert declared == set(block.EXPORTS)
    for name in declared:
        assert hasattr(lib, name), name


def test_constants_match_the_header():
    values = {k: int(v) for k, v in re.findall(r"#define\s+CCONV_((?:TYPE|ACT)_\w+)\s+(\d+)", header())}
    assert values == {k: getattr(block, k) for k in ("TYPE_BF16", "TYPE_FP16", "TYPE_FP32", "ACT_SILU", "ACT_GELU",
                                                     "ACT_GELU_TANH", "ACT_RELU")}


def struct_of(name):
    """The header's structure as a ctypes one."""
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, header()).group(1)
    types = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "uint64_t": ctypes.c_uint64, "float": ctypes.c_float,
             "void*": ctypes.c_void_p, "const void*": ctypes.c_void_p}
    if name != "cconv_matrix":
        types["cconv_matrix"] = struct_of("cconv_matrix")
    fields = []
    for decl in body.split(";"):
        decl = " ".join(decl.split())
        if not decl:
            continue
        m = re.match(r"((?:const )?\w+ ?\*?) ?(\w+(?:, \w+)*)$", decl)
        assert m, decl
        for field in m.group(2).split(", "):
            fields.append((field, types[m.group(1).replace(" *", "*").strip()]))
    return type(name, (ctypes.Structure,), {"_fields_": fields})


@pytest.mark.parametrize("name,packed", [("cconv_ffn_args", block._FFN), ("cconv_residual_norm_args", block._NORM),
                                         ("cconv_fp8_product_args", block._FP8), ("cconv_quantize_args", block._QUANT)])
def test_packed_arguments_have_the_header_s_layout(name, packed):
    s = struct_of(name)
    space = 0 if name == "cconv_quantize_args" else block._SPACE.size
    assert ctypes.sizeof(s) == packed.size + space
    # numbers 1, 2, ... in the order of the fields come back from the fields
    leaves = []
    for field, ty in s._fields_:
        leaves += [(field, f) for f, _ in ty._fields_] if issubclass(ty, ctypes.Structure) else [(field, None)]
    n = len(leaves) - (2 if space else 0)
    raw = packed.pack(*range(1, n + 1)) + (block._SPACE.pack(n + 1, n + 2) if space else b"")
    got = s.from_buffer_copy(raw)
    for i, (field, sub) in enumerate(leaves):
        v = getattr(got, field) if sub is None else getattr(getattr(got, field), sub)
        assert v == i + 1, (field, sub)


def ffn(lib, **kw):
    s = struct_of("cconv_ffn_args")()
    s.T, s.D, s.F = 4, 16, 32
    base = 1 << 20
    shapes = dict(x=(4, 16), w_gate=(32, 16), w_up=(32, 16), w_down=(16, 32), out=(4, 16), dout=(4, 16), dx=(4, 16),
                  dw_gate=(32, 16), dw_up=(32, 16), dw_down=(16, 32), gate_pre=(4, 32), up_pre=(4, 32))
    for i, (name, (_, cols)) in enumerate(shapes.items()):
        m = getattr(s, name)
        m.data, m.row_stride, m.col_stride = base * (i + 1), cols, 1
    for k, v in kw.items():
        if isinstance(v, tuple):
            m = getattr(s, k)
            m.data, m.row_stride, m.col_stride = v
        else:
            setattr(s, k, v)
    return s


# every refusal is made before the device is looked at
@pytest.mark.parametrize("bad", [dict(T=-1), dict(D=1 << 31), dict(F=-5), dict(dtype=2), dict(dtype=-1), dict(act=4),
                                 dict(x=(0, 16, 1)), dict(x=((1 << 20) + 1, 16, 1)), dict(x=(1 << 20, -16, 1)),
                                 dict(out=(1 << 25, 0, 1)), dict(out=(1 << 25, 8, 1)), dict(out=(1 << 25, 16, 0)),
                                 dict(gate_pre=(0, 0, 0)), dict(w_gate=(1 << 22, 1 << 41, 1))])
def test_ffn_forward_refuses(lib, bad):
    f = lib.cconv_ffn_forward
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    s = ffn(lib, **bad)
    assert f(ctypes.addressof(s), None) == binding.EINVAL


def test_null_arguments_are_refused(lib):
    for name in block.EXPORTS:
        if name == "cconv_block_status":
            continue
        f = getattr(lib, name)
        f.restype = ctypes.c_int64 if name.endswith("_workspace") else ctypes.c_int
        f.argtypes = [ctypes.c_void_p] if name.endswith("_workspace") else [ctypes.c_void_p, ctypes.c_void_p]
        assert f(*([None] * len(f.argtypes))) == binding.EINVAL, name


def test_other_entry_points_refuse(lib):
    def call(name, struct, **kw):
        s = struct_of(struct)()
        for k, v in kw.items():
            if isinstance(v, tuple):
                m = getattr(s, k)
                m.data, m.row_stride, m.col_stride = v
            else:
                setattr(s, k, v)
        f = getattr(lib, name)
        f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
        return f(ctypes.addressof(s), None)
    a, b, c, d, e = ((i << 20, 256, 1) for i in range(1, 6))
    norm = dict(T=4, D=256, dtype=0, scale=1.0, eps=1e-6, resid=a, resid_out=b)
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(dtype=3), dict(rows_per_gate=-1),
                dict(norm_out=b), dict(gate=c), dict(w_post=3 << 20), dict(w_pre=3 << 20), dict(block=(c[0] + 1, 256, 1)),
                dict(resid=(a[0], 256, 2)), dict(resid_out=(b[0], 255, 1))):
        assert call("cconv_residual_norm_forward", "cconv_residual_norm_args", **{**norm, **bad}) == binding.EINVAL, bad
    fp8 = dict(M=4, N=256, K=256, dtype=0, a=a, b=b, a_scale=(3 << 20, 2, 1), b_scale=(4 << 20, 2, 1), c=e)
    for bad in (dict(reserved=1), dict(dtype=5), dict(M=-1), dict(a_scale=((3 << 20) + 2, 2, 1)), dict(c=(a[0], 256, 1))):
        assert call("cconv_fp8_product", "cconv_fp8_product_args", **{**fp8, **bad}) == binding.EINVAL, bad
    quant = dict(T=4, D=256, dtype=0, block_rows=1, x=a, q=b, scale=(3 << 20, 2, 1))
    for bad in (dict(block_rows=2), dict(dtype=-1), dict(T=-4), dict(q=(a[0], 256, 1)), dict(scale=(3 << 20, 0, 1))):
        assert call("cconv_quantize_blocks", "cconv_quantize_args", **{**quant, **bad}) == binding.EINVAL, bad


def test_column_slices_of_one_array_are_distinct(lib):
    """gate_pre and up_pre side by side in one array pass the checks; overlapping ones do not.  (What passes
    goes on to the device, which a machine without one answers with another code.)"""
    f = lib.cconv_ffn_forward
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    at = 1 << 26
    s = ffn(lib, gate_pre=(at, 64, 1), up_pre=(at + 62, 64, 1))
    assert f(ctypes.addressof(s), None) == binding.EINVAL
    import torch
    if not torch.cuda.is_available():
        s = ffn(lib, gate_pre=(at, 64, 1), up_pre=(at + 64, 64, 1))
        assert f(ctypes.addressof(s), None) in (binding.ECUDA, binding.EUNSUPPORTED)


def call(lib, name, struct, stream=None, **kw):
    """The code of entry point `name` with these arguments; tuples are matrices (address, strides)."""
    s = struct_of(struct)()
    for k, v in kw.items():
        if isinstance(v, tuple):
            m = getattr(s, k)
            m.data, m.row_stride, m.col_stride = v
        else:
            setattr(s, k, v)
    f = getattr(lib, name)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    return f(ctypes.addressof(s), stream)


def at(i, pitch=256):
    return (i << 20, pitch, 1)


EMPTY = [
    ("cconv_ffn_forward", "cconv_ffn_args",
     dict(T=0, D=16, F=32, x=at(1), w_gate=at(2), w_up=at(3), w_down=at(4), out=at(5), gate_pre=at(6), up_pre=at(7))),
    ("cconv_ffn_forward", "cconv_ffn_args", dict(T=4, D=0, F=32, x=at(1), w_gate=at(2), w_up=at(3), w_down=at(4), out=at(5))),
    ("cconv_ffn_backward", "cconv_ffn_args",
     dict(T=4, D=0, F=32, x=at(1), dout=at(2), gate_pre=at(3), up_pre=at(4), dx=at(5), dw_gate=at(6), dw_up=at(7), dw_down=at(8))),
    ("cconv_ffn_backward", "cconv_ffn_args", dict(T=0, D=16, F=0, dx=at(1))),
    ("cconv_residual_norm_forward", "cconv_residual_norm_args",
     dict(T=0, D=256, scale=1.0, eps=1e-6, resid=at(1), resid_out=at(2), norm_out=at(3))),
    ("cconv_residual_norm_backward", "cconv_residual_norm_args",
     dict(T=0, D=256, scale=1.0, eps=1e-6, resid_out=at(1), dnorm_out=at(2), dresid=at(3))),
    ("cconv_residual_norm_backward", "cconv_residual_norm_args",
     dict(T=4, D=0, scale=1.0, eps=1e-6, resid_out=at(1), dnorm_out=at(2), dresid=at(3))),
    ("cconv_fp8_product", "cconv_fp8_product_args",
     dict(M=0, N=256, K=256, a=at(1), b=at(2), a_scale=at(3, 2), b_scale=at(4, 2), c=at(5))),
    ("cconv_fp8_product", "cconv_fp8_product_args",
     dict(M=4, N=0, K=256, a=at(1), b=at(2), a_scale=at(3, 2), b_scale=at(4, 2), c=at(5))),
    ("cconv_quantize_blocks", "cconv_quantize_args", dict(T=0, D=256, block_rows=1, x=at(1), q=at(2), scale=at(3, 2))),
]


@pytest.mark.parametrize("name,struct,args", EMPTY)
def test_a_call_without_results_leaves_the_stream_alone(lib, name, struct, args):
    """It launches nothing, so that it needs no device and completes nothing: a convolution in front of it may
    still be running afterwards, and one that reads its Out has to wait."""
    key = 0x7E560000 + 256 * EMPTY.index((name, struct, args))
    far = 1 << 40

    def probe(image, out):
        return binding.stream_order_probe(key, (far + image, far + image + 4096), (far, far + 16), (far + out, far + out + 4096),
                                          2, 28.0, 0.0, 148)
    assert probe(1 << 20, 2 << 20) == 0
    assert call(lib, name, struct, stream=key, **args) == binding.OK
    assert probe(2 << 20, 3 << 20) == 1


FORWARD_IN_PLACE = dict(T=8, D=256, scale=1.0, eps=1e-6, resid=at(1), resid_out=at(1), norm_out=at(2), block=at(3))
BACKWARD_IN_PLACE = dict(T=8, D=256, scale=1.0, eps=1e-6, resid_out=at(1), dnorm_out=at(2), dresid_out=at(3), dresid=at(3),
                         block=at(4), dblock=at(5))


@pytest.mark.parametrize("name,args,bad", [
    ("forward", FORWARD_IN_PLACE, dict(block=at(1, 0))),                        # row 0 for every token
    ("forward", FORWARD_IN_PLACE, dict(block=at(1))),
    ("forward", FORWARD_IN_PLACE, dict(gate=at(1))),
    ("forward", FORWARD_IN_PLACE, dict(gate=at(1), rows_per_gate=2)),
    ("forward", FORWARD_IN_PLACE, dict(w_post=1 << 20)),
    ("forward", FORWARD_IN_PLACE, dict(w_pre=1 << 20)),
    ("forward", FORWARD_IN_PLACE, dict(resid=at(1, 0))),
    ("forward", FORWARD_IN_PLACE, dict(resid=at(1, 512))),
    ("forward", FORWARD_IN_PLACE, dict(norm_out=at(1))),
    ("backward", BACKWARD_IN_PLACE, dict(resid_out=at(3, 0))),
    ("backward", BACKWARD_IN_PLACE, dict(dnorm_out=at(3, 512))),
    ("backward", BACKWARD_IN_PLACE, dict(dnorm_out=at(3))),
    ("backward", BACKWARD_IN_PLACE, dict(block=at(3, 0))),
    ("backward", BACKWARD_IN_PLACE, dict(gate=at(3), dgate=at(6))),
    ("backward", BACKWARD_IN_PLACE, dict(w_post=3 << 20, dw_post=6 << 20)),
    ("backward", BACKWARD_IN_PLACE, dict(w_pre=3 << 20, dw_pre=6 << 20)),
    ("backward", BACKWARD_IN_PLACE, dict(dresid_out=at(3, 0))),
])
def test_only_the_named_matrix_may_be_written_in_place(lib, name, args, bad):
    entry = "cconv_residual_norm_" + name
    assert call(lib, entry, "cconv_residual_norm_args", **{**args, **bad}) == binding.EINVAL
    import torch
    if not torch.cuda.is_available():  # in place as the header allows it: goes on to the device
        assert call(lib, entry, "cconv_residual_norm_args", **args) in (binding.ECUDA, binding.EUNSUPPORTED)
        one = {k: (v[0], 7, 1) if isinstance(v, tuple) and k != "norm_out" else v for k, v in args.items()}
        assert call(lib, entry, "cconv_residual_norm_args", **{**one, "T": 1}) in (binding.ECUDA, binding.EUNSUPPORTED)


def test_columns_of_one_array_in_turn_are_distinct(lib):
    """gate_pre in the even columns of an array and up_pre in the odd ones; likewise in turn by threes, with rows
    of any pitch, and by rows.  Those that share an element are refused."""
    f = lib.cconv_ffn_forward
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    a = 1 << 26
    import torch
    for gate, up in (((a, 64, 2), (a + 2, 64, 2)), ((a + 2, 64, 2), (a, 64, 2)), ((a, 96, 3), (a + 4, 96, 3)),
                     ((a, 64, 2), (a + 128 + 2, 128, 2)), ((a, 2, 8), (a + 2, 2, 8)), ((a, 1, 8), (a + 8, 1, 8))):
        s = ffn(lib, gate_pre=gate, up_pre=up)
        if not torch.cuda.is_available():
            assert f(ctypes.addressof(s), None) in (binding.ECUDA, binding.EUNSUPPORTED), (gate, up)
    for gate, up in (((a, 64, 2), (a + 4, 64, 2)), ((a, 64, 2), (a + 2, 65, 2)), ((a, 64, 2), (a + 2, 64, 1)),
                     ((a, 96, 3), (a + 2, 64, 2)), ((a, 64, 2), (a, 64, 2)), ((a, 2, 8), (a + 4, 2, 8))):
        s = ffn(lib, gate_pre=gate, up_pre=up)
        assert f(ctypes.addressof(s), None) == binding.EINVAL, (gate, up)


def test_without_tokens_the_second_norm_s_gradient_may_be_absent(lib):
    """dw_pre belongs to dnorm_out, which may be absent; of no tokens neither has an address."""
    none = dict(T=0, D=256, scale=1.0, eps=1e-6, dresid=at(1))
    assert call(lib, "cconv_residual_norm_backward", "cconv_residual_norm_args", **none, w_pre=2 << 20) == binding.OK
    assert call(lib, "cconv_residual_norm_backward", "cconv_residual_norm_args", **none, dw_pre=2 << 20) == binding.EINVAL
    for more in (dict(w_pre=2 << 20, dresid_out=at(3), dw_pre=4 << 20), dict(w_pre=2 << 20, dnorm_out=at(3), resid_out=at(5)),
                 dict(dnorm_out=at(3), resid_out=at(5), dw_pre=4 << 20)):
        assert call(lib, "cconv_residual_norm_backward", "cconv_residual_norm_args", **{**none, "T": 4}, **more) == binding.EINVAL
