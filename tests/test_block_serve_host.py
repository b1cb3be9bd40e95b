"""Host-side checks of the operators that serve the sub-block and clip its gradients: structures, refusals, stream
bookkeeping.  No compute calls: every refusal is made before the device is looked at."""
import ctypes
import re

import pytest
import torch

from paper_1802_06905_b200 import binding, block
from test_block_host import at, header, lib, struct_of  # noqa: F401

NO_DEVICE = (binding.ECUDA, binding.EUNSUPPORTED)


def nested(name):
    """As struct_of, of structures that hold others or point to them."""
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, header()).group(1)
    types = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "uint64_t": ctypes.c_uint64, "float": ctypes.c_float,
             "void*": ctypes.c_void_p, "const void*": ctypes.c_void_p, "const cconv_tensor*": ctypes.c_void_p,
             "cconv_matrix": struct_of("cconv_matrix")}
    if "cconv_residual_norm_args" in body:
        types["cconv_residual_norm_args"] = struct_of("cconv_residual_norm_args")
    fields = []
    for decl in body.split(";"):
        decl = " ".join(decl.split())
        if decl:
            m = re.match(r"((?:const )?\w+ ?\*?) ?(\w+(?:, \w+)*)$", decl)
            fields += [(f, types[m.group(1).replace(" *", "*").strip()]) for f in m.group(2).split(", ")]
    return type(name, (ctypes.Structure,), {"_fields_": fields})


def leaves(s, path=()):
    for field, ty in s._fields_:
        if issubclass(ty, ctypes.Structure):
            yield from leaves(ty, path + (field,))
        else:
            yield path + (field,)


@pytest.mark.parametrize("name,formats", [
    ("cconv_residual_norm_quantize_args", (block._NORM, block._SPACE, block._TWO)),
    ("cconv_int4_product_args", (block._INT4, block._SPACE)), ("cconv_quantize_groups_args", (block._GROUPS,)),
    ("cconv_moe_args", (block._MOE, block._SPACE)), ("cconv_tensor", (block._TENSOR,)),
    ("cconv_clip_args", (block._CLIP, block._SPACE))])
def test_packed_arguments_have_the_header_s_layout(name, formats):
    s = nested(name)
    assert ctypes.sizeof(s) == sum(f.size for f in formats)
    raw, n = b"", 0
    for f in formats:
        k = len(f.unpack(bytes(f.size)))
        raw += f.pack(*range(n + 1, n + k + 1))
        n += k
    got = s.from_buffer_copy(raw)
    paths = list(leaves(s))
    assert len(paths) == n
    for i, path in enumerate(paths):
        v = got
        for field in path:
            v = getattr(v, field)
        assert v == i + 1, path


def call(lib, name, struct, stream=None, **kw):
    s = nested(struct)()
    for k, v in kw.items():
        m = s.norm if struct == "cconv_residual_norm_quantize_args" and k not in ("q", "q_scale") else s
        if isinstance(v, tuple):
            m = getattr(m, k)
            m.data, m.row_stride, m.col_stride = v
        else:
            setattr(m, k, v)
    f = getattr(lib, name)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    return f(ctypes.addressof(s), stream)


QNORM = ("cconv_residual_norm_quantize", "cconv_residual_norm_quantize_args",
         dict(T=4, D=256, dtype=0, scale=1.0, eps=1e-6, resid=at(1), resid_out=at(2), q=at(3), q_scale=at(4, 2)))
INT4 = ("cconv_int4_product", "cconv_int4_product_args",
        dict(M=4, N=64, K=256, dtype=0, scale_dtype=0, group=128, x=at(1), q=at(2, 128), scale=at(3, 2), c=at(4, 64)))
GROUPS = ("cconv_quantize_groups", "cconv_quantize_groups_args",
          dict(N=64, K=256, dtype=0, scale_dtype=0, group=128, w=at(1), q=at(2, 128), scale=at(3, 2)))
MOE = ("cconv_moe_forward", "cconv_moe_args",
       dict(T=4, D=64, F=32, E=8, dtype=0, act=0, top_k=2, normalize=1, x=at(1, 64), router=at(2, 64), w_gate=at(3, 64),
            w_up=at(4, 64), w_down=at(5, 32), gate_stride=2048, up_stride=2048, down_stride=2048, ids=at(6, 2), weights=at(7, 2),
            out=at(8, 64)))


@pytest.mark.parametrize("entry,bad", [
    (QNORM, dict(eps=0.0)), (QNORM, dict(dtype=3)), (QNORM, dict(T=-1)), (QNORM, dict(q=(0, 256, 1))), (QNORM, dict(q=(3 << 20, 256, 2))),
    (QNORM, dict(q=(3 << 20, 255, 1))), (QNORM, dict(q_scale=(0, 2, 1))), (QNORM, dict(q_scale=((4 << 20) + 2, 2, 1))),
    (QNORM, dict(q_scale=(4 << 20, 0, 1))), (QNORM, dict(q=at(1))), (QNORM, dict(q=at(2))), (QNORM, dict(q_scale=at(3, 2))),
    (QNORM, dict(gate=at(5))), (QNORM, dict(w_post=5 << 20)), (QNORM, dict(norm_out=at(2))), (QNORM, dict(norm_out=at(3))),
    (INT4, dict(dtype=2)), (INT4, dict(scale_dtype=3)), (INT4, dict(group=16)), (INT4, dict(group=0)), (INT4, dict(reserved=1)),
    (INT4, dict(M=-1)), (INT4, dict(K=1 << 31)), (INT4, dict(x=(0, 256, 1))), (INT4, dict(x=((1 << 20) + 1, 256, 1))),
    (INT4, dict(q=(2 << 20, -1, 1))), (INT4, dict(scale=((3 << 20) + 1, 2, 1))), (INT4, dict(c=at(1, 64))), (INT4, dict(c=at(2, 64))),
    (INT4, dict(c=at(3, 64))), (INT4, dict(zero=at(4, 2))), (INT4, dict(c=(4 << 20, 32, 1))), (INT4, dict(c=(4 << 20, 64, 0))),
    (GROUPS, dict(dtype=3)), (GROUPS, dict(scale_dtype=-1)), (GROUPS, dict(group=48)), (GROUPS, dict(reserved=7)), (GROUPS, dict(N=-3)),
    (GROUPS, dict(q=at(1, 128))), (GROUPS, dict(scale=at(2, 2))), (GROUPS, dict(zero=at(3, 2))), (GROUPS, dict(q=(2 << 20, 64, 1))),
    (GROUPS, dict(w=(0, 256, 1))), (GROUPS, dict(scale=((3 << 20) + 1, 2, 1))),
    (MOE, dict(T=-1)), (MOE, dict(T=(1 << 20) + 1)), (MOE, dict(E=1025)), (MOE, dict(D=(1 << 29) + 1)), (MOE, dict(F=(1 << 29) + 1)), (MOE, dict(E=-1)), (MOE, dict(dtype=2)), (MOE, dict(act=4)),
    (MOE, dict(top_k=0)), (MOE, dict(top_k=33)), (MOE, dict(top_k=9)), (MOE, dict(normalize=2)), (MOE, dict(x=(0, 64, 1))),
    (MOE, dict(w_gate=(0, 64, 1))), (MOE, dict(w_up=((4 << 20) + 1, 64, 1))), (MOE, dict(w_down=(5 << 20, -1, 1))),
    (MOE, dict(gate_stride=-1)), (MOE, dict(up_stride=1 << 41)), (MOE, dict(ids=(0, 2, 1))), (MOE, dict(ids=((6 << 20) + 2, 2, 1))),
    (MOE, dict(weights=at(6, 2))), (MOE, dict(out=at(1, 64))), (MOE, dict(out=at(3, 64))), (MOE, dict(out=(8 << 20, 32, 1))),
    (MOE, dict(out=((3 << 20) + 2 * 2048 * 7, 64, 1))), (MOE, dict(ids=(6 << 20, 1, 1))), (MOE, dict(E=0)), (MOE, dict(D=0)),
])
def test_refusals(lib, entry, bad):  # noqa: F811
    name, struct, args = entry
    assert call(lib, name, struct, **{**args, **bad}) == binding.EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a device")
@pytest.mark.parametrize("entry,good", [
    (QNORM, {}), (QNORM, dict(resid_out=at(1))), (QNORM, dict(norm_out=at(5), w_pre=6 << 20)), (QNORM, dict(q_scale=(4 << 20, 1, 4))),
    (INT4, {}), (INT4, dict(zero=at(5, 2))), (INT4, dict(x=(1 << 20, 0, 1))), (INT4, dict(K=255)), (GROUPS, {}), (GROUPS, dict(zero=at(4, 2))),
    (MOE, {}), (MOE, dict(router=(0, 0, 0), top_k=9)), (MOE, dict(w_up=((3 << 20) + 2 * 64 * 32, 64, 1), gate_stride=4096, up_stride=4096)),
    (MOE, dict(gate_stride=0, up_stride=0, down_stride=0)), (MOE, dict(ids=(6 << 20, 1, 4)))])
def test_what_passes_goes_on_to_the_device(lib, entry, good):  # noqa: F811
    name, struct, args = entry
    assert call(lib, name, struct, **{**args, **good}) in NO_DEVICE


def tensors(*ts):
    s = nested("cconv_tensor")
    a = (s * max(1, len(ts)))()
    for t, (data, rows, cols, rs, cs, dtype) in zip(a, ts):
        t.data, t.rows, t.cols, t.row_stride, t.col_stride, t.dtype = data, rows, cols, rs, cs, dtype
    return a


def clip(lib, grads, outs=None, name="cconv_clip_gradients", stream=None, **kw):  # noqa: F811
    s = nested("cconv_clip_args")()
    g, o = (None if ts is None else tensors(*ts) for ts in (grads, outs))
    s.count, s.grads, s.outs = len(grads or []), *(None if ts is None else ctypes.addressof(ts) for ts in (g, o))
    s.max_norm, s.eps, s.norm = 1.0, 1e-6, 99 << 20
    for k, v in kw.items():
        setattr(s, k, v)
    f = getattr(lib, name)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    return f(ctypes.addressof(s), stream)


A, B = (1 << 20, 4, 100, 100, 1, 0), (2 << 20, 1, 333, 333, 1, 2)


@pytest.mark.parametrize("grads,outs,kw", [
    ([A, A], None, {}), ([A, ((1 << 20) + 200, 1, 10, 10, 1, 0)], None, {}), ([A], [(3 << 20, 4, 99, 100, 1, 0)], {}),
    ([A], [(3 << 20, 4, 100, 100, 1, 1)], {}), ([A], [((1 << 20) + 2, 4, 100, 100, 1, 0)], {}), ([A, B], [B[:1] + A[1:], A[:1] + B[1:]], {}),
    ([A], None, dict(max_norm=-1.0)), ([A], None, dict(max_norm=float("nan"))), ([A], None, dict(eps=float("inf"))),
    ([A], None, dict(max_norm=0.0, eps=0.0)), ([A], None, dict(norm=0)), ([A], None, dict(norm=(99 << 20) + 2)), ([A], None, dict(norm=1 << 20)),
    ([A], None, dict(reserved=1)), ([A], None, dict(norm_given=2)), ([A], None, dict(count=-1)), (None, None, dict(count=1)),
    ([(0, 4, 100, 100, 1, 0)], None, {}), ([((1 << 20) + 1, 4, 100, 100, 1, 0)], None, {}), ([(1 << 20, -1, 100, 100, 1, 0)], None, {}),
    ([(1 << 20, 4, 100, 100, 1, 3)], None, {}), ([(1 << 20, 4, 100, 99, 1, 0)], None, {}), ([(1 << 20, 4, 100, 0, 1, 0)], None, {}),
])
def test_clip_refuses(lib, grads, outs, kw):  # noqa: F811
    assert clip(lib, grads, outs, **kw) == binding.EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a device")
def test_clip_accepts(lib):  # noqa: F811
    for grads, outs, kw in (([A, B], None, {}), ([A, A], [(3 << 20,) + A[1:], (4 << 20,) + A[1:]], {}), ([A, B], [A, B], {}),
                            ([(1 << 20, 4, 100, 0, 1, 0)], [(3 << 20, 4, 100, 100, 1, 0)], {}), ([A, B], None, dict(norm_given=1)),
                            ([A, ((1 << 20) + 200, 4, 20, 150, 1, 0)][:1], None, {}), ([], None, {}), ([A], None, dict(max_norm=float("inf"))),
                            # columns of one array, side by side
                            ([(1 << 20, 8, 40, 100, 1, 0), ((1 << 20) + 80, 8, 60, 100, 1, 0)], None, {})):
        assert clip(lib, grads, outs, **kw) in NO_DEVICE, (grads, outs, kw)
        assert clip(lib, grads, None, name="cconv_gradient_norm", max_norm=-1.0) in NO_DEVICE  # (the limit is not looked at)


EMPTY = [(*QNORM[:2], {**QNORM[2], "T": 0}), (*INT4[:2], {**INT4[2], "M": 0}), (*INT4[:2], {**INT4[2], "N": 0}),
         (*GROUPS[:2], {**GROUPS[2], "K": 0}), (*MOE[:2], {**MOE[2], "T": 0})]


@pytest.mark.parametrize("i", range(len(EMPTY) + 1))
def test_a_call_without_results_leaves_the_stream_alone(lib, i):  # noqa: F811
    key, far = 0x7E5A0000 + 256 * i, 1 << 40

    def probe(image, out):
        return binding.stream_order_probe(key, (far + image, far + image + 4096), (far, far + 16), (far + out, far + out + 4096),
                                          2, 28.0, 0.0, 148)
    assert probe(1 << 20, 2 << 20) == 0
    if i < len(EMPTY):
        name, struct, args = EMPTY[i]
        assert call(lib, name, struct, stream=key, **args) == binding.OK
    else:  # nothing to scale, and the norm is given
        assert clip(lib, [(1 << 20, 0, 100, 100, 1, 0)], None, norm_given=1, stream=key) == binding.OK
    assert probe(2 << 20, 3 << 20) == 1


def test_the_binding_says_what_is_wrong():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    u8 = torch.zeros((8, 32), dtype=torch.uint8)
    for f in (lambda: block.int4_product(x, u8, x, x), lambda: block.quantize_groups(x, u8, x),
              lambda: block.residual_norm_quantize(x, x, x, x), lambda: block.moe_forward(x, None, x, x, x, x, x, x)):
        with pytest.raises(ValueError, match="must be a CUDA tensor"):
            f()
    with pytest.raises(ValueError, match="must be a bf16"):
        block.clip_gradients([x], 1.0, x)
    with pytest.raises(ValueError, match="at least one"):
        block.gradient_norm([], x)
