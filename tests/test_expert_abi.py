"""CPU checks of the products, the experts and the rows in 8 bits: struct layouts, and what host and binding refuse.  Nothing
is launched."""
import ctypes as C
import shutil
import subprocess

import pytest

from paper_2509_06362_amd import instance as I
from tests.test_instance_abi import HEADER, INVALID, PTR, SHAPE, inst, lib  # noqa: F401


def filled(struct, values, over):
    a = struct(**values)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def quantize(**over):
    return C.byref(filled(I.QuantizeArgs, dict(type=0, form=1, n=3, width=100, eps=1e-6, x_stride=104, q_stride=112, x=PTR, weight=PTR, q=PTR, scale=PTR), over))


def matrix(**over):
    return filled(I.ProductArgs, dict(type=4, out_type=0, n_a=3, n_in=100, n_out=50, gated=1, a_stride=112, w_stride=112, out_stride=50, a=PTR, w=PTR, a_scale=PTR,
                                      w_scale=PTR, bias=PTR, out=PTR), over)


def experts(product=None, **over):
    return C.byref(filled(I.ExpertProductArgs, dict(product=matrix(**(product or {})), n_rows=6, n_experts=4, expert_stride=100 * 112, start=PTR, token=PTR), over))


def route(**over):
    return C.byref(filled(I.RouteArgs, dict(type=0, n=3, n_experts=8, k=2, sigmoid=1, renorm=1, scale=1.0, stride=8, logits=PTR, bias=PTR, expert=PTR, weight=PTR,
                                            start=PTR, token=PTR, place=PTR), over))


def combine(**over):
    return C.byref(filled(I.CombineArgs, dict(type=0, n=3, k=2, width=100, n_rows=6, y_stride=104, residual_stride=104, out_stride=112, y=PTR, residual=PTR, out=PTR * 2,
                                              place=PTR, weight=PTR), over))


def test_layouts_agree_with_the_binding(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    structs = {"maaso_rows_quantize_args": I.QuantizeArgs, "maaso_product": I.ProductArgs, "maaso_expert_route_args": I.RouteArgs,
               "maaso_expert_product_args": I.ExpertProductArgs, "maaso_expert_combine_args": I.CombineArgs}
    lines = []
    for name, struct in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        lines += [f'  printf("%zu\\n", offsetof({name}, {f}));' for f, _ in struct._fields_]
    src = tmp_path / "abi.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "maaso_instance.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "abi"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", f"-I{HEADER.parent}", str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for struct in structs.values():
        want += [C.sizeof(struct)] + [getattr(struct, f).offset for f, _ in struct._fields_]
    assert got == want
    text = HEADER.read_text()
    assert f"MAASO_INT8 = {I.MAASO_INT8} " in text
    assert f"MAASO_ROWS_PLAIN = {I.MAASO_ROWS_PLAIN}, MAASO_ROWS_NORM = {I.MAASO_ROWS_NORM}, MAASO_ROWS_GATED = {I.MAASO_ROWS_GATED} " in text


def test_no_instance(lib):  # noqa: F811
    assert lib.maaso_rows_quantize(None, quantize(), None) == INVALID
    assert lib.maaso_scaled_product(None, C.byref(matrix()), None) == INVALID
    assert lib.maaso_expert_route(None, route(), None) == INVALID
    assert lib.maaso_expert_product(None, experts(), None) == INVALID
    assert lib.maaso_expert_combine(None, combine(), None) == INVALID


def test_no_arguments(lib, inst):  # noqa: F811
    for call in (lib.maaso_rows_quantize, lib.maaso_scaled_product, lib.maaso_expert_route, lib.maaso_expert_product, lib.maaso_expert_combine):
        assert call(inst, None, None) == INVALID


@pytest.mark.parametrize("over, status", [
    (dict(type=3), INVALID), (dict(type=4), INVALID), (dict(form=3), INVALID), (dict(form=0), INVALID), (dict(form=2), INVALID), (dict(x=None), INVALID),
    (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(width=0), SHAPE), (dict(width=1 << 30), SHAPE), (dict(n=1 << 31), SHAPE), (dict(x=PTR + 1), SHAPE), (dict(q=PTR + 8), SHAPE), (dict(weight=PTR + 1), SHAPE),
    (dict(type=2, x=PTR + 2), SHAPE), (dict(x_stride=96), SHAPE), (dict(q_stride=104), SHAPE), (dict(q_stride=96), SHAPE),
    (dict(form=2, weight=None, x_stride=104), SHAPE), (dict(n=0, x=None), 0)])
def test_quantizing_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_rows_quantize(inst, quantize(**over), None) == status


PRODUCTS = [
    (dict(type=2), INVALID), (dict(type=3), INVALID), (dict(out_type=3), INVALID), (dict(out_type=4), INVALID), (dict(a=None), INVALID), (dict(w=None), INVALID),
    (dict(out=None), INVALID), (dict(n_in=0), SHAPE), (dict(n_in=131072, a_stride=1 << 18, w_stride=1 << 18), SHAPE), (dict(n_out=0), SHAPE),
    (dict(n_out=1 << 30), SHAPE), (dict(n_out=1 << 27, out_stride=1 << 27), SHAPE), (dict(n_a=1 << 31), SHAPE), (dict(a_stride=104), SHAPE), (dict(a_stride=96), SHAPE), (dict(w_stride=104), SHAPE),
    (dict(w_stride=96), SHAPE), (dict(out_stride=49), SHAPE), (dict(a=PTR + 8), SHAPE), (dict(w=PTR + 8), SHAPE), (dict(out=PTR + 1), SHAPE),
    (dict(out=PTR + 2, out_type=2), SHAPE)]


@pytest.mark.parametrize("over, status", PRODUCTS + [(dict(type=0, a_scale=None, w_scale=None), INVALID), (dict(n_a=0, a=None), 0)])
def test_scaled_products_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_scaled_product(inst, C.byref(matrix(**over)), None) == status


@pytest.mark.parametrize("over, status", PRODUCTS + [
    (dict(type=0), INVALID), (dict(type=0, a_scale=None), INVALID), (dict(type=0, w_scale=None), INVALID), (dict(type=0, a_scale=None, w_scale=None, out_type=1), INVALID),
    (dict(type=1, a_scale=None, w_scale=None), INVALID), (dict(n_a=0), INVALID)])
def test_experts_operands_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_expert_product(inst, experts(product=over), None) == status


@pytest.mark.parametrize("over, status", [
    (dict(start=None), INVALID), (dict(n_experts=0), SHAPE), (dict(n_experts=1025), SHAPE), (dict(n_rows=1 << 31), SHAPE), (dict(expert_stride=100 * 112 - 32), SHAPE),
    (dict(expert_stride=100 * 112 + 8), SHAPE), (dict(n_rows=0, start=None), 0)])
def test_experts_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_expert_product(inst, experts(**over), None) == status


@pytest.mark.parametrize("over, status", [
    (dict(type=3), INVALID), (dict(sigmoid=0), INVALID), (dict(scale=float("nan")), INVALID), (dict(logits=None), INVALID), (dict(expert=None), INVALID),
    (dict(weight=None), INVALID), (dict(start=None), INVALID), (dict(token=None), INVALID), (dict(place=None), INVALID), (dict(start=None, token=None), INVALID),
    (dict(n_experts=0), SHAPE), (dict(n_experts=1025, stride=2000), SHAPE), (dict(k=0), SHAPE), (dict(k=9), SHAPE), (dict(k=33, n_experts=64, stride=64), SHAPE),
    (dict(stride=7), SHAPE), (dict(n=1 << 30), SHAPE), (dict(n=1 << 26, k=1), SHAPE), (dict(n=1 << 28, k=1, start=None, token=None, place=None), SHAPE), (dict(n=0, start=None, token=None, place=None), 0)])
def test_routing_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_expert_route(inst, route(**over), None) == status


@pytest.mark.parametrize("over, status", [
    (dict(type=3), INVALID), (dict(type=4), INVALID), (dict(y=None), INVALID), (dict(out=None), INVALID), (dict(place=None), INVALID), (dict(out=PTR), INVALID),
    (dict(width=0), SHAPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(n=1 << 31), SHAPE), (dict(n_rows=1 << 31), SHAPE), (dict(y=PTR + 1), SHAPE),
    (dict(residual=PTR + 1), SHAPE), (dict(out=PTR * 2 + 1), SHAPE), (dict(type=2, y=PTR + 2), SHAPE), (dict(y_stride=99), SHAPE), (dict(residual_stride=99), SHAPE),
    (dict(out_stride=96), SHAPE), (dict(n=0, out=None), 0)])
def test_joining_refused(lib, inst, over, status):  # noqa: F811
    assert lib.maaso_expert_combine(inst, combine(**over), None) == status


def test_calls_look_at_tensors(lib):  # noqa: F811
    """What a call refuses before the library sees it: tensors on the host, of other types or shapes, no tensors at all."""
    torch = pytest.importorskip("torch")
    i32, bf16 = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 16, dtype=torch.bfloat16)
    inst = I.Instance(0, 0)  # noqa: F811
    calls = [lambda x: I.maaso_rows_quantize(inst, x=x, q=x, scale=x), lambda x: I.maaso_scaled_product(inst, a=x, w=x, out=x),
             lambda x: I.maaso_expert_route(inst, logits=x, expert=x, weight=x), lambda x: I.maaso_expert_product(inst, a=x, w=x, out=x, start=x),
             lambda x: I.maaso_expert_combine(inst, y=x, place=i32, out=x)]
    for call in calls:
        for x in (i32, bf16, bf16[0], 3, "rows", None):
            with pytest.raises(AssertionError):
                call(x)
    inst.handle = None
