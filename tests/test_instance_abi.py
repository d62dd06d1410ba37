"""CPU checks of the instance's operators: declared symbols, struct layouts, and what the host refuses.  Nothing is
launched: a call whose arguments are good ends with the status of a machine without a GPU."""
import ctypes as C
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from paper_2509_06362_amd import binding, instance as I

HEADER = Path(__file__).resolve().parent.parent / "include" / "maaso_instance.h"

INVALID, SHAPE = -1, -2


@pytest.fixture(scope="module")
def lib():
    if not binding.LIB_PATH.exists():
        from paper_2509_06362_amd import build
        build.build_library()
    return I._library()


@pytest.fixture
def inst():
    """Stands for an instance: arguments are looked at before anything of it is."""
    return C.create_string_buffer(4096)


PTR = 0x10000  # an address that is never followed


def pages(**over):
    a = I.PagesArgs(64, 16, 4, 8, PTR, PTR, PTR)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


def cache(**over):
    a = I.CacheArgs(0, 2, 64, 2, 16, 64, 2 * 16 * 64, 64 * 2 * 16 * 64, PTR, PTR, None, None)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


def append(**over):
    a = I.AppendArgs(0, 3, 4, 64, 0, 100, 1e-6, PTR, PTR, PTR, 256, 128, 128, 256, PTR, None, None, PTR, PTR, PTR)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


def attention(**over):
    a = I.AttentionArgs(0, 2, 3, 4, 0, 2, 100, 0, 0, 0.125, PTR, PTR, 256, 256, None, PTR, None, None, None)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


def logits(**over):
    a = I.LogitsArgs(0, 2, 2, 100, 104, 104, PTR, PTR, PTR, None, None, None, None, None, None, 0, 0, None, None, None, None, None, 0)
    for k, v in over.items():
        setattr(a, k, v)
    return C.byref(a)


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(maaso_[a-z_]+)\s*\(", text)))
    assert sorted(I.EXPORTS) == names
    for n in names:
        assert getattr(lib, n).argtypes is not None


def test_header_is_plain_c_and_layouts_agree_with_the_binding(lib, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    structs = {"maaso_kv_pages": I.PagesArgs, "maaso_kv_cache": I.CacheArgs, "maaso_kv_append_args": I.AppendArgs,
               "maaso_kv_attention_args": I.AttentionArgs, "maaso_logits_args": I.LogitsArgs}
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


def test_constants_agree_with_the_header():
    text = HEADER.read_text()
    for name, value in (("BAD_PAGE", I.BAD_PAGE), ("BAD_ROW", I.BAD_ROW), ("NO_PAGES", I.NO_PAGES), ("BAD_BOUND", I.BAD_BOUND),
                        ("BAD_TOKEN", I.BAD_TOKEN), ("BAD_POS", I.BAD_POS)):
        assert re.search(rf"MAASO_INST_{name} {value}u", text)
    for name in ("BF16", "FP16", "FP32", "E4M3"):
        assert re.search(rf"MAASO_{name} = {getattr(I, 'MAASO_' + name)}\b", text)


def test_no_instance(lib):
    assert lib.maaso_instance_create(0, 0, None) == INVALID
    lib.maaso_instance_destroy(None)
    assert lib.maaso_instance_status(None, None) == INVALID
    assert lib.maaso_kv_extend(None, pages(), PTR, 1, PTR, 1, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_fork(None, pages(), PTR, PTR, 1, None) == INVALID
    assert lib.maaso_kv_trim(None, pages(), PTR, PTR, 1, None) == INVALID
    assert lib.maaso_kv_compact(None, pages(), PTR, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_copy(None, cache(), PTR, 1, None) == INVALID
    assert lib.maaso_kv_append(None, cache(), 0, append(), None) == INVALID
    assert lib.maaso_kv_attention(None, cache(), 0, pages(), attention(), None) == INVALID
    assert lib.maaso_logits_adjust(None, logits(), None) == INVALID


def test_an_instance_without_a_gpu_is_an_error(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    out = C.c_void_p(5)
    assert lib.maaso_instance_create(0, 0, C.byref(out)) == -4 and out.value is None


@pytest.mark.parametrize("over, status", [
    (dict(refs=None), INVALID), (dict(table=None), INVALID), (dict(length=None), INVALID), (dict(n_pages=0), INVALID),
    (dict(width=0), INVALID), (dict(n_rows=0), INVALID), (dict(page_size=24), SHAPE), (dict(page_size=256), SHAPE),
    (dict(page_size=0), SHAPE), (dict(n_pages=(1 << 24) + 1), SHAPE), (dict(width=1 << 27), SHAPE)])
def test_pages_refused(lib, inst, over, status):
    assert lib.maaso_kv_extend(inst, pages(**over), PTR, 1, PTR, 1, PTR, PTR, PTR, None) == status
    assert lib.maaso_kv_fork(inst, pages(**over), PTR, PTR, 1, None) == status
    assert lib.maaso_kv_trim(inst, pages(**over), PTR, PTR, 1, None) == status
    assert lib.maaso_kv_compact(inst, pages(**over), PTR, PTR, PTR, PTR, None) == status
    assert lib.maaso_kv_attention(inst, cache(), 0, pages(**over), attention(), None) == status


def test_page_calls_refused(lib, inst):
    assert lib.maaso_kv_extend(inst, None, PTR, 1, PTR, 1, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), None, 1, PTR, 1, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), PTR, 1, None, 1, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), PTR, 1, PTR, 1, None, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), PTR, 1, PTR, 1, PTR, PTR, None, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), PTR, 0, PTR, 1, PTR, PTR, PTR, None) == INVALID
    assert lib.maaso_kv_extend(inst, pages(), PTR, 65537, PTR, 1, PTR, PTR, PTR, None) == SHAPE
    assert lib.maaso_kv_extend(inst, pages(), None, 0, None, 0, None, None, None, None) == 0
    for call in (lib.maaso_kv_fork, lib.maaso_kv_trim):
        assert call(inst, pages(), None, PTR, 1, None) == INVALID
        assert call(inst, pages(), PTR, None, 1, None) == INVALID
        assert call(inst, pages(), PTR, PTR, 65537, None) == SHAPE
        assert call(inst, pages(), None, None, 0, None) == 0
    for k in range(4):
        args = [PTR] * 4
        args[k] = None
        assert lib.maaso_kv_compact(inst, pages(), *args, None) == INVALID
    assert lib.maaso_kv_copy(inst, cache(), None, 1, None) == INVALID
    assert lib.maaso_kv_copy(inst, cache(), None, 0, None) == 0


@pytest.mark.parametrize("over, status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(type=2), INVALID), (dict(type=9), INVALID), (dict(k_scale=PTR), INVALID),
    (dict(n_layers=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(page_size=8), SHAPE), (dict(k=PTR + 8), SHAPE), (dict(v=PTR + 2), SHAPE), (dict(page_stride=2 * 16 * 64 - 8), SHAPE),
    (dict(page_stride=2 * 16 * 64 + 4), SHAPE), (dict(layer_stride=64), SHAPE)])
def test_caches_refused(lib, inst, over, status):
    assert lib.maaso_kv_copy(inst, cache(**over), PTR, 1, None) == status
    assert lib.maaso_kv_append(inst, cache(**over), 0, append(), None) == status
    assert lib.maaso_kv_attention(inst, cache(**over), 0, pages(), attention(), None) == status


@pytest.mark.parametrize("over, status", [
    (dict(type=2), INVALID), (dict(type=1), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(q_out=None), INVALID), (dict(slot=None), INVALID), (dict(cos_sin=None), INVALID), (dict(pos=None), INVALID),
    (dict(n_pos=0), INVALID), (dict(cos_sin=PTR + 4), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(rotary=24), SHAPE), (dict(rotary=80), SHAPE), (dict(n_heads=0), SHAPE), (dict(q_stride=255), SHAPE), (dict(k_stride=64), SHAPE),
    (dict(q_out_stride=128), SHAPE), (dict(v_stride=0), SHAPE), (dict(n_tok=0, q=None), 0)])
def test_appends_refused(lib, inst, over, status):
    assert lib.maaso_kv_append(inst, cache(), 0, append(**over), None) == status


def test_append_in_place_keeps_its_stride(lib, inst):
    assert lib.maaso_kv_append(inst, cache(), 0, append(q_stride=512), None) == INVALID  # q_out is q
    assert lib.maaso_kv_append(inst, cache(), 2, append(), None) == INVALID  # a layer too far


@pytest.mark.parametrize("over, status", [
    (dict(type=2), INVALID), (dict(type=1), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q_start=None), INVALID),
    (dict(n=0), INVALID), (dict(scale=float("inf")), INVALID), (dict(n_groups=1, max_shared=16), INVALID), (dict(n_heads=3), SHAPE),
    (dict(n_heads=0), SHAPE), (dict(n_groups=3), SHAPE), (dict(max_q=0), SHAPE), (dict(max_q=4), SHAPE), (dict(q=PTR + 8), SHAPE),
    (dict(out=PTR + 2), SHAPE), (dict(q_stride=260), SHAPE), (dict(out_stride=128), SHAPE), (dict(max_len=1 << 31), SHAPE),
    (dict(n_tok=0, n=0), 0)])
def test_attention_refused(lib, inst, over, status):
    assert lib.maaso_kv_attention(inst, cache(), 0, pages(), attention(**over), None) == status


def test_attention_and_its_pages_belong_together(lib, inst):
    assert lib.maaso_kv_attention(inst, cache(), 0, pages(page_size=32), attention(), None) == INVALID
    assert lib.maaso_kv_attention(inst, cache(), 0, pages(n_pages=63), attention(), None) == INVALID
    assert lib.maaso_kv_attention(inst, cache(), 2, pages(), attention(), None) == INVALID
    assert lib.maaso_kv_attention(inst, cache(), 0, pages(), None, None) == INVALID


@pytest.mark.parametrize("over, status", [
    (dict(type=3), INVALID), (dict(out_type=1), INVALID), (dict(logits=None), INVALID), (dict(out=None, chosen=None), INVALID),
    (dict(out=PTR), INVALID), (dict(n_bias=3), INVALID), (dict(n_history=3, history=PTR), INVALID), (dict(mask=PTR), INVALID),
    (dict(vocab=0), SHAPE), (dict(vocab=1 << 31), SHAPE), (dict(stride=99), SHAPE), (dict(out_stride=99, out=PTR * 2), SHAPE), (dict(n=0), 0)])
def test_logits_refused(lib, inst, over, status):
    over = {"out": PTR * 2, **over}
    assert lib.maaso_logits_adjust(inst, logits(**over), None) == status


def test_the_binding_looks_at_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(AssertionError):
        I.KvPages(torch.zeros(4, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 16)
    with pytest.raises(AssertionError):
        I.KvCache(torch.zeros(1, 2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 1, 16, 64, dtype=torch.bfloat16))
    with pytest.raises(AssertionError):
        I._type(torch.zeros(2, dtype=torch.int64))


def test_calls_look_at_tensors(lib):
    """What a call refuses before the library sees it: tensors on the host, too few elements, other types, no tensors at all."""
    torch = pytest.importorskip("torch")
    i32, bf16 = torch.int32, torch.bfloat16
    inst, view = I.Instance(0, 0), type("View", (), {"at": C.addressof(I.CacheArgs(n_kv_heads=1, head_dim=64))})()
    rows, heads = torch.zeros(2, dtype=i32), torch.zeros(2, 1, 64, dtype=bf16)
    calls = [lambda x: I.maaso_kv_extend(inst, view, rows=x, q_start=x, slot=x, copies=x), lambda x: I.maaso_kv_fork(inst, view, parents=x, children=x),
             lambda x: I.maaso_kv_trim(inst, view, rows=x, keep=x), lambda x: I.maaso_kv_copy(inst, view, pairs=rows if x is None else x),
             lambda x: I.maaso_kv_append(inst, view, layer=0, q=x, k=x, v=x, q_out=x, slot=rows),
             lambda x: I.maaso_kv_attention(inst, view, view, layer=0, q=x, out=x, q_start=rows, scale=1.0, max_q=1, max_len=1),
             lambda x: I.maaso_logits_adjust(inst, logits=x, chosen=rows)]
    for call in calls:
        for x in (rows, heads, heads[0], 3, "rows", None):
            with pytest.raises(AssertionError):
                call(x)
    with pytest.raises((AssertionError, OverflowError, ValueError, TypeError)):
        I.maaso_kv_attention(inst, view, view, layer=-1, q=heads, out=heads, q_start=rows, scale=1.0, max_q=1, max_len=1)
    inst.handle = None
