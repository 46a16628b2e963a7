"""CPU: the calls around the method (embedding, norm, AdamW) refuse what atomo.h does not allow, before anything touches a GPU, and
the ctypes mirrors of their structs match the header."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_1806_04090_amd import binding
from paper_1806_04090_amd.binding import ATOMO_EINVAL, ATOMO_EHIP, ATOMO_F32, ATOMO_BF16

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = [binding.atomo_rows, binding.atomo_tokens, binding.atomo_adamw_tensor, binding.atomo_adamw_options]

# Bytes that stand for a context and a plan of a device that there is none of: a call whose arguments pass ends at that device.
DUMMY = C.create_string_buffer(b"\1" * 4096, 4096)
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="for machines without a GPU")


def address(k):
    """A number that looks like the address of a buffer of its own."""
    return 0x7f00_0000_0000 + k * (1 << 36)


def rows(n=10, cols=8, type=ATOMO_F32, ld=8, data=address(0)):
    return binding.atomo_rows(n, cols, type, ld, data)


def tokens(n=5, data=address(1), nbytes=8, padding=-1):
    return binding.atomo_tokens(n, data, nbytes, padding)


def lookup(table=None, toks=None, out=None, ctx=DUMMY):
    return binding.lib().atomo_embedding(ctx, C.byref(table or rows()), C.byref(toks or tokens()), 1.0, C.byref(out or rows(5, data=address(2))), None)


def grad(toks=None, dy=None, g=None, ctx=DUMMY):
    return binding.lib().atomo_embedding_grad(ctx, C.byref(toks or tokens()), C.byref(dy or rows(5, data=address(2))), 1.0, C.byref(g or rows()), 0, None)


@no_gpu
@pytest.mark.parametrize("call, ok", [
    (lambda: lookup(), True),
    (lambda: lookup(rows(ld=0), None, rows(7, data=address(2), ld=9)), True),              # every row the same; rows behind the last token
    (lambda: lookup(None, tokens(0, None), rows(0, data=None)), True),
    (lambda: lookup(rows(1, ld=-3), tokens(1), rows(1, ld=0, data=address(2))), True),     # strides of single rows
    (lambda: grad(), True),
    (lambda: grad(None, rows(5, data=address(2), ld=0)), True),
    (lambda: grad(tokens(0, None), rows(0, data=None)), True),
    (lambda: lookup(ctx=None), False), (lambda: grad(ctx=None), False),
    (lambda: lookup(rows(0)), False), (lambda: lookup(rows(2 ** 31 - 1)), False), (lambda: lookup(rows(cols=0, ld=1)), False), (lambda: lookup(rows(cols=2 ** 30 + 1, ld=2 ** 31), None, rows(5, 2 ** 30 + 1, ATOMO_F32, 2 ** 31, address(2))), False),
    (lambda: lookup(rows(type=3)), False), (lambda: lookup(rows(type=-1)), False), (lambda: lookup(rows(data=None)), False),
    (lambda: lookup(rows(ld=7)), False), (lambda: lookup(rows(ld=-8)), False),
    (lambda: lookup(None, tokens(-1)), False), (lambda: lookup(None, tokens(2 ** 31)), False), (lambda: lookup(None, tokens(data=None)), False),
    (lambda: lookup(None, tokens(nbytes=2)), False), (lambda: lookup(None, tokens(6)), False),
    (lambda: lookup(None, None, rows(5, cols=7, data=address(2))), False), (lambda: lookup(None, None, rows(5, ld=0, data=address(2))), False),
    (lambda: grad(None, rows(4, data=address(2))), False), (lambda: grad(None, rows(5, cols=9, ld=9, data=address(2))), False),
    (lambda: grad(None, None, rows(ld=0)), False), (lambda: grad(None, None, rows(0)), False), (lambda: grad(None, None, rows(data=None)), False),
])
def test_embedding_calls(call, ok):
    assert call() == (ATOMO_EHIP if ok else ATOMO_EINVAL)


def tensor(k=0, n=1000, **other):
    at = [address(8 * k + j) for j in range(6)]
    t = binding.atomo_adamw_tensor(n, at[0], at[1], at[2], at[3], None, None, None, ATOMO_F32, ATOMO_F32, 1.0, 0.1)
    for name, value in other.items():
        setattr(t, name, value)
    return t


def create(*tensors, n=None, ctx=DUMMY, out=True):
    array = (binding.atomo_adamw_tensor * max(1, len(tensors)))(*tensors)
    h = C.c_void_p(5)
    rc = binding.lib().atomo_adamw_create(ctx, array if tensors else None, len(tensors) if n is None else n, C.byref(h) if out else None)
    assert rc != 0 and (not out or h.value is None)
    return rc


EIGHT = dict(m_scale=address(100), v_scale=address(101))


@no_gpu
@pytest.mark.parametrize("call, ok", [
    (lambda: create(tensor()), True),
    (lambda: create(tensor(0), tensor(1, **EIGHT), tensor(2, copy=address(102), copy_type=ATOMO_BF16)), True),
    (lambda: create(tensor(0, param=None, m=None, v=None), tensor(1, param=None)), True),
    (lambda: create(tensor(0), tensor(1, grad=address(1))), True),                         # one gradient read by two tensors
    (lambda: create(tensor(0, param=None), tensor(1, param=None, grad=address(1) + 40)), True),
    (lambda: create(tensor(0), tensor(1, param=address(0) + 4000)), True),                 # side by side
    (lambda: create(tensor(), ctx=None), False), (lambda: create(tensor(), out=False), False), (lambda: create(), False), (lambda: create(tensor(), n=0), False),
    (lambda: create(tensor(n=0)), False), (lambda: create(tensor(n=2 ** 40)), False), (lambda: create(tensor(n=2 ** 39)), False),
    (lambda: create(tensor(grad=None)), False), (lambda: create(tensor(grad_type=3)), False), (lambda: create(tensor(copy=address(7), copy_type=9)), False),
    (lambda: create(tensor(m=None)), False), (lambda: create(tensor(v=None)), False), (lambda: create(tensor(m_scale=address(7))), False),
    (lambda: create(tensor(v_scale=address(7))), False), (lambda: create(tensor(0), tensor(1, param=None)), False),
    (lambda: create(tensor(lr_mult=-1.0)), False), (lambda: create(tensor(lr_mult=float("nan"))), False),
    (lambda: create(tensor(weight_decay=float("inf"))), False),
    # what a step writes lies apart from everything else: the same tensor twice, a tensor over the end of another, a gradient or scales in them
    (lambda: create(tensor(0), tensor(0)), False), (lambda: create(tensor(0), tensor(1, param=address(0) + 3996)), False),
    (lambda: create(tensor(0, grad=address(0))), False), (lambda: create(tensor(0), tensor(1, grad=address(2) + 3999)), False),
    (lambda: create(tensor(0, v=address(2) + 100)), False), (lambda: create(tensor(0, m_scale=address(3), v_scale=address(7))), False),
    (lambda: create(tensor(0, copy=address(1) + 3998, copy_type=ATOMO_BF16)), False),
    (lambda: create(tensor(0, grad=address(0) + 100, n=10), tensor(1, n=1000, param=address(0) + 90)), False),
])
def test_plans(call, ok):
    assert call() == (ATOMO_EHIP if ok else ATOMO_EINVAL)


def step(ctx=DUMMY, plan=DUMMY, **other):
    o = binding.atomo_adamw_options(1e-3, 0.9, 0.999, 1e-8, 1, None, None, None, 0.0, 1.0, 0)
    for name, value in other.items():
        setattr(o, name, value)
    return binding.lib().atomo_adamw_step(ctx, plan, C.byref(o), None)


@no_gpu
@pytest.mark.parametrize("options, ok", [
    ({}, True), (dict(lr=0.0, eps=0.0, beta1=0.0, beta2=0.0), True), (dict(step=0, step_dev=address(0)), True), (dict(max_norm=1.0, grad_norm=address(0)), True),
    (dict(grad_scale=-1.0), True),
    (dict(ctx=None), False), (dict(plan=None), False), (dict(lr=-1.0), False), (dict(lr=float("nan")), False), (dict(lr=float("inf")), False), (dict(beta1=1.0), False),
    (dict(beta2=-0.1), False), (dict(beta2=float("nan")), False), (dict(eps=-1e-9), False), (dict(eps=float("inf")), False), (dict(step=0), False), (dict(step=-5), False),
    (dict(max_norm=1.0), False), (dict(max_norm=-1.0, grad_norm=address(0)), False), (dict(max_norm=float("nan"), grad_norm=address(0)), False),
    (dict(grad_scale=float("nan")), False), (dict(grad_scale=float("inf")), False),
])
def test_steps(options, ok):
    assert step(**options) == (ATOMO_EHIP if ok else ATOMO_EINVAL)


@no_gpu
def test_the_other_calls():
    L = binding.lib()
    a = [address(k) for k in range(4)]
    assert L.atomo_adamw_grad_norm(DUMMY, DUMMY, 1.0, a[0], None) == ATOMO_EHIP
    for args in ((None, DUMMY, 1.0, a[0]), (DUMMY, None, 1.0, a[0]), (DUMMY, DUMMY, float("nan"), a[0]), (DUMMY, DUMMY, 1.0, None)):
        assert L.atomo_adamw_grad_norm(*args, None) == ATOMO_EINVAL
    assert L.atomo_adamw_destroy(DUMMY, None) == ATOMO_EINVAL and L.atomo_adamw_destroy(None, DUMMY) == ATOMO_EINVAL
    good = (DUMMY, 0, a[0], a[1], 10, ATOMO_F32, a[2])
    assert L.atomo_state8_unpack(*good, None) == ATOMO_EHIP
    for at, bad in ((0, None), (1, 2), (1, -1), (2, None), (3, None), (4, 0), (4, 2 ** 34), (5, 3), (6, None)):
        assert L.atomo_state8_unpack(*good[:at], bad, *good[at + 1:], None) == ATOMO_EINVAL, (at, bad)


def test_workspace_query():
    L, size = binding.lib(), C.c_size_t(0)
    for n, r in ((0, 1), (1, 1), (5, 2 ** 31 - 2), (2 ** 31 - 1, 1000)):
        assert L.atomo_embedding_workspace_bytes(n, r, 64, C.byref(size)) == 0
        assert size.value >= 8 * n
    assert binding.embedding_workspace_bytes(4096, 1000, 64) > 0
    for n, r, c in ((-1, 1, 1), (2 ** 31, 1, 1), (1, 0, 1), (1, 2 ** 31 - 1, 1), (1, 1, 0), (1, 1, 2 ** 30 + 1)):
        assert L.atomo_embedding_workspace_bytes(n, r, c, C.byref(size)) == ATOMO_EINVAL
    assert L.atomo_embedding_workspace_bytes(1, 1, 1, None) == ATOMO_EINVAL


def test_struct_layouts_match_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "atomo.h"', "int main(void) {"]
    for st in STRUCTS:
        lines.append(f'  printf("%zu\\n", sizeof({st.__name__}));')
        lines += [f'  printf("%zu\\n", offsetof({st.__name__}, {name}));' for name, _ in st._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run([cc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    seen = list(map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()))
    assert seen == [x for st in STRUCTS for x in [C.sizeof(st)] + [getattr(st, name).offset for name, _ in st._fields_]]
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "atomo.h")).read(), flags=re.S)
    for st in STRUCTS:
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (st.__name__, st.__name__), text, flags=re.S).group(1)
        declared = [part.replace("*", " ").split()[-1] for stmt in body.split(";") if stmt.strip() for part in stmt.split(",")]
        assert declared == [name for name, _ in st._fields_], st.__name__


def test_kernels_are_launched_by_name():
    # called through a pointer, a kernel's launch was dropped by the optimizer in the build with the host sanitizer, whose check of such
    # calls reads in front of the kernel's handle: the second digit of the sort was missing, and what followed read rows from memory never written
    for name in ("embedding.hip", "adamw.hip"):
        text = re.sub(r"//.*", "", open(os.path.join(ROOT, "paper_1806_04090_amd", "csrc", name)).read())
        kernels = set(re.findall(r"__global__[^;{]*?\bvoid\s+(\w+)\s*\(", text))
        launched = []
        for m in re.finditer("<<<", text):
            head, depth = text[:m.start()].rstrip(), 0
            while head.endswith(">") or depth:                   # template arguments
                depth += (head[-1] == ">") - (head[-1] == "<")
                head = head[:-1].rstrip()
            launched.append(re.search(r"(\w+)$", head)[1])
        assert launched and set(launched) <= kernels, set(launched) - kernels
