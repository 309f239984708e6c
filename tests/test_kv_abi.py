"""The KV page operators' C ABI without a GPU: structure layouts, workspace
sizes, constants, and the refusals that come before any device work."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("no nvcc")
    from paper_2608_01657_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def config(B, **kw):
    c = dict(k=1 << 20, v=1 << 21, num_pages=64, first_page=16, layer_stride=64 * 16 * 2 * 64, page_stride=16 * 2 * 64,
             token_stride=2 * 64, head_stride=64, num_layers=1, page_size=16, num_kv_heads=2, num_q_heads=4, head_dim=64,
             dtype=B.PS_KV_BF16, max_requests=8, max_tokens=64, max_row_pages=32)
    return B.PsKvConfig(**(c | kw))


def size(B, **kw):
    return B.load().ps_kv_workspace_bytes(C.byref(config(B, **kw)))


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    """sizeof and every field's offset, from a C compiler on the header itself."""
    from paper_2608_01657_gb300 import binding as B
    pairs = [("ps_kv_config_t", B.PsKvConfig), ("ps_kv_append_t", B.PsKvAppend), ("ps_kv_batch_t", B.PsKvBatch),
             ("ps_kv_attention_t", B.PsKvAttention), ("ps_kv_rows_t", B.PsKvRows)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "prefixshield_kv.h"', "int main(void) {"]
    for name, cls in pairs:
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in pairs:
        assert int(got[name]) == C.sizeof(cls)
        for f in cls._fields_:
            assert int(got[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset, (name, f[0])


def test_constants_match_the_header():
    from paper_2608_01657_gb300 import binding as B
    txt = open(os.path.join(ROOT, "include", "prefixshield_kv.h")).read()
    for name in ("PS_KV_MAX_HEAD_DIM", "PS_KV_MAX_HEADS"):
        assert getattr(B, name) == int(re.search(rf"#define {name} (\d+)", txt).group(1))
    for name in ("PS_KV_BF16", "PS_KV_F16"):
        assert getattr(B, name) == int(re.search(rf"{name} = (\d+)", txt).group(1))


def test_workspace_grows_with_the_bounds(B):
    base = size(B)
    assert base > 0 and base % 256 == 0
    assert size(B, num_pages=1 << 20) >= base + 12 * ((1 << 20) - 64)
    assert size(B, max_tokens=4096) > base and size(B, max_requests=1024) > base
    assert size(B, max_row_pages=1 << 20) == base


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(k=(1 << 20) + 8), dict(num_pages=0), dict(num_pages=(1 << 30) + 1), dict(first_page=-1),
    dict(page_size=0), dict(page_size=12), dict(page_size=128), dict(page_stride=-8),
    dict(token_stride=12), dict(head_stride=63), dict(layer_stride=4), dict(num_layers=0), dict(num_kv_heads=0),
    dict(num_q_heads=3), dict(num_q_heads=1), dict(num_q_heads=1026), dict(head_dim=0), dict(head_dim=12), dict(head_dim=136),
    dict(dtype=2), dict(max_requests=0), dict(max_requests=1 << 18), dict(max_tokens=0), dict(max_tokens=(1 << 22) + 1),
    dict(num_q_heads=1024, max_tokens=1 << 21), dict(max_row_pages=0), dict(max_row_pages=1 << 26)])
def test_invalid_configurations_have_no_size(B, bad):
    assert size(B, **bad) == 0


def test_null_and_misaligned_arguments_are_refused(B):
    L, bad = B.load(), B.PS_ERR_INVALID_ARG
    c, h = config(B), C.c_void_p()
    n = size(B)
    assert L.ps_kv_create(None, C.byref(c), 1 << 20, n, None) == bad
    assert L.ps_kv_create(C.byref(h), None, 1 << 20, n, None) == bad
    assert L.ps_kv_create(C.byref(h), C.byref(c), None, n, None) == bad
    assert L.ps_kv_create(C.byref(h), C.byref(c), (1 << 20) + 16, n, None) == bad
    assert L.ps_kv_create(C.byref(h), C.byref(c), 1 << 20, n - 1, None) == bad
    assert L.ps_kv_append(None, None, 0, C.byref(B.PsKvAppend()), None) == bad
    assert L.ps_kv_plan(None, None, C.byref(B.PsKvBatch()), None) == bad
    assert L.ps_kv_attention(None, None, 0, C.byref(B.PsKvAttention()), None) == bad
    assert L.ps_kv_copy(None, None, 0, None, None, None) == bad
    assert L.ps_kv_fork(None, None, 0, None, None, None, C.byref(B.PsKvRows()), None, None, None) == bad
    assert L.ps_kv_release(None, None, 0, None, C.byref(B.PsKvRows()), None, None) == bad
    assert L.ps_kv_compact(None, None, C.byref(B.PsKvRows()), None, None, None, None, None) == bad
    assert L.ps_step_blocks(None, None, 0, None, None, 0, None, None) == bad
    L.ps_kv_destroy(None)


@pytest.mark.parametrize("bad", [dict(head_stride=0), dict(token_stride=0), dict(page_stride=0), dict(head_stride=56),
                                 dict(page_stride=32), dict(num_layers=2, layer_stride=0), dict(num_layers=3, layer_stride=8)])
def test_pools_whose_elements_share_addresses_have_no_size(B, bad):
    """An axis of several places steps over a head's elements at least (an expanded tensor does not)."""
    assert size(B, **bad) == 0


def test_axes_of_one_place_may_have_any_stride(B):
    base = size(B)
    assert size(B, layer_stride=0) == base and size(B, num_pages=1, first_page=1, page_stride=0) > 0
    assert size(B, num_kv_heads=1, head_stride=0) > 0
