"""Beam search's C ABI without a GPU: structure layouts, constants, workspace sizes,
and the refusals that come before any device work."""
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


def config(B, end=(), **kw):
    c = B.PsBeamConfig(**(dict(max_requests=4, beams=4, vocab=1000, dtype=B.PS_BEAM_BF16, num_end=len(end)) | kw))
    for i, t in enumerate(end):
        c.end_tokens[i] = t
    return c


def size(B, **kw):
    return B.load().ps_beam_workspace_bytes(C.byref(config(B, **kw)))


def test_structures_are_laid_out_as_in_the_header(tmp_path):
    from paper_2608_01657_gb300 import binding as B
    pairs = [("ps_beam_config_t", B.PsBeamConfig), ("ps_beam_select_t", B.PsBeamSelect), ("ps_beam_trace_t", B.PsBeamTrace),
             ("ps_kv_layout_t", B.PsKvLayout)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "prefixshield_kv.h"', '#include "prefixshield_beam.h"', "int main(void) {"]
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


def test_constants_match_the_headers():
    from paper_2608_01657_gb300 import binding as B
    txt = open(os.path.join(ROOT, "include", "prefixshield_beam.h")).read()
    for name in ("PS_BEAM_MAX_BEAMS", "PS_BEAM_MAX_END"):
        assert getattr(B, name) == int(re.search(rf"#define {name} (\d+)", txt).group(1))
    for name in ("PS_BEAM_BF16", "PS_BEAM_F16", "PS_BEAM_F32"):
        assert getattr(B, name) == int(re.search(rf"{name} = (\d+)", txt).group(1))
    kv = open(os.path.join(ROOT, "include", "prefixshield_kv.h")).read()
    assert B.PS_KV_MAX_BEAMS == int(re.search(r"#define PS_KV_MAX_BEAMS (\d+)", kv).group(1)) == B.PS_BEAM_MAX_BEAMS


def test_workspace_sizes(B):
    assert size(B) > 0 and size(B) % 256 == 0 and size(B, max_requests=1000) > size(B)
    assert size(B, vocab=1) > 0 and size(B, vocab=1 << 24) == size(B)  # partial results do not grow with the vocabulary
    assert size(B, beams=32, max_requests=1 << 15) > 0


@pytest.mark.parametrize("bad", [
    dict(max_requests=0), dict(max_requests=1 << 18, beams=5), dict(beams=0), dict(beams=33), dict(vocab=0), dict(vocab=(1 << 24) + 1),
    dict(dtype=3), dict(dtype=-1), dict(num_end=-1), dict(num_end=9), dict(end=(1000,)), dict(end=(-1,)), dict(end=(3, 4, 3))])
def test_invalid_configurations_have_no_size(B, bad):
    assert size(B, **bad) == 0


def test_arguments_are_refused(B):
    L, bad = B.load(), B.PS_ERR_INVALID_ARG
    c, h, n = config(B), C.c_void_p(), size(B)
    assert L.ps_beam_create(None, C.byref(c), 1 << 20, n) == bad
    assert L.ps_beam_create(C.byref(h), None, 1 << 20, n) == bad
    assert L.ps_beam_create(C.byref(h), C.byref(c), None, n) == bad
    assert L.ps_beam_create(C.byref(h), C.byref(c), (1 << 20) + 16, n) == bad
    assert L.ps_beam_create(C.byref(h), C.byref(c), 1 << 20, n - 1) == bad
    assert L.ps_beam_select(None, None, C.byref(B.PsBeamSelect()), None) == bad
    assert L.ps_beam_trace(None, None, C.byref(B.PsBeamTrace()), None) == bad
    assert L.ps_kv_layout(None, None, C.byref(B.PsKvRows()), C.byref(B.PsKvLayout()), None) == bad
    assert L.ps_kv_reorder(None, None, 0, 1, None, None, 0, C.byref(B.PsKvRows()), None, None, None) == bad
    L.ps_beam_destroy(None)
