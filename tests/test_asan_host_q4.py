"""The 4-bit entry points' host code under AddressSanitizer, and the binding's
mirrors of their structs (CPU only).

The sources are compiled with AddressSanitizer on their host side only and
linked with tests/asan/abi_errors_q4.cpp, which drives the argument checks of
every 4-bit entry point with pointers that are never dereferenced, so it runs
only where no GPU is visible.
"""

import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_09240_amd import tq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG = "/opt/rocm/llvm/bin/clang++"
SOURCES = ("q4", "kvcache", "kvpages", "kvattn", "q4_api")


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers missing")
@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake-pointer calls run only without a GPU")
def test_q4_host_code_under_address_sanitizer(tmp_path):
    inc = os.path.join(ROOT, "include")
    flags = ["--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fno-omit-frame-pointer", "-I", inc]
    objs, procs = [], []
    for s in SOURCES:
        objs.append(str(tmp_path / (s + ".o")))
        procs.append(subprocess.Popen([HIPCC, *flags, "-c", os.path.join(ROOT, "paper_2609_09240_amd", "csrc", s + ".hip"),
                                       "-o", objs[-1]], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for s, p in zip(SOURCES, procs):
        out, _ = p.communicate(timeout=600)
        assert p.returncode == 0, f"{s}:\n{out[-2000:]}"
    exe = str(tmp_path / "abi_errors_q4")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-g", "-fsanitize=address", "-I", inc,
                    os.path.join(ROOT, "tests", "asan", "abi_errors_q4.cpp"), *objs, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    assert "Sanitizer" not in r.stderr, r.stderr[-4000:]
    assert r.returncode == 0 and r.stdout.strip().endswith("ok: 0 failure(s)"), r.stdout[-4000:] + r.stderr[-2000:]


@pytest.mark.parametrize("name,mirror", [("tq_q4_matrix", tq.TqQ4Matrix), ("tq_kv_cache", tq.TqKvCache),
                                         ("tq_kv_rows", tq.TqKvRows), ("tq_kv_attn", tq.TqKvAttn)])
def test_structs_match_the_header(tmp_path, name, mirror):
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "tq.h"\nint main(void) {\n'
                   f'  printf("size %zu\\n", sizeof({name}));\n'
                   + "".join(f'  printf("{f[0]} %zu\\n", offsetof({name}, {f[0]}));\n' for f in mirror._fields_)
                   + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True,
                                                       check=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(mirror)
    for f in mirror._fields_:
        assert int(out[f[0]]) == getattr(mirror, f[0]).offset, f[0]


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros((2, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        tq.tq_q4_quantize(x)
    with pytest.raises(ValueError):
        tq.KVCache(torch.zeros((1, 2, 3), dtype=torch.uint8), *(torch.zeros(2, dtype=torch.int32),) * 3, 1, 64)
