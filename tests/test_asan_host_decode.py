"""The host code of rotary positions, log probabilities and attention with sinks
or shared prefixes under AddressSanitizer, and the binding's mirrors of their
structs (CPU only).

The sources are compiled with AddressSanitizer on their host side only and
linked with tests/asan/abi_errors_decode.cpp, which drives the argument checks
with pointers that are never dereferenced, so it runs only where no GPU is
visible.
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
SOURCES = ("rope", "logprobs", "kvattn", "kvscope", "decode_api")


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers missing")
@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake-pointer calls run only without a GPU")
def test_decode_host_code_under_address_sanitizer(tmp_path):
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
    exe = str(tmp_path / "abi_errors_decode")
    subprocess.run([CLANG, "-std=c++17", "-O1", "-g", "-fsanitize=address", "-I", inc,
                    os.path.join(ROOT, "tests", "asan", "abi_errors_decode.cpp"), *objs, "-L/opt/rocm/lib", "-lamdhip64",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    assert "Sanitizer" not in r.stderr, r.stderr[-4000:]
    assert r.returncode == 0 and r.stdout.strip().endswith("ok: 0 failure(s)"), r.stdout[-4000:] + r.stderr[-2000:]


@pytest.mark.parametrize("name,mirror", [("tq_kv_scope", tq.TqKvScope), ("tq_rope_call", tq.TqRopeCall),
                                         ("tq_logprobs_call", tq.TqLogprobsCall)])
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


def test_packed_calls_have_the_layout_of_their_structs():
    for packed, mirror in ((tq._ROPE_CALL, tq.TqRopeCall), (tq._LOGPROBS_CALL, tq.TqLogprobsCall),
                           (tq._ATTN_CALL, tq.TqKvAttn), (tq._SCOPE_CALL, tq.TqKvScope)):
        assert packed.size == ctypes.sizeof(mirror)
    # every member its own number, through the struct's names
    n = iter(range(1, 100))
    members = [next(n) for _ in range(7)] + [0.5] + [next(n) for _ in range(16)]
    call = tq.TqRopeCall.from_buffer_copy(tq._ROPE_CALL.pack(*members))
    assert (call.n_tokens, call.n_heads, call.n_kv_heads, call.head_dim, call.rot, call.n_axes, call.flags) == (
        1, 2, 3, 4, 5, 6, 7)
    assert (call.scale, call.positions, call.axis_stride, call.freq, call.axis) == (0.5, 8, 9, 10, 11)
    assert [(r.data, r.token_stride, r.head_stride) for r in (call.q, call.k, call.q_out, call.k_out)] == [
        (12, 13, 14), (15, 16, 17), (18, 19, 20), (21, 22, 23)]
    members = list(range(1, 6)) + [0.5] + list(range(6, 16))
    call = tq.TqLogprobsCall.from_buffer_copy(tq._LOGPROBS_CALL.pack(*members))
    assert (call.n_rows, call.n_vocab, call.n_ids, call.n_top, call.flags, call.scale) == (1, 2, 3, 4, 5, 0.5)
    assert (call.logits, call.ld, call.ids, call.logp, call.entropy, call.top_ids, call.top_logp, call.d_err,
            call.workspace, call.workspace_bytes) == tuple(range(6, 16))
    members = list(range(1, 7)) + [0.5] + list(range(7, 17))
    call = tq.TqKvAttn.from_buffer_copy(tq._ATTN_CALL.pack(*members))
    assert (call.n_rows, call.n_tokens, call.max_q, call.n_heads, call.max_len, call.window, call.scale, call.flags) == (
        1, 2, 3, 4, 5, 6, 0.5, 7)
    assert (call.seqs, call.cu_q, call.q.data, call.q.token_stride, call.q.head_stride, call.o, call.lse, call.workspace,
            call.workspace_bytes) == tuple(range(8, 17))
    call = tq.TqKvScope.from_buffer_copy(tq._SCOPE_CALL.pack(*range(1, 7)))
    assert (call.sinks, call.n_groups, call.max_prefix, call.max_tail, call.cu_rows, call.prefix) == tuple(range(1, 7))


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros((2, 4, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        tq.tq_rope(x, None, torch.zeros(2, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(ValueError):
        tq.tq_logprobs(x[0], top=3)
