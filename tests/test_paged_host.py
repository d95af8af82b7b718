"""Host-only checks of the paged operators' C ABI: every refusal happens before any HIP call and says why; struct layouts; the
header as plain C."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2601_17917_amd as sd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(1 << 20)           # aligned, never read: validation ends before any launch
ODD = ctypes.c_void_p((1 << 20) + 2)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sd.LIB_PATH):
        from paper_2601_17917_amd.build import build
        build(verbose=False)
    return sd.load_library()


def refused(lib, rc, code, word):
    text = lib.sdllm_last_error().decode()
    assert rc == code and word in text, (rc, text)


def test_layouts_and_plain_c(tmp_path, lib):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    src = tmp_path / "c.c"
    src.write_text('''#include <stdio.h>
#include "sdllm_paged.h"
int main(void) {
  sdllm_paged_extend_params e = {4, 1, 16, 8, 100};
  printf("%zu %zu %zu %zu\\n", sizeof(sdllm_paged_extend_params), sizeof(sdllm_qk_norm_rope_params),
         sizeof(sdllm_paged_append_params), sizeof(sdllm_paged_attn_params));
  if (sdllm_paged_extend_workspace_bytes(&e) == (size_t)-1) return 1;
  e.page_size = 24;
  if (sdllm_paged_extend_workspace_bytes(&e) != (size_t)-1) return 2;
  return 0;
}
''')
    exe = tmp_path / "c_prog"
    libdir = os.path.dirname(sd.LIB_PATH)
    r = subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                        str(exe), "-L", libdir, "-l:libsdllm.so", "-Wl,-rpath," + libdir, "-Wl,-rpath,/opt/rocm/lib"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    sizes = [ctypes.sizeof(c) for c in (sd.PagedExtendParams, sd.QkNormRopeParams, sd.PagedAppendParams, sd.PagedAttnParams)]
    assert r.stdout.split() == [str(n) for n in sizes]


EXTEND = dict(B=4, K=2, page_size=16, max_pages=8, n_pages=100)


@pytest.mark.parametrize("change,code,word", [
    (dict(B=0), sd.ERR_INVALID_ARG, "must be >= 1"), (dict(K=0), sd.ERR_INVALID_ARG, "must be >= 1"),
    (dict(max_pages=0), sd.ERR_INVALID_ARG, "must be >= 1"), (dict(n_pages=0), sd.ERR_INVALID_ARG, "n_pages"),
    (dict(page_size=24), sd.ERR_UNSUPPORTED, "page_size"), (dict(page_size=8), sd.ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=2048), sd.ERR_UNSUPPORTED, "page_size"), (dict(page_size=-16), sd.ERR_UNSUPPORTED, "page_size"),
    (dict(n_pages=1 << 27), sd.ERR_UNSUPPORTED, "2^31"), (dict(B=65537), sd.ERR_UNSUPPORTED, "too large"),
    (dict(B=65536, K=1 << 15), sd.ERR_UNSUPPORTED, "too large"), (dict(max_pages=1 << 27), sd.ERR_UNSUPPORTED, "too large"),
    (dict(B=65536, max_pages=1 << 14), sd.ERR_UNSUPPORTED, "too large"),
])
def test_extend_refuses(lib, change, code, word):
    p = sd.PagedExtendParams(**dict(EXTEND, **change))
    refused(lib, lib.sdllm_paged_extend(ctypes.byref(p), *[P] * 11, P, 1 << 30, None), code, word)
    assert lib.sdllm_paged_extend_workspace_bytes(ctypes.byref(p)) == ctypes.c_size_t(-1).value


def test_extend_refuses_pointers(lib):
    p = sd.PagedExtendParams(**EXTEND)
    for i in (0, 1, 5, 6, 7, 8, 9, 10):
        args = [P] * 11
        args[i] = None
        refused(lib, lib.sdllm_paged_extend(ctypes.byref(p), *args, None, 0, None), sd.ERR_INVALID_ARG, "NULL")
        args[i] = ODD
        refused(lib, lib.sdllm_paged_extend(ctypes.byref(p), *args, None, 0, None), sd.ERR_INVALID_ARG, "aligned")
    refused(lib, lib.sdllm_paged_extend(None, *[P] * 11, None, 0, None), sd.ERR_INVALID_ARG, "NULL")
    p.B, p.K = 100, 4000
    need = lib.sdllm_paged_extend_workspace_bytes(ctypes.byref(p))
    if need:
        refused(lib, lib.sdllm_paged_extend(ctypes.byref(p), *[P] * 11, P, need - 1, None), sd.ERR_WORKSPACE, "workspace")
        refused(lib, lib.sdllm_paged_extend(ctypes.byref(p), *[P] * 11, None, need, None), sd.ERR_WORKSPACE, "workspace")


NORM = dict(dtype=sd.BF16, B=2, K=3, Hq=4, Hkv=2, D=64, rotary_dim=64, page_size=16, n_pages=10, eps=1e-6, theta_base=1e4,
            scale_factor=1.0, low_turns=1.0, high_turns=32.0, amplitude=1.0)
S3 = ctypes.c_int64 * 3


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=2), sd.ERR_UNSUPPORTED, "dtype"), (dict(B=0), sd.ERR_INVALID_ARG, ">= 1"), (dict(Hkv=0), sd.ERR_INVALID_ARG, ">= 1"),
    (dict(D=72), sd.ERR_UNSUPPORTED, "head_dim"), (dict(D=272), sd.ERR_UNSUPPORTED, "head_dim"), (dict(D=0), sd.ERR_UNSUPPORTED, "head_dim"),
    (dict(rotary_dim=80), sd.ERR_INVALID_ARG, "rotary_dim"), (dict(rotary_dim=24), sd.ERR_INVALID_ARG, "rotary_dim"),
    (dict(rotary_dim=-16), sd.ERR_INVALID_ARG, "rotary_dim"), (dict(eps=-1.0), sd.ERR_INVALID_ARG, "eps"),
    (dict(eps=float("nan")), sd.ERR_INVALID_ARG, "eps"), (dict(theta_base=1.0), sd.ERR_INVALID_ARG, "theta_base"),
    (dict(scale_factor=0.5), sd.ERR_INVALID_ARG, "scale_factor"), (dict(scale_factor=float("inf")), sd.ERR_INVALID_ARG, "scale_factor"),
    (dict(amplitude=float("nan")), sd.ERR_INVALID_ARG, "amplitude"), (dict(original_len=-1), sd.ERR_INVALID_ARG, "original_len"),
    (dict(original_len=100, low_turns=32.0), sd.ERR_INVALID_ARG, "low_turns"), (dict(B=1 << 12, K=1 << 12), sd.ERR_UNSUPPORTED, "too large"),
    (dict(q_stride=S3(4, 0, 0)), sd.ERR_INVALID_ARG, "16 bytes"), (dict(k_stride=S3(-8, 0, 0)), sd.ERR_INVALID_ARG, "negative"),
    (dict(q_out_stride=S3(192, 64, 64)), sd.ERR_INVALID_ARG, "overlap"), (dict(k_out_stride=S3(1 << 41, 64, 128)), sd.ERR_UNSUPPORTED, "large"),
])
def test_norm_rope_refuses(lib, change, code, word):
    p = sd.QkNormRopeParams(**dict(NORM, **change))
    dense = [P, P, None, P, P, P, P, P, None, None, None]
    refused(lib, lib.sdllm_qk_norm_rope(ctypes.byref(p), *dense, None), code, word)


def test_norm_rope_refuses_pointers(lib):
    p = sd.QkNormRopeParams(**NORM)
    call = lambda args: lib.sdllm_qk_norm_rope(ctypes.byref(p), *args, None)
    dense, paged = [P, P, None, P, P, P, P, P, None, None, None], [P, P, P, P, P, P, P, None, P, P, P]
    for i in (0, 1, 3, 6):
        refused(lib, call(dense[:i] + [None] + dense[i + 1:]), sd.ERR_INVALID_ARG, "NULL")
    for i in (2, 8, 9):
        refused(lib, call(dense[:i] + [P] + dense[i + 1:]), sd.ERR_INVALID_ARG, "either")
        refused(lib, call(paged[:i] + [None] + paged[i + 1:]), sd.ERR_INVALID_ARG, "either")
    refused(lib, call(dense[:7] + [None] * 4), sd.ERR_INVALID_ARG, "either")
    refused(lib, call(paged[:7] + [P] + paged[8:]), sd.ERR_INVALID_ARG, "either")
    for i in (0, 1, 2, 4, 5, 6, 8, 9):
        refused(lib, call(paged[:i] + [ODD] + paged[i + 1:]), sd.ERR_INVALID_ARG, "aligned")
    p.page_size = 17
    refused(lib, call(paged), sd.ERR_UNSUPPORTED, "page_size")


APPEND = dict(dtype=sd.BF16, n_layers=2, B=2, Hkv=2, D=64, K=3, page_size=16, n_pages=10)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=5), sd.ERR_UNSUPPORTED, "dtype"), (dict(n_layers=0), sd.ERR_INVALID_ARG, ">= 1"), (dict(K=0), sd.ERR_INVALID_ARG, ">= 1"),
    (dict(D=12), sd.ERR_UNSUPPORTED, "row size"), (dict(page_size=40), sd.ERR_UNSUPPORTED, "page_size"),
    (dict(n_pages=1 << 28), sd.ERR_UNSUPPORTED, "2^31"), (dict(K=1 << 30, Hkv=64), sd.ERR_UNSUPPORTED, "too large"),
    (dict(pages_layer_stride=10 * 16 * 2 * 64 - 8), sd.ERR_INVALID_ARG, "pages_layer_stride"),
    (dict(pages_layer_stride=10 * 16 * 2 * 64 + 4), sd.ERR_INVALID_ARG, "pages_layer_stride"),
    (dict(block_layer_stride=2 * 2 * 3 * 64 - 8), sd.ERR_INVALID_ARG, "block_layer_stride"),
])
def test_append_refuses(lib, change, code, word):
    p = sd.PagedAppendParams(**dict(APPEND, **change))
    refused(lib, lib.sdllm_paged_kv_append(ctypes.byref(p), *[P] * 5, None), code, word)


def test_append_refuses_pointers(lib):
    p = sd.PagedAppendParams(**APPEND)
    for i in range(5):
        for bad, word in ((None, "NULL"), (ODD, "aligned")):
            args = [P] * 5
            args[i] = bad
            refused(lib, lib.sdllm_paged_kv_append(ctypes.byref(p), *args, None), sd.ERR_INVALID_ARG, word)


ATTN = dict(dtype=sd.BF16, B=2, Hq=4, Hkv=2, D=64, K=1, page_size=16, n_pages=10, max_pages=5, max_kv_len=80)


@pytest.mark.parametrize("change,code,word", [
    (dict(dtype=3), sd.ERR_UNSUPPORTED, "dtype"), (dict(K=0), sd.ERR_INVALID_ARG, ">= 1"), (dict(Hq=5), sd.ERR_INVALID_ARG, "multiple"),
    (dict(D=96), sd.ERR_UNSUPPORTED, "head_dim"), (dict(page_size=48), sd.ERR_UNSUPPORTED, "page_size"),
    (dict(max_pages=0, max_kv_len=0), sd.ERR_INVALID_ARG, "max_pages"), (dict(max_kv_len=81), sd.ERR_INVALID_ARG, "max_kv_len"),
    (dict(max_kv_len=-1), sd.ERR_INVALID_ARG, "max_kv_len"), (dict(window=-1), sd.ERR_INVALID_ARG, "window"),
    (dict(sinks=-1), sd.ERR_INVALID_ARG, "sinks"), (dict(kv_splits=-1), sd.ERR_INVALID_ARG, "kv_splits"),
    (dict(scale=float("nan")), sd.ERR_INVALID_ARG, "scale"), (dict(B=1 << 22, Hq=1, Hkv=1), sd.ERR_UNSUPPORTED, "too large"),
    (dict(K=(1 << 30) - 79, Hq=2), sd.ERR_UNSUPPORTED, "too large"), (dict(out_stride=S3(0, 64, 64)), sd.ERR_INVALID_ARG, "overlap"),
    (dict(q_stride=S3(0, 0, 4)), sd.ERR_INVALID_ARG, "16 bytes"), (dict(k_block_stride=S3(12, 0, 0)), sd.ERR_INVALID_ARG, "16 bytes"),
])
def test_attention_refuses(lib, change, code, word):
    p = sd.PagedAttnParams(**dict(ATTN, **change))
    refused(lib, lib.sdllm_paged_attention(ctypes.byref(p), *[P] * 9, P, 1 << 40, None), code, word)
    assert lib.sdllm_paged_attention_workspace_bytes(ctypes.byref(p), 1) == ctypes.c_size_t(-1).value


def test_attention_refuses_pointers(lib):
    p = sd.PagedAttnParams(**ATTN)
    call = lambda args: lib.sdllm_paged_attention(ctypes.byref(p), *args, P, 1 << 40, None)
    for i in (0, 1, 2, 3, 4, 8):
        refused(lib, call([P] * i + [None] + [P] * (8 - i)), sd.ERR_INVALID_ARG, "NULL")
    for i in (5, 6):
        refused(lib, call([P] * i + [None] + [P] * (8 - i)), sd.ERR_INVALID_ARG, "both")
    for i in range(9):
        refused(lib, call([P] * i + [ODD] + [P] * (8 - i)), sd.ERR_INVALID_ARG, "aligned")
    p = sd.PagedAttnParams(**dict(ATTN, B=4, max_pages=5000, max_kv_len=80000, n_pages=20000))
    need = lib.sdllm_paged_attention_workspace_bytes(ctypes.byref(p), 0)
    if need:
        args = [P, P, P, P, P, None, None, None, P]
        refused(lib, lib.sdllm_paged_attention(ctypes.byref(p), *args, P, need - 1, None), sd.ERR_WORKSPACE, "workspace")
        refused(lib, lib.sdllm_paged_attention(ctypes.byref(p), *args, None, need, None), sd.ERR_WORKSPACE, "workspace")


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    q, pages = torch.zeros(1, 2, 1, 64), torch.zeros(3, 1, 16, 64)
    table, lens = torch.zeros(1, 3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: sd.paged_attention(q, pages, pages, table, lens, 16, out=q),
                 lambda: sd.paged_attention(q, pages, pages, table, lens, 16, k_block=q, out=q),
                 lambda: sd.paged_kv_append(pages[None], pages[None], q[None], q[None], table[:, :1]),
                 lambda: sd.qk_norm_rope(q, q, lens, 1e4, q_out=q, k_out=q),
                 lambda: sd.qk_norm_rope(q, q, lens, 1e4, q_out=q, k_out=q, v=q),
                 lambda: sd.paged_extend(table, lens, lens, lens, 16, 1, slots=table, granted=lens)):
        with pytest.raises(sd.SdllmError):
            call()
