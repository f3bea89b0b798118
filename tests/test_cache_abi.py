"""Host side of include/fly_cache.h without a GPU: every refusal comes before any CUDA call."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_22972_b200 import binding as Bd, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = Bd.FLY_ERR_INVALID_ARG, Bd.FLY_ERR_UNSUPPORTED
A = 1 << 20     # an address that is never followed


def test_every_declared_symbol_is_exported_and_listed():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "fly_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(fly_[a-z_]+)\s*\(", text)))
    assert names == sorted(cache.EXPORTS)
    assert all(hasattr(cache.lib(), n) for n in names)


def test_struct_layout_matches_the_header(tmp_path):
    src = tmp_path / "h.c"
    src.write_text('#include <stddef.h>\n#include "fly_cache.h"\n#define S(c, e) typedef char t_##c[(e) ? 1 : -1]\n'
                   f"S(a, sizeof(fly_cache_t) == {C.sizeof(cache.fly_cache_t)}); S(b, offsetof(fly_cache_t, lengths) == {cache.fly_cache_t.lengths.offset});\n"
                   f"S(c, offsetof(fly_cache_t, page_stride) == {cache.fly_cache_t.page_stride.offset}); S(d, sizeof(fly_rows_t) == {C.sizeof(cache.fly_rows_t)});\n"
                   f"S(e, sizeof(fly_attention_args_t) == {C.sizeof(cache.fly_attention_args_t)}); S(f, offsetof(fly_attention_args_t, scale) == {cache.fly_attention_args_t.scale.offset});\n"
                   f"S(g, offsetof(fly_attention_args_t, counts) == {cache.fly_attention_args_t.counts.offset}); S(h, sizeof(fly_attention_config_t) == 24);\n"
                   "int main(void) { return 0; }\n")
    inc = os.path.join(ROOT, "include")
    if shutil.which("gcc"):
        subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", inc, "-fsyntax-only", str(src)], check=True)
    if shutil.which("g++"):
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-I", inc, "-fsyntax-only", "-x", "c++", str(src)], check=True)


def good(**kw):
    v = dict(device=0, format=0, k_pages=A, v_pages=A, k_scales=None, v_scales=None, num_pages=10, page_size=16, kv_heads=2, head_dim=64,
             page_stride=2048, token_stride=128, head_stride=64, block_table=A, table_stride=4, max_pages=4, sequences=3, lengths=A)
    v.update(kw)
    return cache.fly_cache_t(**v)


CACHES = [
    (dict(device=-1), INVALID), (dict(format=2), INVALID), (dict(k_pages=None), INVALID), (dict(v_pages=None), INVALID),
    (dict(block_table=None), INVALID), (dict(lengths=None), INVALID), (dict(k_scales=A, v_scales=A), INVALID), (dict(format=1), INVALID),
    (dict(format=1, k_scales=A), INVALID), (dict(num_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(head_dim=0), INVALID), (dict(max_pages=0), INVALID), (dict(sequences=0), INVALID), (dict(table_stride=3), INVALID), (dict(sequences=1), INVALID),
    (dict(token_stride=-128), INVALID), (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(page_size=4), UNSUPPORTED),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=131072), UNSUPPORTED), (dict(max_pages=1 << 27, table_stride=1 << 27), UNSUPPORTED),
    (dict(k_pages=A + 8), UNSUPPORTED), (dict(page_stride=2052), UNSUPPORTED), (dict(token_stride=132), UNSUPPORTED), (dict(head_stride=68), UNSUPPORTED),
    (dict(block_table=A + 2), UNSUPPORTED), (dict(lengths=A + 1), UNSUPPORTED), (dict(format=1, k_scales=A + 4, v_scales=A), UNSUPPORTED), (dict(format=1, k_scales=A, v_scales=A, head_stride=72), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", CACHES)
def test_caches_that_are_refused(kw, status):
    L, c = cache.lib(), good(**kw)
    r = cache.fly_rows_t(A, 512, 128, 64)
    assert L.fly_cache_append(C.byref(c), 2, 4, C.byref(r), C.byref(r), None, None, None) == status
    assert L.fly_cache_read(C.byref(c), 2, 4, None, C.byref(r), C.byref(r), None) == status


@pytest.mark.parametrize("B,n,r,status", [
    (0, 4, (A, 512, 128, 64), INVALID), (4, 4, (A, 512, 128, 64), INVALID), (2, 0, (A, 512, 128, 64), INVALID), (2, 4, (None, 512, 128, 64), INVALID),
    (2, 4, (A, -512, 128, 64), INVALID), (2, 4, (A, 512, -1, 64), INVALID), (2, 4, (A + 1, 512, 128, 64), UNSUPPORTED),
    (2, (1 << 30) + 1, (A, 512, 128, 64), UNSUPPORTED)])
def test_rows_that_are_refused(B, n, r, status):
    L, c, r = cache.lib(), good(), cache.fly_rows_t(*r)
    assert L.fly_cache_append(C.byref(c), B, n, C.byref(r), C.byref(r), None, None, None) == status
    assert L.fly_cache_read(C.byref(c), B, n, None, C.byref(r), C.byref(r), None) == status
    r = cache.fly_rows_t(A, 512, 128, 64)
    assert L.fly_cache_append(None, 1, 1, C.byref(r), C.byref(r), None, None, None) == INVALID
    assert L.fly_cache_append(C.byref(c), 1, 1, None, C.byref(r), None, None, None) == INVALID
    assert L.fly_cache_read(C.byref(c), 1, 1, None, C.byref(r), None, None) == INVALID


@pytest.mark.parametrize("cfg,status", [
    ((-1, 1, 1, 8, 1, 64), INVALID), ((0, 0, 1, 8, 1, 64), INVALID), ((0, 1, 0, 8, 1, 64), INVALID), ((0, 1, 1, 0, 1, 64), INVALID),
    ((0, 1, 1, 8, 0, 64), INVALID), ((0, 1, 1, 8, 3, 64), INVALID), ((0, 1, 1, 8, 1, 0), INVALID), ((0, 1, 1, 8, 1, 96), UNSUPPORTED),
    ((0, 1, 1, 129, 1, 64), UNSUPPORTED)])
def test_attention_shapes_that_are_refused(cfg, status):
    L, h, c = cache.lib(), C.c_void_p(123), cache.fly_attention_config_t(*cfg)
    assert L.fly_attention_create(C.byref(c), C.byref(h)) == status and not h.value
    assert L.fly_attention_create(None, C.byref(h)) == INVALID and L.fly_attention_create(C.byref(c), None) == INVALID


def test_null_handles():
    L, c = cache.lib(), good()
    assert L.fly_attention_run(None, C.byref(c), None, None) == INVALID
    assert L.fly_attention_destroy(None) == Bd.FLY_OK
    assert L.fly_attention_last_launch_count(None) == 0 and L.fly_attention_last_cuda_error(None) == 0


def test_tensors_on_the_host_are_refused_in_python():
    import torch
    p = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA device"):
        cache.PagedCache(p, p.clone(), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    c = good()
    for bad in (p, None, torch.nested.nested_tensor([torch.zeros(2, 2, 64), torch.zeros(1, 2, 64)]), p.to_sparse(), 5):
        with pytest.raises((ValueError, RuntimeError)):
            Bd._native.cache_append(C.addressof(c), bad, bad, None, None, 0)
        with pytest.raises((ValueError, RuntimeError)):
            Bd._native.attention_run(0, C.addressof(c), 4, bad, bad, 0, 0, 0.0, None, None, 0)
    assert Bd._native.cache_append(0, p, p, None, None, 0) == INVALID


@pytest.mark.parametrize("kw", [dict(token_stride=0), dict(token_stride=56), dict(head_stride=0), dict(page_stride=0), dict(page_stride=56)])
def test_caches_whose_rows_overlap_are_refused(kw):
    test_caches_that_are_refused(kw, UNSUPPORTED)


@pytest.mark.parametrize("strides", [(0, 128, 64), (512, 0, 64), (512, 128, 0), (512, 128, 56)])
def test_rows_that_are_written_do_not_overlap(strides):
    L, c, r, ok = cache.lib(), good(), cache.fly_rows_t(A, *strides), cache.fly_rows_t(A, 512, 128, 64)
    assert L.fly_cache_read(C.byref(c), 2, 4, None, C.byref(r), C.byref(ok), None) == UNSUPPORTED
    assert L.fly_cache_read(C.byref(c), 2, 4, None, C.byref(ok), C.byref(r), None) == UNSUPPORTED


def test_device_integers_off_their_alignment_are_refused():
    L, c, r = cache.lib(), good(), cache.fly_rows_t(A, 512, 128, 64)
    assert L.fly_cache_append(C.byref(c), 2, 4, C.byref(r), C.byref(r), A + 1, None, None) == UNSUPPORTED
    assert L.fly_cache_append(C.byref(c), 2, 4, C.byref(r), C.byref(r), None, A + 2, None) == UNSUPPORTED
    assert L.fly_cache_read(C.byref(c), 2, 4, A + 3, C.byref(r), C.byref(r), None) == UNSUPPORTED
