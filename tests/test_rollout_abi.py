"""The rollout operators' header as plain C99, its structures against the binding's, and the
refusals that come before any device call. No GPU is used."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ro():
    from paper_2608_17310_gb300 import build, rollout
    build.build_library()
    rollout._lib()
    return rollout


def test_structures_match_the_header(ro, tmp_path):
    names = {"es_cache_desc_t": ro.es_cache_desc_t, "es_batch_t": ro.es_batch_t, "es_append_t": ro.es_append_t,
             "es_attention_t": ro.es_attention_t}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "es_rollout.h"', "int main(void) {"]
    want = []
    for n, s in names.items():
        lines.append(f'  printf("%zu\\n", sizeof({n}));')
        want.append(ctypes.sizeof(s))
        for f, _ in s._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({n}, {f}));')
            want.append(getattr(s, f).offset)
    lines += ["  return ES_MAX_SEQUENCES == 4096 ? 0 : 1;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [int(x) for x in out.split()] == want


def desc(ro, **kw):
    d = dict(k=0x10000, v=0x20000, k_scale=0, v_scale=0, num_pages=4, page_stride=2 * 16 * 128, scale_stride=0,
             page_size=16, kv_heads=2, head_dim=128, dtype=ro.ES_BF16) | kw
    return ro.es_cache_desc_t(**d)


def create(ro, d):
    handle = ctypes.c_void_p(1)
    status = ro._lib().es_cache_create(None if d is None else ctypes.byref(d), ctypes.byref(handle))
    assert handle.value is None
    return status


def test_cache_descriptions_are_checked_before_the_device(ro):
    from paper_2608_17310_gb300 import esopt as es
    bad, align = es.ES_ERR_INVALID_ARG, es.ES_ERR_ALIGNMENT
    assert create(ro, None) == bad
    for kw in (dict(dtype=es.ES_FP32), dict(page_size=8), dict(page_size=48), dict(page_size=256), dict(head_dim=96),
               dict(kv_heads=0), dict(kv_heads=1025), dict(num_pages=0), dict(num_pages=2 ** 31),
               dict(page_stride=2 * 16 * 128 - 8), dict(page_stride=2 ** 60), dict(k=0), dict(v=0), dict(k_scale=0x30000),
               dict(dtype=es.ES_FP8_E4M3), dict(dtype=es.ES_FP8_E4M3, k_scale=64, v_scale=64, scale_stride=31),
               dict(dtype=es.ES_FP8_E4M3, scale_stride=32)):
        assert create(ro, desc(ro, **kw)) == bad, kw
    for kw in (dict(k=0x10008), dict(v=0x20002), dict(page_stride=2 * 16 * 128 + 4),
               dict(dtype=es.ES_FP8_E4M3, k_scale=64, v_scale=64, scale_stride=32, page_stride=2 * 16 * 128 + 8)):
        assert create(ro, desc(ro, **kw)) == align, kw
    # addresses that pass every host check fail at the device: there is none here, and with one
    # they are no device memory
    assert create(ro, desc(ro)) in (es.ES_ERR_CUDA, bad)


def test_calls_without_a_cache_are_refused(ro):
    from paper_2608_17310_gb300 import esopt as es
    L, b = ro._lib(), ro.es_batch_t()
    assert L.es_cache_append(None, ctypes.byref(b), ctypes.byref(ro.es_append_t()), None) == es.ES_ERR_INVALID_ARG
    assert L.es_cache_read(None, ctypes.byref(b), None, None, None) == es.ES_ERR_INVALID_ARG
    assert L.es_attention(None, ctypes.byref(b), ctypes.byref(ro.es_attention_t()), None, 0, None) == es.ES_ERR_INVALID_ARG
    assert "cache is NULL" in es.es_last_error()
    assert L.es_attention_workspace(None, 8) == 0
    assert L.es_cache_destroy(None) == es.ES_OK
