"""The header of the products whose rows choose their weights as plain C99, its structures and
constants against the binding's, and the refusals that come before any device call. No GPU is used."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pj():
    from paper_2608_17310_gb300 import build, project
    build.build_library()
    project._lib()
    return project


def test_structures_match_the_header(pj, tmp_path):
    names = {n: getattr(pj, n) for n in ("es_weights_desc_t", "es_adapters_desc_t", "es_project_t", "es_project_experts_t",
                                         "es_route_t", "es_combine_t")}
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "es_project.h"', "int main(void) {"]
    want = []
    for n, s in names.items():
        lines.append(f'  printf("%zu\\n", sizeof({n}));')
        want.append(ctypes.sizeof(s))
        for f, _ in s._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({n}, {f}));')
            want.append(getattr(s, f).offset)
    lines += ["  return 0;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", f"-I{os.path.join(ROOT, 'include')}", str(src), "-o",
                    str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [int(x) for x in out.split()] == want


def test_constants_are_the_headers(pj):
    with open(os.path.join(ROOT, "include", "es_project.h")) as f:
        defined = dict(re.findall(r"#define (ES_\w+) (\d+)", f.read()))
    assert {k: int(v) for k, v in defined.items()} == {k: getattr(pj, k) for k in defined}
    assert set(defined) == {"ES_MAX_EXPERTS", "ES_MAX_ROWS", "ES_PROJECT_GAVE_UP"}


def create(call, structure):
    handle = ctypes.c_void_p(1)
    status = call(None if structure is None else ctypes.byref(structure), ctypes.byref(handle))
    assert handle.value is None
    return status


def test_descriptions_are_checked_before_the_device(pj):
    from paper_2608_17310_gb300 import esopt as es
    bad, align = es.ES_ERR_INVALID_ARG, es.ES_ERR_ALIGNMENT
    L = pj._lib()

    def weights(**kw):
        return create(L.es_weights_create, pj.es_weights_desc_t(**(dict(
            data=0x10000, scale=0, group_stride=64 * 128, row_stride=128, groups=2, out_features=64, in_features=128, dtype=es.ES_BF16) | kw)))

    def adapters(**kw):
        return create(L.es_adapters_create, pj.es_adapters_desc_t(**(dict(
            a=0x10000, b=0x20000, scale=0, a_stride=16 * 128, b_stride=16 * 64, count=2, rank=16, out_features=64, in_features=128) | kw)))

    assert create(L.es_weights_create, None) == bad and create(L.es_adapters_create, None) == bad
    fp8 = dict(dtype=es.ES_FP8_E4M3, scale=0x40)
    for kw in (dict(dtype=es.ES_FP32), dict(data=0), dict(groups=0), dict(groups=1025), dict(out_features=0), dict(out_features=60),
               dict(out_features=2 ** 20 + 8), dict(in_features=4), dict(in_features=0), dict(in_features=2 ** 17 + 8), dict(row_stride=120),
               dict(group_stride=64 * 128 - 8), dict(group_stride=2 ** 40), dict(scale=0x40), dict(dtype=es.ES_FP8_E4M3),
               fp8 | dict(in_features=120)):
        assert weights(**kw) == bad, kw
    for kw in (dict(data=0x10008), dict(row_stride=132, group_stride=64 * 132), dict(group_stride=64 * 128 + 4),
               fp8 | dict(row_stride=136, group_stride=64 * 136)):
        assert weights(**kw) == align, kw
    for kw in (dict(a=0), dict(b=0), dict(count=0), dict(count=65537), dict(rank=0), dict(rank=12), dict(rank=136), dict(out_features=4),
               dict(in_features=12), dict(a_stride=16 * 128 - 8), dict(b_stride=16 * 64 - 8)):
        assert adapters(**kw) == bad, kw
    for kw in (dict(a=0x10008), dict(b=0x20002), dict(a_stride=16 * 128 + 4), dict(b_stride=16 * 64 + 4)):
        assert adapters(**kw) == align, kw
    # what passes every host check fails at the device: there is none here, and with one these
    # addresses are no device memory
    assert weights() in (es.ES_ERR_CUDA, bad) and adapters() in (es.ES_ERR_CUDA, bad)
    assert weights(**fp8) in (es.ES_ERR_CUDA, bad)
    # a single matrix has no group_stride
    assert weights(groups=1, group_stride=1) in (es.ES_ERR_CUDA, bad)


def test_calls_without_handles_are_refused(pj):
    from paper_2608_17310_gb300 import esopt as es
    L = pj._lib()
    for layout, call in ((pj._PROJECT, lambda a: L.es_project(None, None, a, None, 0, None)),
                         (pj._EXPERTS, lambda a: L.es_project_experts(None, a, None, 0, None))):
        assert call(bytes(layout.size)) == es.ES_ERR_INVALID_ARG
        assert "weights is NULL" in es.es_last_error()
    assert L.es_route(None, None, 0, None) == es.ES_ERR_INVALID_ARG
    assert L.es_combine(None, None) == es.ES_ERR_INVALID_ARG
    assert L.es_project_workspace(None, None, 8) == 0
    assert L.es_weights_destroy(None) == es.ES_OK and L.es_adapters_destroy(None) == es.ES_OK


def test_route_and_combine_check_their_numbers_before_the_device(pj):
    from paper_2608_17310_gb300 import esopt as es
    L = pj._lib()
    L.es_route.argtypes, saved = [ctypes.POINTER(pj.es_route_t), ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p], L.es_route.argtypes
    try:
        for kw in (dict(experts=0), dict(experts=1025), dict(top=0), dict(top=33), dict(top=9), dict(tokens=-1), dict(tokens=2 ** 24),
                   dict(normalise=2), dict(dtype=es.ES_FP8_E4M3), dict(scores_stride=7), dict(scores_stride=2 ** 41)):
            a = pj.es_route_t(**(dict(scores=64, chosen=64, weights=64, start=64, rows=64, places=64, scores_stride=8, tokens=4,
                                      experts=8, top=2, normalise=1, dtype=es.ES_FP32) | kw))
            assert L.es_route(ctypes.byref(a), None, 0, None) == es.ES_ERR_INVALID_ARG, kw
    finally:
        L.es_route.argtypes = saved
    for kw, status in ((dict(features=4), 1), (dict(features=2 ** 20 + 8), 1), (dict(top=0), 1), (dict(top=33), 1), (dict(slots=-1), 1),
                       (dict(tokens=2 ** 24 + 1), 1), (dict(y_stride=56), 1), (dict(out_stride=68), 2), (dict(add=64, add_stride=0), 1)):
        a = pj.es_combine_t(**(dict(y=64, places=64, weights=64, add=0, out=64, y_stride=64, add_stride=0, out_stride=64, slots=4,
                                    tokens=4, top=2, features=64) | kw))
        assert L.es_combine(bytes(a), None) == status, kw
    assert L.es_route_workspace(10, 8, 9) == 0 and L.es_route_workspace(-1, 8, 2) == 0 and L.es_route_workspace(10, 8, 2) > 0


def test_numbers_that_c_does_not_hold_are_value_errors(pj):
    w = pj.Weights(None, ())
    for rows in (2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            pj.es_project_workspace(w, rows)
        with pytest.raises(ValueError):
            pj.es_route_workspace(rows, 8, 2)
