"""The backend's C-ABI without a GPU: everything its header declares is exported and bound, records have the header's layout, and bad
configurations are refused before any CUDA call."""
import ctypes as C
import os
import re

import pytest

from paper_2603_20661_b200 import backend
from paper_2603_20661_b200 import build as cuda_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD = dict(n_heads=8, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=10, max_seqs=4, max_tokens=100, max_pages=5, max_rows=3, dtype=0, cache=1)


@pytest.fixture(scope="module")
def lib():
    cuda_build.build()
    return backend._lib()


def test_every_declared_function_is_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "wwws_backend.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(wwws_[a-z_0-9]+)\s*\(", text))
    assert names == set(backend.EXPORTS)
    for n in names:
        assert hasattr(lib, n), n


def test_struct_layouts_match_the_header():
    assert C.sizeof(backend.BackendConfig) == 11 * 4 and C.sizeof(backend.KvPages) == 32
    assert C.sizeof(backend.SeqBatch) == 3 * 8 + 4 * 4 and C.sizeof(backend.ShapingRecord) == 11 * 8 + 2 * 8 + 2 * 4


def test_configurations_are_checked_on_the_host(lib):
    n = C.c_uint64()
    ask = lambda **more: lib.wwws_backend_workspace_bytes(C.byref(backend.BackendConfig(**{**GOOD, **more})), C.byref(n))     # noqa: E731
    assert ask() == 0 and n.value > 0 and n.value % 256 == 0
    assert ask(n_heads=0) == 0                                      # logits alone
    for bad in (dict(n_heads=0, max_rows=0), dict(n_heads=9), dict(n_kv_heads=0), dict(n_heads=34), dict(head_dim=96), dict(page_tokens=8), dict(page_tokens=48),
                dict(page_tokens=256), dict(n_pages=0), dict(n_pages=1 << 26), dict(max_seqs=0), dict(max_seqs=2049), dict(max_tokens=0), dict(max_tokens=1 << 27),
                dict(max_pages=0), dict(max_pages=1 << 26), dict(max_rows=65536), dict(dtype=2), dict(cache=3), dict(n_heads=2048, n_kv_heads=1024)):
        assert ask(**bad) == 1, bad
        assert len(lib.wwws_backend_last_error(None)) > 0
    assert lib.wwws_backend_workspace_bytes(None, C.byref(n)) == 1 and lib.wwws_backend_workspace_bytes(C.byref(backend.BackendConfig(**GOOD)), None) == 1


def test_creation_and_null_handles(lib):
    cfg, h = backend.BackendConfig(**GOOD), C.c_void_p()
    assert lib.wwws_create_backend(C.byref(cfg), None, 0, None, C.byref(h)) == 2 and h.value is None
    assert lib.wwws_create_backend(C.byref(cfg), 8, 1 << 40, None, C.byref(h)) == 2               # misaligned
    assert lib.wwws_create_backend(C.byref(cfg), 256, 16, None, C.byref(h)) == 2                  # too small
    assert lib.wwws_create_backend(C.byref(cfg), 256, 1 << 40, None, None) == 1
    assert lib.wwws_create_backend(None, 256, 1 << 40, None, C.byref(h)) == 1
    assert lib.wwws_destroy_backend(None) == 0 and lib.wwws_backend_sync(None) == 1
    assert lib.wwws_attend(None, None, None, None, 0, None, 0, 1.0, 0, 0) == 1
    assert lib.wwws_cache_append(None, None, None, None, 0, None, 0) == 1 and lib.wwws_cache_read(None, None, None, None, 0, None, None) == 1
    assert lib.wwws_shape_logits(None, None, 0, 0, 0, None, 0, None, 0, None) == 1
