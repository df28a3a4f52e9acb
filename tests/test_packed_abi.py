"""The calls of the 4-bit cache without a GPU: arguments that are refused on the host before
any device call."""

import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_21827_amd", "librheo.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="librheo.so not built")


def test_null_handles_are_refused():
    from paper_2609_21827_amd import binding
    lib = binding.load_library()
    for rc in (lib.rheo_packed_append(None, None, None, None),
               lib.rheo_packed_read(None, None, None, None),
               lib.rheo_packed_attention(None, None, None),
               lib.rheo_packed_commit(None, None, None)):
        assert rc == binding.RHEO_EINVAL and lib.rheo_last_error().decode()


@pytest.mark.parametrize("D,page,want", [(128, 64, 64 * 68), (8, 16, 16 * 17), (80, 16, 16 * 51),
                                         (256, 4096, 4096 * 136)])
def test_page_bytes(D, page, want):
    from paper_2609_21827_amd import binding
    assert binding.load_library().rheo_packed_page_bytes(D, page) == want


def test_small_pages_are_refused():
    from paper_2609_21827_amd import binding
    binding.load_library()
    with pytest.raises(binding.RheoError, match="page_size") as e:
        binding.PackedCache(1, 1, 1, 64, 8, 4, 1)
    assert e.value.code == binding.RHEO_EINVAL
