"""Page sizes of the 4-bit cache, asked for before there is a handle."""

import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_21827_amd", "librheo.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="librheo.so not built")


def _bytes(D, page):
    from paper_2609_21827_amd import binding
    return binding.load_library().rheo_packed_page_bytes(D, page)


def test_every_size_that_a_handle_may_have():
    for D in range(8, 257, 8):
        for page in (16, 32, 64, 128, 256, 512, 1024, 2048, 4096):
            assert _bytes(D, page) == page * -(-D // 32) * 17


@pytest.mark.parametrize("D,page", [(128, 8), (128, 0), (128, -64), (128, 48), (128, 8192), (0, 64),
                                    (-128, 64), (12, 64), (264, 64), (256, 1 << 24), (1 << 30, 1 << 30),
                                    (2 ** 31 - 1, 64), (-2 ** 31, -2 ** 31), (128, 2 ** 31 - 1)])
def test_other_sizes_have_no_bytes(D, page):
    """None of these is a handle's; products of the larger ones do not fit 32 bits."""
    assert _bytes(D, page) == 0
