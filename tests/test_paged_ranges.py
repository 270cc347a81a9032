"""Caps and scales at the ends of float32, over prompts and pages: refused on the host where a factor of the kernels would be infinite."""
import ctypes as C

import pytest

import paper_2508_06526_amd as pk
from test_paged_abi import FAKE, UNSUPPORTED, WORKSPACE, desc, mass, pages, prompt

RANGES = [  # scale, cap, whether 1 / cap and scale / cap are numbers of float32
    (0.0, 1e-37, True), (0.0, 2.0 ** -127, True), (0.0, 2.0 ** -128, False), (0.0, 1e-39, False), (0.0, 1e-45, False), (1.0, 3.4e38, True), (0.0, 0.0, True),
    (1e30, 1e-8, True), (1e30, 1e-9, False), (3e38, 1.0, True), (3e38, 0.5, False), (1e-45, 3.4e38, True), (1e-38, 0.0, True), (3e38, 0.0, True)]


@pytest.fixture(scope="module")
def lib():
    return pk.load_library()


@pytest.mark.parametrize("scale,cap,fine", RANGES)
def test_utilities_of_a_prompt(lib, scale, cap, fine):
    assert mass(lib, scale=scale, cap=cap, ws=None) == (WORKSPACE if fine else UNSUPPORTED)


@pytest.mark.parametrize("scale,cap,fine", RANGES)
def test_attention_over_pages(lib, scale, cap, fine):
    args = [FAKE] * 7, [2, 0, scale, cap, None, 0, None, FAKE, FAKE, FAKE], [None] * 5, [0, None]
    assert lib.pikv_paged_attn(C.byref(desc()), C.byref(pages()), *sum(args, [])) == (WORKSPACE if fine else UNSUPPORTED)


@pytest.mark.parametrize("scale,cap,fine", RANGES)
def test_attention_of_a_prompt(lib, scale, cap, fine):
    """Its scores are kept in units of the cap, or of the scale, which go to the base 2."""
    unit = cap if cap > 0 else max(scale, 1.0)
    assert prompt(lib, scale=scale, cap=cap, tokens=0) == (0 if fine and unit < 2.3e38 else UNSUPPORTED)
    f = lambda slopes: lib.pikv_prompt_attn(FAKE, FAKE, FAKE, 0, 512, 256, 256, 8, 4, 64, 1, FAKE, 2, 6, None, scale, cap, slopes, 0, FAKE, None, None, None)
    assert f(FAKE) == (0 if fine else UNSUPPORTED)
