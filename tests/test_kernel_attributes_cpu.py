"""What is asked of a kernel once a device before its first launch: a question that failed is asked again, and a kernel with fewer registers
than its warps move among themselves is not launched.  The host's code alone, without a GPU."""
import ctypes

import pytest

from test_rules_cpu import compile_host

SUCCESS, NOT_READY, OUT_OF_RESOURCES = 0, 600, 701


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    return compile_host(str(tmp_path_factory.mktemp("attributes")), """
        #include "kvd_internal.h"
        using namespace kvd;
        extern "C" int enough(int warps, int needed, int registers, int answer)
        {
            return enough_registers(warps, needed, [&](int* n) { *n = registers; return (cudaError_t)answer; });
        }
        static int asked;
        extern "C" int times_asked() { return asked; }
        extern "C" int launch(int registers, int answer)
        {
            static OncePerDevice once;
            return once(0, [&] { return enough_registers(12, 2016, [&](int* n) { ++asked; *n = registers; return (cudaError_t)answer; }); });
        }
        """)


def test_registers_are_compared_as_they_are_handed_out(shim):
    for registers, fits in ((168, 1), (167, 1), (161, 1), (160, 0), (128, 0), (176, 1), (255, 1), (0, 0)):
        assert shim.enough(12, 8 * 208 + 4 * 88, registers, SUCCESS) == (SUCCESS if fits else OUT_OF_RESOURCES), registers
    assert shim.enough(12, 2016, 168, NOT_READY) == NOT_READY


def test_a_failed_question_is_asked_again(shim):
    """Also where the failure left nothing, or something, in place of the answer."""
    assert shim.launch(0, NOT_READY) == NOT_READY
    assert shim.launch(168, NOT_READY) == NOT_READY
    assert shim.launch(160, SUCCESS) == OUT_OF_RESOURCES
    assert shim.launch(168, SUCCESS) == SUCCESS and shim.times_asked() == 4
    assert shim.launch(0, NOT_READY) == SUCCESS and shim.times_asked() == 4
