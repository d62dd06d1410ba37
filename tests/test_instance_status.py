"""CPU checks of the instance's status call."""
import ctypes as C

import pytest

from paper_2509_06362_amd import binding, instance as I


@pytest.fixture(scope="module")
def lib():
    if not binding.LIB_PATH.exists():
        from paper_2509_06362_amd import build
        build.build_library()
    return I._library()


def test_the_status_waits_for_nobody_elses_call(lib):
    """An instance of which every word is taken: some call is in it.  Nothing else of it is looked at."""
    taken, bits = C.create_string_buffer(b"\1" * 4096, 4096), C.c_uint32(7)
    assert lib.maaso_instance_status(taken, C.byref(bits)) == -8 and bits.value == 0


def test_a_closed_instance_has_no_status(lib):
    with pytest.raises(I.MaasoError) as e:
        I.maaso_instance_status(I.Instance(None, 0))
    assert e.value.status == -1
