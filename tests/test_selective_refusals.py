"""Descriptors of the 8-bit product that no call accepts, next to ones that are and need room.  No GPU: a refused call looks at nothing
else."""
import ctypes as C

import pytest

from paper_1606_03401_amd import binding as mb

GOOD = (512, 4096, 1022, mb.FP32)


def _call(desc):
    """The product's status, every pointer NULL: EINVAL either way, with its own words for a descriptor."""
    lib = mb.lib()
    rc = lib.mebptt_int8_product(C.byref(desc), None, desc.K, None, None, desc.K, None, None, None, desc.N, None, 0, None)
    return rc, mb.mebptt_last_error()


def test_a_descriptor_that_is_accepted_needs_room():
    assert mb.mebptt_int8_workspace_bytes(mb.make_int8_desc(*GOOD)) == (512 + 4096) * 1024
    rc, said = _call(mb.make_int8_desc(*GOOD))
    assert rc == mb.EINVAL and "pointer" in said


@pytest.mark.parametrize("at,value,word", [(0, -1, "M"), (0, (1 << 28) + 1, "M"), (1, 0, "N"), (1, (1 << 21) + 1, "N"), (2, -2, "K"), (2, 131073, "K"),
                                           (3, mb.INT8, "out_dtype"), (3, 7, "out_dtype")])
def test_a_descriptor_that_no_call_accepts(at, value, word):
    desc = list(GOOD)
    desc[at] = value
    desc = mb.make_int8_desc(*desc)
    assert mb.mebptt_int8_workspace_bytes(desc) == 0
    rc, said = _call(desc)
    assert rc == mb.EINVAL and said.startswith(word), said


def test_an_output_of_too_many_values():
    desc = mb.make_int8_desc(1 << 28, 1 << 11, 1022, mb.FP32)
    assert mb.mebptt_int8_workspace_bytes(desc) == 0
    rc, said = _call(desc)
    assert rc == mb.EINVAL and "2^38" in said
