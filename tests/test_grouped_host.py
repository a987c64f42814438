"""The grouped products' entry points as far as they go without a GPU: declared, bound, and refusing a null handle."""
import ctypes
import inspect


def test_null_handles_are_refused():
    from paper_2203_03341_amd import binding
    lib = binding._lib
    assert lib.ecgemm_sgemm_grouped(None, 1, 0, 1, 8, 8, 8, 1.0, None, 8, 64, None, 8, None, 0.0, None, 8, 0) == binding.ERR_INVALID_ARG
    assert lib.ecgemm_sgemm_grouped_depth(None, 0, 1, 1, 8, 8, 8, 1.0, None, 8, None, 8, None, 0.0, None, 8, 64, 0) == binding.ERR_INVALID_ARG
    assert lib.ecgemm_sgemm_adapters(None, 1, 0, 8, 8, 8, 1.0, None, 8, None, 8, 1, None, None, 1, 4, 1, None, 8, 32, 1, None, 4, 32, None, None,
                                     4, 0.0, None, 8, 0) == binding.ERR_INVALID_ARG


def test_methods_take_the_arguments_of_the_c_functions():
    """As many as the C functions have, the handle being the object."""
    import paper_2203_03341_amd as ec
    from paper_2203_03341_amd import binding
    for name in ("sgemm_grouped", "sgemm_grouped_depth", "sgemm_adapters"):
        types = getattr(binding._lib, "ecgemm_" + name).argtypes
        assert len(inspect.signature(getattr(ec.Handle, name)).parameters) == len(types)
        assert types[0] is ctypes.c_void_p
    assert ec.GROUPED_WORKSPACE_BYTES == 256 * 128 * 128 * 4    # partial sums of as many tiles as the chip has units


def test_the_header_says_the_same_constants():
    import os
    import re
    import paper_2203_03341_amd as ec
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "ecgemm.h")).read()
    mib = int(re.search(r"#define ECGEMM_GROUPED_WORKSPACE_BYTES \(\(size_t\)(\d+) << 20\)", text)[1])
    assert mib << 20 == ec.GROUPED_WORKSPACE_BYTES
