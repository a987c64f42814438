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


def _run_on_the_sizes(tmp_path, body):
    """Compiles `body` as the main function of a program that includes the sizes' header, with the host compiler, and runs it."""
    import os
    import shutil
    import subprocess
    import pytest
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    (tmp_path / "sizes.cpp").write_text(
        '#include "grouped_sizes.hpp"\n#include <cstdio>\n#include <initializer_list>\nusing namespace ecgemm;\n'
        '#define CHECK(cond) do { if (!(cond)) { std::printf("line %d: %s\\n", __LINE__, #cond); return 1; } } while (0)\n'
        "int main() {\n" + body + "\nreturn 0;\n}\n")
    exe = str(tmp_path / "sizes")
    built = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I",
                            os.path.join(root, "paper_2203_03341_amd", "csrc"), str(tmp_path / "sizes.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout + run.stderr


def test_tiles_of_groups_next_to_the_largest(tmp_path):
    """What the kernels count from two 32-bit offsets: as many tiles as there are, up to the largest group there can be."""
    _run_on_the_sizes(tmp_path, """
      const int begins[] = {0, 1, 127, 128, 1 << 20};
      for (int begin : begins)
        for (long long columns : {0ll, 1ll, 127ll, 128ll, 129ll, 2147483519ll, 2147483520ll, 2147483521ll, 2147483646ll, 2147483647ll}) {
          if (begin + columns > 2147483647ll) continue;
          const int end = (int)(begin + columns);
          const long long tiles = grouped_tiles(end - begin);
          CHECK(tiles >= 0 && tiles * 128 >= columns && (tiles - 1) * 128 < columns);
        }
      CHECK(grouped_tiles(2147483521) == 16777216);
    """)


def test_kernels_count_tiles_nowhere_else():
    """The tiles of a group are counted by the function tested above, on either side."""
    import glob
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    files = glob.glob(os.path.join(root, "paper_2203_03341_amd", "csrc", "grouped_*.hpp"))
    text = {os.path.basename(f): open(f).read() for f in files}
    assert "grouped_tiles(end - begin)" in text["grouped_kernel.hpp"]
    assert [f for f, t in text.items() if "kGroupedTile - 1) / kGroupedTile" in t] == ["grouped_sizes.hpp"]


def test_calls_go_only_to_launches_that_hold_them(tmp_path):
    """A launch has fewer than 2^32 threads along x.  The kernels of few columns and shallow groups, from both sides of that."""
    _run_on_the_sizes(tmp_path, """
      CHECK(launchable(8388607, 512) && !launchable(8388608, 512) && launchable(16777215, 256) && !launchable(16777216, 256));
      CHECK(!launchable((long long)1 << 62, 1));
      // 131072 groups of 1024 rows, depth contiguous: 64 blocks of 16 rows each; rows contiguous: 16 of 64
      CHECK(!narrow_fits(true, 131072, 1024, 1, 0) && narrow_fits(true, 131071, 1024, 1, 0) && !narrow_fits(true, 131071, 1024, 1, 1));
      CHECK(narrow_fits(false, 131072, 1024, 1, 1) && !narrow_fits(false, 524288, 1024, 1, 0));
      CHECK(!narrow_fits(true, 131072, 1024, 1, 1) && narrow_fits(true, 131072, 512, 1, 1));
      CHECK(narrow_fits(true, 1, 134217712, 1, 0) && !narrow_fits(true, 1, 134217713, 1, 0) && narrow_fits(true, 1, 134217713, 17, 0));
      CHECK(!narrow_fits(true, 2147483647, 2147483647, 1, 1));
      // groups of one value, of 256 x 64, of 257 x 64
      CHECK(!shallow_fits(16777216, 1, 1) && shallow_fits(16777215, 1, 1) && shallow_fits(16777215, 256, 64));
      CHECK(!shallow_fits(16777215, 257, 64) && shallow_fits(8388607, 257, 64) && !shallow_fits(2147483647, 1 << 22, 1 << 22));
      CHECK(adapter_up_blocks(257, 65, 64) == 4 && adapter_up_blocks(256, 64, 8) == 8);
      CHECK(launchable(adapter_up_blocks(1 << 20, 262080, 64), 256) && !launchable(adapter_up_blocks(1 << 20, 262144, 64), 256));
      CHECK(adapter_up_blocks(0, 5, 64) == 0);
      // as many rows as the columns of adapters that a call of one launch can have
      CHECK(launchable(narrow_row_blocks(narrow_fr(true, 1, 134217712, 16), 134217712), kNarrowThreads));
      CHECK(!launchable(narrow_row_blocks(narrow_fr(true, 1, 134217713, 16), 134217713), kNarrowThreads));
      CHECK(launchable(narrow_row_blocks(narrow_fr(false, 1, 536870848, 16), 536870848), kNarrowThreads));
    """)


def _calls():
    """Of each method: its arguments by name, sound but for the null handle and operands that are not on a GPU"""
    import torch
    f, offs, index = torch.zeros(4096), torch.zeros(4, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    values = dict(transA=1, transB=0, groups=3, M=8, N=8, K=8, alpha=1.0, A=f, lda=8, strideA=64, B=f, ldb=8, offsets=offs, beta=0.0, C=f, ldc=8,
                  strideC=64, mode=0, index=index, adapters=2, rank=4, transD=1, D=f, ldd=8, strideD=32, transU=1, U=f, ldu=4, strideU=32,
                  scales=torch.ones(2), H=f, ldh=4)
    import paper_2203_03341_amd as ec
    for name in ("sgemm_grouped", "sgemm_grouped_depth", "sgemm_adapters"):
        order = list(inspect.signature(getattr(ec.Handle, name)).parameters)[1:]
        yield name, {k: values[k] for k in order}


def test_operands_of_the_wrong_type_length_or_device_are_refused():
    """Before the library sees an address: index in torch's default type, offsets in 32 bits, tables that end too early or have
    gaps, weights in another type, what lies in host memory."""
    import pytest
    import torch
    import paper_2203_03341_amd as ec
    handle = ec.Handle.__new__(ec.Handle)
    handle._h = None
    wrong = {"offsets": [torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(3, dtype=torch.int64), torch.zeros(8, dtype=torch.int64)[::2]],
             "index": [torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]],
             "scales": [torch.ones(2, dtype=torch.float64), torch.ones(1), torch.ones(4)[::2]]}
    for operand in "ABCDUH":
        wrong[operand] = [torch.zeros(4096, dtype=t) for t in (torch.float64, torch.float16, torch.bfloat16, torch.int32)]
    for name, sound in _calls():
        order = list(sound)
        on_gpu = {k: 4096 if isinstance(v, torch.Tensor) else v for k, v in sound.items()}      # (addresses are taken as they are)
        with pytest.raises(ec.EcgemmError) as err:
            getattr(handle, name)(*on_gpu.values())
        assert "null handle" in str(err.value)      # got as far as the library
        for operand, values in wrong.items():
            if operand not in sound:
                continue
            for value in [*values, sound[operand]]:     # (the last: of the right type, in host memory)
                with pytest.raises(ec.EcgemmError) as err:
                    getattr(handle, name)(*{**on_gpu, operand: value}.values())
                assert err.value.status == ec.ERR_INVALID_ARG and err.value.argument == order.index(operand) + 2, (name, operand, err.value)
                assert operand + ":" in str(err.value)


def test_counts_that_the_library_refuses_are_left_to_it():
    """A negative or far too large number of groups or adapters is that argument's fault, not its table's."""
    import pytest
    import torch
    from paper_2203_03341_amd import binding
    table = torch.zeros(4, dtype=torch.int64)
    for count in (-(1 << 62), -1, 0, 1 << 31, (1 << 31) + 1, 1 << 62):
        with pytest.raises(binding.EcgemmError) as err:
            binding._typed(table, "offsets", 14, torch.int64, count)
        assert "not in GPU memory" in str(err.value)     # (its length was not what is wrong)
    with pytest.raises(binding.EcgemmError) as err:
        binding._typed(table, "offsets", 14, torch.int64, (1 << 31) - 1)
    assert "contiguous entries" in str(err.value)
