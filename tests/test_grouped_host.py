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
