"""Memory that the block calls ask for, and what the timing report writes (CPU)."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def p():
    import paper_2608_22526_amd as pkg
    pkg.lib()
    return pkg


def test_timing_report_writes_as_many_entries_as_its_caller_has(p):
    lib = p.lib()

    def arrays(n):
        ms, count = np.full(32, -7.0), np.full(32, -7, np.int64)
        return ms, count, n
    # the entry without a length fills the 14 kernels that its header had
    for n, fill in ((14, lambda ms, c: lib.rs3_profile_report(ms.ctypes.data, c.ctypes.data, None)),
                    (18, lambda ms, c: lib.rs3_profile_report_n(18, ms.ctypes.data, c.ctypes.data, None)),
                    (0, lambda ms, c: lib.rs3_profile_report_n(0, ms.ctypes.data, c.ctypes.data, None)),
                    (30, lambda ms, c: lib.rs3_profile_report_n(30, ms.ctypes.data, c.ctypes.data, None))):
        ms, count, _ = arrays(n)
        assert fill(ms, count) == p.RS3_OK
        assert (ms[:n] == 0).all() and (count[:n] == 0).all()
        assert (ms[n:] == -7).all() and (count[n:] == -7).all()
    ms, count, _ = arrays(18)
    assert lib.rs3_profile_report_n(-1, ms.ctypes.data, count.ctypes.data, None) == p.RS3_E_INVALID
    assert lib.rs3_profile_report_n(18, None, count.ctypes.data, None) == p.RS3_E_INVALID


def test_timing_report_of_a_program_built_on_the_header(p, tmp_path):
    """In C the plain name passes RS3_K_COUNT along."""
    import os
    import shutil
    import subprocess
    from conftest import ROOT
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    src = tmp_path / "report.c"
    src.write_text("#include <stdio.h>\n#include \"rs3.h\"\nint main(void) {\n"
                   "  double ms[RS3_K_COUNT + 1]; int64_t n[RS3_K_COUNT + 1];\n"
                   "  for (int i = 0; i <= RS3_K_COUNT; ++i) ms[i] = -7, n[i] = -7;\n"
                   "  int st = rs3_profile_report(ms, n, NULL), bad = 0;\n"
                   "  for (int i = 0; i < RS3_K_COUNT; ++i) bad += ms[i] != 0 || n[i] != 0;\n"
                   "  printf(\"%d %d %d\", st, bad, (int)n[RS3_K_COUNT]);\n  return 0;\n}\n")
    exe = tmp_path / "report"
    lib = os.path.join(ROOT, "paper_2608_22526_amd")
    subprocess.check_call([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe), os.path.join(lib, "librs3.so"),
                           "-Wl,-rpath," + lib, "-Wl,-rpath,/opt/rocm/lib", "-Wl,--allow-shlib-undefined"])
    assert subprocess.check_output([str(exe)]) == b"0 0 -7"


def select_bytes(p, n_q, n_kv, H, H_kv, d_h, block, top_k, n_obj=1, dt=1):
    return p.block_select_workspace_size(p.block_shape(p.RS3_BF16 if dt else p.RS3_F32, n_obj, n_q, n_kv, H, H_kv, d_h, block,
                                                       top_k))


def test_select_workspace_does_not_grow_with_the_queries(p):
    """At most 256 MiB of scores, at any size that is accepted."""
    for case in ((4096, 524289, 32, 8, 128, 32, 16), (32768, 1100000, 32, 8, 128, 64, 16), (1 << 22, 1 << 26, 256, 256, 32, 32, 256),
                 (32768, 1 << 22, 8, 8, 128, 64, 16), (1, 1 << 26, 256, 256, 32, 32, 256), (1, 1 << 20, 8, 8, 64, 64, 8, 4096),
                 (100, 1 << 24, 4, 2, 64, 32, 9, 77, 0)):
        assert select_bytes(p, *case) <= 256 << 20, case
    assert select_bytes(p, 0, 1 << 26, 8, 8, 128, 32, 16) == 0
    # as long as they fit, the scores of all rows
    assert select_bytes(p, 1, 1 << 20, 8, 8, 128, 64, 16) == 8 * (1 << 14) * 8
