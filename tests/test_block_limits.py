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


def attend_bytes(p, n_q, n_kv, H, H_kv, d_h, block, top_k, n_obj=1, dt=1):
    return p.block_attend_workspace_size(p.block_shape(p.RS3_BF16 if dt else p.RS3_F32, n_obj, n_q, n_kv, H, H_kv, d_h, block,
                                                       top_k))


def test_attend_workspace_does_not_grow_with_the_queries(p):
    """1 GiB of partial rows, and lists and (m, l) pairs of 256 MiB; or those of one
    chunk of queries, whose lists have a few queries' places per block of the
    keys (an eighth of the bytes of their keys and values)."""
    rng = np.random.default_rng(4)
    cases = [(131072, 131072, 32, 8, 128, 64, 64), (1 << 22, 262144, 256, 256, 32, 32, 255), (1 << 22, 8192, 8, 8, 32, 32, 256),
             (65536, 131072, 32, 8, 128, 64, 64), (1024, 262144, 8, 8, 64, 32, 100, 4096), (300000, 5000, 40, 8, 64, 64, 17, 2, 0)]
    for _ in range(3000):
        H_kv = int(rng.choice([1, 2, 4, 8, 32, 256]))
        H = H_kv * int(rng.choice([1, 3, 8]))
        n_obj = int(rng.choice([1, 1, 3, 64, 4096]))
        n_q = int(2 ** rng.uniform(3, 22)) // n_obj
        if H <= 256 and n_q:
            cases.append((n_q, int(2 ** rng.uniform(4, 24)), H, H_kv, int(rng.choice([32, 64, 128, 256])),
                          int(rng.choice([32, 64, 128, 256])), int(2 ** rng.uniform(0, 8)), n_obj, int(rng.integers(0, 2))))
    for c in cases:
        n_kv, H_kv, d_h, n_obj = c[1], c[3], c[4], c[7] if len(c) > 7 else 1
        keys = 2 * n_obj * H_kv * n_kv * d_h * (2 if len(c) < 9 or c[8] else 4)
        assert attend_bytes(p, *c) <= (1 << 30) + max(256 << 20, (320 << 20) + keys // 8), c


def test_binding_refuses_a_pairing_past_32_bits(p):
    with pytest.raises(ValueError):
        p.qk_norm_rope(1, None, 0, None, 0, 64, p.RS3_BF16, None, None, pairing=2 ** 32 + 1)
