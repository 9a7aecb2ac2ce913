"""Refusals of the norm and rotation and of the block-sparse attention, on the
host before any device work (CPU)."""
import ctypes

import pytest

from conftest import ROOT

PTR = 1 << 20      # never dereferenced: every call here is refused


@pytest.fixture(scope="module")
def p():
    import paper_2608_22526_amd as pkg
    pkg.lib()
    return pkg


def norm(p, **kw):
    a = dict(n=4, Q=PTR, qs=256, H=4, K=PTR, ks=128, Hk=2, d=64, dt=p.RS3_BF16, gq=None, gk=None, eps=1e-6, table=PTR,
             n_pos=8, d_rot=64, pairing=0, pos=PTR, Qo=PTR, qos=256, Ko=PTR, kos=128)
    a.update(kw)
    return p.lib().rs3_qk_norm_rope(a["n"], a["Q"], a["qs"], a["H"], a["K"], a["ks"], a["Hk"], a["d"], a["dt"], a["gq"],
                                    a["gk"], a["eps"], a["table"], a["n_pos"], a["d_rot"], a["pairing"], a["pos"],
                                    a["Qo"], a["qos"], a["Ko"], a["kos"], None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(n=(1 << 24) + 1), dict(dt=7), dict(H=-1), dict(H=1024), dict(d=8), dict(d=72), dict(d=272),
    dict(eps=0.0), dict(eps=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(d_rot=72), dict(d_rot=80),
    dict(d_rot=8), dict(table=None), dict(d_rot=0), dict(pairing=2), dict(n_pos=0), dict(pos=None, n_pos=3),
    dict(Q=None), dict(Ko=None), dict(Q=PTR + 8), dict(Ko=PTR + 2), dict(table=PTR + 4), dict(gq=PTR + 4),
    dict(qs=248), dict(qs=260), dict(kos=64), dict(ks=-128), dict(Q=PTR, Qo=PTR, qos=512)])
def test_norm_refuses(p, kw):
    assert norm(p, **kw) == p.RS3_E_INVALID


def test_nothing_to_do_is_ok(p):
    assert norm(p, n=0, Q=None, Qo=None, K=None, Ko=None) == p.RS3_OK
    assert norm(p, H=0, Hk=0, Q=None, K=None) == p.RS3_OK
    s = p.block_shape(p.RS3_BF16, 2, 0, 100, 4, 2, 64, 32, 4)
    lib = p.lib()
    assert lib.rs3_block_select(ctypes.byref(s), None, PTR, None, None, None, None, 0, None) == p.RS3_OK
    assert lib.rs3_block_attend(ctypes.byref(s), None, PTR, PTR, None, None, None, None, None, 0, None) == p.RS3_OK
    s = p.block_shape(p.RS3_BF16, 2, 3, 0, 4, 2, 64, 32, 4)
    assert lib.rs3_block_means(ctypes.byref(s), None, None, 0, None, None) == p.RS3_OK


def calls(p, s):
    lib, r = p.lib(), ctypes.byref(s)
    size = ctypes.c_size_t()
    big = 1 << 62
    return dict(means=lib.rs3_block_means(r, PTR, None, 0, PTR, None),
                select=lib.rs3_block_select(r, PTR, PTR, None, PTR, PTR, PTR, big, None),
                attend=lib.rs3_block_attend(r, PTR, PTR, PTR, PTR, PTR, None, PTR * 2, PTR, big, None),
                select_size=lib.rs3_block_select_workspace_size(r, ctypes.byref(size)),
                attend_size=lib.rs3_block_attend_workspace_size(r, ctypes.byref(size)))


def shape(p, **kw):
    s = p.block_shape(p.RS3_BF16, 2, 5, 100, 4, 2, 64, 32, 4, 1, 1)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("kw", [
    dict(n_obj=0), dict(n_obj=4097), dict(n_q=-1), dict(n_q=1 << 22), dict(n_kv=-1), dict(n_kv=(1 << 26) + 1), dict(H=0),
    dict(H=3), dict(H=512), dict(H_kv=0), dict(d_h=48), dict(d_h=512), dict(block=16), dict(block=48), dict(block=512),
    dict(top_k=0), dict(top_k=257), dict(n_first=-1), dict(n_last=-1), dict(n_first=3, n_last=2), dict(dt=5),
    dict(n_first=2 ** 31 - 1, n_last=2 ** 31 - 1), dict(reserved=1)])
def test_every_call_refuses_the_shape(p, kw):
    assert set(calls(p, shape(p, **kw)).values()) == {p.RS3_E_INVALID}


@pytest.mark.parametrize("kw,who", [
    (dict(k_stride=120), ("means", "attend")), (dict(k_stride=132), ("means", "attend")),
    (dict(k_obj_stride=-128), ("means", "attend")), (dict(v_stride=64), ("attend",)), (dict(q_stride=248), ("select", "attend")),
    (dict(q_obj_stride=4), ("select", "attend")), (dict(o_stride=8), ("attend",)), (dict(o_obj_stride=0), ("attend",)),
    (dict(o_obj_stride=256), ("attend",)), (dict(k_stride=1 << 40), ("means", "attend")), (dict(v_stride=1 << 22), ("attend",))])
def test_row_layouts_refused(p, kw, who):
    s = shape(p, **kw)
    # only the calls that must refuse are made: the others would launch
    lib, r = p.lib(), ctypes.byref(s)
    if "means" in who:
        assert lib.rs3_block_means(r, PTR, None, 0, PTR, None) == p.RS3_E_INVALID
    if "select" in who:
        assert lib.rs3_block_select(r, PTR, PTR, None, PTR, PTR, PTR, 1 << 62, None) == p.RS3_E_INVALID
    if "attend" in who:
        assert lib.rs3_block_attend(r, PTR, PTR, PTR, PTR, PTR, None, PTR * 2, PTR, 1 << 62, None) == p.RS3_E_INVALID


def test_pointers_and_workspaces_refused(p):
    s, lib = shape(p), p.lib()
    r, big = ctypes.byref(s), 1 << 62
    size = ctypes.c_size_t()
    inv = p.RS3_E_INVALID
    assert lib.rs3_block_means(None, PTR, None, 0, PTR, None) == inv
    for args in ((None, None, 0, PTR), (PTR, None, 0, None), (PTR + 4, None, 0, PTR), (PTR, None, 0, PTR + 8),
                 (PTR, None, -1, PTR)):
        assert lib.rs3_block_means(r, *args, None) == inv
    for args in ((None, PTR, None, PTR, PTR, PTR, big), (PTR, None, None, PTR, PTR, PTR, big),
                 (PTR, PTR, None, None, PTR, PTR, big), (PTR, PTR, None, PTR, None, PTR, big),
                 (PTR + 8, PTR, None, PTR, PTR, PTR, big), (PTR, PTR, None, PTR, PTR, PTR + 4, big)):
        assert lib.rs3_block_select(r, *args, None) == inv
    for at in (0, 1, 2, 3, 4, 6):
        args = [PTR, PTR, PTR, PTR, PTR, None, PTR * 2, PTR, big]
        args[at] = None
        assert lib.rs3_block_attend(r, *args, None) == inv
    for at in (0, 1, 2, 6, 7):
        args = [PTR, PTR, PTR, PTR, PTR, None, PTR * 2, PTR, big]
        args[at] += 4
        assert lib.rs3_block_attend(r, *args, None) == inv
    assert lib.rs3_block_attend(r, PTR, PTR, PTR, PTR, PTR, None, PTR, PTR, big, None) == inv       # O is Q
    assert lib.rs3_block_select_workspace_size(r, None) == inv
    assert lib.rs3_block_attend_workspace_size(r, None) == inv
    assert lib.rs3_block_select_workspace_size(r, ctypes.byref(size)) == p.RS3_OK
    if size.value:
        assert lib.rs3_block_select(r, PTR, PTR, None, PTR, PTR, PTR, size.value - 1, None) == inv
        assert lib.rs3_block_select(r, PTR, PTR, None, PTR, PTR, None, big, None) == inv
    assert lib.rs3_block_attend_workspace_size(r, ctypes.byref(size)) == p.RS3_OK
    if size.value:
        assert lib.rs3_block_attend(r, PTR, PTR, PTR, PTR, PTR, None, PTR * 2, PTR, size.value - 1, None) == inv
        assert lib.rs3_block_attend(r, PTR, PTR, PTR, PTR, PTR, None, PTR * 2, None, big, None) == inv


def test_block_shape_layout_matches_header(p, tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    names = [n for n, _ in p.BlockShape._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"rs3.h\"\nint main(void) {\n"
                   "  printf(\"%zu\", sizeof(rs3_block_shape));\n"
                   + "".join("  printf(\" %%zu\", offsetof(rs3_block_shape, %s));\n" % n for n in names)
                   + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.check_call([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    assert got == [ctypes.sizeof(p.BlockShape)] + [getattr(p.BlockShape, n).offset for n in names]


def test_binding_refuses_tensors():
    """Shapes, types and devices that the kernels would read past are refused
    before the library is called."""
    torch = pytest.importorskip("torch")
    from paper_2608_22526_amd import _binding as b
    cpu = torch.device("cpu")
    t = torch.zeros(10, dtype=torch.int32)
    b._check_tensor("t", t, 10, torch.int32, cpu)
    for args in ((t, 11, torch.int32, cpu), (t, 10, torch.float32, cpu), (t, 10, torch.int32, torch.device("cuda", 0)),
                 (t[::2], 5, torch.int32, cpu)):
        with pytest.raises(ValueError):
            b._check_tensor("t", *args)
    b._check_rows("t", t[4:], 6, torch.int32, cpu)
    for args in ((t[4:], 7, torch.int32, cpu), (t, 10, torch.float32, cpu), (t, 1, torch.int32, torch.device("cuda", 0))):
        with pytest.raises(ValueError):
            b._check_rows("t", *args)
    with pytest.raises(TypeError):
        b.block_shape(b.RS3_BF16, 1, 1, 1, 1, 1, 32, 32, 1, x_stride=3)


def test_binding_refuses_integers_past_32_bits(p):
    with pytest.raises(ValueError):
        p.block_shape(p.RS3_BF16, 1, 1, 2 ** 32 + 5, 1, 1, 32, 32, 1)
    with pytest.raises(ValueError):
        p.block_means(shape(p), None, None, n_new=2 ** 32)
    with pytest.raises(ValueError):
        p.qk_norm_rope(2 ** 32, None, 0, None, 0, 64, p.RS3_BF16, None, None)


def test_norm_refuses_more_heads_than_a_launch_holds(p):
    n = 1 << 24
    wide = dict(n=n, n_pos=n, qs=1024, ks=1024, qos=1024, kos=1024)
    assert norm(p, **wide, H=7, Hk=2) == p.RS3_E_INVALID
    assert norm(p, **wide, H=9, Hk=0) == p.RS3_E_INVALID
