"""Norm, block means, block choice and block-sparse attention where values are
not finite, ties lie close or a call is taken in parts, against the fp64 oracle.

Finite values are held to the bounds of test_gpu_block.py; a value that the
formula makes an infinity or no number has to be that."""
import numpy as np
import pytest

import test_gpu_block
from oracle import block as B
from test_gpu_block import U, check_attend, dev, dt_of, host, huge, not_finite, rs3, run_attend, run_select
from workloads import storage_to_f64, to_storage

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- select --------------------------------------------------------------------
@pytest.mark.parametrize("make", [not_finite, huge])
@pytest.mark.parametrize("n_obj,n_q,n_kv,top_k,first,last,vis", [
    (2, 37, 1500, 4, 2, 2, "ragged"), (2, 37, 1500, 3, 0, 3, "causal"), (3, 300, 5000, 2, 2, 0, "ragged"),
    (2, 1, 1500, 4, 2, 2, "ragged")])
def test_forced_blocks_alone_fill_the_list(make, n_obj, n_q, n_kv, top_k, first, last, vis):
    """No block is chosen, whatever its score: the list is the forced ones and
    its count no more than top_k."""
    run_select(n_obj, n_q, n_kv, 4, 2, 64, 32, top_k, first, last, vis, "bf16", seed=n_q + top_k, make=make)


# ---- attend --------------------------------------------------------------------
def check_values(got, Q, K, V, idx, count, v, block, dtype):
    """check_attend where the result is finite, else the same infinity or no number."""
    with np.errstate(all="ignore"):
        O = B.block_attend(Q, K, V, idx, count, v, block)[0]
    assert np.array_equal(np.isnan(got), np.isnan(O))
    inf = np.isinf(O)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(np.sign(got[inf]), np.sign(O[inf]))
    W = np.where(np.isfinite(V), V, 0.0)
    check_attend(np.where(np.isfinite(O), got, B.block_attend(Q, K, W, idx, count, v, block)[0]), Q, K, W, idx, count, v,
                 block, dtype)
    return O


def every_block(rng, n_obj, n_q, H_kv, nb, top_k, wrong):
    idx = np.broadcast_to(np.arange(nb, dtype=np.int32), (n_obj, n_q, H_kv, nb))
    return idx.copy(), np.full((n_obj, n_q, H_kv), nb, np.int32)


def infinite_values(at):
    def edit(rng, Q, K, V, v):
        inf = np.array([0x7F80, 0xFF80], np.uint16) if V.dtype == np.uint16 else np.array([np.inf, -np.inf], np.float32)
        V[:, at, :, 5], V[:, at, :, V.shape[-1] - 1] = inf[0], inf[1]
        return Q, K, V
    return edit


# Queries, keys, heads, width, block: a query per work-group, and (many rows) a block per work-group.
@pytest.mark.parametrize("n_obj,n_q,n_kv,H,H_kv,d_h,block,dtype", [
    (1, 1, 81, 2, 1, 64, 64, "bf16"), (2, 3, 333, 6, 2, 32, 32, "bf16"), (1, 2, 2017, 4, 2, 128, 64, "bf16"),
    (3, 1, 70, 5, 1, 256, 128, "bf16"), (1, 40, 129, 2, 2, 128, 256, "bf16"), (1, 1, 81, 2, 1, 64, 64, "f32"),
    (2, 3, 119, 4, 2, 128, 64, "f32"), (1, 2, 1001, 4, 1, 256, 64, "f32"), (3, 5, 60, 2, 2, 32, 128, "f32"),
    (30, 60, 90, 4, 4, 64, 64, "bf16"), (8, 150, 333, 8, 4, 128, 128, "bf16"), (30, 60, 90, 2, 2, 64, 32, "f32")])
def test_infinite_last_value(monkeypatch, n_obj, n_q, n_kv, H, H_kv, d_h, block, dtype):
    """The last key that a query sees, inside a block, has an infinite value: those
    channels of the row are infinite, the others as ever."""
    monkeypatch.setattr(test_gpu_block, "lists", every_block)
    for vis, at in (("all", n_kv - 1), ("ragged", n_kv * 2 // 3 | 1)):
        some = infinite_values(at)

        def edit(rng, Q, K, V, v):
            if v is not None:   # not seen, last, or with keys behind it
                v[:] = at + np.arange(1, v.size + 1).reshape(v.shape) % 4
            return some(rng, Q, K, V, v)
        got, args = run_attend(n_obj, n_q, n_kv, H, H_kv, d_h, block, -(-n_kv // block), vis, dtype, seed=n_kv + d_h, edit=edit)
        assert np.isinf(check_values(got, *args)[..., 5]).any()


@pytest.mark.parametrize("n_obj", [1, 30])
@pytest.mark.parametrize("dtype,d_h,G", [("bf16", 64, 1), ("bf16", 128, 4), ("f32", 64, 2)])
def test_infinite_value_under_a_weight_of_0(monkeypatch, n_obj, dtype, d_h, G):
    """A key that a query sees at a logit of -inf has weight 0, and 0 times an
    infinite value is no number, whether or not the query sees all of the block."""
    monkeypatch.setattr(test_gpu_block, "lists", every_block)
    n_q = 96

    def edit(rng, Q, K, V, v):
        q, k = storage_to_f64(Q, dtype), storage_to_f64(K, dtype)
        q[..., 1], k[..., 1], k[:, 70, :, 1] = 8.0, 0.0, -3e38     # below the fp32 range
        v[0, -1] = 128
        infinite_values(70)(rng, Q, K, V, v)
        return to_storage(q.astype(np.float32), dtype), to_storage(k.astype(np.float32), dtype), V
    got, args = run_attend(n_obj, n_q, 128, G, 1, d_h, 64, 2, "causal", dtype, seed=d_h, edit=edit)
    v = args[5]
    check_values(got, *args)
    assert np.isnan(got[v > 70][..., 5]).all() and np.isfinite(got[v <= 70]).all() and (v <= 70).any()


# ---- norm and rotation ---------------------------------------------------------
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("n,heads,d_h,d_rot,dtype", [
    (5, 3, 64, 32, "bf16"), (5, 3, 256, 128, "bf16"), (4100, 9, 256, 128, "bf16"), (5, 2, 80, 48, "f32"),
    (5, 2, 128, 64, "f32"), (3000, 5, 240, 16, "f32"), (5, 3, 96, 0, "bf16")])
def test_norm_rope_infinite_channel(halves, n, heads, d_h, d_rot, dtype):
    """An infinite value makes its own channel, and the one that it is turned
    with, no number (the row's root is infinite, and the others are 0)."""
    p, rng = rs3(), np.random.default_rng(d_h)
    x = to_storage(rng.standard_normal((n, heads, d_h), dtype=np.float32), dtype)
    at = rng.integers(0, d_h, (n, heads))
    inf = np.where(rng.random((n, heads)) < 0.5, np.inf, -np.inf).astype(np.float32)
    np.put_along_axis(x, at[..., None], to_storage(inf, dtype)[..., None], -1)
    table = rng.uniform(0.5, 1.0, (n, max(d_rot, 2) // 2, 2)).astype(np.float32)
    X, Y = dev(x), torch.full(x.shape, 7.0, dtype=dev(x).dtype, device="cuda")
    p.qk_norm_rope(n, X, heads, None, 0, d_h, dt_of(dtype), Y, None, eps=1e-5, table=dev(table) if d_rot else None,
                   d_rot=d_rot, pairing=p.RS3_PAIRS_HALVES if halves else p.RS3_PAIRS_ADJACENT)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        exp = B.norm_rope(storage_to_f64(x, dtype), None, 1e-5, table if d_rot else None, None, halves)
    got = host(Y, dtype)
    assert np.array_equal(np.isnan(got), np.isnan(exp)) and (got[~np.isnan(exp)] == 0).all()


# ---- means ---------------------------------------------------------------------
def bf16_of(x):
    """fp64 to the nearest bf16 in one rounding, ties to even (normal results)."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def run_means(K, block, kv_len=None):
    p = rs3()
    n_obj, n_kv, H_kv, d_h = K.shape
    M = torch.full((n_obj, H_kv, -(-n_kv // block), d_h), 9.0, device="cuda", dtype=torch.bfloat16)
    p.block_means(p.block_shape(p.RS3_BF16, n_obj, 1, n_kv, H_kv, H_kv, d_h, block, 1), dev(K), M,
                  kv_len=None if kv_len is None else dev(kv_len))
    torch.cuda.synchronize()
    return host(M, "bf16"), B.block_means(storage_to_f64(K, "bf16"), [n_kv] * n_obj if kv_len is None else kv_len, block)


def test_means_are_rounded_once():
    """Means a little beside the middle of two bf16 numbers, by less than fp32
    tells apart, and on it; of either sign and of any size."""
    rng = np.random.default_rng(1)
    k = np.zeros((1, 4, 3, 64))
    k[0, :2] = rng.choice([(2.0, 2.015625), (2.015625, 2.03125), (2.5, 2.515625)], (3, 64)).transpose(2, 0, 1)
    k[0, 2] = rng.choice([-1, 0, 1], (3, 64)) * 2.0 ** -rng.integers(24, 40, (3, 64))
    k *= rng.choice([-1, 1], (3, 64)) * 2.0 ** rng.integers(-60, 100, (3, 64))
    got, exp = run_means(to_storage(k.astype(np.float32), "bf16"), 32)
    assert (bf16_of(exp) != bf16_of(exp.astype(np.float32).astype(np.float64))).any()
    assert np.array_equal(got, bf16_of(exp))


@pytest.mark.parametrize("d_h,block", [(32, 32), (64, 64), (128, 128), (256, 256)])
def test_means_of_ordinary_keys_are_the_nearest(d_h, block):
    rng = np.random.default_rng(block)
    K = to_storage(rng.standard_normal((3, 700, 2, d_h), dtype=np.float32), "bf16")
    got, exp = run_means(K, block, np.array([700, 0, 333], np.int32))
    assert np.array_equal(got, bf16_of(exp))


def test_means_of_infinite_and_largest_keys():
    big = storage_to_f64(np.array([0x7F7F], np.uint16), "bf16")[0]
    k = np.zeros((1, 2, 1, 32))
    k[0, :, 0, :6] = np.array([(np.inf, 1), (-np.inf, 1), (np.inf, -np.inf), (np.nan, 1), (big, big), (-big, -big)]).T
    with np.errstate(invalid="ignore"):
        got = run_means(to_storage(k.astype(np.float32), "bf16"), 32)[0][0, 0, 0]
    assert np.array_equal(got[:6], [np.inf, -np.inf, np.nan, np.nan, big, -big], equal_nan=True) and (got[6:] == 0).all()


# ---- calls that are taken in parts ------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_select_of_more_rows_than_the_scores_workspace_holds(dtype):
    """2,406 rows of 16,385 blocks: the same lists as object by object, and at the
    parts' border those of the oracle."""
    p, rng = rs3(), np.random.default_rng(3)
    n_obj, n_q, H, H_kv, d_h, block, top_k, n_kv = 3, 401, 4, 2, 32, 32, 11, 524289
    nb = -(-n_kv // block)
    Q = to_storage(rng.standard_normal((n_obj, n_q, H, d_h), dtype=np.float32), dtype)
    M = to_storage(rng.standard_normal((n_obj, H_kv, nb, d_h), dtype=np.float32), dtype)
    v = rng.integers(0, n_kv + 1, (n_obj, n_q)).astype(np.int32)
    v[:, ::7] = n_kv

    def run(o):
        n = Q[o].shape[0]
        s = p.block_shape(dt_of(dtype), n, n_q, n_kv, H, H_kv, d_h, block, top_k, 1, 2)
        idx = torch.full((n, n_q, H_kv, top_k), 77, dtype=torch.int32, device="cuda")
        count = torch.full((n, n_q, H_kv), 77, dtype=torch.int32, device="cuda")
        ws = torch.full((p.block_select_workspace_size(s),), 0xFF, dtype=torch.uint8, device="cuda")
        p.block_select(s, dev(Q[o]), dev(M[o]), idx, count, n_vis=dev(v[o]), ws=ws)
        torch.cuda.synchronize()
        return idx.cpu().numpy(), count.cpu().numpy(), ws.numel()
    idx, count, size = run(slice(0, n_obj))
    assert size < n_obj * n_q * H_kv * nb * 8      # more than one part
    for o in range(n_obj):
        i1, c1, _ = run(slice(o, o + 1))
        assert np.array_equal(idx[o:o + 1], i1) and np.array_equal(count[o:o + 1], c1)
    border = size // (nb * 8) // H_kv
    for at in (0, border - 1, border, border + 1, n_obj * n_q - 1):
        o, i = divmod(at, n_q)
        ei, ec = B.block_select(storage_to_f64(Q[o:o + 1, i:i + 1], dtype), storage_to_f64(M[o:o + 1], dtype),
                                v[o:o + 1, i:i + 1], block, top_k, 1, 2, n_kv)
        assert np.array_equal(idx[o, i], ei[0, 0]) and np.array_equal(count[o, i], ec[0, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_attend_of_more_queries_than_the_lists_workspace_holds(dtype):
    """1,200,001 queries, whose lists are made in parts: the same bits as for a part
    of the queries in a call of its own, and at the parts' border the oracle's."""
    p = rs3()
    n_q, n_kv, H, H_kv, d_h, block, top_k = 1200001, 500, 4, 4, 32, 32, 8
    gen = torch.Generator(device="cuda").manual_seed(6)
    dt, nb = (torch.bfloat16 if dtype == "bf16" else torch.float32), -(-n_kv // block)
    Q = torch.randn((1, n_q, H, d_h), generator=gen, device="cuda", dtype=dt)
    K, V = (torch.randn((1, n_kv, H_kv, d_h), generator=gen, device="cuda", dtype=dt) for _ in range(2))
    idx = torch.rand((1, n_q, H_kv, nb), generator=gen, device="cuda").argsort(-1)[..., :top_k].sort(-1).values.int()
    count = torch.randint(0, top_k + 1, (1, n_q, H_kv), generator=gen, device="cuda", dtype=torch.int32)
    v = torch.randint(0, n_kv + 1, (1, n_q), generator=gen, device="cuda", dtype=torch.int32)

    def run(a, b):
        s = p.block_shape(dt_of(dtype), 1, b - a, n_kv, H, H_kv, d_h, block, top_k)
        O = torch.full((1, b - a, H, d_h), float("nan"), dtype=dt, device="cuda")
        ws = torch.full((p.block_attend_workspace_size(s),), 0xFF, dtype=torch.uint8, device="cuda")
        p.block_attend(s, Q[:, a:b], K, V, idx[:, a:b], count[:, a:b], O, n_vis=v[:, a:b], ws=ws)
        torch.cuda.synchronize()
        return O, ws.numel()
    O, size = run(0, n_q)
    assert size < (1 << 30) + n_q * top_k * H * 16        # not the lists and pairs of all queries
    for a in range(0, n_q, 150001):   # each of them many queries too
        b = min(a + 150001, n_q)
        assert torch.equal(O[:, a:b], run(a, b)[0]), a
    at = np.unique(np.clip(np.concatenate([np.arange(-3, 4) + k * n_q // 12 for k in range(13)]), 0, n_q - 1))
    f = lambda t: host(t.contiguous(), dtype)  # noqa: E731
    check_attend(f(O[:, at]), f(Q[:, at]), f(K), f(V), idx[:, at].cpu().numpy(), count[:, at].cpu().numpy(),
                 v[:, at].cpu().numpy(), block, dtype)


# ---- layouts -----------------------------------------------------------------------
@pytest.mark.parametrize("n_q", [1, 2000])
def test_keys_and_values_past_32_bit_offsets(n_q):
    """Rows almost 2^22 elements apart (9 GB): the same bits as with packed rows."""
    p = rs3()
    n_kv, H, H_kv, d_h, block, top_k, row = 1100, 4, 2, 64, 32, 12, (1 << 22) - 8
    gen = torch.Generator(device="cuda").manual_seed(n_q)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    Q, K, V = rand(1, n_q, H, d_h), rand(1, n_kv, H_kv, d_h), rand(1, n_kv, H_kv, d_h)
    far = torch.empty((n_kv, row), dtype=torch.bfloat16, device="cuda")
    at = row - 2 * H_kv * d_h
    far[:, at:at + H_kv * d_h], far[:, at + H_kv * d_h:] = K.view(n_kv, -1), V.view(n_kv, -1)

    def run(K, V, **strides):
        s = p.block_shape(p.RS3_BF16, 1, n_q, n_kv, H, H_kv, d_h, block, top_k, 1, 1, **strides)
        M = torch.full((1, H_kv, -(-n_kv // block), d_h), 9.0, dtype=torch.bfloat16, device="cuda")
        idx = torch.full((1, n_q, H_kv, top_k), 77, dtype=torch.int32, device="cuda")
        count, O = torch.full((1, n_q, H_kv), 77, dtype=torch.int32, device="cuda"), torch.full_like(Q, float("nan"))
        ws = torch.empty(max(p.block_select_workspace_size(s), p.block_attend_workspace_size(s), 16), dtype=torch.uint8,
                         device="cuda")
        p.block_means(s, K, M)
        p.block_select(s, Q, M, idx, count, ws=ws)
        p.block_attend(s, Q, K, V, idx, count, O, ws=ws)
        torch.cuda.synchronize()
        return M, idx, count, O
    packed = run(K, V)
    assert torch.isfinite(packed[3]).all()
    apart = run(far[:, at:], far[:, at + H_kv * d_h:], k_stride=row, v_stride=row, k_obj_stride=0, v_obj_stride=0)
    for a, b in zip(packed, apart):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """The same calls in flight on two streams, with outputs and workspaces of their
    own, against one after the other."""
    p = rs3()
    n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k = 2, 1500, 2000, 4, 2, 128, 64, 9
    s = p.block_shape(p.RS3_BF16, n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k, 1, 1)
    gen = torch.Generator(device="cuda").manual_seed(8)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    sides = []
    for _ in range(2):
        Q, K, V = rand(n_obj, n_q, H, d_h), rand(n_obj, n_kv, H_kv, d_h), rand(n_obj, n_kv, H_kv, d_h)
        need = max(p.block_select_workspace_size(s), p.block_attend_workspace_size(s), 16)
        outs = lambda: (torch.zeros((n_obj, H_kv, -(-n_kv // block), d_h), dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                        torch.zeros((n_obj, n_q, H_kv, top_k), dtype=torch.int32, device="cuda"),
                        torch.zeros((n_obj, n_q, H_kv), dtype=torch.int32, device="cuda"), torch.zeros_like(Q),
                        torch.empty(need, dtype=torch.uint8, device="cuda"))
        sides.append((Q, K, V, outs(), outs(), torch.cuda.Stream()))

    def calls(Q, K, V, out):
        M, idx, count, O, ws = out
        p.block_means(s, K, M)
        p.block_select(s, Q, M, idx, count, ws=ws)
        p.block_attend(s, Q, K, V, idx, count, O, ws=ws)
    for Q, K, V, one, _, _ in sides:
        calls(Q, K, V, one)
    torch.cuda.synchronize()
    for _ in range(3):
        for Q, K, V, _, two, st in sides:
            with torch.cuda.stream(st):
                for t in two[:4]:
                    t.zero_()
                calls(Q, K, V, two)
    torch.cuda.synchronize()
    for _, _, _, one, two, _ in sides:
        for a, b in zip(one[:4], two[:4]):
            assert torch.equal(a, b)
