"""The work that the block-sparse attention is timed on: the norm and rotation
of queries and keys, the block means of the keys, the choice of a query's
blocks, and the attention over them.  `kind` says which call a case makes:

  norm    rs3_qk_norm_rope: RMS norm of each head of the queries and keys and
          the rotation by the token's position.  A position of -1 is padding:
          that row of the outputs stays as it is.
  means   rs3_block_means: the mean key of every block of `block` keys, or
          (n_new > 0) of the blocks that hold the last n_new keys only.
  select  rs3_block_select: each query's top_k blocks by the product of the
          query (summed over the heads that share the keys) with the mean key,
          its first and last visible blocks always among them.
  attend  rs3_block_attend: softmax attention over the keys of those blocks.

`vis` says which keys a query sees: "all", "causal" (the queries are the last
n_q tokens) or "ragged" (a length of its own, some of them 0).

Keys are Gaussian around a centre that drifts from block to block, and a query
lies near the centres of a few blocks, so that some blocks are read by many
queries and others by none, as with text or the frames of a clip.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
THETA = 10000.0
LOGIT_SCALE = 3.0   # standard deviation of the attention logits


# ---- the cases ---------------------------------------------------------------
def _norm(name, n, H, H_kv, d_h, d_rot, halves, dtype="bf16", pad=0.0):
    return dict(name=name, kind="norm", n=n, H=H, H_kv=H_kv, d_h=d_h, d_rot=d_rot, halves=halves, dtype=dtype, pad=pad)


def _block(name, kind, n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k=1, n_first=0, n_last=0, vis="all", dtype="bf16",
           n_new=0):
    return dict(name=name, kind=kind, n_obj=n_obj, n_q=n_q, n_kv=n_kv, H=H, H_kv=H_kv, d_h=d_h, block=block,
                top_k=top_k, n_first=n_first, n_last=n_last, vis=vis, dtype=dtype, n_new=n_new)


def listed():
    return [
        # one new token of each of 64 streams: launch and memory latency
        _norm("norm_tokens", 64, 32, 8, 128, 128, True),
        # the tokens of a 128x128 grid in eight heads of 32, turned by row and column
        _norm("norm_grid", 16384, 8, 8, 32, 32, False),
        # long prompts of several streams, padded to one length
        _norm("norm_prompt", 16384, 32, 8, 128, 128, True, pad=0.1),
        # 64 caches that grew by one token each
        _block("means_append", "means", 64, 1, 4096, 8, 8, 64, 64, n_new=1, vis="ragged"),
        # the whole of a long cache, once after it was filled
        _block("means_cache", "means", 1, 1, 65536, 8, 8, 128, 64),
        # one token of 32 streams against caches of up to 131,072 keys
        _block("select_token", "select", 32, 1, 131072, 32, 8, 128, 64, 32, 1, 1, "ragged"),
        # fp32: a 32x32 grid against a bank that ends inside a block
        _block("select_grid_f32", "select", 1, 1024, 8170, 4, 4, 64, 32, 16, dtype="f32"),
        # 4,096 prompt tokens behind 28,672 earlier ones, four heads to a key head
        _block("select_prompt", "select", 1, 4096, 32768, 16, 4, 128, 64, 16, 1, 2, "causal"),
        # one token of 32 streams, 2,048 of up to 16,384 keys each
        _block("attend_token", "attend", 32, 1, 16384, 32, 8, 128, 64, 32, 1, 1, "ragged"),
        # fp32: the 32x32 grid, 512 of 4,100 keys
        _block("attend_grid_f32", "attend", 1, 1024, 4100, 4, 4, 64, 32, 16, dtype="f32"),
        # every cell of a 64x64 grid against 2,048 keys of seven whole frames
        _block("attend_grid", "attend", 1, 4096, 28672, 2, 2, 128, 64, 32),
        # a long prompt: 8,192 tokens, 1,024 of up to 32,768 keys; the largest
        _block("attend_prompt", "attend", 1, 8192, 32768, 16, 4, 128, 64, 16, 1, 2, "causal"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    kind = rng.choice(["norm", "means", "select", "select", "attend", "attend", "attend"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "norm":
        d_h = rng.choice([32, 64, 80, 96, 128, 256])
        H_kv = rng.choice([1, 2, 3, 4, 8])
        return dict(_norm("", _log_int(rng, 1, 16384), H_kv * rng.choice([1, 1, 2, 3, 4, 8]), H_kv, d_h,
                          rng.choice([0, d_h // 2, d_h, d_h]) // 16 * 16, rng.random() < 0.5, dtype,
                          rng.choice([0.0, 0.0, 0.2])))
    d_h = rng.choice([32, 64, 128, 128, 256])
    H_kv = rng.choice([1, 2, 3, 4, 8])
    H = H_kv * rng.choice([1, 1, 2, 3, 4, 6, 8, 16])
    block = rng.choice([32, 64, 64, 128, 256])
    if kind == "means":
        n_obj = rng.choice([1, _log_int(rng, 1, 64)])
        n_kv = _log_int(rng, 1, 65536)
        return dict(_block("", kind, n_obj, 1, n_kv, H_kv, H_kv, d_h, block, dtype=dtype,
                           n_new=rng.choice([0, 0, 1, min(n_kv, _log_int(rng, 1, 300))]),
                           vis=rng.choice(["all", "ragged"])))
    if rng.random() < 0.4:
        n_obj, n_q = _log_int(rng, 1, 48), rng.choice([1, 1, 1, 2, 4])
    else:
        n_obj, n_q = rng.choice([1, 1, 1, 2, 3]), _log_int(rng, 5, 8192)
    n_kv = _log_int(rng, 1, 131072 if kind == "select" else 40000)
    vis = rng.choice(["all", "ragged", "causal", "causal"])
    top_k = max(1, min(_log_int(rng, 1, 64), (4096 if kind == "attend" else 1 << 20) // block))
    forced = rng.choice([(0, 0), (0, 1), (1, 1), (1, 2)])
    if sum(forced) > top_k:
        forced = (0, 0)
    return dict(_block("", kind, n_obj, n_q, n_kv, H, H_kv, d_h, block, top_k, *forced, vis, dtype))


def draw(rng):
    """One more case of the same ranges, no larger than the largest listed."""
    every = [work(c) for c in listed()]
    most, flops = max(w["bytes"] for w in every), max(w["flops"] for w in every)
    while True:
        c = _draw_one(rng)
        c.pop("name", None)
        w = work(c)
        if w["bytes"] > most or w["flops"] > flops:
            continue
        es = 4 if c["dtype"] == "f32" else 2
        if c["kind"] != "norm" and c["n_obj"] * c["n_kv"] * c["H_kv"] * c["d_h"] * es > 1 << 31:
            continue   # caches of 2 GB at most
        if c["kind"] == "attend" and c["n_obj"] * c["n_q"] * c["H_kv"] * c["top_k"] * c["block"] * c["d_h"] > 1 << 32:
            continue   # the plain form gathers every query's keys
        if c["kind"] == "select" and c["n_obj"] * c["n_q"] * c["H_kv"] * _blocks(c) > 1 << 26:
            continue
        if c["kind"] == "select" and (_blocks(c) < max(16, 2 * c["top_k"]) or c["top_k"] <= c["n_first"] + c["n_last"]):
            continue   # nothing to choose
        return c


def _blocks(case):
    return -(-case["n_kv"] // case["block"])


def work(case):
    """The bytes (every input read once, every output written once) and the
    operations that one pass cannot do without."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        vals = case["n"] * (case["H"] + case["H_kv"]) * case["d_h"]
        return dict(bytes=2 * vals * es + case["n"] * (4 + case["d_rot"] * 4), flops=8 * vals)
    n_obj, n_q, n_kv, H, H_kv = (case[k] for k in ("n_obj", "n_q", "n_kv", "H", "H_kv"))
    d_h, block, top_k, nb = case["d_h"], case["block"], case["top_k"], _blocks(case)
    mean_len = {"all": 1.0, "ragged": 0.6, "causal": 1.0 - 0.5 * min(n_q, n_kv) / n_kv}[case["vis"]]
    if case["kind"] == "means":
        keys = n_obj * min(n_kv, case["n_new"] + block / 2 if case["n_new"] else n_kv * mean_len)
        return dict(bytes=(keys + keys / block) * H_kv * d_h * es, flops=keys * H_kv * d_h)
    rows = n_obj * n_q
    if case["kind"] == "select":
        return dict(bytes=(rows * H + n_obj * H_kv * nb * (mean_len if n_q == 1 else 1.0)) * d_h * es +
                    rows * H_kv * (top_k + 1) * 4, flops=2 * rows * H_kv * nb * mean_len * d_h)
    keys = max(1.0, min(top_k * block, n_kv * mean_len))
    read = min(n_kv, n_q * keys) * n_obj * H_kv
    return dict(bytes=(2 * rows * H + 2 * read) * d_h * es + rows * H_kv * (top_k + 1) * 4,
                flops=4 * rows * H * keys * d_h)


# ---- inputs ------------------------------------------------------------------
def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + stream)


def _randn(shape, dt, gen):
    return torch.randn(shape, dtype=dt, device="cuda", generator=gen)


def _lengths(case, gen):
    """Visible keys of every query, int32 [n_obj][n_q], or None for all."""
    n_obj, n_q, n_kv = case["n_obj"], case["n_q"], case["n_kv"]
    if case["vis"] == "all":
        return None
    if case["vis"] == "causal":
        v = torch.arange(n_q, device="cuda", dtype=torch.int32) + (n_kv - n_q + 1)
        return v.clamp_(0, n_kv).expand(n_obj, n_q).contiguous()
    u = torch.rand((n_obj, n_q), device="cuda", generator=gen)
    v = ((0.2 + 0.8 * u) * n_kv).clamp_(min=1)
    v[1:][u[1:] < 0.03] = 0   # streams and rows that see nothing
    v[:, 1:][u[:, 1:] < 0.03] = 0
    return v.to(torch.int32)


def _norm_state(case, seed):
    n, H, H_kv, d_h, dt = case["n"], case["H"], case["H_kv"], case["d_h"], DT[case["dtype"]]
    g = _gen(seed, 1)
    st = dict(case=case)
    # an fp32 table of (cos, sin) of every position and pair
    pairs = case["d_rot"] // 2
    n_pos = max(16, n)
    p = torch.arange(n_pos, device="cuda", dtype=torch.float64)
    f = THETA ** (-torch.arange(max(pairs, 1), device="cuda", dtype=torch.float64) / max(pairs, 1))
    a = p[:, None] * f[None]
    if not case["halves"]:   # a grid: half of the pairs turn by the column, half by the row
        side = max(1, math.isqrt(n_pos))
        half = max(1, (pairs + 1) // 2)
        a = torch.cat([(p % side)[:, None] * f[None, :half], (p // side)[:, None] * f[None, :half]], 1)[:, :max(pairs, 1)]
    st["table"] = torch.stack([a.cos(), a.sin()], -1).float().contiguous() if pairs else None
    st["Q"] = _randn((n, H, d_h), dt, g)
    st["K"] = _randn((n, H_kv, d_h), dt, g) * 2
    st["gain_q"] = 1 + 0.2 * _randn((d_h,), torch.float32, g)
    st["gain_k"] = 1 + 0.2 * _randn((d_h,), torch.float32, g)
    pos = torch.randperm(n_pos, device="cuda", generator=g)[:n].to(torch.int32)
    if case["halves"]:
        pos = pos.sort().values
    pad = torch.rand((n,), device="cuda", generator=g) < case["pad"]
    pad[0] = False
    st["pos"] = torch.where(pad, torch.full_like(pos, -1), pos)
    st["Qo"], st["Ko"] = torch.zeros_like(st["Q"]), torch.zeros_like(st["K"])
    return st


def _block_state(case, seed):
    n_obj, n_q, n_kv, H, H_kv = (case[k] for k in ("n_obj", "n_q", "n_kv", "H", "H_kv"))
    d_h, block, nb, dt = case["d_h"], case["block"], _blocks(case), DT[case["dtype"]]
    g = _gen(seed, 2)
    st = dict(case=case, n_vis=_lengths(case, g))
    # centres that drift from block to block
    c = _randn((n_obj, nb, H_kv, d_h), torch.float32, g)
    c = 0.6 * (c + torch.roll(c, 1, 1) + torch.roll(c, 2, 1))
    if case["kind"] == "select":
        # the mean of `block` keys around a centre
        m = c + _randn((n_obj, nb, H_kv, d_h), torch.float32, g) / math.sqrt(block)
        st["Kmean"] = m.transpose(1, 2).to(dt).contiguous()
    else:
        K = torch.empty((n_obj, nb * block, H_kv, d_h), dtype=dt, device="cuda")
        K.normal_(generator=g)
        K.view(n_obj, nb, block, H_kv, d_h).mul_(0.7).add_(0.7 * c.to(dt)[:, :, None])
        st["K"] = K[:, :n_kv].contiguous() if nb * block > n_kv else K
        del K
    if case["kind"] == "means":
        st["Kmean"] = torch.zeros((n_obj, H_kv, nb, d_h), dtype=dt, device="cuda")
        return st
    # a query near the centres of a few blocks
    near = torch.randint(0, nb, (3, n_obj, n_q), device="cuda", generator=g)
    o = torch.arange(n_obj, device="cuda")[:, None]
    q = (c[o, near[0]] + c[o, near[1]] + 0.5 * c[o, near[2]])[:, :, :, None].expand(n_obj, n_q, H_kv, H // H_kv, d_h)
    q = q + _randn(q.shape, torch.float32, g)
    st["Q"] = (q * (LOGIT_SCALE / q.std())).reshape(n_obj, n_q, H, d_h).to(dt)
    shape = (n_obj, n_q, H_kv, case["top_k"])
    if case["kind"] == "select":
        st["idx"] = torch.zeros(shape, dtype=torch.int32, device="cuda")
        st["count"] = torch.zeros(shape[:3], dtype=torch.int32, device="cuda")
        return st
    st["V"] = torch.empty_like(st["K"]).normal_(generator=g)
    st["O"] = torch.zeros_like(st["Q"])
    qs = st["Q"].view(n_obj, n_q, H_kv, H // H_kv, d_h).float().sum(3)
    st["idx"], st["count"] = _pick(case, qs.transpose(1, 2) @ c.permute(0, 2, 3, 1), st["n_vis"])
    return st


def prepare(case, seed):
    st = (_norm_state if case["kind"] == "norm" else _block_state)(case, seed)
    if own:   # the shape and the workspace that a program keeps beside its cache
        import paper_2608_22526_amd as rs3
        dt = {"bf16": rs3.RS3_BF16, "f32": rs3.RS3_F32}[case["dtype"]]
        st["dt"] = dt
        if case["kind"] != "norm":
            st["shape"] = s = rs3.block_shape(dt, *(case[k] for k in ("n_obj", "n_q", "n_kv", "H", "H_kv", "d_h",
                                                                      "block", "top_k", "n_first", "n_last")))
            size = {"select": rs3.block_select_workspace_size, "attend": rs3.block_attend_workspace_size}
            need = size[case["kind"]](s) if case["kind"] in size else 0
            st["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return st


# ---- the plain forms ---------------------------------------------------------
def _turn(x, table, pos, d_rot, halves):
    """Rotation of the first d_rot channels of fp32 x [n][heads][d_h]."""
    cs = table[pos.clamp(min=0).long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    r, rest = x[..., :d_rot], x[..., d_rot:]
    if halves:
        a, b = r[..., :d_rot // 2], r[..., d_rot // 2:]
        r = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _plain_norm(st):
    c = st["case"]
    keep = (st["pos"] >= 0)[:, None, None]

    def one(x, gain, out):
        f = x.float()
        y = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * gain
        if c["d_rot"]:
            y = _turn(y, st["table"], st["pos"], c["d_rot"], c["halves"])
        return torch.where(keep, y.to(x.dtype), out)

    return [one(st["Q"], st["gain_q"], st["Qo"]), one(st["K"], st["gain_k"], st["Ko"])]


def _plain_means(st):
    c, K, out = st["case"], st["K"], st["Kmean"]
    n_obj, n_kv, block, nb = c["n_obj"], c["n_kv"], c["block"], _blocks(c)
    dev = K.device
    length = st["n_vis"][:, 0].long() if st["n_vis"] is not None else torch.full((n_obj,), n_kv, device=dev)
    # the blocks to compute: all of them, or those of the last n_new keys
    new = c["n_new"]
    first = (length - new).clamp(min=0) // block if new else torch.zeros_like(length)
    count = min(nb, (new + block - 2) // block + 1) if new else nb
    b = first[:, None] + torch.arange(count, device=dev)
    j = b[:, :, None] * block + torch.arange(block, device=dev)      # [n_obj][count][block]
    there = j < length[:, None, None]
    rows = K[torch.arange(n_obj, device=dev)[:, None, None], j.clamp(max=n_kv - 1)].double()
    total = torch.where(there[..., None, None], rows, torch.zeros((), dtype=torch.float64, device=dev)).sum(2)
    n = there.sum(2)
    mean = (total / n.clamp(min=1)[..., None, None]).to(K.dtype).transpose(1, 2)      # [n_obj][H_kv][count][d_h]
    # a block past an object's last key has a mean of 0 where all are computed
    use = (b < nb) & ((n > 0) | (new == 0))
    o = torch.arange(n_obj, device=dev)[:, None].expand_as(b)
    out[o[use], :, b[use]] = mean.transpose(1, 2)[use]
    return out


def _pick(c, scores, n_vis):
    """The lists of the scores [n_obj][H_kv][n_q][n_blk], ties to the lower block."""
    n_obj, n_q, nb, top_k, block = c["n_obj"], c["n_q"], _blocks(c), c["top_k"], c["block"]
    dev = scores.device
    seen = torch.full((n_obj, n_q), c["n_kv"], device=dev) if n_vis is None else n_vis.long()
    seen = ((seen + block - 1) // block)[:, None, :, None]          # visible blocks
    b = torch.arange(nb, device=dev)
    s = torch.where((b < c["n_first"]) | (b >= seen - c["n_last"]), torch.full_like(scores, math.inf), scores)
    s = torch.where(b < seen, s, torch.full_like(scores, -math.inf))
    k = min(top_k, nb)
    at = torch.sort(s, dim=-1, descending=True, stable=True).indices[..., :k]
    n = seen.clamp(max=top_k)
    at = torch.where(torch.arange(k, device=dev) < n, at, torch.full_like(at, nb)).sort(-1).values
    at = torch.where(at < nb, at, torch.full_like(at, -1))
    idx = torch.full((*at.shape[:3], top_k), -1, dtype=torch.int32, device=dev)
    idx[..., :k] = at.to(torch.int32)
    count = n.squeeze(-1).expand(at.shape[:3]).to(torch.int32)
    return idx.transpose(1, 2).contiguous(), count.transpose(1, 2).contiguous()


def _plain_select(st):
    c = st["case"]
    n_obj, n_q, H, H_kv, d_h = (c[k] for k in ("n_obj", "n_q", "H", "H_kv", "d_h"))
    # in 64 bits: two blocks' scores can lie closer than 32 bits tell apart
    q = st["Q"].view(n_obj, n_q, H_kv, H // H_kv, d_h).double().sum(3).transpose(1, 2)
    return list(_pick(c, q @ st["Kmean"].double().transpose(2, 3), st["n_vis"]))


def _plain_attend(st):
    c = st["case"]
    n_obj, n_q, n_kv, H, H_kv, d_h, block = (c[k] for k in ("n_obj", "n_q", "n_kv", "H", "H_kv", "d_h", "block"))
    dev = st["Q"].device
    idx = st["idx"].long()
    j = (idx[..., None] * block + torch.arange(block, device=dev)).flatten(3)   # [n_obj][n_q][H_kv][keys]
    seen = torch.full((n_obj, n_q), n_kv, device=dev) if st["n_vis"] is None else st["n_vis"].long()
    there = (j >= 0) & (j < seen[:, :, None, None])
    j = j.clamp(0, n_kv - 1)
    o = torch.arange(n_obj, device=dev)[:, None, None, None]
    h = torch.arange(H_kv, device=dev)[:, None]
    q = st["Q"].view(n_obj, n_q, H_kv, H // H_kv, d_h).float()
    logits = (q @ st["K"][o, j, h].float().transpose(-1, -2)) * (1.0 / math.sqrt(d_h))
    logits = torch.where(there[:, :, :, None], logits, torch.full_like(logits, -math.inf))
    top = logits.amax(-1, keepdim=True)
    w = torch.exp(logits - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = w.sum(-1, keepdim=True)
    out = (w @ st["V"][o, j, h].float()) / torch.where(total > 0, total, torch.ones_like(total))
    return out.reshape(n_obj, n_q, H, d_h).to(st["Q"].dtype)


# ---- one pass ----------------------------------------------------------------
def _own(st):
    import paper_2608_22526_amd as rs3
    c = st["case"]
    if c["kind"] == "norm":
        rs3.qk_norm_rope(c["n"], st["Q"], c["H"], st["K"], c["H_kv"], c["d_h"], st["dt"], st["Qo"], st["Ko"],
                         gain_q=st["gain_q"], gain_k=st["gain_k"], eps=EPS, table=st["table"], d_rot=c["d_rot"],
                         pairing=rs3.RS3_PAIRS_HALVES if c["halves"] else rs3.RS3_PAIRS_ADJACENT, pos=st["pos"])
        return [st["Qo"], st["Ko"]]
    if c["kind"] == "means":
        rs3.block_means(st["shape"], st["K"], st["Kmean"], kv_len=st["n_vis"], n_new=c["n_new"])
        return st["Kmean"]
    if c["kind"] == "select":
        rs3.block_select(st["shape"], st["Q"], st["Kmean"], st["idx"], st["count"], n_vis=st["n_vis"], ws=st["ws"])
        return [st["idx"], st["count"]]
    rs3.block_attend(st["shape"], st["Q"], st["K"], st["V"], st["idx"], st["count"], st["O"], n_vis=st["n_vis"],
                     ws=st["ws"])
    return st["O"]


PLAIN = dict(norm=_plain_norm, means=_plain_means, select=_plain_select, attend=_plain_attend)


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["kind"]](state)


# ---- the definition in 64 bits -------------------------------------------------
def exact(case, seed):
    def norm(st):
        c = st["case"]
        outs = []
        for x, gain in ((st["Q"], st["gain_q"]), (st["K"], st["gain_k"])):
            y = x.double()
            y = y / (y.square().sum(-1, keepdim=True) / c["d_h"] + EPS).sqrt() * gain.double()
            half = c["d_rot"] // 2
            for p in range(half):   # pair p as a complex number, times its factor
                a, b = (p, p + half) if c["halves"] else (2 * p, 2 * p + 1)
                f = torch.view_as_complex(st["table"][:, p].double())[st["pos"].clamp(min=0).long()][:, None]
                z = torch.complex(y[..., a], y[..., b]) * f
                y[..., a], y[..., b] = z.real, z.imag
            y[st["pos"] < 0] = 0.0
            outs.append(y)
        return outs

    def means(st):
        c, K = st["case"], st["K"]
        out = torch.zeros((c["n_obj"], c["H_kv"], _blocks(c), c["d_h"]), dtype=torch.float64, device=K.device)
        for o in range(c["n_obj"]):
            length = c["n_kv"] if st["n_vis"] is None else int(st["n_vis"][o, 0])
            b0 = max(0, length - c["n_new"]) // c["block"] if c["n_new"] else 0
            for b in range(b0, -(-length // c["block"])):
                out[o, :, b] = K[o, b * c["block"]:min(length, (b + 1) * c["block"])].double().mean(0)
        return out

    def attend(st):
        """Every query against every key, the keys outside its blocks masked."""
        c = st["case"]
        n_kv, H, H_kv, d_h, block, nb = (*(c[k] for k in ("n_kv", "H", "H_kv", "d_h", "block")), _blocks(c))
        out = torch.zeros(st["Q"].shape, dtype=torch.float64, device=st["Q"].device)
        step = max(1, (1 << 27) // n_kv)
        for o in range(c["n_obj"]):
            for hk in range(H_kv):
                kt, v = st["K"][o, :, hk].double().t().contiguous(), st["V"][o, :, hk].double()
                for a in range(0, c["n_q"], step):
                    idx = st["idx"][o, a:a + step, hk].long()
                    on = torch.zeros((idx.shape[0], nb + 1), dtype=torch.bool, device=idx.device)
                    on.scatter_(1, torch.where(idx < 0, torch.full_like(idx, nb), idx), True)
                    on = on[:, :nb].repeat_interleave(block, 1)[:, :n_kv]
                    if st["n_vis"] is not None:
                        on &= torch.arange(n_kv, device=idx.device) < st["n_vis"][o, a:a + step, None]
                    for h in range(hk * (H // H_kv), (hk + 1) * (H // H_kv)):
                        z = (st["Q"][o, a:a + step, h].double() @ kt) / math.sqrt(d_h)
                        z = torch.softmax(z.masked_fill_(~on, -math.inf), -1)
                        z[~on.any(1)] = 0.0
                        out[o, a:a + step, h] = z @ v
        return out

    if case["kind"] == "select":
        return None   # whole numbers
    st = (_norm_state if case["kind"] == "norm" else _block_state)(case, seed)
    return dict(norm=norm, means=means, attend=attend)[case["kind"]](st)
