"""The 4-bit operators of the draft-and-verify step, as cases that can be measured.

Four operators let the step's two largest reads stand in 4 bits: the draft head over 4-bit weights (`draft`), tree
attention over a 4-bit cache (`attention`), the history update that appends to such a cache (`commit`) and storing a
prompt's rows in it (`store`); what the last two wrote is read back as values by the call that does so.  Every case
is a dict of plain values:

  draft      dtype, M (rows), H, V, T, k, group (weights that share a scale), mapped (rows picked by a row map)
  attention  dtype, B, Hq, Hkv, D, nodes (tree rows per sequence), live ("all", "ragged", "one"), kv_lo, kv_hi
  commit     dtype, B, Hkv, D, nodes, T (longest accepted path), kv_lo, kv_hi
  store      dtype, B, Hkv, D, rows_lo, rows_hi (rows of a prompt), at (cached rows before it)

The format.  A row is cut into groups (32 values in a cache) with a bfloat16 scale and origin each; level q = 0..15
stands for origin + scale * (16 + q), rounded to the activations' type.  Quantising, in float32: scale =
bf16((max - min) / 15), origin = bf16(min - 16 scale), q = (v - origin) / scale - 16 rounded half to even and
clamped, 0 where the scale is 0.

With `own` false run() computes the operators in elementary torch operations in 32 bits; with `own` true it
calls the library.  exact() restates the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
LARGEST = 1.58e9       # weights of the largest listed draft case
GROUP = 32             # values of a cached row that share a scale


def listed():
    return [
        # the tiny float32 configuration: pure latency
        dict(name="draft-tiny-fp32", op="draft", dtype="fp32", M=1, H=256, V=1000, T=4, k=3, group=32, mapped=False),
        # the headline step's draft head
        dict(name="draft-7b", op="draft", dtype="bf16", M=1, H=4096, V=32000, T=5, k=4, group=128, mapped=False),
        # the batched 13B step, chained: rows picked from the previous step's tree
        dict(name="draft-13b-chained", op="draft", dtype="bf16", M=4, H=5120, V=32000, T=8, k=5, group=64, mapped=True),
        # the 70B step at batch 32: the largest
        dict(name="draft-70b", op="draft", dtype="bf16", M=32, H=8192, V=32000, T=6, k=4, group=128, mapped=False),
        # the tiny float32 configuration's tree over its cache
        dict(name="attn-tiny-fp32", op="attention", dtype="fp32", B=1, Hq=4, Hkv=4, D=64, nodes=32, live="all",
             kv_lo=128, kv_hi=128),
        # plain decoding over long caches, one token per sequence, 13B heads, odd lengths
        dict(name="attn-token-13b", op="attention", dtype="bf16", B=4, Hq=40, Hkv=40, D=128, nodes=2, live="one",
             kv_lo=16001, kv_hi=32767),
        # the batched 7B step with its 64-node trees
        dict(name="attn-tree-7b", op="attention", dtype="bf16", B=8, Hq=32, Hkv=32, D=128, nodes=64, live="ragged",
             kv_lo=512, kv_hi=2048),
        # the grouped 70B step at batch 32
        dict(name="attn-tree-70b", op="attention", dtype="bf16", B=32, Hq=64, Hkv=8, D=128, nodes=64, live="ragged",
             kv_lo=1024, kv_hi=4096),
        # every step of the batched 7B configuration: a path joins the cache
        dict(name="commit-7b", op="commit", dtype="bf16", B=8, Hkv=32, D=128, nodes=64, T=6, kv_lo=512, kv_hi=2048),
        # the tiny float32 configuration's
        dict(name="commit-tiny-fp32", op="commit", dtype="fp32", B=1, Hkv=4, D=64, nodes=32, T=4, kv_lo=128, kv_hi=128),
        # one short odd prompt
        dict(name="store-odd", op="store", dtype="bf16", B=3, Hkv=7, D=64, rows_lo=1, rows_hi=333, at=65),
        # the prompts of the grouped 70B batch
        dict(name="store-70b", op="store", dtype="bf16", B=32, Hkv=8, D=128, rows_lo=1024, rows_hi=4096, at=0),
    ]


HEADS = [(4, 4, 64), (12, 3, 64), (8, 1, 64), (28, 4, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (64, 8, 128),
         (15, 3, 128), (16, 1, 128)]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["draft", "draft", "attention", "attention", "commit", "store"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "draft":
        while True:
            T = rng.randint(1, 8)
            c = dict(op=op, dtype=dtype, M=_log(rng, 1, 32), H=8 * _log(rng, 8, 1024), V=_log(rng, 200, 128000), T=T,
                     k=rng.randint(1, min(8, 64 // T)), group=rng.choice([32, 64, 128]), mapped=rng.random() < 0.4)
            if c["T"] * c["V"] * c["H"] <= LARGEST / (1 if dtype == "bf16" else 8) and work(c)["bytes"] <= 8.36e8:
                return c
    Hq, Hkv, D = rng.choice(HEADS)
    if op == "attention":
        while True:
            c = dict(op=op, dtype=dtype, B=_log(rng, 1, 48), Hq=Hq, Hkv=Hkv, D=D,
                     nodes=rng.choice([2, 7, 32, 33, 64, 100, 128, 256]), live=rng.choice(["all", "ragged", "one"]),
                     kv_lo=1, kv_hi=_log(rng, 1, 32768))
            c["kv_lo"] = rng.randint(0, c["kv_hi"])
            # the plain form's scores and widened cache, and float32 without tensor cores, bound what a case may cost
            cells = c["B"] * (c["kv_hi"] + c["nodes"])
            if work(c)["flops"] <= 1.35e11 / (1 if dtype == "bf16" else 8) and cells * c["nodes"] * Hq <= 8e8 \
                    and cells * Hkv * D <= 7e8:
                return c
    while True:
        if op == "commit":
            nodes = rng.choice([8, 33, 64, 128])
            hi = _log(rng, 1, 8192)
            c = dict(op=op, dtype=dtype, B=_log(rng, 1, 48), Hkv=Hkv, D=D, nodes=nodes, T=rng.randint(1, 8),
                     kv_lo=rng.randint(0, hi), kv_hi=hi)
            if c["B"] * (hi + nodes) * Hkv * D <= 7e8:
                return c
        else:
            hi = _log(rng, 1, 32768)
            c = dict(op=op, dtype=dtype, B=_log(rng, 1, 32), Hkv=Hkv, D=D, rows_lo=rng.randint(0, hi), rows_hi=hi,
                     at=rng.choice([0, rng.randint(1, 500)]))
            if c["B"] * (hi + c["at"]) * Hkv * D * (1 if dtype == "bf16" else 2) <= 1.4e8:
                return c


# ---- lengths: part of the case, not of the seed ---------------------------------------------------
def _spread(lo, hi, n, phase):
    """n whole numbers over [lo, hi], scattered; the last is hi."""
    g = [(phase + 0.6180339887498949 * i) % 1.0 for i in range(n)]
    return [hi if i == n - 1 else lo + int(x * (hi - lo + 1)) for i, x in enumerate(g)]


def _lengths(c):
    B = c["B"]
    if c["op"] == "attention":
        n = {"all": [c["nodes"]] * B, "one": [1] * B, "ragged": _spread((c["nodes"] + 1) // 2, c["nodes"], B, 0.3)}[c["live"]]
        return n, _spread(c["kv_lo"], c["kv_hi"], B, 0.1)
    if c["op"] == "commit":                # accepted draft tokens, and cached rows before the update
        return _spread(0, min(c["T"], c["nodes"] - 1), B, 0.4), _spread(c["kv_lo"], c["kv_hi"], B, 0.1)
    return _spread(c["rows_lo"], c["rows_hi"], B, 0.2), [c["at"]] * B


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "draft":
        rows = c["T"] * (c["V"] + 1)
        return {"bytes": rows * (c["H"] / 2 + 4 * math.ceil(c["H"] / c["group"])) + c["M"] * (c["H"] * e + c["T"] * (8 * c["k"] + 4)),
                "flops": 2.0 * rows * c["H"] * c["M"]}
    a, kv = _lengths(c)
    D, Hkv, B = c["D"], c["Hkv"], c["B"]
    row = D / 2 + 4 * D / GROUP            # a cached row: levels, scales and origins
    if c["op"] == "attention":
        q = sum(a) * c["Hq"] * D * e
        out = B * c["nodes"] * c["Hq"] * (D * e + 4)
        pairs = sum(n * k + n * min(n, 6) for n, k in zip(a, kv))       # a node sees a short path of the tree
        return {"bytes": 2 * Hkv * (sum(kv) * row + sum(a) * D * e) + q + out, "flops": 4.0 * pairs * c["Hq"] * D}
    rows = sum(n + 1 for n in a) if c["op"] == "commit" else sum(a)
    back = B * ((c["T"] + 1) if c["op"] == "commit" else max(a))        # rows read back, the unused ones zero
    return {"bytes": 2 * Hkv * (rows * (D * e + row) + back * D * e), "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------
def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEVICE)


def _trees(rng, n_live, nodes):
    """Random trees as parents[i] < i, as their ancestor bit masks [B,nodes,W] (a row's own bit set)."""
    B, W = len(n_live), (nodes + 63) // 64
    mask = np.zeros((B, nodes, W), dtype=np.uint64)
    u = rng.random((B, nodes))
    for i in range(nodes):
        if i:
            parent = np.minimum((u[:, i] ** 2 * i).astype(np.int64), i - 1)
            mask[:, i] = mask[np.arange(B), parent]
        mask[:, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    for b, n in enumerate(n_live):
        mask[b, n:] = 0
    return mask


def _levels(v, group):
    """Levels (uint8, padded with level 0 to whole groups), scales and origins (bfloat16) of the rows of v [..., n]."""
    n = v.shape[-1]
    groups = (n + group - 1) // group
    f = v.float()
    if groups * group != n:                # (padded with the row's last value, which moves no limit)
        f = torch.cat([f, f[..., -1:].expand(*f.shape[:-1], groups * group - n)], -1)
    f = f.reshape(*f.shape[:-1], groups, group)
    lo, hi = f.amin(-1), f.amax(-1)
    scale = ((hi - lo) / 15.0).to(torch.bfloat16)
    origin = (lo - 16.0 * scale.float()).to(torch.bfloat16)
    q = ((f - origin.float()[..., None]) / scale.float()[..., None] - 16.0).round_().clamp_(0.0, 15.0)
    q = torch.where((scale > 0)[..., None], q, 0.0)
    return q.to(torch.uint8).flatten(-2), scale, origin


def _values(q, scale, origin, n, act):
    """What levels stand for, in float32 (values of the type `act`)."""
    q = q.unflatten(-1, (scale.shape[-1], -1)).float()
    v = (q + 16.0) * scale.float()[..., None] + origin.float()[..., None]
    return v.flatten(-2)[..., :n].to(act).float()


def prepare(case, seed):
    c = dict(case)
    act = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 23)
    rng = np.random.default_rng([int(seed), 43])

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32).to(act)

    s = dict(case=c, act=act)
    if c["op"] == "draft":
        return _prepare_draft(c, s, normal, rng)
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    a, kv = _lengths(c)

    def keys(*shape):      # channels of their own mean and spread, a few keys that draw most of the attention
        k = torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32)
        k.mul_(torch.rand(shape[-1], generator=gen, device=DEVICE).mul_(1.5).add_(0.25))
        k.mul_(torch.rand(shape[:-1] + (1,), generator=gen, device=DEVICE).pow_(6).mul_(2.0).add_(0.5))
        return k.add_(torch.randn(shape[-1], generator=gen, device=DEVICE).mul_(0.5)).to(act)

    if c["op"] == "attention":
        Lcap = max(kv) + 9
        nodes = c["nodes"]
        s.update(Q=normal(B, nodes, c["Hq"], D), Kt=keys(B, Hkv, nodes, D), Vt=normal(B, Hkv, nodes, D), kv_len=_i32(kv),
                 n_nodes=_i32(a), mask=torch.from_numpy(_trees(rng, a, nodes).view(np.int64)).to(DEVICE), scale=1.0 / math.sqrt(D),
                 out_O=torch.empty(B, nodes, c["Hq"], D, dtype=act, device=DEVICE),
                 out_lse=torch.empty(B, nodes, c["Hq"], dtype=torch.float32, device=DEVICE))
        _fill_cache(s, keys(B, Hkv, Lcap, D), normal(B, Hkv, Lcap, D), [Lcap] * B, Lcap)
        if own:
            s["plan"] = s["h"].make_q4_attention()
    elif c["op"] == "commit":
        Lcap = max(kv) + c["T"] + 1
        s.update(Kt=keys(B, Hkv, c["nodes"], D), Vt=normal(B, Hkv, c["nodes"], D), kv_len=_i32(kv), acc_len=_i32(a),
                 out_kv_len=_i32([0] * B), out_sel_row=_i32([0] * B), n_new=_i32([n + 1 for n in a]),
                 out_K=torch.empty(B, Hkv, c["T"] + 1, D, dtype=act, device=DEVICE),
                 out_V=torch.empty(B, Hkv, c["T"] + 1, D, dtype=act, device=DEVICE))
        path = np.full((B, c["T"]), -1, dtype=np.int64)
        for b, n in enumerate(a):
            path[b, :n] = np.sort(rng.choice(np.arange(1, c["nodes"]), size=n, replace=False))
        s["acc_nodes"] = _i32(path)
        _fill_cache(s, None, None, None, Lcap)
    else:
        rows, Lcap = max(a), max(a) + c["at"] + 3
        s.update(K=keys(B, Hkv, max(1, rows), D), V=normal(B, Hkv, max(1, rows), D), n_rows=_i32(a), at=_i32([c["at"]] * B),
                 out_K=torch.empty(B, Hkv, max(1, rows), D, dtype=act, device=DEVICE),
                 out_V=torch.empty(B, Hkv, max(1, rows), D, dtype=act, device=DEVICE))
        _fill_cache(s, None, None, None, Lcap)
    return s


def _handle(c):
    from paper_2412_00061_b200 import binding
    return binding.Handle(c.get("B", c.get("M")), c.get("H", 256), c.get("V", 1000), c.get("T", 5), c.get("k", 3), 16, 8,
                          c.get("nodes", 2), c.get("Hq", c.get("Hkv", 1)), c.get("Hkv", 1), c.get("D", 64),
                          binding.DTYPE_BF16 if c["dtype"] == "bf16" else binding.DTYPE_F32, device=DEVICE)


def _prepare_draft(c, s, normal, rng):
    """Weights in 4 bits, as the program holds them; x: hidden states, with a row map when `mapped`."""
    M, H, V, T = c["M"], c["H"], c["V"], c["T"]
    rows = M if not c["mapped"] else 7 * M
    s.update(x=normal(rows, H), x_rows=_i32(rng.permutation(rows)[:M]) if c["mapped"] else None,
             blank_bias=_i32(rng.integers(0, 3, M)).float(),
             out_topk_id=torch.empty(M, T, c["k"], dtype=torch.int32, device=DEVICE),
             out_topk_lp=torch.empty(M, T, c["k"], dtype=torch.float32, device=DEVICE),
             out_lse=torch.empty(M, T, dtype=torch.float32, device=DEVICE))
    if own:
        Wd = torch.empty(T, V + 1, H, dtype=s["act"], device=DEVICE)
    else:
        s.update(q=[], q_scale=[], q_origin=[])
    for t in range(T):
        w = normal(V + 1, H).mul_(0.02)
        if own:
            Wd[t] = w
        else:
            for name, v in zip(("q", "q_scale", "q_origin"), _levels(w, c["group"])):
                s[name].append(v)
    if own:
        s["h"] = _handle(c)
        s["Wq"] = s["h"].quantize_weights_q4(Wd, c["group"])
    return s


def _fill_cache(s, K, V, n, Lcap):
    """A cache of Lcap rows a sequence, its first n[b] rows filled."""
    c = s["case"]
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    if own:
        s["h"] = _handle(c)
        s["cache"] = s["h"].make_q4_cache(Lcap)
        if K is not None:
            s["h"].store_rows_q4(s["cache"], K, V, _i32(n), _i32([0] * B))
        return
    for name, v in (("K", K), ("V", V)):
        if v is not None:
            s[name + "q"], s[name + "s"], s[name + "o"] = _levels(v, GROUP)
        else:
            s[name + "q"] = torch.zeros(B, Hkv, Lcap, D, dtype=torch.uint8, device=DEVICE)
            s[name + "s"] = torch.zeros(B, Hkv, Lcap, D // GROUP, dtype=torch.bfloat16, device=DEVICE)
            s[name + "o"] = torch.zeros(B, Hkv, Lcap, D // GROUP, dtype=torch.bfloat16, device=DEVICE)


# ---- one pass ---------------------------------------------------------------------------------------
def run(s):
    return {"draft": _draft, "attention": _attention, "commit": _commit, "store": _store}[s["case"]["op"]](s)


def _draft(s):
    c = s["case"]
    if own:
        s["h"].draft_logits_q4(s["x"], s["x_rows"], s["Wq"], None, s["blank_bias"], s["out_topk_id"], s["out_topk_lp"], s["out_lse"])
        return {"topk_id": s["out_topk_id"], "topk_lp": s["out_topk_lp"], "lse": s["out_lse"]}
    x = (s["x"] if s["x_rows"] is None else s["x"][s["x_rows"].long()]).float()
    ids, lps, lses = [], [], []
    for t in range(c["T"]):
        w = _values(s["q"][t], s["q_scale"][t], s["q_origin"][t], c["H"], s["act"])
        z = torch.matmul(x, w.t())
        z[:, -1] += s["blank_bias"]
        top = z.amax(-1, keepdim=True)
        lse = (z - top).exp_().sum(-1).log_() + top[:, 0]
        z, i = z.sort(dim=-1, descending=True, stable=True)
        ids.append(i[:, :c["k"]].int())
        lps.append(z[:, :c["k"]] - lse[:, None])
        lses.append(lse)
    return {"topk_id": torch.stack(ids, 1), "topk_lp": torch.stack(lps, 1), "lse": torch.stack(lses, 1)}


def _attention(s):
    if own:
        s["h"].tree_attention_q4(s["plan"], s["Q"], s["cache"], s["Kt"], s["Vt"], s["kv_len"], s["n_nodes"], s["mask"], s["scale"],
                                 s["out_O"], s["out_lse"])
        return {"O": s["out_O"], "lse": s["out_lse"]}
    c = s["case"]
    B, n, Hq, Hkv, D = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"]
    G, Lcap = Hq // Hkv, s["Kq"].shape[2]
    q = s["Q"].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    kc, vc = (_values(s[a + "q"], s[a + "s"], s[a + "o"], D, s["act"]) for a in "KV")
    xc = torch.matmul(q, kc.transpose(2, 3)).view(B, Hkv, n, G, Lcap)
    xt = torch.matmul(q, s["Kt"].float().transpose(2, 3)).view(B, Hkv, n, G, n)
    seen_c = torch.arange(Lcap, device=DEVICE)[None] < s["kv_len"][:, None]                # [B,Lcap]
    j = torch.arange(n, device=DEVICE)
    bits = s["mask"][:, :, j >> 6] >> (j & 63)
    seen_t = ((bits & 1) != 0) & (j < s["n_nodes"][:, None])[:, None]                      # [B,n,n]
    xc.mul_(s["scale"]).masked_fill_(~seen_c[:, None, None, None], -math.inf)
    xt.mul_(s["scale"]).masked_fill_(~seen_t[:, None, :, None], -math.inf)
    top = torch.maximum(xc.amax(-1, keepdim=True), xt.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    xc.sub_(top).exp_()
    xt.sub_(top).exp_()
    total = xc.sum(-1, keepdim=True) + xt.sum(-1, keepdim=True)
    o = torch.matmul(xc.view(B, Hkv, n * G, Lcap), vc) + torch.matmul(xt.view(B, Hkv, n * G, n), s["Vt"].float())
    live = (j < s["n_nodes"][:, None])[:, None, :, None, None] & (total > 0)
    o = torch.where(live, o.view(B, Hkv, n, G, D) / total, 0.0)
    lse = torch.where(live, top + total.log(), -math.inf)
    return {"O": o.permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D).to(s["act"]),
            "lse": lse.permute(0, 2, 1, 3, 4).reshape(B, n, Hq)}


def _put(s, name, rows, at, n):
    """Rows [B,Hkv,R,D] to cache rows at .. at+n-1, and what then stands there (zero from row n on)."""
    c = s["case"]
    parts = _levels(rows, GROUP)
    R = rows.shape[2]
    b, r = torch.nonzero(torch.arange(R, device=DEVICE)[None] < n[:, None], as_tuple=True)
    to = at.long()[b] + r
    for part, v in zip("qso", parts):
        s[name + part][b, :, to] = v[b, :, r]
    out = torch.zeros(c["B"], c["Hkv"], R, c["D"], dtype=s["act"], device=DEVICE)
    out[b, :, r] = _values(*(s[name + part][b, :, to] for part in "qso"), c["D"], s["act"]).to(s["act"])
    return out


def _commit(s):
    c = s["case"]
    if own:
        s["h"].commit_accepted_q4(s["Kt"], s["Vt"], s["cache"], s["kv_len"], s["acc_len"], s["acc_nodes"], s["out_kv_len"], s["out_sel_row"])
        s["h"].load_rows_q4(s["cache"], s["kv_len"], s["n_new"], s["out_K"], s["out_V"])
        return {"K": s["out_K"], "V": s["out_V"], "kv_len": s["out_kv_len"], "sel_row": s["out_sel_row"]}
    b = torch.arange(c["B"], device=DEVICE)
    nodes = torch.cat([torch.zeros(c["B"], 1, dtype=torch.int64, device=DEVICE), s["acc_nodes"].long().clamp(min=0)], 1)
    out = {}
    for name, t in (("K", s["Kt"]), ("V", s["Vt"])):
        rows = t.gather(2, nodes[:, None, :, None].expand(-1, c["Hkv"], -1, c["D"]))
        out[name] = _put(s, name, rows, s["kv_len"], s["n_new"])
    out["kv_len"] = s["kv_len"] + 1 + s["acc_len"]
    out["sel_row"] = (b * c["nodes"] + nodes[b, s["acc_len"].long()]).int()
    return out


def _store(s):
    if own:
        s["h"].store_rows_q4(s["cache"], s["K"], s["V"], s["n_rows"], s["at"])
        s["h"].load_rows_q4(s["cache"], s["at"], s["n_rows"], s["out_K"], s["out_V"])
        return {"K": s["out_K"], "V": s["out_V"]}
    return {name: _put(s, name, s[name], s["at"], s["n_rows"]) for name in "KV"}


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def _stands_for(v, group, act):
    """The values, in float64, that the rows of v [R,n] have in 4 bits.  Scale, origin and level are defined by their
    float32 steps; the value is formed in 64 bits and rounded to `act`."""
    R, n = v.shape
    out = torch.empty(R, n, dtype=torch.float64, device=v.device)
    for g0 in range(0, n, group):
        w = v[:, g0:g0 + group].to(torch.float32)
        low = w.min(dim=1, keepdim=True).values
        step = torch.sub(w.max(dim=1, keepdim=True).values, low).div(15.0).bfloat16().float()
        base = torch.sub(low, step * 16.0).bfloat16().float()
        level = torch.sub(w, base).div(step).sub(16.0).round().clamp(0, 15)
        level[step[:, 0] == 0] = 0
        out[:, g0:g0 + group] = (base.double() + step.double() * (level.double() + 16)).to(act).double()
    return out


def exact(case, seed):
    c = dict(case)
    act = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 23)
    if c["op"] == "draft":
        return _exact_draft(c, act, gen, seed)
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    s = _inputs_alone(case, seed)
    if c["op"] == "store":
        out = {}
        for name in "KV":
            out[name] = torch.zeros(s[name].shape, dtype=torch.float64, device=DEVICE)
            for b, n in enumerate(s["n_rows"].tolist()):
                out[name][b, :, :n] = _stands_for(s[name][b, :, :n].reshape(-1, D), GROUP, act).view(Hkv, n, D)
        return out
    if c["op"] == "commit":
        acc, kv, path = s["acc_len"].tolist(), s["kv_len"].tolist(), s["acc_nodes"].tolist()
        out = {name: torch.zeros(B, Hkv, c["T"] + 1, D, dtype=torch.float64, device=DEVICE) for name in "KV"}
        for b in range(B):
            at = [0] + path[b][:acc[b]]
            for name in "KV":
                rows = s[name + "t"][b, :, at].reshape(-1, D)
                out[name][b, :, :len(at)] = _stands_for(rows, GROUP, act).view(Hkv, len(at), D)
        out["kv_len"] = torch.tensor([k + 1 + n for k, n in zip(kv, acc)], dtype=torch.int32, device=DEVICE)
        out["sel_row"] = torch.tensor([b * c["nodes"] + ([0] + path[b])[acc[b]] for b in range(B)], dtype=torch.int32, device=DEVICE)
        return out
    n, Hq = c["nodes"], c["Hq"]
    G = Hq // Hkv
    O = torch.zeros(B, n, Hq, D, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device=DEVICE)
    words = s["mask"].cpu().numpy().view(np.uint64)
    for b, (m, L) in enumerate(zip(s["n_nodes"].tolist(), s["kv_len"].tolist())):
        anc = np.unpackbits(words[b, :m].view(np.uint8), axis=1, bitorder="little")[:, :m].astype(bool)
        hidden = torch.from_numpy(~anc).to(DEVICE)
        for g in range(Hkv):
            q = s["Q"][b, :m, g * G:(g + 1) * G].double().reshape(m * G, D)
            k = torch.cat([_stands_for(s["Kc"][b, g, :L], GROUP, act), s["Kt"][b, g, :m].double()])
            v = torch.cat([_stands_for(s["Vc"][b, g, :L], GROUP, act), s["Vt"][b, g, :m].double()])
            x = (q @ k.t() * s["scale"]).view(m, G, -1)
            x[:, :, L:] = x[:, :, L:].masked_fill(hidden[:, None], -math.inf)
            O[b, :m, g * G:(g + 1) * G] = (torch.softmax(x, -1).view(m * G, -1) @ v).view(m, G, D)
            lse[b, :m, g * G:(g + 1) * G] = torch.logsumexp(x, -1)
    return {"O": O, "lse": lse}


def _inputs_alone(case, seed):
    """The case's inputs, with the rows that the cache was filled from in place of the cache."""
    global own, _fill_cache
    was, fill, rows = own, _fill_cache, {}
    try:
        own, _fill_cache = False, lambda s, K, V, n, Lcap: rows.update(Kc=K, Vc=V)
        s = prepare(case, seed)
    finally:
        own, _fill_cache = was, fill
    s.update(rows)
    return s


def _exact_draft(c, act, gen, seed):
    M, H, V, T, k = c["M"], c["H"], c["V"], c["T"], c["k"]
    rng = np.random.default_rng([int(seed), 43])
    rows = 7 * M if c["mapped"] else M
    x = torch.randn(rows, H, generator=gen, device=DEVICE, dtype=torch.float32).to(act).double()
    if c["mapped"]:
        x = x[torch.from_numpy(rng.permutation(rows)[:M]).to(DEVICE)]
    bias = torch.from_numpy(rng.integers(0, 3, M)).to(DEVICE).double()
    ids = torch.empty(M, T, k, dtype=torch.int32, device=DEVICE)
    lps = torch.empty(M, T, k, dtype=torch.float64, device=DEVICE)
    lses = torch.empty(M, T, dtype=torch.float64, device=DEVICE)
    for t in range(T):
        w = torch.randn(V + 1, H, generator=gen, device=DEVICE, dtype=torch.float32).to(act) * 0.02
        z = torch.cat([x @ _stands_for(part, c["group"], act).t() for part in w.split(4096)], 1)
        z[:, V] += bias
        lses[:, t] = torch.logsumexp(z, 1)
        for j in range(k):                 # the largest, ties to the lowest id
            best = z.max(dim=1, keepdim=True).values
            i = torch.where(z == best, torch.arange(V + 1, device=DEVICE), V + 1).min(dim=1).values
            ids[:, t, j] = i.int()
            lps[:, t, j] = best[:, 0] - lses[:, t]
            z.scatter_(1, i[:, None], -math.inf)
    return {"topk_id": ids, "topk_lp": lps, "lse": lses}
