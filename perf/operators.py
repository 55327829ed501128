"""The cache operators of the draft-and-verify step, as cases that can be measured.

Three operators stand behind a batch that decodes for a long time: tree attention over a prefix that all
sequences share and their own caches (`attention`), the attention weight that every cached row has gathered
(`mass`), and the eviction of the rows that gathered least (`evict`).  Every case is a dict of plain values:

  attention  dtype, B, Hq, Hkv, D, nodes (tree rows per sequence), live ("all", "ragged", "one"), prefix (longest
             shared prefix), spread (sequences share different lengths of it), kv_lo, kv_hi (own cached rows)
  mass       dtype, B, Hq, Hkv, D, nodes, T (longest accepted path), kv_lo, kv_hi, decay
  evict      dtype, B, Hkv, D, budget, over_lo, over_hi (rows above the budget), sinks, recent

With `own` false run() computes the operators in elementary torch operations in 32 bits; with `own` true it
calls the library.  exact() restates the definitions in 64 bits, one sequence and kv head at a time.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
LARGEST = 5.6e11       # flops of the largest listed attention case


def listed():
    return [
        # the tiny float32 configuration, one sequence: pure latency
        dict(name="attn-tiny-fp32", op="attention", dtype="fp32", B=1, Hq=4, Hkv=4, D=64, nodes=32, live="all",
             prefix=128, spread=False, kv_lo=128, kv_hi=128),
        # 7B heads, one token per sequence behind a long system prompt: the prefix's rows are the traffic
        dict(name="attn-token-7b", op="attention", dtype="bf16", B=8, Hq=32, Hkv=32, D=128, nodes=2, live="one",
             prefix=8192, spread=False, kv_lo=512, kv_hi=2048),
        # the batched 7B step: 64-node trees, few-shot prompt shared by all
        dict(name="attn-tree-7b", op="attention", dtype="bf16", B=8, Hq=32, Hkv=32, D=128, nodes=64, live="ragged",
             prefix=2048, spread=False, kv_lo=512, kv_hi=2048),
        # the grouped 70B step at batch 32 behind a long shared document: the largest
        dict(name="attn-tree-70b", op="attention", dtype="bf16", B=32, Hq=64, Hkv=8, D=128, nodes=64, live="ragged",
             prefix=8192, spread=False, kv_lo=1024, kv_hi=4096),
        # odd everything: seven heads per kv head, 33 nodes, sequences that share different lengths
        dict(name="attn-odd", op="attention", dtype="bf16", B=5, Hq=28, Hkv=4, D=64, nodes=33, live="ragged",
             prefix=1537, spread=True, kv_lo=1, kv_hi=777),
        # the headline step's cache, accepted path of the longest kind: latency
        dict(name="mass-7b", op="mass", dtype="bf16", B=1, Hq=32, Hkv=32, D=128, nodes=64, T=5, kv_lo=1024,
             kv_hi=1024, decay=1.0),
        # the grouped batch-32 step
        dict(name="mass-70b", op="mass", dtype="bf16", B=32, Hq=64, Hkv=8, D=128, nodes=64, T=6, kv_lo=1024,
             kv_hi=4096, decay=1.0),
        # 13B heads over long caches
        dict(name="mass-13b-long", op="mass", dtype="bf16", B=2, Hq=40, Hkv=40, D=128, nodes=128, T=8, kv_lo=30001,
             kv_hi=32768, decay=0.99),
        # the tiny float32 configuration's cache, cut by a quarter
        dict(name="evict-tiny-fp32", op="evict", dtype="fp32", B=1, Hkv=4, D=64, budget=96, over_lo=32, over_hi=32,
             sinks=4, recent=16),
        # every step once the budget is reached: a handful of rows leave
        dict(name="evict-step-7b", op="evict", dtype="bf16", B=8, Hkv=32, D=128, budget=2048, over_lo=1, over_hi=7,
             sinks=4, recent=256),
        # a prompt's cache cut to a quarter after prefill, batch 32
        dict(name="evict-cut-70b", op="evict", dtype="bf16", B=32, Hkv=8, D=128, budget=1024, over_lo=500,
             over_hi=7168, sinks=4, recent=128),
        # one very long prompt
        dict(name="evict-long", op="evict", dtype="bf16", B=1, Hkv=8, D=128, budget=16384, over_lo=49152,
             over_hi=49152, sinks=16, recent=1024),
    ]


HEADS = [(4, 4, 64), (12, 3, 64), (8, 1, 64), (28, 4, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (64, 8, 128),
         (15, 3, 128), (16, 1, 128)]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "mass", "evict"])
    Hq, Hkv, D = rng.choice(HEADS)
    if op == "attention":
        while True:
            c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), B=_log(rng, 1, 48), Hq=Hq, Hkv=Hkv, D=D,
                     nodes=rng.choice([2, 7, 32, 33, 64, 100, 128, 256]), live=rng.choice(["all", "ragged", "one"]),
                     prefix=_log(rng, 1, 32768), spread=rng.random() < 0.3, kv_lo=1, kv_hi=1)
            c["kv_hi"] = _log(rng, 1, 8192)
            c["kv_lo"] = rng.randint(0, c["kv_hi"])
            # the plain form's score matrices, and float32 without tensor cores, bound what a case may cost
            rows = c["B"] * c["nodes"] * Hq * (c["prefix"] + c["kv_hi"] + c["nodes"])
            if work(c)["flops"] <= LARGEST / (1 if c["dtype"] == "bf16" else 8) and rows <= 1.7e9:
                return c
    if op == "mass":
        while True:
            hi = _log(rng, 1, 65536)
            c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), B=_log(rng, 1, 32), Hq=Hq, Hkv=Hkv, D=D,
                     nodes=rng.choice([8, 33, 64, 128]), T=rng.randint(1, 8), kv_lo=rng.randint(0, hi), kv_hi=hi,
                     decay=rng.choice([1.0, 1.0, 0.9]))
            if work(c)["bytes"] <= 8e8 and c["B"] * (c["T"] + 1) * Hq * hi <= 4e8:
                return c
    while True:
        budget = _log(rng, 16, 32768)
        steady = rng.random() < 0.5
        hi = rng.randint(1, 9) if steady else _log(rng, 1, 4 * budget)
        recent = rng.randint(0, budget // 2)
        c = dict(op="evict", dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), B=_log(rng, 1, 32), Hkv=Hkv, D=D,
                 budget=budget, over_lo=rng.randint(-min(9, budget // 2), hi), over_hi=hi,
                 sinks=rng.randint(0, min(8, budget - recent)), recent=recent)
        if c["B"] * Hkv * (budget + hi) * (D * 4 + 64) <= 1.2e9:
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
        pre = _spread(0, c["prefix"], B, 0.55) if c["spread"] else [c["prefix"]] * B
        return n, pre, _spread(c["kv_lo"], c["kv_hi"], B, 0.1)
    if c["op"] == "mass":                 # accepted draft tokens, and cached rows before the step
        top = min(c["T"], c["nodes"] - 1)
        return _spread(0, top, B, 0.4), None, _spread(c["kv_lo"], c["kv_hi"], B, 0.1)
    return None, None, [c["budget"] + o for o in _spread(c["over_lo"], c["over_hi"], B, 0.2)]


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    a, pre, kv = _lengths(c)
    D, Hkv, B = c["D"], c["Hkv"], c["B"]
    if c["op"] == "attention":
        rows = max(pre) + sum(k + n for k, n in zip(kv, a))
        q = sum(a) * c["Hq"] * D * e
        out = B * c["nodes"] * c["Hq"] * (D * e + 4)
        pairs = sum(n * (p + k) + n * min(n, 6) for n, p, k in zip(a, pre, kv))     # a node sees a short path of the tree
        return {"bytes": 2 * rows * Hkv * D * e + q + out, "flops": 4 * pairs * c["Hq"] * D}
    if c["op"] == "mass":
        rows = [k + 1 + n for k, n in zip(kv, a)]
        q = sum(n + 1 for n in a) * c["Hq"] * (D * e + 4)
        return {"bytes": sum(rows) * Hkv * (D * e + 8) + q + 4 * sum(n + 1 for n in a) * Hkv,
                "flops": 2 * sum((n + 1) * r for n, r in zip(a, rows)) * c["Hq"] * D}
    total = 0.0
    for L in kv:
        new = min(L, c["budget"])
        total += 8.0 * (L + new)
        e_rows, free = L - new, max(1, L - c["sinks"] - c["recent"])
        if e_rows > 0:                    # rows behind the budget that stay, and have to move (expected)
            kept = min(c["recent"], e_rows) + max(0, e_rows - c["recent"]) * (new - c["sinks"] - c["recent"]) / free
            total += 4.0 * kept * D * e   # K and V, read and written
    return {"bytes": total * Hkv, "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------
def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEVICE)


def _trees(rng, n_live, nodes):
    """Random trees as parents[i] < i, and their ancestor bit masks [B,nodes,W] (a row's own bit set)."""
    B, W = len(n_live), (nodes + 63) // 64
    mask = np.zeros((B, nodes, W), dtype=np.uint64)
    parent = np.full((B, nodes), -1, dtype=np.int64)
    u = rng.random((B, nodes))
    for i in range(nodes):
        if i:
            parent[:, i] = np.minimum((u[:, i] ** 2 * i).astype(np.int64), i - 1)
            mask[:, i] = mask[np.arange(B), parent[:, i]]
        mask[:, i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    for b, n in enumerate(n_live):
        mask[b, n:] = 0
        parent[b, n:] = -1
    return parent, mask


def _paths(rng, acc, nodes, T):
    """An accepted path per sequence: increasing node ids, -1 behind its end."""
    out = np.full((len(acc), T), -1, dtype=np.int64)
    for b, n in enumerate(acc):
        out[b, :n] = np.sort(rng.choice(np.arange(1, nodes), size=n, replace=False))
    return out


def prepare(case, seed):
    c = dict(case)
    act = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 17)
    rng = np.random.default_rng([int(seed), 41])
    B, Hkv, D = c["B"], c["Hkv"], c["D"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32).to(act)

    def keys(*shape):      # a few keys draw most of the attention, as in a trained model
        k = torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32)
        return k.mul_(torch.rand(shape[:-1] + (1,), generator=gen, device=DEVICE).pow_(6).mul_(2.0).add_(0.5)).to(act)

    a, pre, kv = _lengths(c)
    s = dict(case=c, kv_len=_i32(kv))
    if c["op"] == "attention":
        Lcap = max(kv) + c["nodes"] + 5
        parent, mask = _trees(rng, a, c["nodes"])
        s.update(Q=normal(B, c["nodes"], c["Hq"], D), Kp=keys(Hkv, c["prefix"], D), Vp=normal(Hkv, c["prefix"], D),
                 K=keys(B, Hkv, Lcap, D), V=normal(B, Hkv, Lcap, D), n_nodes=_i32(a), prefix_len=_i32(pre),
                 mask=torch.from_numpy(mask.view(np.int64)).to(DEVICE), scale=1.0 / math.sqrt(D),
                 out_O=torch.empty(B, c["nodes"], c["Hq"], D, dtype=act, device=DEVICE),
                 out_lse=torch.empty(B, c["nodes"], c["Hq"], dtype=torch.float32, device=DEVICE))
    elif c["op"] == "mass":
        Lcap = max(k + 1 + n for k, n in zip(kv, a)) + c["nodes"]
        s.update(Q=normal(B, c["nodes"], c["Hq"], D), K=keys(B, Hkv, Lcap, D), acc_len=_i32(a),
                 acc_nodes=_i32(_paths(rng, a, c["nodes"], c["T"])), scale=1.0 / math.sqrt(D),
                 kv_len=_i32([k + 1 + n for k, n in zip(kv, a)]),
                 mass=torch.rand(B, Hkv, Lcap, generator=gen, device=DEVICE).pow_(4),
                 row_pos=torch.arange(Lcap, dtype=torch.int32, device=DEVICE).repeat(B, Hkv, 1),
                 n_evicted=_i32(rng.integers(0, 1000, B)))
        s["lse"] = _path_lse(s)
    else:
        Lcap = max(kv) + 9
        n_ev = rng.integers(0, 2 * c["budget"], B)
        # rows of the budget hold old positions in any order, the rows above it the newest in order
        row_pos = torch.empty(B, Hkv, Lcap, dtype=torch.int32, device=DEVICE)
        j = torch.arange(Lcap, dtype=torch.int32, device=DEVICE)
        front = torch.rand(B, Hkv, Lcap, generator=gen, device=DEVICE)
        front = torch.where((j < s["kv_len"][:, None, None]) & (j < c["budget"]), front, 2.0)
        order = front.argsort(dim=-1).argsort(dim=-1).to(torch.int32)
        row_pos.copy_(order + torch.where(j < c["budget"], 0, 1) * _i32(n_ev)[:, None, None])
        row_pos[:, :, c["budget"]:] = (j[None] + _i32(n_ev)[:, None])[:, None, c["budget"]:]
        # weights with ties among them: rows that nobody looked at hold nothing
        m = torch.rand(B, Hkv, Lcap, generator=gen, device=DEVICE)
        m = torch.where(m < 0.2, 0.0, m.pow(8) * 10)
        s.update(K=normal(B, Hkv, Lcap, D), V=normal(B, Hkv, Lcap, D), mass=m, row_pos=row_pos, n_evicted=_i32(n_ev),
                 out_mass=torch.zeros_like(m), out_row_pos=torch.zeros_like(row_pos),
                 out_kv_len=torch.zeros_like(s["kv_len"]), out_n_evicted=torch.zeros_like(s["kv_len"]))
    if own:
        s["h"], s["plan"] = _handle(c, Lcap)
    return s


def _handle(c, Lcap):
    from paper_2412_00061_b200 import binding
    h = binding.Handle(c["B"], 256, 1000, c.get("T", 5), 3, 16, 8, c.get("nodes", 2), c.get("Hq", c["Hkv"]), c["Hkv"], c["D"],
                       binding.DTYPE_BF16 if c["dtype"] == "bf16" else binding.DTYPE_F32, device=DEVICE)
    if c["op"] == "evict":
        return h, h.make_eviction(Lcap)
    return h, (h.make_shared_attention() if c["op"] == "attention" else None)


def _path_rows(s):
    """Accepted queries of every sequence, root first: [B,T+1,Hq,D] and which of them exist."""
    c, T1 = s["case"], s["case"]["T"] + 1
    nodes = torch.cat([torch.zeros(c["B"], 1, dtype=torch.int64, device=DEVICE), s["acc_nodes"].long().clamp(min=0)], 1)
    live = torch.arange(T1, device=DEVICE)[None] <= s["acc_len"][:, None]
    return nodes, live


def _path_scores(s):
    """Scaled scores [B,Hkv,G,T+1,Lcap] of the accepted queries, -inf where a row is not seen."""
    c = s["case"]
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    G, T1 = c["Hq"] // Hkv, c["T"] + 1
    nodes, live = _path_rows(s)
    q = s["Q"][torch.arange(B, device=DEVICE)[:, None], nodes].float()                    # [B,T1,Hq,D]
    q = q.view(B, T1, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * T1, D)
    x = torch.matmul(q, s["K"].float().transpose(2, 3)).view(B, Hkv, G, T1, -1) * s["scale"]
    j = torch.arange(s["K"].shape[2], device=DEVICE)
    base = (s["kv_len"] - 1 - s["acc_len"])[:, None, None]
    seen = (j <= base + torch.arange(T1, device=DEVICE)[None, :, None]) & live[:, :, None]
    return x.masked_fill_(~seen[:, None, None], -math.inf)


def _path_lse(s):
    """Log-sum-exp of the accepted queries as the attention would have returned it (their sequence's shared
    prefix takes a part of the weight); other nodes' entries are not read."""
    c = s["case"]
    nodes, live = _path_rows(s)
    own_part = torch.logsumexp(_path_scores(s), dim=-1)                                   # [B,Hkv,G,T1]
    own_part = own_part.permute(0, 3, 1, 2).reshape(c["B"], c["T"] + 1, c["Hq"]) + 0.4
    lse = torch.zeros(c["B"], c["nodes"], c["Hq"], device=DEVICE)
    b, l = torch.nonzero(live, as_tuple=True)
    lse[b, nodes[b, l]] = own_part[b, l]
    return lse


# ---- one pass ---------------------------------------------------------------------------------------
def run(s):
    return {"attention": _attention, "mass": _mass, "evict": _evict}[s["case"]["op"]](s)


def _attention(s):
    if own:
        s["h"].tree_attention_shared(s["plan"], s["Q"], s["Kp"], s["Vp"], s["prefix_len"], s["K"], s["V"], s["kv_len"],
                                     s["n_nodes"], s["mask"], s["scale"], s["out_O"], s["out_lse"])
        return {"O": s["out_O"], "lse": s["out_lse"]}
    c = s["case"]
    B, n, Hq, Hkv, D = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"]
    G, P, Lcap = Hq // Hkv, c["prefix"], s["K"].shape[2]
    q = s["Q"].float().view(B, n, Hkv, G, D).permute(2, 0, 1, 3, 4)                        # [Hkv,B,n,G,D]
    xp = torch.matmul(q.reshape(Hkv, B * n * G, D), s["Kp"].float().transpose(1, 2)).view(Hkv, B, n, G, P)
    xo = torch.matmul(q.reshape(Hkv, B, n * G, D), s["K"].float().permute(1, 0, 3, 2)).view(Hkv, B, n, G, Lcap)
    seen_p = torch.arange(P, device=DEVICE)[None] < s["prefix_len"][:, None]               # [B,P]
    rel = torch.arange(Lcap, device=DEVICE)[None] - s["kv_len"][:, None]                   # [B,Lcap]
    at = rel.clamp(0, n - 1).long()
    bits = torch.gather(s["mask"], 2, (at >> 6)[:, None].expand(B, n, Lcap)) >> (at & 63)[:, None]
    seen_o = (rel < 0)[:, None] | (((bits & 1) != 0) & (rel < s["n_nodes"][:, None])[:, None])   # [B,n,Lcap]
    xp.mul_(s["scale"]).masked_fill_(~seen_p[None, :, None, None], -math.inf)
    xo.mul_(s["scale"]).masked_fill_(~seen_o[None, :, :, None], -math.inf)
    top = torch.maximum(xp.amax(-1, keepdim=True), xo.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    xp.sub_(top).exp_()
    xo.sub_(top).exp_()
    total = xp.sum(-1, keepdim=True) + xo.sum(-1, keepdim=True)
    vp = torch.where(seen_p.any(0)[None, :, None], s["Vp"].float(), 0.0)
    vo = torch.where((rel < s["n_nodes"][:, None])[:, None, :, None], s["V"].float(), 0.0)
    o = torch.matmul(xp.view(Hkv, B * n * G, P), vp).view(Hkv, B, n, G, D)
    o += torch.matmul(xo.view(Hkv, B, n * G, Lcap), vo.permute(1, 0, 2, 3)).view(Hkv, B, n, G, D)
    live = (torch.arange(n, device=DEVICE)[None] < s["n_nodes"][:, None])[None, :, :, None, None] & (total > 0)
    o = torch.where(live, o / total, 0.0)
    lse = torch.where(live, top + total.log(), -math.inf)
    return {"O": o.permute(1, 2, 0, 3, 4).reshape(B, n, Hq, D).to(s["Q"].dtype),
            "lse": lse.permute(1, 2, 0, 3, 4).reshape(B, n, Hq)}


def _mass(s):
    c = s["case"]
    if own:
        s["h"].attention_mass(s["Q"], s["K"], s["kv_len"], s["acc_len"], s["acc_nodes"], s["lse"], s["scale"], s["mass"],
                              s["row_pos"], s["n_evicted"], decay=c["decay"])
        return {"mass": s["mass"], "row_pos": s["row_pos"]}
    B, Hkv, T1 = c["B"], c["Hkv"], c["T"] + 1
    nodes, live = _path_rows(s)
    lse = s["lse"][torch.arange(B, device=DEVICE)[:, None], nodes]                         # [B,T1,Hq]
    lse = torch.where(live[:, :, None], lse, 0.0).view(B, T1, Hkv, -1).permute(0, 2, 3, 1)
    w = _path_scores(s).sub_(lse[..., None]).exp_().sum((2, 3))                            # [B,Hkv,Lcap]
    j = torch.arange(w.shape[2], dtype=torch.int32, device=DEVICE)
    base, end = (s["kv_len"] - 1 - s["acc_len"])[:, None, None], s["kv_len"][:, None, None]
    mass = torch.where(j < base, s["mass"] * c["decay"] + w, torch.where(j < end, w, s["mass"]))
    pos = torch.where((j >= base) & (j < end), j + s["n_evicted"][:, None, None], s["row_pos"])
    s["mass"].copy_(mass)
    s["row_pos"].copy_(pos)
    return {"mass": s["mass"], "row_pos": s["row_pos"]}


def _evict(s):
    c = s["case"]
    budget = c["budget"]
    out = {"K": s["K"][:, :, :budget], "V": s["V"][:, :, :budget], "mass": s["out_mass"][:, :, :budget],
           "row_pos": s["out_row_pos"][:, :, :budget], "kv_len": s["out_kv_len"], "n_evicted": s["out_n_evicted"]}
    if own:
        s["h"].evict_rows(s["plan"], s["K"], s["V"], s["mass"], s["row_pos"], s["kv_len"], s["n_evicted"], budget,
                          c["sinks"], c["recent"], s["out_mass"], s["out_row_pos"], s["out_kv_len"], s["out_n_evicted"])
        return out
    Lcap = s["mass"].shape[2]
    j = torch.arange(Lcap, device=DEVICE)
    L, ev = s["kv_len"][:, None, None], s["n_evicted"][:, None, None]
    new = L.clamp(max=budget)
    kept_for_sure = (s["row_pos"] < c["sinks"]) | (s["row_pos"] >= ev + L - c["recent"])
    rank = torch.where(kept_for_sure, math.inf, s["mass"]).masked_fill(j >= L, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(2, order, j.expand_as(order).contiguous())
    kept = place < new                                                                     # [B,Hkv,Lcap]
    # the k-th kept row behind the new length fills the k-th dropped row before it
    holes = torch.where(~kept & (j < new), j, j + Lcap).argsort(dim=-1)
    movers = torch.where(kept & (j >= new), j, j + Lcap).argsort(dim=-1)
    count = (kept & (j >= new)).sum(-1, keepdim=True)
    src = j.expand_as(order).clone()
    src.scatter_(2, holes, torch.where(j < count, movers, holes))
    src = src[:, :, :budget]
    rows = src[..., None].expand(-1, -1, -1, c["D"])
    s["K"][:, :, :budget] = s["K"].gather(2, rows)
    s["V"][:, :, :budget] = s["V"].gather(2, rows)
    written = j[:budget] < new
    s["out_mass"][:, :, :budget] = torch.where(written, s["mass"].gather(2, src), s["out_mass"][:, :, :budget])
    s["out_row_pos"][:, :, :budget] = torch.where(written, s["row_pos"].gather(2, src), s["out_row_pos"][:, :, :budget])
    s["out_kv_len"].copy_(new.view(-1))
    s["out_n_evicted"].copy_((ev + L - new).view(-1))
    return out


# ---- the definitions in 64 bits -----------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = dict(case)
    if c["op"] == "attention":
        return _exact_attention(c, s)
    if c["op"] == "mass":
        return _exact_mass(c, s)
    return _exact_evict(c, s)


def _exact_attention(c, s):
    B, n, Hq, Hkv, D = c["B"], c["nodes"], c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    O = torch.zeros(B, n, Hq, D, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, n, Hq), -math.inf, dtype=torch.float64, device=DEVICE)
    words = s["mask"].cpu().numpy().view(np.uint64)
    ns, pre, kv = s["n_nodes"].tolist(), s["prefix_len"].tolist(), s["kv_len"].tolist()
    for b in range(B):
        m, p, L = ns[b], pre[b], kv[b]
        anc = np.unpackbits(words[b, :m].view(np.uint8), axis=1, bitorder="little")[:, :m].astype(bool)
        hidden = torch.from_numpy(~anc).to(DEVICE)
        for g in range(Hkv):
            q = s["Q"][b, :m, g * G:(g + 1) * G].double().reshape(m * G, D)
            k = torch.cat([s["Kp"][g, :p], s["K"][b, g, :L + m]]).double()
            v = torch.cat([s["Vp"][g, :p], s["V"][b, g, :L + m]]).double()
            x = (q @ k.t() * s["scale"]).view(m, G, -1)
            x[:, :, p + L:] = x[:, :, p + L:].masked_fill(hidden[:, None], -math.inf)
            O[b, :m, g * G:(g + 1) * G] = (torch.softmax(x, -1).view(m * G, -1) @ v).view(m, G, D)
            lse[b, :m, g * G:(g + 1) * G] = torch.logsumexp(x, -1)
    return {"O": O, "lse": lse}


def _exact_mass(c, s):
    B, Hkv = c["B"], c["Hkv"]
    G = c["Hq"] // Hkv
    mass, pos = s["mass"].double(), s["row_pos"].clone()
    acc, kv, path = s["acc_len"].tolist(), s["kv_len"].tolist(), s["acc_nodes"].tolist()
    for b in range(B):
        base = kv[b] - 1 - acc[b]
        q = s["Q"][b, [0] + path[b][:acc[b]]].double()                                     # [rows,Hq,D]
        lse = s["lse"][b, [0] + path[b][:acc[b]]].double()
        mass[b, :, :base] *= c["decay"]
        mass[b, :, base:kv[b]] = 0
        pos[b, :, base:kv[b]] = torch.arange(base, kv[b], dtype=torch.int32, device=DEVICE) + s["n_evicted"][b]
        for g in range(Hkv):
            k = s["K"][b, g, :kv[b]].double()
            for l in range(acc[b] + 1):
                x = q[l, g * G:(g + 1) * G] @ k[:base + l + 1].t() * s["scale"] - lse[l, g * G:(g + 1) * G, None]
                mass[b, g, :base + l + 1] += x.exp().sum(0)
    return {"mass": mass, "row_pos": pos}


def _exact_evict(c, s):
    """By sorting (kept for sure, weight, row) on the host; the copied values are the inputs' own."""
    B, Hkv, budget = c["B"], c["Hkv"], c["budget"]
    mass, pos = s["mass"].double().cpu().numpy(), s["row_pos"].cpu().numpy()
    kv, ev = s["kv_len"].tolist(), s["n_evicted"].tolist()
    src = np.tile(np.arange(budget), (B, Hkv, 1))
    out_mass, out_pos = np.zeros((B, Hkv, budget)), np.zeros((B, Hkv, budget), dtype=np.int32)
    for b in range(B):
        L, new = kv[b], min(kv[b], budget)
        for g in range(Hkv):
            sure = (pos[b, g, :L] < c["sinks"]) | (pos[b, g, :L] >= ev[b] + L - c["recent"])
            order = np.lexsort((np.arange(L), -mass[b, g, :L], ~sure))
            kept = np.zeros(L, dtype=bool)
            kept[order[:new]] = True
            free = np.nonzero(~kept[:new])[0]
            src[b, g, free] = new + np.nonzero(kept[new:])[0]
            out_mass[b, g, :new] = mass[b, g, src[b, g, :new]]
            out_pos[b, g, :new] = pos[b, g, src[b, g, :new]]
    rows = torch.from_numpy(src).to(DEVICE)[..., None].expand(-1, -1, -1, c["D"])
    return {"K": s["K"].gather(2, rows).double(), "V": s["V"].gather(2, rows).double(),
            "mass": torch.from_numpy(out_mass).to(DEVICE), "row_pos": torch.from_numpy(out_pos).to(DEVICE),
            "kv_len": torch.tensor([min(k, budget) for k in kv], dtype=torch.int32, device=DEVICE),
            "n_evicted": torch.tensor([e + k - min(k, budget) for e, k in zip(ev, kv)], dtype=torch.int32, device=DEVICE)}
