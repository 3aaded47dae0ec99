"""The gated delta rule layer and the norm of its queries and keys, as measurable cases.

Three operators that are used one behind another in a layer of a drafter: the norm of every query and key head, with the
position rotation in the same pass ("norm"); the context encode of the gated delta rule over packed sequences ("encode"); and
its one-token step over the nodes of draft trees, each from its parent's state ("step").  Shapes go by the 130M drafter of this
repository (1536 channels = 12 heads of 128 values), its contexts (one sequence of 2048 or 32768 tokens, 32 packed ones of 1k to
8k), its trees (15, 150 and 32 x 32 nodes) and its tiny fp32 configuration.

The plain forms are written in elementary torch operations, in 32 bits (angles and running sums of log decays in 64).  The
recurrence over tokens is taken in chunks of 64, which leaves one loop over the chunks and one over the rows of a chunk.
"""

from __future__ import annotations

import math
import random

import torch

own = False   # whether run() calls the package's operators

Q = 64                   # tokens per chunk of the plain encode
DT_BIAS = -4.579712      # softplus(bias + 0.5 N(0, 1)) stays inside [1e-3, 1e-1]
DT_CLIP = 2.3125
LARGEST_ENCODE = 32 * 4608 * 12 * 128 * 128   # tokens x heads x entries of a state
LARGEST_STEP = 1024 * 12 * 128 * 128          # nodes x heads x entries of a state
LARGEST_NORM = 141000 * 16 * 128              # rows x heads x values
EPS = 1e-5


def listed():
    return [
        # One level of a draft tree on its way into a delta layer: q and k of 18 nodes brought to unit length.
        {"name": "norm 18 nodes", "kind": "norm", "rows": 18, "q_heads": 12, "k_heads": 12, "d": 128, "act": "bf16", "norm": "l2",
         "weights": False, "rot": 0, "layout": "half", "first": 0, "tree": False},
        # A context of 2048 tokens on its way into an attention layer: RMS norm with weights, the whole head rotated by halves.
        {"name": "norm rotate 2k", "kind": "norm", "rows": 2048, "q_heads": 12, "k_heads": 4, "d": 128, "act": "bf16", "norm": "rms",
         "weights": True, "rot": 128, "layout": "half", "first": 0, "tree": False},
        # The packed batch (141k tokens), small heads, half of each rotated in neighbouring pairs, at positions far into a long context.
        {"name": "norm rotate 141k far", "kind": "norm", "rows": 141000, "q_heads": 12, "k_heads": 4, "d": 64, "act": "bf16",
         "norm": "rms", "weights": True, "rot": 32, "layout": "pairs", "first": 1000003, "tree": False},
        # fp32 and odd: 777 rows of 6 + 3 heads of 96 values, no norm, rotation only.
        {"name": "norm fp32 odd", "kind": "norm", "rows": 777, "q_heads": 6, "k_heads": 3, "d": 96, "act": "f32", "norm": "none",
         "weights": False, "rot": 48, "layout": "half", "first": 77, "tree": True},
        # Context encode of one layer, the benchmark's own context length; gate and output norm inside.
        {"name": "encode 2k", "kind": "encode", "k_heads": 12, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 1,
         "lo": 2048, "hi": 2048, "lens_seed": 0, "init": False, "gate": True, "norm": True},
        # The long context, key heads shared by three value heads each, no output norm.
        {"name": "encode 32k shared keys", "kind": "encode", "k_heads": 4, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 1,
         "lo": 32768, "hi": 32768, "lens_seed": 0, "init": False, "gate": True, "norm": False},
        # The batched configuration: 32 packed sequences of 1k to 8k tokens.
        {"name": "encode packed 32", "kind": "encode", "k_heads": 12, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 32,
         "lo": 1024, "hi": 8192, "lens_seed": 0, "init": False, "gate": True, "norm": True},
        # Catching up with what verification accepted: eight sequences of 1 to 9 tokens, each from its slot.
        {"name": "encode accepted 8", "kind": "encode", "k_heads": 12, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 8,
         "lo": 1, "hi": 9, "lens_seed": 0, "init": True, "gate": True, "norm": True},
        # fp32, small heads, three ragged sequences from slots, nothing behind the rule.
        {"name": "encode fp32 ragged", "kind": "encode", "k_heads": 3, "v_heads": 6, "dk": 64, "dv": 64, "act": "f32", "n_seq": 3,
         "lo": 100, "hi": 500, "lens_seed": 1, "init": True, "gate": False, "norm": False},
        # Chain decoding at batch 1: a single node.
        {"name": "step 1 node", "kind": "step", "k_heads": 12, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 1,
         "branching": "", "cap": 0, "nodes": 0, "tree_seed": 0, "gate": True, "norm": True},
        # The 150-node round (6 levels in one call).
        {"name": "step round 150", "kind": "step", "k_heads": 12, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 1,
         "branching": "4,4,2,2,2", "cap": 150, "nodes": 0, "tree_seed": 0, "gate": True, "norm": True},
        # The batched configuration's round: a random 32-node tree below each of 32 sequences, shared key heads.
        {"name": "step round 32 x 32", "kind": "step", "k_heads": 4, "v_heads": 12, "dk": 128, "dv": 128, "act": "bf16", "n_seq": 32,
         "branching": "", "cap": 0, "nodes": 32, "tree_seed": 0, "gate": True, "norm": False},
    ]


# ---------------------------------------------------------------- more cases of the same ranges
def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _branching(rng):
    """Branching factors of a tree of at most 150 nodes."""
    while True:
        b = [rng.randint(1, 4) for _ in range(rng.randint(1, 6))]
        n, w = 1, 1
        for f in b:
            w *= f
            n += w
        if n <= 150:
            return ",".join(str(f) for f in b)


def draw(rng):
    kind = rng.choice(["norm", "encode", "encode", "step", "step"])
    act = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "norm":
        d = rng.choice([32, 64, 80, 96, 128, 192, 256])
        layout = rng.choice(["half", "pairs"])
        rot = 16 * rng.randint(0, d // 16) if layout == "half" else 2 * rng.randint(0, d // 2)
        k = rng.randint(1, 8)
        c = {"kind": kind, "rows": _log(rng, 1, 141000), "q_heads": k * rng.randint(1, 4), "k_heads": k, "d": d, "act": act,
             "norm": rng.choice(["none", "l2", "rms"]), "weights": rng.random() < 0.5, "rot": rot, "layout": layout,
             "first": rng.choice([0, rng.randrange(5000), rng.randrange(4000000)]), "tree": rng.random() < 0.5}
        while c["rows"] * (c["q_heads"] + c["k_heads"]) * d * (2 if act == "f32" else 1) > LARGEST_NORM:
            c["rows"] = max(1, c["rows"] * 2 // 3)
        return c
    k = rng.randint(1, 8)
    c = {"kind": kind, "k_heads": k, "v_heads": k * rng.randint(1, 4), "dk": rng.choice([64, 128, 128]), "dv": rng.choice([64, 128, 128]),
         "act": act, "n_seq": _log(rng, 1, 32), "gate": rng.random() < 0.7, "norm": rng.random() < 0.5}
    state = c["v_heads"] * c["dk"] * c["dv"]
    if kind == "encode":
        c.update(hi=_log(rng, 1, 32768), lens_seed=rng.randrange(1000), init=rng.random() < 0.4)
        if act == "f32":   # the encode of a small fp32 drafter
            c["hi"] = min(c["hi"], 1024)
        while c["n_seq"] * c["hi"] * state > LARGEST_ENCODE // 2:
            c["hi"] = c["hi"] * 2 // 3
        c["lo"] = max(1, c["hi"] // rng.randint(1, 4))
        return c
    if rng.random() < 0.5:
        c.update(n_seq=1, branching=_branching(rng), cap=0, nodes=0, tree_seed=0)
    else:
        c.update(branching="", cap=0, nodes=rng.choice([0, rng.randint(2, 40)]), tree_seed=rng.randrange(1000))
        while c["n_seq"] * max(1, c["nodes"]) * state > LARGEST_STEP:
            c["n_seq"] = max(1, c["n_seq"] * 2 // 3)
    return c


# ---------------------------------------------------------------- what a case's sizes mean
def _lens(c):
    r = random.Random(c["lens_seed"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["n_seq"])]


def _one_tree(c, rng):
    """Lists of parents per level, breadth first: fixed branching factors (the deepest level cut to `cap` nodes in all), or `nodes`
    nodes on at most 5 levels with 1 to 3 children each, or a single node."""
    levels, first = [[-1]], 0
    if c["branching"]:
        for f in (int(v) for v in c["branching"].split(",")):
            prev = levels[-1]
            levels.append([first + j for j in range(len(prev)) for _ in range(f)])
            first += len(prev)
        total = sum(len(v) for v in levels)
        if c["cap"] and total > c["cap"]:
            levels[-1] = sorted(rng.sample(levels[-1], len(levels[-1]) - (total - c["cap"])))
        return levels
    total = 1
    for l in range(4):
        prev, left = levels[-1], c["nodes"] - total
        nxt = [first + j for j in range(len(prev)) for _ in range(rng.randint(1, 3))]
        if l == 3 and len(nxt) < left:
            nxt = sorted(nxt + [first + rng.randrange(len(prev)) for _ in range(left - len(nxt))])
        first += len(prev)
        nxt = nxt[:max(left, 0)]
        if not nxt:
            break
        levels.append(nxt)
        total += len(nxt)
    return levels


def _trees(c):
    """All sequences' trees merged level by level: (sequence, parent's index or -1) of every node, and the level offsets."""
    rng = random.Random(c["tree_seed"])
    trees = [_one_tree(c, rng) for _ in range(c["n_seq"])]
    nodes, off, index = [], [0], {}
    for l in range(max(len(t) for t in trees)):
        for s, t in enumerate(trees):
            if l >= len(t):
                continue
            base = sum(len(v) for v in t[:l])
            for j, p in enumerate(t[l]):
                index[s, base + j] = len(nodes)
                nodes.append((s, -1 if p < 0 else index[s, p]))
        off.append(len(nodes))
    return nodes, off


# ---------------------------------------------------------------- inputs
def _act(c):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[c["act"]]


def _normal(g, shape, scale=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g).mul_(scale)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"norm": _prepare_norm, "encode": _prepare_encode, "step": _prepare_step}[case["kind"]](case, g)


def _prepare_norm(c, g):
    """q and k are column ranges of one projection output, next to v's channels; one position per row."""
    n, d, hq, hk, act = c["rows"], c["d"], c["q_heads"], c["k_heads"], _act(c)
    u = _normal(g, (n, (hq + 2 * hk) * d), 2.0).to(act)
    if c["tree"]:   # positions of tree nodes: the level below the context's end, in no special order
        pos = c["first"] + torch.randint(0, 8, (n,), generator=g, device="cuda")
    else:
        pos = c["first"] + torch.arange(n, device="cuda")
    freqs = None
    if c["rot"]:
        freqs = (10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])).float()
    w = [1.0 + 0.2 * _normal(g, (d,)) if c["weights"] and c["norm"] != "none" else None for _ in range(2)]
    s = {"case": c, "q": u[:, :hq * d], "k": u[:, hq * d:(hq + hk) * d], "pos": pos.to(torch.int32), "freqs": freqs, "q_w": w[0], "k_w": w[1],
         "rot_scale": 1.0 if c["first"] < 100000 else 1.1}   # long contexts come with a scale on the rotation
    if own:   # the description that a program keeps
        import paper_2506_01206_b200 as md
        s["spec"] = md.QkNorm(d, hq, hk, act, {"none": md.MDRAFT_NORM_NONE, "l2": md.MDRAFT_NORM_L2, "rms": md.MDRAFT_NORM_RMS}[c["norm"]],
                              q_w=w[0], k_w=w[1], eps=EPS, rot_dim=c["rot"],
                              rot_layout=md.MDRAFT_ROT_HALF if c["layout"] == "half" else md.MDRAFT_ROT_PAIRS, freqs=freqs,
                              rot_scale=s["rot_scale"])
        s["q_out"], s["k_out"] = (torch.empty((n, h * d), dtype=act, device="cuda") for h in (hq, hk))
    return s


def _prepare_rule(c, g, rows, slots):
    """Constants and activations of a delta layer: keys and queries of unit length, q | k | v side by side as the conv leaves them."""
    hk, hv, dk, dv, act = c["k_heads"], c["v_heads"], c["dk"], c["dv"], _act(c)
    u = _normal(g, (rows, 2 * hk * dk + hv * dv))
    qk = u[:, :2 * hk * dk].view(rows, 2 * hk, dk)
    qk.mul_(torch.rsqrt(qk.square().sum(-1, keepdim=True) + 1e-6))
    u = u.to(act)
    A = -(1.0 + 15.0 * torch.rand((hv,), generator=g, device="cuda"))
    s = {"case": c, "q": u[:, :hk * dk], "k": u[:, hk * dk:2 * hk * dk], "v": u[:, 2 * hk * dk:],
         "z": _normal(g, (rows, hv * dv)).to(act) if c["gate"] else None,
         "dt": _normal(g, (rows, hv), 0.5).clamp_(-DT_CLIP, DT_CLIP).to(act), "b": _normal(g, (rows, hv)).to(act),
         "A": A, "dt_bias": torch.full((hv,), DT_BIAS, device="cuda"),
         "norm_w": 1.0 + 0.2 * _normal(g, (dv,)) if c["norm"] else None, "scale": dk ** -0.5}
    if own:   # the layer and the state pool that a program keeps
        import paper_2506_01206_b200 as md
        s["layer"] = md.GdrLayer(A, s["dt_bias"], s["norm_w"], hk, dk, dv, act, md.MDRAFT_DT_SOFTPLUS | md.MDRAFT_BETA_SIGMOID, s["scale"], EPS)
        s["cache"] = md.StateCache(1, slots, hv * dv, d_state=dk, act=act)
        s["ssm"] = s["cache"].ssm[0]
        s["out"] = torch.zeros((rows, hv * dv), dtype=act, device="cuda")
        s["status"] = _i32([0])
    else:
        s["ssm"] = torch.zeros((slots, hv * dv, dk), device="cuda")
    return s


def _prepare_encode(c, g):
    lens = _lens(c)
    n, cu = len(lens), [0]
    for v in lens:
        cu.append(cu[-1] + v)
    s = _prepare_rule(c, g, cu[-1], 2 * n)   # slots 0 .. n-1 start the sequences, the others take their final states
    if c["init"]:
        s["ssm"][:n] = _normal(g, s["ssm"][:n].shape, 0.1)
    s.update(lens=lens, cu=_i32(cu) if n > 1 else None, longest=max(lens), init=_i32(list(range(n))) if c["init"] else None,
             final=_i32(list(range(n, 2 * n))))
    if own:
        import paper_2506_01206_b200 as md
        s["ws"] = torch.empty(max(256, md.mdraft_gdr_prefill_workspace_bytes(s["layer"], cu[-1], n, s["longest"])), dtype=torch.uint8, device="cuda")
    return s


def _prepare_step(c, g):
    nodes, off = _trees(c)
    n, m = c["n_seq"], len(nodes)
    s = _prepare_rule(c, g, m, n + m)   # slots 0 .. n-1: the sequences' committed states; n + i: node i
    s["ssm"][:n] = _normal(g, s["ssm"][:n].shape, 0.1)
    parent = [q if p < 0 else n + p for q, p in nodes]
    s.update(levels=off, parent=_i32(parent), node=_i32(list(range(n, n + m))), parents_host=parent)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2506_01206_b200 as md
        if kind == "norm":
            md.mdraft_qk_norm(s["spec"], s["q"], s["k"], s["q_out"], s["k_out"], s["pos"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if kind == "encode":
            n = s["case"]["n_seq"]
            md.mdraft_gdr_prefill(s["layer"], s["cache"], 0, s["q"], s["k"], s["v"], s["z"], s["dt"], s["b"], s["out"], s["cu"], s["longest"],
                                  s["init"], s["final"], s["ws"], s["status"])
            return {"out": s["out"], "states": s["ssm"][n:]}
        md.mdraft_gdr_tree_step(s["layer"], s["cache"], 0, s["q"], s["k"], s["v"], s["z"], s["dt"], s["b"], s["out"], s["parent"], s["node"],
                                s["levels"], s["status"])
        return {"out": s["out"], "states": s["ssm"][s["case"]["n_seq"]:]}
    return {"norm": _plain_norm, "encode": _plain_encode, "step": _plain_step}[kind](s)


def _plain_norm(s):
    c, d, r = s["case"], s["case"]["d"], s["case"]["rot"]

    def one(x, w):
        y = x.float().reshape(x.shape[0], -1, d)
        if c["norm"] != "none":
            y2 = y.square()
            y = y * torch.rsqrt((y2.sum(-1, keepdim=True) if c["norm"] == "l2" else y2.mean(-1, keepdim=True)) + EPS)
            y = y if w is None else y * w
        if r:
            angle = s["pos"].double()[:, None] * s["freqs"].double()   # positions of a million times a frequency need more than 32 bits
            cos, sin = ((f(angle) * s["rot_scale"]).float()[:, None] for f in (torch.cos, torch.sin))
            a, b = (y[..., :r // 2], y[..., r // 2:r]) if c["layout"] == "half" else (y[..., 0:r:2], y[..., 1:r:2])
            a, b = a * cos - b * sin, b * cos + a * sin
            turned = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
            y = torch.cat([turned, y[..., r:]], -1)
        return y.reshape(x.shape).to(x.dtype)

    return {"q": one(s["q"], s["q_w"]), "k": one(s["k"], s["k_w"])}


def _gates(s):
    """(log of the decay, beta) of every row and head."""
    delta = torch.log1p(torch.exp(s["dt"].float() + s["dt_bias"]))
    return delta * s["A"], torch.sigmoid(s["b"].float())


def _behind(s, o):
    """Output norm and gate of rows of heads (rows, heads, dv), rounded to the activation type."""
    if s["norm_w"] is not None:
        o = o * torch.rsqrt(o.square().mean(-1, keepdim=True) + EPS) * s["norm_w"]
    o = o.reshape(o.shape[0], -1)
    if s["z"] is not None:
        z = s["z"].float()
        o = o * (z * torch.sigmoid(z))
    return o.to(s["v"].dtype)


def _plain_encode(s):
    c = s["case"]
    hk, hv, dk, dv, lens = c["k_heads"], c["v_heads"], c["dk"], c["dv"], s["lens"]
    n, dev = len(lens), s["v"].device
    chunks = -(-max(lens) // Q)
    length = torch.tensor(lens, device=dev)
    first = torch.cumsum(length, 0) - length
    t = torch.arange(chunks * Q, device=dev)
    there = t[None] < length[:, None]                                   # (sequence, padded token)
    row = torch.where(there, first[:, None] + t, 0)
    g, beta = _gates(s)

    def padded(x, heads):   # (sequence, head, chunk, token, value), zeros behind a sequence's end
        x = x.float().reshape(x.shape[0], heads, -1)[row] * there[..., None, None]
        x = x.permute(0, 2, 1, 3).reshape(n, heads, chunks, Q, -1)
        return x if heads == hv else x.repeat_interleave(hv // heads, 1)

    q, k, v = padded(s["q"], hk), padded(s["k"], hk), padded(s["v"], hv)
    g, beta = padded(g, hv)[..., 0], padded(beta, hv)[..., 0]
    G = torch.cumsum(g.double(), -1)
    upto = torch.ones((Q, Q), dtype=torch.bool, device=dev).tril()
    decay = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~upto, -math.inf)).float()
    eG, rest = torch.exp(G).float(), torch.exp(G[..., -1:] - G).float()
    A = (beta[..., None] * (k @ k.transpose(-1, -2)) * decay).tril(-1)
    T = torch.eye(Q, device=dev).expand_as(A).contiguous()               # (1 + A)^-1, row by row
    for i in range(1, Q):
        T[..., i, :i] = -(A[..., i, None, :i] @ T[..., :i, :i])[..., 0, :]
    T = T * beta[..., None, :]
    M = (q @ k.transpose(-1, -2)) * decay
    S = torch.zeros((n, hv, dk, dv), device=dev) if s["init"] is None else s["ssm"][s["init"].long()].view(n, hv, dv, dk).transpose(-1, -2)
    o = torch.empty_like(v)
    for i in range(chunks):
        x = T[:, :, i] @ (v[:, :, i] - eG[:, :, i, :, None] * (k[:, :, i] @ S))
        o[:, :, i] = eG[:, :, i, :, None] * (q[:, :, i] @ S) + M[:, :, i] @ x
        S = eG[:, :, i, -1, None, None] * S + k[:, :, i].transpose(-1, -2) @ (rest[:, :, i, :, None] * x)
    o = o.reshape(n, hv, chunks * Q, dv).transpose(1, 2)[there] * s["scale"]
    states = S.transpose(-1, -2).reshape(n, hv * dv, dk)
    s["ssm"][s["final"].long()] = states
    return {"out": _behind(s, o), "states": s["ssm"][n:]}


def _plain_step(s):
    c = s["case"]
    hk, hv, dk, dv = c["k_heads"], c["v_heads"], c["dk"], c["dv"]
    m = s["v"].shape[0]
    g, beta = _gates(s)
    q, k = (s[x].float().view(m, hk, dk).repeat_interleave(hv // hk, 1) for x in ("q", "k"))
    v = s["v"].float().view(m, hv, dv)
    pool = s["ssm"].view(-1, hv, dv, dk)
    o = torch.empty_like(v)
    for a, b in zip(s["levels"][:-1], s["levels"][1:]):   # a level's parents are in the levels before it
        S = torch.exp(g[a:b])[..., None, None] * pool[s["parent"][a:b].long()]
        r = beta[a:b, :, None] * (v[a:b] - (S @ k[a:b, ..., None])[..., 0])
        S = S + r[..., None] * k[a:b, :, None]
        o[a:b] = (S @ q[a:b, ..., None])[..., 0]
        pool[s["node"][a:b].long()] = S
    return {"out": _behind(s, o * s["scale"]), "states": s["ssm"][c["n_seq"]:]}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c, es = case, 4 if case["act"] == "f32" else 2
    if c["kind"] == "norm":
        values = c["rows"] * (c["q_heads"] + c["k_heads"]) * c["d"]
        return {"bytes": 2 * values * es + c["rows"] * 4, "flops": 8 * values}
    hk, hv, dk, dv = c["k_heads"], c["v_heads"], c["dk"], c["dv"]
    row = (2 * hk * dk + (3 if c["gate"] else 2) * hv * dv + 2 * hv) * es   # q, k, v, out, the gates
    if c["kind"] == "encode":
        tokens = sum(_lens(c))
        chunk = min(Q, c["hi"])
        return {"bytes": tokens * row + (2 if c["init"] else 1) * c["n_seq"] * hv * dk * dv * 4,
                "flops": tokens * hv * 2 * (chunk * (dk + dv) + 3 * dk * dv)}   # triangles of a chunk count half
    nodes, _ = _trees(c)
    read = len(set(nodes[i][0] if nodes[i][1] < 0 else (-1, nodes[i][1]) for i in range(len(nodes))))   # states that some node forks
    return {"bytes": len(nodes) * row + (len(nodes) + read) * hv * dk * dv * 4, "flops": len(nodes) * hv * dk * dv * 7}


# ---------------------------------------------------------------- the same from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(case, s)
    return _exact_encode(case, s) if case["kind"] == "encode" else _exact_step(case, s)


def _exact_norm(c, s):
    n, d, r = c["rows"], c["d"], c["rot"]
    out = {}
    for name in ("q", "k"):
        x = s[name].double().reshape(n, -1, d)
        if c["norm"] != "none":
            size = (x * x).sum(-1, keepdim=True) / (1 if c["norm"] == "l2" else d)
            x = x / torch.sqrt(size + EPS)
            if s[name + "_w"] is not None:
                x = x * s[name + "_w"].double()
        if r:   # pairs of values as complex numbers, turned
            i = torch.arange(r // 2, device=x.device)
            lo, hi = (i, i + r // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            turn = torch.polar(torch.full((n, 1, r // 2), float(s["rot_scale"]), dtype=torch.float64, device=x.device),
                               (s["pos"].double()[:, None] * s["freqs"].double()[None])[:, None])
            p = torch.complex(x[..., lo], x[..., hi]) * turn
            x = x.clone()
            x[..., lo], x[..., hi] = p.real, p.imag
        out[name] = x.reshape(n, -1)
    return out


def _token(s, c, rows, S):
    """One token of the rule for the given rows from states S (rows, heads, dv, dk): (outputs before norm and gate, states)."""
    hk, hv, dk, dv = c["k_heads"], c["v_heads"], c["dk"], c["dv"]
    of_key = torch.arange(hv, device=S.device) // (hv // hk)
    q, k = (s[x][rows].double().reshape(-1, hk, dk)[:, of_key] for x in ("q", "k"))
    v = s["v"][rows].double().reshape(-1, hv, dv)
    alpha = torch.exp(s["A"].double() * torch.log(1 + torch.exp(s["dt"][rows].double() + s["dt_bias"].double())))[..., None, None]
    beta = 1 / (1 + torch.exp(-s["b"][rows].double()))
    held = torch.einsum("nhvk,nhk->nhv", S, k)
    new = beta[..., None] * (v - alpha[..., 0] * held)
    S = alpha * S + torch.einsum("nhv,nhk->nhvk", new, k)
    return torch.einsum("nhvk,nhk->nhv", S, q) * s["scale"], S


def _exact_behind(s, o):
    if s["norm_w"] is not None:
        o = s["norm_w"].double() * o / torch.sqrt((o * o).mean(-1, keepdim=True) + EPS)
    o = o.reshape(o.shape[0], -1)
    return o if s["z"] is None else o * s["z"].double() / (1 + torch.exp(-s["z"].double()))


def _exact_encode(c, s):
    hv, dk, dv, lens = c["v_heads"], c["dk"], c["dv"], s["lens"]
    dev = s["v"].device
    order = sorted(range(len(lens)), key=lambda i: -lens[i])   # longest first: those still running are a prefix
    start = [sum(lens[:i]) for i in order]
    S = torch.zeros((len(lens), hv, dv, dk), dtype=torch.float64, device=dev)
    if s["init"] is not None:
        S = s["ssm"][:len(lens)].double().view(-1, hv, dv, dk)[order].clone()
    base = torch.tensor(start, device=dev)
    o = torch.zeros((sum(lens), hv, dv), dtype=torch.float64, device=dev)
    running = len(lens)
    for t in range(max(lens)):
        while lens[order[running - 1]] <= t:
            running -= 1
        rows = base[:running] + t
        o[rows], S[:running] = _token(s, c, rows, S[:running])
    states = torch.empty_like(S)
    states[order] = S
    return {"out": _exact_behind(s, o), "states": states.reshape(len(lens), hv * dv, dk)}


def _exact_step(c, s):
    hv, dk, dv, n = c["v_heads"], c["dk"], c["dv"], c["n_seq"]
    pool = s["ssm"].double().view(-1, hv, dv, dk)
    outs = []
    for a, b in zip(s["levels"][:-1], s["levels"][1:]):
        rows = torch.arange(a, b, device=pool.device)
        y, pool[n + rows] = _token(s, c, rows, pool[torch.tensor(s["parents_host"][a:b], device=pool.device)])
        outs.append(y)
    return {"out": _exact_behind(s, torch.cat(outs)), "states": pool[n:].reshape(-1, hv * dv, dk)}
