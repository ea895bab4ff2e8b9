"""Operators around a verification block's MoE layers, as measurable cases.

  norm     residual addition with the root-mean-square norm behind it, in the
           layer's type or in 8 bits with scales (`ops.residual_norm`)
  sample   a token per row of logits: temperature, top-k, top-p and min-p from
           given random numbers (`ops.sample`)
  accept   the accepted path of each draft tree, given the target's token at
           every node (`ops.accept`)
  q4       the grouped SwiGLU expert FFN with weights in 4 bits and group scales
           (`ops.moe_forward_q4`)

`run` computes them in plain torch operations, or with `own` set by the
package's own kernels.  Inputs come from the seed alone.

Fields of a case: "op" and

  norm     rows, hidden, dtype; add (whether there is an addend); group (0: output
           in `dtype`; else codes of 8 bits with one scale per `group` columns, -1:
           per row)
  sample   rows, vocab, dtype, spread (standard deviation of the bulk of the
           logits), greedy (share of rows with temperature 0), top_k, top_p,
           min_p (largest values drawn; 0 or 1: off), masked (share of tokens at
           minus infinity, as a grammar's mask leaves them)
  accept   trees, nodes, branch (most children of a node), hit (probability that
           a node's token is the target's)
  q4       tokens, hidden, inner, experts, top_k, eligible (experts the rows are
           routed within), idle (share of rows that are routed nowhere)
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
GROUP = 32  # columns per scale of a 4-bit weight


def listed():
    return [
        # one token between two layers: launches and latency
        {"name": "norm_decode_1", "op": "norm", "rows": 1, "hidden": 2048, "dtype": "bf16", "add": True, "group": 0},
        # a ragged block of an fp32 layer, width no power of two
        {"name": "norm_fp32_37", "op": "norm", "rows": 37, "hidden": 1100, "dtype": "f32", "add": True, "group": 0},
        # a full server's verification batch, handed on in 8 bits
        {"name": "norm_8bit_32x60", "op": "norm", "rows": 1920, "hidden": 2048, "dtype": "bf16", "add": True,
         "group": 128},
        # a long prompt's rows through the wide layer
        {"name": "norm_16384", "op": "norm", "rows": 16384, "hidden": 4096, "dtype": "bf16", "add": True, "group": 0},
        # plain decoding: one row of logits, all filters on
        {"name": "sample_decode_1", "op": "sample", "rows": 1, "vocab": 32000, "dtype": "f32", "spread": 2.0,
         "greedy": 0.0, "top_k": 64, "top_p": 0.95, "min_p": 0.02, "masked": 0.0},
        # every node of one draft tree, large vocabulary, top-p alone on the most part
        {"name": "sample_tree_64", "op": "sample", "rows": 64, "vocab": 131072, "dtype": "f32", "spread": 2.5,
         "greedy": 0.0, "top_k": 0, "top_p": 0.98, "min_p": 0.0, "masked": 0.0},
        # eight trees of 64 nodes with settings of their own, odd vocabulary, a grammar's mask
        {"name": "sample_batch_8x64", "op": "sample", "rows": 512, "vocab": 100003, "dtype": "bf16", "spread": 2.5,
         "greedy": 0.2, "top_k": 100, "top_p": 0.98, "min_p": 0.05, "masked": 0.3},
        # one request's draft tree
        {"name": "accept_tree_64", "op": "accept", "trees": 1, "nodes": 64, "branch": 4, "hit": 0.5},
        # a full server's trees
        {"name": "accept_32x60", "op": "accept", "trees": 32, "nodes": 60, "branch": 4, "hit": 0.6},
        # plain decoding through 4-bit experts
        {"name": "q4_decode_1", "op": "q4", "tokens": 1, "hidden": 2048, "inner": 768, "experts": 128, "top_k": 8,
         "eligible": 128, "idle": 0.0},
        # a draft tree on the wide layer, routed within the eligible set
        {"name": "q4_wide_64", "op": "q4", "tokens": 64, "hidden": 4096, "inner": 1536, "experts": 128, "top_k": 8,
         "eligible": 26, "idle": 0.0},
        # a full server: 32 trees of 60 nodes
        {"name": "q4_batch_32x60", "op": "q4", "tokens": 1920, "hidden": 2048, "inner": 768, "experts": 128,
         "top_k": 8, "eligible": 128, "idle": 0.0},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("norm", "sample", "accept", "q4"))
    if op == "norm":
        while True:
            group = rng.choice((0, 0, -1, 32, 64, 128))
            step = group if group > 0 else 4
            c = {"op": op, "rows": _log_uniform(rng, 1, 16384), "hidden": step * _log_uniform(rng, 256 // step, 8192 // step),
                 "dtype": rng.choice(("bf16", "bf16", "f32")), "add": rng.random() < 0.8, "group": group}
            if c["rows"] * c["hidden"] * (2 if c["dtype"] == "f32" else 1) <= 16384 * 4096:
                return c
    if op == "sample":
        while True:
            c = {"op": op, "rows": _log_uniform(rng, 1, 512), "vocab": _log_uniform(rng, 1000, 200000),
                 "dtype": rng.choice(("bf16", "f32")), "spread": round(rng.uniform(1.0, 4.0), 2),
                 "greedy": rng.choice((0.0, 0.3)), "top_k": rng.choice((0, 20, 100, 1000)),
                 "top_p": rng.choice((1.0, 0.9, 0.99)), "min_p": rng.choice((0.0, 0.0, 0.1)),
                 "masked": rng.choice((0.0, 0.5))}
            if c["rows"] * c["vocab"] <= 512 * 100003:
                return c
    if op == "accept":
        return {"op": op, "trees": _log_uniform(rng, 1, 32), "nodes": _log_uniform(rng, 1, 64),
                "branch": rng.randint(1, 6), "hit": round(rng.uniform(0.2, 0.9), 2)}
    while True:
        experts = _log_uniform(rng, 8, 256)
        c = {"op": op, "tokens": _log_uniform(rng, 1, 1920), "hidden": 32 * _log_uniform(rng, 8, 128),
             "inner": 32 * _log_uniform(rng, 4, 48), "experts": experts, "top_k": rng.randint(1, 8),
             "eligible": rng.randint(8, experts), "idle": rng.choice((0.0, 0.0, 0.2))}
        w = c["experts"] * c["hidden"] * c["inner"]
        if w <= 128 * 4096 * 1536 and w * c["tokens"] <= 128 * 2048 * 768 * 1920:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs_norm(case, gen):
    T, H = case["rows"], case["hidden"]
    # a residual stream grows with depth and has a few large channels
    channel = 1.0 + 20.0 * (torch.rand(H, generator=gen, device=DEVICE) < 0.004)
    hidden = torch.randn(T, H, generator=gen, device=DEVICE) * 2.0 * channel
    y = torch.randn(T, H, generator=gen, device=DEVICE) * 0.5
    weight = 1.0 + 0.3 * torch.randn(H, generator=gen, device=DEVICE)
    dt = _dtype(case)
    return {"hidden": hidden.to(dt), "y": y if case["add"] else None, "weight": weight.to(dt)}


def _inputs_sample(case, gen):
    R, V = case["rows"], case["vocab"]
    logits = torch.randn(R, V, generator=gen, device=DEVICE) * case["spread"]
    # a context favours a handful of tokens
    top = torch.randint(0, V, (R, 12), generator=gen, device=DEVICE)
    lift = 4.0 * case["spread"] + 4.0 * torch.rand(R, 12, generator=gen, device=DEVICE)
    logits.scatter_(1, top, lift)
    if case["masked"]:
        gone = torch.rand(R, V, generator=gen, device=DEVICE) < case["masked"]
        logits = torch.where(gone, -math.inf, logits)
    rand = lambda: torch.rand(R, generator=gen, device=DEVICE)  # noqa: E731
    temperature = torch.where(rand() < case["greedy"], 0.0, 0.5 + rand())
    k, p, m = case["top_k"], case["top_p"], case["min_p"]
    return {"logits": logits.to(_dtype(case)), "uniform": rand(), "temperature": temperature,
            "top_k": (1 + rand() * k).int() if k else None,
            "top_p": p - 0.2 * rand() if p < 1.0 else None,
            "min_p": m * rand() if m else None}


def _inputs_accept(case, seed):
    rng = np.random.default_rng(seed)
    parent, token, offsets, n = [], [], [0], case["nodes"]
    for _ in range(case["trees"]):
        first, par, head = offsets[-1], [-1], 0
        while len(par) < n:  # breadth-first, 1 .. branch children a node
            par += [head] * min(int(rng.integers(1, case["branch"] + 1)), n - len(par))
            head += 1
        parent += [p if p < 0 else p + first for p in par]
        token += [int(v) for v in rng.integers(0, 32000, n)]
        offsets.append(first + n)
    T = len(parent)
    target = rng.integers(0, 32000, T)
    for t in range(T):  # the target agrees with a node's draft token in a share `hit` of the nodes
        if parent[t] >= 0 and rng.random() < case["hit"]:
            target[parent[t]] = token[t]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEVICE)  # noqa: E731
    return {"token": dev(token), "parent": dev(parent), "target": dev(target), "offsets": offsets}


def _inputs_q4(case, gen):
    T, H, I, E, k = (case[f] for f in ("tokens", "hidden", "inner", "experts", "top_k"))
    # what quantising weights of N(0, 0.02^2) leaves: two codes a byte, scales of 2^-7 and 2^-6
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEVICE)
    w = torch.randn(2, 65536, generator=gen, device=DEVICE) * 2.2
    code = (w.abs()[..., None] - values).abs().argmin(-1) + 8 * (w < 0)
    pair = (code[0] + 16 * code[1]).to(torch.uint8)

    def stack(N, K):
        pick = torch.randint(0, 65536, (E, N, K // 2), generator=gen, device=DEVICE, dtype=torch.int32)
        scales = torch.randint(120, 122, (E, N, K // GROUP), generator=gen, device=DEVICE, dtype=torch.uint8)
        return pair[pick], scales

    experts = torch.randperm(E, generator=gen, device=DEVICE)[:case["eligible"]]
    # rows lean to the same experts, as the nodes of one tree do
    score = torch.randn(T, len(experts), generator=gen, device=DEVICE) + torch.randn(len(experts), generator=gen,
                                                                                   device=DEVICE)
    z, at = score.topk(k, dim=1)
    idx, gate = experts[at].int(), torch.softmax(z, dim=1)
    idle = torch.rand(T, 1, generator=gen, device=DEVICE) < case["idle"]
    return {"hidden": torch.randn(T, H, generator=gen, device=DEVICE).bfloat16(), "gate_w": stack(I, H),
            "up_w": stack(I, H), "down_w": stack(H, I), "idx": torch.where(idle, -1, idx).contiguous(),
            "gate": torch.where(idle, 0.0, gate).contiguous()}


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    if case["op"] == "accept":
        return _inputs_accept(case, seed)
    return {"norm": _inputs_norm, "sample": _inputs_sample, "q4": _inputs_q4}[case["op"]](case, gen)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2608_02989_amd import ops
        if case["op"] == "sample":  # scratch kept beside the logits buffer
            s["workspace"] = ops.sample_workspace(case["rows"], case["vocab"], DEVICE)
        if case["op"] == "q4":  # weights laid out once, scratch of the layer
            s["w_gate_up"] = ops.pack_gate_up_q4(*s["gate_w"], *s["up_w"])
            s["w_down"] = ops.pack_down_q4(*s["down_w"])
            s["workspace"] = ops.forward_q4_workspace(case["tokens"], case["hidden"], case["inner"], case["experts"],
                                                      case["top_k"], DEVICE)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if op == "norm":
        return run_norm(state)
    if op == "sample":
        return run_sample(state)
    return run_accept(state) if op == "accept" else run_q4(state)


def run_norm(s):
    group = s["case"]["group"]
    if own:
        from paper_2608_02989_amd import ops
        return ops.residual_norm(s["hidden"], s["y"], s["weight"], eps=EPS, group=group or None)
    h = s["hidden"].float()
    if s["y"] is not None:
        h = h + s["y"]
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    hidden = s["hidden"] if s["y"] is None else h.to(s["hidden"].dtype)
    if not group:
        return {"hidden": hidden, "norm": n.to(s["hidden"].dtype)}
    T, H = n.shape
    parts = n.view(T, 1 if group < 0 else H // group, -1)
    scale = parts.abs().amax(2) / 448.0
    value = torch.where(scale[..., None] > 0, parts / scale[..., None], 0.0).clamp(-448.0, 448.0)
    return {"hidden": hidden, "codes": value.view(T, H).to(torch.float8_e4m3fn), "scale": scale}


def run_sample(s):
    if own:
        from paper_2608_02989_amd import ops
        return ops.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                          min_p=s["min_p"], workspace=s["workspace"])
    z, order = torch.sort(s["logits"].float() + 0.0, dim=1, descending=True, stable=True)
    V = z.shape[1]
    rank = torch.arange(V, device=z.device)
    tau = s["temperature"].double()[:, None]
    z = z.double()
    w = torch.exp((z - z[:, :1]) / torch.where(tau > 0, tau, 1.0))
    w = torch.where((tau > 0) | (rank == 0), w, 0.0)
    if s["top_k"] is not None:
        w = torch.where(rank < s["top_k"][:, None], w, 0.0)
    cum = w.cumsum(1)
    keep = w > 0
    if s["top_p"] is not None:
        keep &= cum - w < s["top_p"].double()[:, None] * cum[:, -1:]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    last = keep.sum(1, keepdim=True) - 1
    total = cum.gather(1, last)
    at = (cum <= s["uniform"].double()[:, None] * total).sum(1, keepdim=True)
    at = torch.minimum(at, last)
    return {"token": order.gather(1, at)[:, 0].int(), "prob": (w.gather(1, at) / total)[:, 0].float()}


def run_accept(s):
    if own:
        from paper_2608_02989_amd import ops
        return ops.accept(s["token"], s["parent"], s["target"], s["offsets"])
    token, parent, target = s["token"], s["parent"].long(), s["target"]
    T, B = len(token), len(s["offsets"]) - 1
    bounds = torch.tensor(s["offsets"], device=token.device)
    node = torch.arange(T, device=token.device)
    tree = torch.searchsorted(bounds, node, right=True) - 1
    root = node == bounds[tree]
    fits = (parent >= 0) & (token == target[parent.clamp(min=0)])
    # of siblings with the same token the first counts
    earlier = (parent[:, None] == parent) & fits & (node < node[:, None])
    link = fits & ~earlier.any(1)
    # where following the links upwards ends: a node's own tree's root, or nowhere (state T)
    up = torch.where(root, node, torch.where(link, parent, T))
    step = torch.zeros(T + 1, T + 1, device=token.device)
    step[node, up] = 1.0
    step[T, T] = 1.0
    ends = torch.linalg.matrix_power(step, 1 << max(1, (T - 1).bit_length()))
    on_path = ends[node, bounds[tree]] > 0
    # nodes come behind their parents: a node's place on the path is the count before it
    before = torch.cumsum(on_path.int(), 0)
    place = before - 1 - torch.where(bounds[tree] > 0, before[(bounds[tree] - 1).clamp(min=0)], 0)
    length = torch.zeros(B, dtype=torch.int32, device=token.device).index_add_(0, tree, on_path.int())
    longest = max(b - a for a, b in zip(s["offsets"], s["offsets"][1:]))
    path = torch.full((B, longest + 1), -1, dtype=torch.int32, device=token.device)
    path[tree, torch.where(on_path, place, longest)] = torch.where(on_path, node, -1).int()
    path = path[:, :longest].contiguous()
    bonus = target[path.gather(1, (length - 1)[:, None].long())[:, 0].long()]
    return {"on_path": on_path.to(torch.uint8), "path": path, "length": length, "bonus": bonus}


def _dequantise(codes, scales):
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    values = torch.cat([values, -values])
    both = values[torch.stack((codes & 15, codes >> 4), dim=-1).int()]
    E, N, _ = codes.shape
    return (both.view(E, N, -1, GROUP) * torch.exp2(scales.float() - 127.0)[..., None]).view(E, N, -1)


def run_q4(s):
    if own:
        from paper_2608_02989_amd import ops
        return ops.moe_forward_q4(s["hidden"], s["w_gate_up"], s["w_down"], s["idx"], s["gate"],
                                  workspace=s["workspace"])
    x, E = s["hidden"].float(), s["gate_w"][0].shape[0]
    T = x.shape[0]
    # each row's gate for every expert (0: not routed there), then all experts as one matrix
    weight = torch.zeros(T, E + 1, device=x.device).scatter_add_(1, torch.where(s["idx"] < 0, E, s["idx"]).long(),
                                                                s["gate"])[:, :E]
    g = x @ _dequantise(*s["gate_w"]).flatten(0, 1).t()
    u = x @ _dequantise(*s["up_w"]).flatten(0, 1).t()
    act = (g / (1.0 + torch.exp(-g)) * u).view(T, E, -1) * weight[..., None]
    down = _dequantise(*s["down_w"]).transpose(1, 2).flatten(0, 1)
    return act.flatten(1) @ down


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "norm":
        n, eb = case["rows"] * case["hidden"], 2 if case["dtype"] == "bf16" else 4
        scales = 4 * (case["rows"] if case["group"] < 0 else n // case["group"]) if case["group"] else 0
        return {"bytes": n * (eb + (4 + eb if case["add"] else 0) + (1 if case["group"] else eb)) + scales
                + case["hidden"] * eb, "flops": 6 * n}
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + 28 * case["rows"], "flops": 4 * n}
    if op == "accept":
        T = case["trees"] * case["nodes"]
        return {"bytes": 13 * T + 4 * T + 8 * case["trees"], "flops": 2 * T}
    slots = case["tokens"] * case["top_k"] * (1.0 - case["idle"])
    expert = 3 * case["hidden"] * case["inner"]
    touched = min(case["eligible"], slots)  # experts that get a row, at most
    return {"bytes": int(touched * expert * (1 / 2 + 1 / GROUP) + case["tokens"] * (6 * case["hidden"] + 8 * case["top_k"])),
            "flops": int(2 * slots * expert)}


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    if case["op"] == "sample":
        return _exact_sample(s)
    return _exact_accept(s) if case["op"] == "accept" else _exact_q4(s)


def _exact_norm(case, s):
    h = s["hidden"].double() if s["y"] is None else s["hidden"].double() + s["y"].double()
    size = torch.sqrt(h.square().sum(1) / h.shape[1] + EPS)
    n = h / size[:, None] * s["weight"].double()
    if not case["group"]:
        return {"hidden": h, "norm": n}
    width = n.shape[1] if case["group"] < 0 else case["group"]
    largest = n.abs().unfold(1, width, width).amax(-1)
    return {"hidden": h, "codes": n * 448.0 / largest.repeat_interleave(width, 1), "scale": largest / 448.0}


def _exact_sample(s):
    get = lambda f: None if s[f] is None else s[f].double().cpu().numpy()  # noqa: E731
    z, u, tau, k, p, m = (get(f) for f in ("logits", "uniform", "temperature", "top_k", "top_p", "min_p"))
    token, prob = np.zeros(len(z), np.int32), np.zeros(len(z))
    for r in range(len(z)):
        if tau[r] == 0:
            token[r], prob[r] = z[r].argmax(), 1.0
            continue
        live = np.flatnonzero(z[r] > z[r].max() - 60.0 * tau[r])  # exp(-60): nothing beside 64 bits of a sum
        order = live[np.argsort(-z[r][live], kind="stable")]
        w = np.exp((z[r][order] - z[r][order[0]]) / tau[r])
        if k is not None:
            order, w = order[:int(k[r])], w[:int(k[r])]
        c = np.cumsum(w)
        n = len(w) if p is None else 1 + np.searchsorted(c, p[r] * c[-1], side="left")
        n = max(1, min(n, len(w)))
        if m is not None:
            n = min(n, int((w >= m[r]).sum()))
        j = min(int(np.searchsorted(c[:n], u[r] * c[n - 1], side="right")), n - 1)
        token[r], prob[r] = order[j], w[j] / c[n - 1]
    return {"token": torch.from_numpy(token), "prob": torch.from_numpy(prob)}


def _exact_accept(s):
    token, parent, target = (s[f].tolist() for f in ("token", "parent", "target"))
    offs = s["offsets"]
    longest = max(b - a for a, b in zip(offs, offs[1:]))
    on, path, length, bonus = [0] * len(token), [], [], []
    for a, b in zip(offs, offs[1:]):
        walk = [a]
        while True:
            nxt = [t for t in range(walk[-1] + 1, b) if parent[t] == walk[-1] and token[t] == target[walk[-1]]]
            if not nxt:
                break
            walk.append(nxt[0])
        for t in walk:
            on[t] = 1
        path.append(walk + [-1] * (longest - len(walk)))
        length.append(len(walk))
        bonus.append(target[walk[-1]])
    whole = lambda a, t: torch.tensor(a, dtype=t)  # noqa: E731
    return {"on_path": whole(on, torch.uint8), "path": whole(path, torch.int32), "length": whole(length, torch.int32),
            "bonus": whole(bonus, torch.int32)}


def _exact_q4(s):
    def matrix(pair, e):
        codes, scales = pair[0][e].long(), pair[1][e].long()
        q = torch.stack((codes % 16, codes // 16), -1).flatten(1)
        sign, ex, mant = 1 - 2 * (q // 8), q // 2 % 4, q % 2
        value = torch.where(ex == 0, 0.5 * mant, (1.0 + 0.5 * mant) * 2.0 ** (ex - 1).double())
        return sign * value.double() * torch.exp2((scales - 127).double()).repeat_interleave(GROUP, 1)

    x = s["hidden"].double()
    out = torch.zeros_like(x)
    for e in sorted(set(s["idx"].flatten().tolist()) - {-1}):
        t, j = torch.nonzero(s["idx"] == e, as_tuple=True)
        g = x[t] @ matrix(s["gate_w"], e).t()
        a = g * torch.sigmoid(g) * (x[t] @ matrix(s["up_w"], e).t())
        out.index_add_(0, t, (a @ matrix(s["down_w"], e).t()) * s["gate"][t, j].double()[:, None])
    return out
