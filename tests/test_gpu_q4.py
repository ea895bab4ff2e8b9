"""Experts with weights in 4 bits on the GPU: quantisation bit for bit, the forward
against the fp64 oracle with a bound per element, the layer and a whole pass."""
import numpy as np
import pytest
import torch

from oracle import acceptmoe_oracle as O
from oracle import around_oracle as A
from paper_2608_02989_amd import ops
from paper_2608_02989_amd import workload as W

from _util import GATE_RTOL

pytestmark = pytest.mark.gpu
DEV = "cuda"


def say(*a):
    print(*a, flush=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def stack(rng, E, N, K, lo=118, hi=123):
    return (rng.integers(0, 256, (E, N, K // 2)).astype(np.uint8),
            rng.integers(lo, hi, (E, N, K // 32)).astype(np.uint8))


def forward_bound(x, gate, up, down, idx, g):
    """(out, bound): what fp32 accumulation in any order, the activation in 16 bits and
    the fp32 epilogue may add, element by element.  2^-24: a rounding of fp32."""
    u32 = 2.0 ** -24
    x = np.asarray(x, np.float64)
    H, I = x.shape[1], gate.shape[1]
    out, bound = np.zeros_like(x), np.zeros_like(x)
    size = np.zeros_like(x)
    for t, row in enumerate(idx):
        seen = set()
        for j, e in enumerate(row):
            if not 0 <= e < len(gate) or e in seen:
                continue
            seen.add(e)
            z, u = gate[e] @ x[t], up[e] @ x[t]
            dz, du = (H * u32 * (np.abs(m[e]) @ np.abs(x[t])) for m in (gate, up))
            s = z / (1 + np.exp(-z))
            a = s * u
            # |silu'| <= 1.1; exp, reciprocal and products: (|z| + 8) steps of 2^-23; two bf16 planes: 2^-16
            da = 1.1 * dz * (np.abs(u) + du) + np.abs(s) * du
            da += (np.abs(a) + da) * ((np.abs(z) + 8) * 2.0 ** -23 + 2.0 ** -16)
            y, ya = down[e] @ a, np.abs(down[e]) @ (np.abs(a) + da)
            out[t] += g[t][j] * y
            bound[t] += abs(g[t][j]) * (np.abs(down[e]) @ da + (2 * I + 2) * u32 * ya)
            size[t] += abs(g[t][j]) * ya
    return out, bound + (len(idx[0]) + 1) * u32 * size


def case(seed, T, H, I, E, k, eligible=None, odd=True):
    rng = np.random.default_rng(seed)
    stacks = [stack(rng, E, I, H), stack(rng, E, I, H), stack(rng, E, H, I)]
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32)).bfloat16()
    pick = rng.permutation(E)[:eligible or E]
    idx = np.stack([rng.permutation(pick)[:k] if len(pick) >= k else rng.choice(pick, k) for _ in range(T)]).astype(np.int32)
    g = rng.random((T, k)).astype(np.float32)
    if odd and T > 2:
        idx[T // 2] = -1                                 # a row routed nowhere
        idx[T - 1, 0] = E                                # out of range
        idx[0, k - 1] = idx[0, 0]                        # repeated
        idx[1, 0] = -2 ** 31
    return stacks, x, idx, g


def packed(stacks):
    d = [(dev(c), dev(s)) for c, s in stacks]
    return ops.pack_gate_up_q4(*d[0], *d[1]), ops.pack_down_q4(*d[2])


def run_check(T, H, I, E, k, eligible=None, seed=None):
    stacks, x, idx, g = case(T * 31 + H + I if seed is None else seed, T, H, I, E, k, eligible)
    wgu, wd = packed(stacks)
    ws = torch.full((ops.forward_q4_workspace(T, H, I, E, k, DEV).numel(),), 0xFF, dtype=torch.uint8, device=DEV)
    raw = torch.full((T + 2, H), float("nan"), device=DEV)
    out = raw[1:T + 1]
    got = []
    for _ in range(2):
        ops.moe_forward_q4(x.to(DEV), wgu, wd, dev(idx), dev(g), out=out, workspace=ws)
        got.append(out.cpu().numpy().copy())
    assert np.array_equal(got[0], got[1])
    assert torch.isnan(raw[0]).all() and torch.isnan(raw[-1]).all()
    w = [A.dequantize_q4(*s) for s in stacks]
    ref, bound = forward_bound(x.double().numpy(), *w, idx, g)
    err = np.abs(got[0] - ref)
    scale = np.abs(ref).max()
    say(f"q4 T={T} H={H} I={I} E={E} k={k}: error {err.max() / scale:.2e} of the largest output, "
        f"{(err / np.where(bound > 0, bound, 1)).max():.3f} of the bound")
    assert (err <= bound).all()


@pytest.mark.parametrize("T,H,I,E,k,eligible", [
    (1, 32, 32, 1, 1, None), (1, 256, 96, 8, 3, None), (2, 160, 32, 4, 4, None), (3, 96, 128, 8, 2, None),
    (5, 512, 160, 16, 4, None), (8, 1024, 256, 32, 8, None), (13, 288, 224, 8, 2, 3), (16, 64, 64, 4, 1, None),
    (17, 128, 96, 2, 2, None), (33, 416, 128, 3, 2, None), (40, 256, 64, 64, 8, 20), (64, 544, 192, 16, 8, 12),
    (100, 128, 32, 1, 1, None), (129, 96, 160, 1, 1, None), (130, 256, 128, 5, 3, None), (300, 192, 96, 2, 2, None),
    (257, 64, 64, 8, 8, None), (50, 64, 64, 512, 32, None)])
def test_forward(gpu, T, H, I, E, k, eligible):
    run_check(T, H, I, E, k, eligible)


@pytest.mark.parametrize("T", [1, 4, 9, 20, 60, 150])
def test_forward_at_layer_width(gpu, T):
    run_check(T, 2048, 768, 16, 8)


@pytest.mark.parametrize("T,H,I,E,k", [(2100, 32, 32, 8, 8), (600, 32, 32, 40, 32), (5500, 32, 32, 3, 3),
                                       (32, 64, 64, 64, 1), (4, 2048, 64, 512, 8), (16, 96, 32, 5, 2)])
def test_forward_long_lists(gpu, T, H, I, E, k):
    """More routing entries than the dispatch holds at a time; the largest blocks that need no dispatch."""
    run_check(T, H, I, E, k)


def test_forward_more_tokens_than_a_launch_takes(gpu):
    """2^24 tokens and more, each row a copy of one of the first 1000, some routed nowhere."""
    T, few, H, I, E = 2 ** 24 + 1234, 1000, 32, 32, 3
    stacks, x, idx, g = case(6, few, H, I, E, 1)
    wgu, wd = packed(stacks)
    ref, bound = forward_bound(x.double().numpy(), *[A.dequantize_q4(*s) for s in stacks], idx, g)
    row = torch.arange(T, device=DEV) % few
    out = torch.full((T, H), float("nan"), device=DEV)
    ops.moe_forward_q4(x.to(DEV)[row], wgu, wd, dev(idx)[row], dev(g)[row], out=out)
    worst = torch.zeros(few, H, dtype=torch.float64, device=DEV)
    refd = dev(ref)
    for a in range(0, T - T % few, 1000 * few):
        part = out[a:min(a + 1000 * few, T - T % few)].view(-1, few, H).double()
        worst = torch.maximum(worst, (part - refd).abs().amax(0))
    tail = out[T - T % few:].double()
    worst[:len(tail)] = torch.maximum(worst[:len(tail)], (tail - refd[:len(tail)]).abs())
    assert (worst.cpu().numpy() <= bound).all()


def test_forward_on_its_own_stream_and_in_a_graph(gpu):
    """Calls on a side stream with tensors of their own, and two captured graphs that share a
    workspace, replayed in turn with eager work between."""
    for T, H, I, E, k in ((1, 256, 96, 8, 2), (40, 256, 96, 8, 2), (300, 256, 96, 8, 2)):
        stacks, x, idx, g = case(T, T, H, I, E, k)
        wgu, wd = packed(stacks)
        xs = [x.to(DEV), (x * 0.5).to(DEV)]
        i, gd = dev(idx), dev(g)
        eager = [ops.moe_forward_q4(v, wgu, wd, i, gd).cpu() for v in xs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = [ops.moe_forward_q4(v, wgu, wd, i, gd, stream=side) for v in xs for _ in range(3)]
        side.synchronize()
        for n, y in enumerate(got):
            assert torch.equal(y.cpu(), eager[n // 3])
        ws = ops.forward_q4_workspace(T, H, I, E, k, DEV)
        outs = [torch.empty(T, H, device=DEV) for _ in xs]
        graphs = []
        for v, o in zip(xs, outs):
            torch.cuda.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                ops.moe_forward_q4(v, wgu, wd, i, gd, out=o, workspace=ws)
        for rep in range(3):
            for n in (0, 1):
                outs[n].fill_(float("nan"))
                graphs[n].replay()
                torch.cuda.synchronize()
                assert torch.equal(outs[n].cpu(), eager[n]), (T, rep, n)
            ops.moe_forward_q4(xs[0], wgu, wd, i, gd)


def test_forward_large_items_at_layer_width(gpu):
    """Items of 48 and of 64 rows, several to an expert, at the width of a layer: a sample of the tokens, and that
    equal tokens have equal rows."""
    H, I, E, k, few = 2048, 768, 8, 4, 24
    stacks, x, idx, g = case(77, few, H, I, E, k)
    wgu, wd = packed(stacks)
    ref, bound = forward_bound(x.double().numpy(), *[A.dequantize_q4(*s) for s in stacks], idx, g)
    for T in (700, 1999, 2500):
        row = torch.randint(0, few, (T,), generator=torch.Generator().manual_seed(T)).to(DEV)
        got = ops.moe_forward_q4(x.to(DEV)[row], wgu, wd, dev(idx)[row], dev(g)[row]).cpu().numpy()
        err = np.abs(got - ref[row.cpu()])
        say(f"q4 T={T} at layer width: {(err / np.where(bound > 0, bound, 1)[row.cpu()]).max():.3f} of the bound")
        assert (err <= bound[row.cpu()]).all()


def test_layer_from_codes_and_scales(gpu):
    """VerifyLayerQ4 given (codes, scales) pairs is the layer that quantises the stacks itself."""
    cfg, [(layer, rw, _)] = small(1)
    pairs = [ops.quantize_q4(w.float()) for w in W.expert_weights_torch(cfg, 0, DEV)]
    other = ops.VerifyLayerQ4(dev(rw), *pairs, cfg.k, max_tokens=2 * cfg.T, max_trees=cfg.B)
    blk = W.make_block(cfg, block=0)
    args = [torch.from_numpy(blk.hidden).bfloat16().to(DEV)] + [dev(a) for a in (blk.parent, blk.depth, blk.prob)]
    a, b = (ly.step(*args, tree_offsets=blk.offsets) for ly in (layer, other))
    assert torch.equal(a[2], b[2]) and torch.equal(a[1]["idx"], b[1]["idx"])


@pytest.mark.parametrize("T,H,I,E,k", [(4, 192, 160, 64, 6), (9, 192, 160, 64, 1), (10, 192, 160, 64, 1),
                                       (2, 320, 96, 64, 16), (1, 2048, 768, 64, 32), (3, 96, 224, 40, 10),
                                       (640, 160, 96, 8, 4), (641, 160, 96, 8, 4), (2048, 96, 64, 40, 4),
                                       (2049, 96, 64, 40, 4), (700, 160, 192, 9, 4)])
def test_forward_where_the_kernels_change(gpu, T, H, I, E, k):
    """The last block without a dispatch and the first with one; items of 32, 48 and 64 rows."""
    run_check(T, H, I, E, k)


def test_forward_scales_across_the_range(gpu):
    """Scale bytes from 2 to 252 in one stack: weights from 2^-126 to 6 * 2^125, each row's
    output compared with what its own magnitude allows."""
    T, H, I, E = 6, 64, 64, 2
    rng = np.random.default_rng(3)
    stacks = [stack(rng, E, I, H, 117, 120), stack(rng, E, I, H, 117, 120), stack(rng, E, H, I, 117, 120)]
    down = stacks[2][1]
    down[0, 0::4], down[0, 1::4], down[1, 0::4], down[1, 2::4] = 252, 20, 2, 230
    x = torch.from_numpy(rng.standard_normal((T, H)).astype(np.float32) * 0.01).bfloat16()
    idx = np.int32([[0], [1], [0], [1], [0], [-1]])
    g = np.full((T, 1), 0.5, np.float32)
    got = ops.moe_forward_q4(x.to(DEV), *packed(stacks), dev(idx), dev(g)).cpu().numpy()
    ref, bound = forward_bound(x.double().numpy(), *[A.dequantize_q4(*s) for s in stacks], idx, g)
    assert np.isfinite(got).all()
    # 2^-149: the smallest fp32 step, for sums below the normal range
    assert (np.abs(got - ref) <= bound + I * 2.0 ** -126).all()


@pytest.mark.parametrize("experts", [9, 16])
@pytest.mark.parametrize("shift,first,last", [(20, 0, 200), (-20, 40, 255)])
def test_forward_every_scale_byte(gpu, experts, shift, first, last):
    """Row n of W_d has scale byte n, expert c code c in its first column alone: each output is one product, of
    normal size for the bytes looked at.  9 experts, one token each, take the way without a dispatch."""
    say("scale bytes", experts, shift)
    H = 256
    I = 32
    rng = np.random.default_rng(5)
    one = np.zeros((experts, I, H // 2), np.uint8)
    one[:, 0, 0] = 2  # gate and up: 1.0 in the first row's first column
    plain = np.full((experts, I, H // 32), 127, np.uint8)
    down = np.zeros((experts, H, I // 2), np.uint8)
    down[:, :, 0] = np.arange(experts)[:, None]
    stacks = [(one, plain), (one, plain + np.uint8(shift % 256)),
              (down, np.broadcast_to(np.arange(256, dtype=np.uint8)[None, :, None], (experts, H, 1)).copy())]
    x = np.zeros((experts, H), np.float32)
    x[:, 0] = 60.0 + rng.integers(0, 4, experts)
    idx, g = np.arange(experts, dtype=np.int32)[:, None], np.ones((experts, 1), np.float32)
    x = torch.from_numpy(x).bfloat16()
    got = ops.moe_forward_q4(x.to(DEV), *packed(stacks), dev(idx), dev(g)).cpu().numpy()
    w = [A.dequantize_q4(*s) for s in stacks]
    ref, bound = forward_bound(x.double().numpy(), *w, idx, g)
    sound = np.abs(w[2]).max(axis=2) <= np.finfo(np.float32).max  # [expert, row]
    sound[:, 255] = False
    if experts == 9:  # one sum over all experts, zeros for the tokens that are routed elsewhere
        sound[:] = sound.all(axis=0)
    rows = np.arange(first, last + 1)
    ok = sound[:, rows]
    size = np.abs(ref[:, rows])
    assert (np.isfinite(got[:, rows]) == ok).all()
    assert (np.abs(got[:, rows] - ref[:, rows])[ok] <= bound[:, rows][ok]).all()
    # nothing passes for being small: 2^-126 is the smallest normal number
    code = np.arange(experts) % 8 != 0
    assert (size[code] > 2.0 ** -112).all() and (bound[:, rows] <= 2.0 ** -13 * size).all()


def test_forward_scale_bytes_of_gate_and_up(gpu):
    """Experts whose gate or up stack has one scale byte at an end of the range, against hidden states that bring
    the products back to normal size."""
    H = I = 64
    ends = [(0, 118), (1, 118), (2, 117), (20, 100), (250, -118), (252, -120)]
    cases = [(side, s, e) for side in (0, 1) for s, e in ends]
    E = len(cases)
    rng = np.random.default_rng(9)
    stacks = [stack(rng, E, I, H), stack(rng, E, I, H), stack(rng, E, H, I)]
    x = np.zeros((E, H), np.float32)
    for c, (side, s, e) in enumerate(cases):
        stacks[side][1][c] = s
        stacks[1 - side][1][c] = 125 - e  # the other product: about 1
        x[c] = rng.standard_normal(H) * 2.0 ** e
    idx, g = np.arange(E, dtype=np.int32)[:, None], np.ones((E, 1), np.float32)
    x = torch.from_numpy(x).bfloat16()
    with np.errstate(over="ignore"):  # exp(-z) of a large -z
        ref, bound = forward_bound(x.double().numpy(), *[A.dequantize_q4(*s) for s in stacks], idx, g)
    for order in (np.arange(E), np.arange(9), np.arange(3, E)):  # with and without a dispatch
        got = ops.moe_forward_q4(x[order].to(DEV), *packed(stacks), dev(idx[order]), dev(g[order])).cpu().numpy()
        err = np.abs(got - ref[order])
        say("gate and up bytes: error over bound", (err / bound[order]).max(axis=1))
        assert (err <= bound[order]).all()
    largest = np.abs(ref).max(axis=1)
    assert (largest > 2.0 ** -60).all() and (bound.max(axis=1) < 0.01 * largest).all()
    stacks[0][1][2] = 255  # NaN weights: their expert's token alone
    got = ops.moe_forward_q4(x.to(DEV), *packed(stacks), dev(idx), dev(g)).cpu().numpy()
    assert np.isnan(got[2]).all() and np.isfinite(np.delete(got, 2, axis=0)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize(gpu, dtype):
    rng = np.random.default_rng(4)
    w = rng.standard_normal((6, 5, 160)) * 2.0 ** rng.integers(-30, 30, (6, 5, 1))
    w[0, 0] = 0.0
    w[0, 1, :32] = np.arange(32) * 0.25 - 2.0                       # every tie
    w[0, 2, :8] = 6.0, 6.25, -6.0, 5.0, 3.5, 2.5, 0.25, -0.0
    w[0, 3] = 1e-38
    w[0, 4, :3] = 3e38, -1e30, 2.0 ** -126
    t = torch.from_numpy(w.astype(np.float32)).to(dtype)
    codes, scales = ops.quantize_q4(t.to(DEV))
    ref_c, ref_s = A.quantize_q4(t.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), ref_s)
    assert np.array_equal(codes.cpu().numpy(), ref_c)


def test_refusals(gpu):
    stacks, x, idx, g = case(1, 4, 64, 32, 4, 2, odd=False)
    wgu, wd = packed(stacks)
    xd, i, gd = x.to(DEV), dev(idx), dev(g)
    ops.moe_forward_q4(xd, wgu, wd, i, gd)
    for args, err in (((xd.float(), wgu, wd, i, gd), TypeError), ((xd, wd, wgu, i, gd), TypeError),
                      ((xd[:, :32].contiguous(), wgu, wd, i, gd), ValueError), ((xd, wgu, wd, i[:3], gd), ValueError),
                      ((xd, wgu, wd, i, gd[:, :1].contiguous()), ValueError), ((xd.t(), wgu, wd, i, gd), ValueError)):
        with pytest.raises(err):
            ops.moe_forward_q4(*args)
    with pytest.raises(ops.AcceptMoEError):
        ops.moe_forward_q4(xd, wgu, wd, i, gd, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        ops.quantize_q4(torch.zeros(4, 48, device=DEV))
    d = [(dev(c), dev(s)) for c, s in stacks]
    with pytest.raises(ValueError):
        ops.pack_down_q4(d[0][0], d[2][1])
    with pytest.raises(ValueError):
        ops.pack_gate_up_q4(*d[0], *d[2])
    assert ops.moe_forward_q4(xd[:0], wgu, wd, i[:0], gd[:0]).shape == (0, 64)


# ---------------------------------------------------------------------------
# the layer, and a whole verification pass: norms, 4-bit layers, sampling, acceptance
# ---------------------------------------------------------------------------
def small(layers):
    cfg = W.LayerConfig("q4_small", 131, "bf16", T=24, B=2, H=256, E=32, k=4, I=96, depth_max=5,
                        commit_rule="depth_sibling", hidden_std=1.0)
    out = []
    for l in range(layers):
        stacks = [w.float() for w in W.expert_weights_torch(cfg, l, DEV)]
        rw = W.router_weights(cfg, l)
        out.append((ops.VerifyLayerQ4(dev(rw), *stacks, cfg.k, max_tokens=2 * cfg.T, max_trees=cfg.B), rw,
                    [A.dequantize_q4(*(t.cpu().numpy() for t in ops.quantize_q4(w))) for w in stacks]))
    return cfg, out


def test_layer_is_its_three_steps(gpu):
    cfg, [(layer, rw, w)] = small(1)
    blk = W.make_block(cfg, block=0)
    h = torch.from_numpy(blk.hidden).bfloat16().to(DEV)
    tree = [dev(a) for a in (blk.parent, blk.depth, blk.prob)]
    logits, sel, y = layer.step(h, *tree, tree_offsets=blk.offsets)
    z = logits.cpu().numpy()
    ref = O.select(z, blk.parent, blk.depth, blk.prob, blk.offsets, cfg.k)
    assert np.array_equal(sel["idx"].cpu().numpy(), ref["idx"])
    assert np.allclose(sel["gate"].cpu().numpy(), ref["gate"], rtol=GATE_RTOL, atol=0)
    want, bound = forward_bound(h.double().cpu().numpy(), *w, ref["idx"], sel["gate"].cpu().numpy())
    assert (np.abs(y.cpu().numpy() - want) <= bound).all()


def test_verification_pass(gpu):
    """Stack with norms and 4-bit layers -> logits -> sampled tokens -> accepted path ->
    estimator; every step against the oracle on the step's own inputs, eager and
    captured."""
    cfg, made = small(3)
    layers = [m[0] for m in made]
    rng = np.random.default_rng(8)
    norms = [torch.from_numpy((1 + 0.2 * rng.standard_normal(cfg.H)).astype(np.float32)).bfloat16().to(DEV)
             for _ in range(4)]
    blocks = [W.make_block(cfg, block=b) for b in range(2)]
    T, V = len(blocks[0].parent), 777
    stack = ops.VerifyStack(layers, T, norms=norms)
    head = torch.from_numpy(rng.standard_normal((cfg.H, V)).astype(np.float32) * 0.3).bfloat16().to(DEV)
    offs = blocks[0].offsets
    u = dev(rng.random(T).astype(np.float32))
    k = torch.full((T,), 3, dtype=torch.int32, device=DEV)
    p = torch.full((T,), 0.8, device=DEV)
    ws = ops.sample_workspace(T, V, DEV)
    token = dev(rng.integers(0, V, T).astype(np.int32))
    h_in = torch.empty(T, cfg.H, dtype=torch.bfloat16, device=DEV)
    tree_in = [dev(a) for a in (blocks[0].parent, blocks[0].depth, blocks[0].prob)]

    def load(b):
        h_in.copy_(torch.from_numpy(blocks[b].hidden).bfloat16())
        for dst, a in zip(tree_in, (blocks[b].parent, blocks[b].depth, blocks[b].prob)):
            dst.copy_(torch.from_numpy(a))

    def whole():
        x = stack.step(h_in, *tree_in, tree_offsets=offs)
        z = x @ head
        s = ops.sample(z, u, top_k=k, top_p=p, workspace=ws)
        return z, s, ops.accept(token, tree_in[0], s["token"], offs)

    est = ops.CommitEstimator(cfg.depth_max + 1)
    eager = []
    for b in range(2):
        load(b)
        z, s, acc = whole()
        torch.cuda.synchronize()
        for l in range(3):
            h = stack.h[l][:T].double().cpu().numpy()
            y = layers[l].out[:T]
            assert torch.equal(stack.h[l + 1][:T], (stack.h[l][:T].float() + y).bfloat16())
            for src, add, wn, got in (([(h, None, norms[l], stack.x[l])] if l == 0 else []) +
                                      [(h, y.double().cpu().numpy(), norms[l + 1], stack.x[l + 1])]):
                _, n = A.residual_norm(src, add, wn.double().cpu().numpy(), stack.eps)
                # a rounding to bf16 and fp32 work
                assert (np.abs(got[:T].double().cpu().numpy() - n) <= np.abs(n) * (2.0 ** -8 + 1e-5) + 1e-6).all()
            sel = layers[l].sel_out
            want, bound = forward_bound(stack.x[l][:T].double().cpu().numpy(), *made[l][2],
                                        sel["idx"][:T].cpu().numpy(), sel["gate"][:T].cpu().numpy())
            assert (np.abs(y.cpu().numpy() - want) <= bound).all()
        zh, uh = z.double().cpu().numpy(), u.cpu().numpy()
        for t in range(T):
            tok, prob, margin = A.sample_row(zh[t], uh[t], top_k=3, top_p=np.float32(0.8))
            assert margin <= 1 or int(s["token"][t]) == tok
        on, paths, length, bonus = A.accept(token.tolist(), blocks[b].parent, s["token"].tolist(), offs)
        assert acc["on_path"].cpu().tolist() == on.tolist() and acc["length"].cpu().tolist() == length
        assert acc["bonus"].cpu().tolist() == bonus
        est.add(blocks[b].depth, acc["on_path"].cpu().numpy())
        eager.append([t.cpu().clone() for t in (z, s["token"], s["prob"], acc["path"])])
    assert est.m.sum() == 2 * T and est.estimate()[0] == 1.0

    load(0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        whole()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        z, s, acc = whole()
    for rep in range(4):
        say("replay", rep)
        load(rep % 2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((z, s["token"], s["prob"], acc["path"]), eager[rep % 2]):
            assert torch.equal(a.cpu(), b), rep
        whole()  # eager work between replays
        torch.cuda.synchronize()


def test_stack_twin_and_refused_norms(gpu):
    """Two blocks in flight on two streams give what each gives alone; norms that do not fit."""
    cfg, made = small(2)
    layers = [m[0] for m in made]
    norms = [torch.full((cfg.H,), 0.5 + l, dtype=torch.bfloat16, device=DEV) for l in range(3)]
    blocks = [W.make_block(cfg, block=b) for b in range(2)]
    T = len(blocks[0].parent)
    stack = ops.VerifyStack(layers, T, norms=norms)
    args = [(torch.from_numpy(b.hidden).bfloat16().to(DEV), *(dev(a) for a in (b.parent, b.depth, b.prob)), b.offsets)
            for b in blocks]
    alone = [stack.step(*a).clone() for a in args]
    twin, streams = stack.twin(), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [s.step(*a, stream=st) for s, a, st in zip((stack, twin), args, streams)]
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        assert torch.equal(a, b)
    for bad, err in ((norms[:2], ValueError), ([n[:-1] for n in norms], ValueError), ([n.float() for n in norms], TypeError),
                     ([n.cpu() for n in norms], ValueError)):
        with pytest.raises(err):
            ops.VerifyStack(layers, T, norms=bad)
    with pytest.raises(ValueError):
        layers[0].step(torch.zeros(2 * cfg.T + 1, cfg.H, dtype=torch.bfloat16, device=DEV), *args[0][1:4])
    with pytest.raises(TypeError):
        layers[0].step(args[0][0].float(), *args[0][1:4])
