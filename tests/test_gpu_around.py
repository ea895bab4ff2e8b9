"""The operators around the layer on the GPU (residual norm, sampling, accepted
path) against the fp64 oracle, at sizes and contents where they can go wrong."""
import numpy as np
import pytest
import torch

from oracle import around_oracle as A
from paper_2608_02989_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


def say(*a):
    print(*a, flush=True)


def dev(a, dt=None):
    t = torch.from_numpy(np.array(a))
    return (t if dt is None else t.to(dt)).to(DEV)


def poisoned(shape, dtype):
    """A buffer whose every byte is set, and the words around it to check."""
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    raw = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device=DEV)
    return raw, raw[256:256 + n].view(dtype).view(shape)


def untouched(raw):
    r = raw.cpu().numpy()
    return bool((r[:256] == 0xA5).all() and (r[-256:] == 0xA5).all())


# ---------------------------------------------------------------------------
# residual norm
# ---------------------------------------------------------------------------
# fp32 work of one value, in units of 2^-24 relative: the addition 1; the sum of
# squares, whose terms all have one sign: half of (3 for s^2, at most 4 NV + 1 adds in
# a thread, 6 + 16 over lanes and waves), NV <= 4 for H <= 16384 and 16 for 65536;
# the mean's product and eps 1, the reciprocal root 2, two products 2.
def norm_units(H):
    nv = max(1, -(-H // 4 // 1024))
    nv = 1 << (nv - 1).bit_length()
    return 1 + (3 + 4 * nv + 1 + 22) / 2 + 1 + 2 + 2


@pytest.mark.parametrize("T,H,dtype,group", [
    (1, 4, torch.float32, None), (1, 64, torch.bfloat16, 32), (3, 36, torch.float32, -1), (37, 1100, torch.float32, None),
    (5, 1100, torch.bfloat16, -1), (60, 2048, torch.bfloat16, None), (33, 2048, torch.bfloat16, 128),
    (7, 4096, torch.float32, 256), (64, 4096, torch.bfloat16, 64), (2, 4100, torch.bfloat16, None),
    (3, 5120, torch.bfloat16, 32), (2, 16384, torch.float32, -1), (1, 65536, torch.bfloat16, None),
    (4097, 256, torch.bfloat16, 128)])
@pytest.mark.parametrize("add", [True, False])
def test_residual_norm(gpu, T, H, dtype, group, add):
    say("norm", T, H, dtype, group, add)
    gen = torch.Generator().manual_seed(T * 131 + H)
    h = (torch.randn(T, H, generator=gen) * 3).to(dtype)
    y = torch.randn(T, H, generator=gen) if add else None
    w = (1 + 0.5 * torch.randn(H, generator=gen)).to(dtype)
    got = ops.residual_norm(h.to(DEV), None if y is None else y.to(DEV), w.to(DEV), eps=1e-6, group=group)
    s, n = A.residual_norm(h.double().numpy(), None if y is None else y.double().numpy(), w.double().numpy(), 1e-6)
    if add:  # the fp32 sum rounded once, bit for bit
        assert torch.equal(got["hidden"].cpu(), (h.float() + y).to(dtype))
    else:
        assert torch.equal(got["hidden"].cpu(), h)
    # the fp32 sum's own rounding counts against |h| + |y| where they cancel
    size = np.abs(h.double().numpy()) + (np.abs(y.double().numpy()) if add else 0)
    cancel = np.divide(size, np.abs(s), out=np.ones_like(s), where=s != 0)
    rel = (norm_units(H) + cancel) * 2.0 ** -24
    if group is None:
        half = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0
        err = np.abs(got["norm"].cpu().double().numpy() - n)
        assert (err <= np.abs(n) * (half + (1 + half) * rel)).all(), float((err / np.abs(n)).max())
        return
    width = H if group < 0 else group
    largest = np.abs(n).reshape(T, -1, width).max(axis=2)
    scale = got["scale"].cpu().double().numpy()
    worst = rel.reshape(T, -1, width).max(axis=2)
    assert scale.shape == largest.shape
    assert (np.abs(scale - largest / 448) <= largest / 448 * (worst + 2.0 ** -24)).all()
    code = got["codes"].cpu().double().numpy().reshape(T, -1, width)
    want = n.reshape(T, -1, width) / (largest / 448)[..., None]
    near = np.abs(want) * (rel.reshape(want.shape) + worst[..., None] + 2.0 ** -23)
    assert (np.abs(code - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) + near * (1 + 2.0 ** -4)).all()


def test_residual_norm_beyond_32_bits(gpu):
    """More than 2^31 elements: the last rows as in a call of their own."""
    T, H = 525000, 4096
    gen = torch.Generator(device=DEV).manual_seed(2)
    h = torch.zeros(T, H, dtype=torch.bfloat16, device=DEV)
    y = torch.zeros(T, H, device=DEV)
    h[-3:], y[-3:] = torch.randn(3, H, generator=gen, device=DEV).bfloat16(), torch.randn(3, H, generator=gen, device=DEV)
    w = torch.rand(H, generator=gen, device=DEV).bfloat16()
    for group in (None, 128):
        want = ops.residual_norm(h[-3:].clone(), y[-3:].clone(), w, group=group)
        got = ops.residual_norm(h, y, w, group=group)
        for name in want:
            assert torch.equal(got[name][-3:].view(torch.uint8), want[name].view(torch.uint8)), name
        del got


@pytest.mark.parametrize("group", [None, -1])
def test_residual_norm_more_rows_than_a_launch_takes(gpu, group):
    """2^32 threads and more in all: rows of both launches as in a call of their own."""
    T, H = 2 ** 26 + 70, 4
    gen = torch.Generator(device=DEV).manual_seed(3)
    h = torch.randn(T, H, generator=gen, device=DEV).bfloat16()
    w = torch.rand(H, generator=gen, device=DEV).bfloat16()
    for add in (False, True):
        y = torch.randn(T, H, generator=gen, device=DEV) if add else None
        got = ops.residual_norm(h, y, w, group=group)
        for part in (slice(0, 40), slice(2 ** 26 - 21, 2 ** 26 + 30), slice(T - 9, T)):
            want = ops.residual_norm(h[part].clone(), None if y is None else y[part].clone(), w, group=group)
            for name in want:
                assert torch.equal(got[name][part].view(torch.uint8), want[name].view(torch.uint8)), (add, name, part)


def test_residual_norm_zero_rows_and_in_place(gpu):
    h = torch.zeros(3, 64, dtype=torch.bfloat16)
    h[1] = 2.0
    w = torch.full((64,), 1.5, dtype=torch.bfloat16)
    y = torch.zeros(3, 64)
    hd = h.to(DEV)
    raw, codes = poisoned((3, 64), torch.float8_e4m3fn)
    out = {"hidden": hd, "codes": codes, "scale": torch.empty(3, 2, device=DEV)}
    got = ops.residual_norm(hd, y.to(DEV), w.to(DEV), eps=0.5, group=32, out=out)
    assert got["hidden"].data_ptr() == hd.data_ptr() and torch.equal(hd.cpu(), h)
    c, s = got["codes"].cpu().float(), got["scale"].cpu()
    assert (c[[0, 2]] == 0).all() and (s[[0, 2]] == 0).all()
    assert (c[1] == 448).all() and torch.allclose(s[1], torch.full((2,), 3.0 / 4.5 ** 0.5 / 448), rtol=1e-6)
    assert untouched(raw)
    assert ops.residual_norm(hd[:0], y.to(DEV)[:0], w.to(DEV))["norm"].shape == (0, 64)


@pytest.mark.parametrize("H", [64, 4352, 16640])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [None, 32, 256, -1])
def test_residual_norm_not_finite(gpu, group, dtype, H):
    """NaN and infinities in the stream, the addend and the weight: not finite exactly where the formulas are."""
    if group is not None and H % group:
        group = 64
    say("norm not finite", group, dtype, H)
    gen = torch.Generator().manual_seed(H)
    nan = float("nan")
    h, y, w = torch.randn(9, H, generator=gen).to(dtype), torch.randn(9, H, generator=gen), torch.randn(H, generator=gen)
    h[1, H - 1], h[2, 0], h[3, 33], y[4, H // 2], y[5, 1], h[6, :] = nan, INF, -INF, nan, INF, nan
    h[7, 5], y[7, 5] = INF, -INF  # their sum is NaN
    for weight in (w, torch.where(torch.arange(H) == 40, torch.tensor(INF), w), torch.where(torch.arange(H) == 40, torch.tensor(nan), w)):
        weight = weight.to(dtype)
        got = ops.residual_norm(h.to(DEV), y.to(DEV), weight.to(DEV), group=group)
        with np.errstate(invalid="ignore", over="ignore"):
            s, n = A.residual_norm(h.double().numpy(), y.double().numpy(), weight.double().numpy(), 1e-6)
            assert np.array_equal(np.isfinite(got["hidden"].cpu().double().numpy()), np.isfinite(s))
            # an infinity's row has an infinite mean: zeros beside it, NaN in its place
            if group is None:
                out = got["norm"].cpu().double().numpy()
                assert np.array_equal(np.isnan(out), np.isnan(n)) and np.array_equal(np.isinf(out), np.isinf(n))
                assert (out[n == 0] == 0).all()
                continue
            parts = n.reshape(9, -1, H if group < 0 else group)
            scale = np.abs(parts).max(axis=2) / 448
            code = np.where(scale[..., None] == 0, 0.0, parts / scale[..., None])
        out, got_scale = got["codes"].cpu().double().numpy().reshape(parts.shape), got["scale"].cpu().double().numpy()
        assert np.array_equal(np.isnan(got_scale), np.isnan(scale)) and np.array_equal(np.isinf(got_scale), np.isinf(scale))
        assert np.array_equal(np.isnan(out), np.isnan(code))
        sound = np.isfinite(scale)
        assert (out[sound & (scale == 0)] == 0).all() and (got_scale[sound & (scale == 0)] == 0).all()
        assert (np.abs(out[sound & (scale > 0)]).max(axis=1) == 448).all()
        assert (out[np.isinf(scale)][np.isfinite(parts[np.isinf(scale)])] == 0).all()


@pytest.mark.parametrize("group", [None, 32, -1])
def test_residual_norm_zero_over_zero(gpu, group):
    h = torch.zeros(2, 96, device=DEV)
    h[1] = 1.0
    got = ops.residual_norm(h, None, torch.ones(96, device=DEV), eps=0.0, group=group)
    for name in ("norm",) if group is None else ("codes", "scale"):
        out = got[name].float()
        assert out[0].isnan().all() and out[1].isfinite().all()


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def check_sample(z, u, dtype=torch.float32, stride=None, **rules):
    """Tokens equal to the oracle's, u and top_p's sum being further off any border than 64-bit
    sums may move it (the oracle's margin)."""
    z = torch.as_tensor(z).to(dtype)
    R, V = z.shape
    zd = z.to(DEV)
    if stride:
        wide = torch.full((R, stride), 1e30, dtype=dtype, device=DEV)
        wide[:, :V] = zd
        zd = wide[:, :V]
    names = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    host = {n: np.broadcast_to(np.asarray(rules[n], t), (R,)) for n, t in names.items() if rules.get(n) is not None}
    u = np.asarray(u, np.float32)
    raw_t, token = poisoned((R,), torch.int32)
    raw_p, prob = poisoned((R,), torch.float32)
    ws = torch.full((int(ops.sample_workspace(R, V, DEV).numel()),), 0xA5, dtype=torch.uint8, device=DEV)
    args = {n: dev(a) for n, a in host.items()}
    outs = []
    for _ in range(2):  # the second call finds the first one's workspace
        ops.sample(zd, dev(u), **args, workspace=ws, outputs={"token": token, "prob": prob})
        outs.append((token.cpu().numpy().copy(), prob.cpu().numpy().copy()))
    assert all(np.array_equal(a, b) for a, b in zip(*outs))
    assert untouched(raw_t) and untouched(raw_p)
    for r in range(R):
        t, p, margin = A.sample_row(z[r].double().numpy(), u[r], **{n: a[r] for n, a in host.items()})
        assert margin > 1, (r, margin)
        assert outs[0][0][r] == t, (r, outs[0][0][r], t, margin)
        # V 2^-44 of the sum and 64-bit work, then one rounding
        assert abs(outs[0][1][r] - p) <= p * (2.0 ** -24 + 1e-7), (r, outs[0][1][r], p)


def logits(rng, R, V, spread=2.5):
    z = rng.standard_normal((R, V)) * spread
    z[np.arange(R)[:, None], rng.integers(0, V, (R, min(V, 12)))] += 4 * spread
    return z.astype(np.float32)


@pytest.mark.parametrize("R,V", [(1, 1), (3, 2), (2, 63), (5, 1000), (4, 4099), (1, 32000), (3, 33001), (2, 131072)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rules", [
    {}, {"top_k": 1}, {"top_k": 50, "top_p": 0.9, "min_p": 0.05, "temperature": 0.8}, {"top_p": 0.95},
    {"min_p": 0.01, "temperature": 1.3}, {"temperature": 0.0}, {"top_k": 700, "temperature": 2.0},
    {"top_p": 0.5, "min_p": 0.001, "temperature": 3.0}, {"top_k": 5000, "top_p": 0.99}], ids=str)
def test_sample(gpu, R, V, dtype, rules):
    say("sample", R, V, dtype, rules)
    rng = np.random.default_rng(R * 7 + V)
    check_sample(logits(rng, R, V), rng.random(R), dtype, **rules)


def test_sample_rows_with_their_own_rules(gpu):
    rng = np.random.default_rng(5)
    R, V = 24, 5003
    z = logits(rng, R, V)
    z[rng.random((R, V)) < 0.4] = -INF
    check_sample(z, rng.random(R), stride=5010, temperature=np.where(np.arange(R) % 4 == 0, 0.0, 0.3 + rng.random(R)),
                 top_k=np.where(np.arange(R) % 3 == 0, 0, rng.integers(1, 2000, R)),
                 top_p=np.where(np.arange(R) % 5 == 0, 1.0, 0.6 + 0.3 * rng.random(R)),
                 min_p=np.where(np.arange(R) % 7 == 0, 0.0, 0.1 * rng.random(R)))


@pytest.mark.parametrize("V", [64, 5000, 40000])
def test_sample_hard_rows(gpu, V):
    """Ties, masks that leave one or no token, lowest finite values, infinities, NaN, sorted rows."""
    rng = np.random.default_rng(V)
    low = np.finfo(np.float32).min
    rows = [np.full(V, -INF), np.full(V, np.nan), np.zeros(V), np.full(V, low)]
    one = np.full(V, -INF)
    one[V - 1] = -3.0
    some = np.full(V, low)
    some[[5, 40]] = 1.0, 0.5
    infs = rng.standard_normal(V)
    infs[[3, 17, 50]] = INF
    nans = rng.standard_normal(V)
    nans[::3] = np.nan
    signed = np.where(np.arange(V) % 2 == 0, 0.0, -0.0)
    rows += [one, some, infs, nans, signed, np.linspace(-9, 9, V), np.linspace(9, -9, V),
             np.repeat(rng.standard_normal(-(-V // 8)), 8)[:V], np.round(rng.standard_normal(V))]
    z = np.stack(rows).astype(np.float32)
    R = len(z)
    for i, rules in enumerate(({}, {"top_k": 3}, {"top_k": 60, "top_p": 0.7}, {"top_p": 0.37}, {"min_p": 0.3},
                               {"temperature": 0.0}, {"temperature": 0.01}, {"top_k": 40, "min_p": 1.0},
                               {"top_k": 64, "top_p": 0.93, "min_p": 0.01, "temperature": 5.0})):
        say("hard rows", V, rules)
        check_sample(z, 0.0437 + 0.9 * np.random.default_rng(100 + i).random(R), **rules)


@pytest.mark.parametrize("spread", [0.02, 0.3, 1.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_crowded(gpu, spread, dtype):
    """Many tokens of nearly one weight: thousands within 1/32 of a nat, in bf16 mostly equal."""
    rng = np.random.default_rng(int(spread * 100))
    R, V = 4, 150001
    z = (rng.standard_normal((R, V)) * spread).astype(np.float32)
    for rules in ({}, {"top_p": 0.6}, {"min_p": 0.3}, {"top_p": 0.9, "min_p": 0.5}, {"top_k": 900}, {"top_k": 1000},
                  {"top_k": 1001}, {"top_k": 64, "temperature": 40.0}, {"temperature": 1e4}):
        say("crowded", spread, dtype, rules)
        check_sample(z, rng.random(R), dtype, **rules)


@pytest.mark.parametrize("R,V,dtype", [(33, 1023, torch.bfloat16), (257, 4097, torch.float32), (1100, 515, torch.float32),
                                       (2, 262147, torch.bfloat16), (1, 1000000, torch.float32)])
def test_sample_shapes(gpu, R, V, dtype):
    """Rows spread over one to many workgroups, more rows than one launch takes, every row start's alignment."""
    rng = np.random.default_rng(V)
    z = logits(rng, R, V)
    for rules in ({"top_k": 20, "top_p": 0.9}, {"top_p": 0.95}, {"temperature": 0.0}):
        say("shape", R, V, rules)
        check_sample(z, rng.random(R), dtype, **rules)


def test_sample_far_from_zero(gpu):
    """Logits with a large common part, of which the weights keep nothing."""
    rng = np.random.default_rng(9)
    z = np.round(rng.standard_normal((6, 9001)) * 3 * 64) / 64
    z += np.float64([1e3, -1e3, 3e4, 1e5, -1e5, 0])[:, None]
    for rules in ({}, {"top_p": 0.9, "min_p": 0.01}, {"top_k": 100}, {"temperature": 0.1}):
        say("far", rules)
        check_sample(z.astype(np.float32), rng.random(6), **rules)


def test_sample_on_its_own_stream_and_in_a_graph(gpu):
    rng = np.random.default_rng(12)
    side = torch.cuda.Stream()
    for R, V, rules in ((3, 5000, {"top_k": 30, "top_p": 0.9}), (3, 40000, {"top_p": 0.9}), (40, 9000, {"min_p": 0.02})):
        zs = [dev(logits(rng, R, V)) for _ in range(2)]
        u = dev(rng.random(R).astype(np.float32))
        args = {n: torch.full((R,), v, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV)
                for n, v in rules.items()}
        eager = [ops.sample(z, u, **args) for z in zs]
        eager = [(e["token"].cpu(), e["prob"].cpu()) for e in eager]
        side.wait_stream(torch.cuda.current_stream())
        got = [ops.sample(z, u, **args, stream=side) for z in zs for _ in range(3)]
        side.synchronize()
        for n, o in enumerate(got):
            assert torch.equal(o["token"].cpu(), eager[n // 3][0]) and torch.equal(o["prob"].cpu(), eager[n // 3][1])
        ws = ops.sample_workspace(R, V, DEV)
        graphs = []
        for z in zs:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = ops.sample(z, u, **args, workspace=ws)
            graphs.append((g, out))
        for rep in range(3):
            for n in (0, 1):
                graphs[n][0].replay()
                torch.cuda.synchronize()
                assert torch.equal(graphs[n][1]["token"].cpu(), eager[n][0]), (rep, n)
                assert torch.equal(graphs[n][1]["prob"].cpu(), eager[n][1])
            ops.sample(zs[0], u)


def test_sample_rows_beyond_32_bits(gpu):
    """Rows 2^31 elements apart."""
    V, step = 5000, 2 ** 31
    z = dev(logits(np.random.default_rng(8), 3, V), torch.bfloat16)
    big = torch.empty(2 * step + V, dtype=torch.bfloat16, device=DEV).as_strided((3, V), (step, 1))
    big.copy_(z)
    u = torch.tensor([0.2, 0.5, 0.9], device=DEV)
    for k in (None, torch.full((3,), 40, dtype=torch.int32, device=DEV)):
        a, b = ops.sample(z, u, top_k=k), ops.sample(big, u, top_k=k)
        assert torch.equal(a["token"], b["token"]) and torch.equal(a["prob"], b["prob"])


def test_sample_settings_at_the_ends_of_their_types(gpu):
    """Every row gets one of its tokens, whatever its settings hold."""
    tiny, nan = float(np.finfo(np.float32).smallest_subnormal), float("nan")
    rows = [(t, p, m, k, u) for t in (1.0, tiny, 3e38, INF, nan, -INF) for p in (1.0, 0.5, nan, -INF, INF, tiny)
            for m in (0.0, 0.5, nan, INF, -INF) for k in (0, 3, -2 ** 31, 2 ** 31 - 1) for u in (0.0, 0.7, nan, INF, -1.0)]
    t, p, m, k, u = (dev(np.array(c, np.int32 if i == 3 else np.float32)) for i, c in enumerate(zip(*rows)))
    rng = np.random.default_rng(4)
    for V in (70, 6000):
        z = logits(rng, len(rows), V).astype(np.float32)
        z[::3, 5:60] = -INF
        z[1::7, 9] = INF
        z[2::5, 11] = nan
        for args in ({"top_k": k}, {}):
            out = ops.sample(dev(z), u, temperature=t, top_p=p, min_p=m, **args)
            token, prob = out["token"].cpu().numpy(), out["prob"].cpu().numpy()
            assert ((token >= 0) & (token < V)).all()
            chosen = z[np.arange(len(rows)), token]
            assert (chosen > -INF).all() and ((prob > 0) & (prob <= 1)).all()


@pytest.mark.parametrize("V", [70, 6000])
@pytest.mark.parametrize("with_k", [True, False])
def test_sample_defined_ends_of_settings(gpu, V, with_k):
    """Settings at the ends of their types wherever the header says what they mean: token and probability of the oracle."""
    tiny, nan = float(np.finfo(np.float32).smallest_subnormal), float("nan")
    rows = [(t, p, m, k, u) for t in (1.0, tiny, 3e38, INF, nan, -INF) for p in (1.0, 0.57, 0.0, -INF, INF, tiny)
            for m in (0.0, 0.5, INF, -INF) for k in ((0, 3, -2 ** 31, 2 ** 31 - 1) if with_k else (0,))
            for u in (0.0, 0.7, INF, -1.0)]
    t, p, m, k, u = (np.array(c, np.int32 if i == 3 else np.float32) for i, c in enumerate(zip(*rows)))
    R = len(rows)
    z = logits(np.random.default_rng(4), R, V)
    z[::3, 5:60] = -INF
    z[1::7, [9, 33]] = INF
    z[2::5, 11] = nan
    got = ops.sample(dev(z), dev(u), temperature=dev(t), top_p=dev(p), min_p=dev(m), **({"top_k": dev(k)} if with_k else {}))
    token, prob = got["token"].cpu().numpy(), got["prob"].cpu().numpy()
    unsure = 0
    for r in range(R):
        say("row", r, rows[r]) if r % 500 == 0 else None
        # beside infinite logits every finite temperature gives the same weights, and so does the limit
        tau = 1.0 if np.isposinf(t[r]) and np.isposinf(z[r]).any() else t[r]
        want, prob_want, margin = A.sample_row(z[r], min(max(u[r], 0.0), 1 - 2.0 ** -24), temperature=tau, top_k=k[r],
                                               top_p=p[r], min_p=m[r])
        if margin <= 1:
            unsure += 1
            continue
        assert token[r] == want, (rows[r], token[r], want, margin)
        assert abs(prob[r] - prob_want) <= prob_want * (2.0 ** -24 + 1e-7), (rows[r], prob[r], prob_want)
    assert unsure <= R // 50, unsure


def test_sample_borders_of_u_and_top_p(gpu):
    z = np.log(np.tile(np.float32([4, 2, 1, 1]), (4, 1)))
    z = np.concatenate([z, np.full((4, 300), -INF, np.float32)], axis=1)
    u = dev(np.float32([0.0, -1.0, 1.0 - 2.0 ** -24, 1.0]))
    got = ops.sample(dev(z), u)
    assert got["token"].cpu().tolist() == [0, 0, 3, 3]
    one = torch.ones(4, device=DEV)
    got = ops.sample(dev(z), u, top_p=one * 0.0, min_p=one * 7.0)
    assert got["token"].cpu().tolist() == [0] * 4 and got["prob"].cpu().tolist() == [1.0] * 4
    got = ops.sample(dev(z), u, top_p=one * 2.0, min_p=-one, top_k=torch.full((4,), -5, dtype=torch.int32, device=DEV))
    assert got["token"].cpu().tolist() == [0, 0, 3, 3]
    assert ops.sample(dev(z)[:0], u[:0])["token"].shape == (0,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top_k", [None, 0, 3, 2000, 6000])
def test_sample_top_p_of_nothing_keeps_the_first_token(gpu, dtype, top_k):
    """top_p of 0, below 0 and next to it on rows whose first tokens are equal or nearly so: fewer of them than a
    search's window holds, more, and more than a list holds; every way a row can take."""
    V = 6000
    rng = np.random.default_rng(31)
    z = np.tile((rng.standard_normal(V) - 9).astype(np.float32), (6, 1))
    z[0, [4000, 17, 2500]] = 5.0, 5.0, 1.0
    z[1, [4000, 17, 2500]] = 5.001, 5.0, 4.999
    z[2, rng.permutation(V)[:300]] = 2.0
    z[3, rng.permutation(V)[:300]] = 2.0 + 0.02 * rng.random(300)
    z[4, rng.permutation(V)[:5000]] = -1.0
    z[5, 1234] = 7.0
    for temperature in (None, 50.0):
        for p in (0.0, -1.0, -INF, float(np.finfo(np.float32).smallest_subnormal), 1e-30):
            say("top_p", p, "top_k", top_k, dtype, temperature)
            for u in (0.0, 0.5, 0.9, 1 - 2.0 ** -24):
                check_sample(z, np.full(6, u), dtype, top_p=p, top_k=top_k, temperature=temperature)


# ---------------------------------------------------------------------------
# accepted path
# ---------------------------------------------------------------------------
def tree(rng, n, branch, hit, chain=False):
    par = [-1]
    if chain:
        par += list(range(n - 1))
    head = 0
    while len(par) < n:
        par += [head] * min(int(rng.integers(1, branch + 1)), n - len(par))
        head += 1
    tok = rng.integers(0, 5, n)
    target = rng.integers(0, 5, n)
    for t in range(1, n):
        if rng.random() < hit:
            target[par[t]] = tok[t]
    return par[:n], tok, target


def check_accept(token, parent, target, offsets):
    on, paths, length, bonus = A.accept(token, parent, target, offsets)
    got = ops.accept(dev(token, torch.int32), dev(parent, torch.int32), dev(target, torch.int32), offsets)
    longest = max(b - a for a, b in zip(offsets, offsets[1:]))
    want = [p + [-1] * (longest - len(p)) for p in paths]
    assert got["on_path"].cpu().tolist() == on.tolist()
    assert got["path"].cpu().tolist() == want
    assert got["length"].cpu().tolist() == length and got["bonus"].cpu().tolist() == bonus


@pytest.mark.parametrize("sizes,branch,hit", [
    ([1], 1, 0.5), ([2], 1, 1.0), ([60] * 32, 4, 0.6), ([1, 0, 64, 65, 0, 1024, 3], 3, 0.9), ([1000], 8, 1.0),
    ([0], 1, 0.5), ([13] * 256, 2, 0.8)])
@pytest.mark.parametrize("chain", [False, True])
def test_accept(gpu, sizes, branch, hit, chain):
    say("accept", sizes[:4], len(sizes), chain)
    rng = np.random.default_rng(sum(sizes))
    token, parent, target, offs = [], [], [], [0]
    for n in sizes:
        if n:
            par, tok, tgt = tree(rng, n, branch, hit, chain)
            parent += [p if p < 0 else p + offs[-1] for p in par]
            token += list(tok)
            target += list(tgt)
        offs.append(offs[-1] + n)
    check_accept(np.array(token, int), np.array(parent, int), np.array(target, int), offs)


def test_accept_malformed_parents(gpu):
    """Parents outside the tree, behind the child, the child itself, and the extremes of the type."""
    big = 2 ** 31 - 1
    parent = np.array([7, 0, 1, 3, -5, big, -big - 1, 0, -1, 0, 8, 10, 9])
    token = np.ones(13, int)
    target = np.ones(13, int)
    check_accept(token, parent, target, [0, 8, 13])


def test_accept_ways_to_give_trees(gpu):
    rng = np.random.default_rng(7)
    a, b = tree(rng, 5, 3, 0.6), tree(rng, 9, 3, 0.6)
    parent, token, target = (np.concatenate([x, y]).astype(int) for x, y in zip(a, b))
    parent[6:] += 5
    for offs in ([0, 5, 5, 14], (0, 5, 5, 14), np.array([0, 5, 5, 14]), np.array([0, 5, 5, 14], np.int32),
                 list(np.array([0, 5, 5, 14]))):
        check_accept(token, parent, target, offs)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    got = ops.accept(none, none, none, [0])
    assert got["path"].shape == (0, 0) and got["length"].shape == (0,)


def test_refusals(gpu):
    """Arguments that do not fit together: an exception before any launch."""
    h, y, w = (torch.zeros(s, device=DEV) for s in ((4, 64), (4, 64), (64,)))
    ops.residual_norm(h, y, w)
    for args, kw, err in (((h.half(), y, w.half()), {}, TypeError), ((h, y.bfloat16(), w), {}, TypeError),
                          ((h, y, w.bfloat16()), {}, TypeError), ((h, y, w[:60]), {}, ValueError),
                          ((h, y[:3], w), {}, ValueError), ((h.t(), y, w), {}, ValueError),
                          ((h, y, w), {"group": 48}, ValueError), ((h, y, w), {"group": 128}, ValueError),
                          ((h.cpu(), y, w), {}, ValueError), ((h, y, w), {"eps": -1.0}, ops.AcceptMoEError),
                          ((h, y, w), {"out": {"hidden": h, "norm": y}}, ops.AcceptMoEError),
                          ((h, y, w), {"out": {"hidden": y, "norm": h.clone()}}, ops.AcceptMoEError),
                          ((h, y, w), {"out": {"hidden": h, "norm": h[:3].clone()}}, ValueError),
                          ((h[:, :62].contiguous(), None, w[:62]), {}, ops.AcceptMoEError)):
        with pytest.raises(err):
            ops.residual_norm(*args, **kw)
    z, u = torch.zeros(3, 40, device=DEV), torch.zeros(3, device=DEV)
    f, i = torch.ones(3, device=DEV), torch.ones(3, dtype=torch.int32, device=DEV)
    ops.sample(z, u)
    for args, kw, err in (((z.half(), u), {}, TypeError), ((z[0], u), {}, ValueError), ((z, u[:2]), {}, ValueError),
                          ((z, u.double()), {}, TypeError), ((z.t(), f), {}, ValueError), ((z.cpu(), u), {}, ValueError),
                          ((z, u), {"top_k": f}, TypeError), ((z, u), {"top_p": f[:2]}, ValueError),
                          ((z, u), {"temperature": i}, TypeError),
                          ((z[:1].expand(3, 40), u), {}, ValueError),
                          ((z, u), {"outputs": {"token": i, "prob": f[:2]}}, ValueError),
                          ((z, u), {"workspace": torch.empty(256, dtype=torch.uint8, device=DEV)}, ops.AcceptMoEError),
                          ((z[:, :0], u), {}, ops.AcceptMoEError)):
        with pytest.raises(err):
            ops.sample(*args, **kw)
    t = torch.zeros(6, dtype=torch.int32, device=DEV)
    ops.accept(t, t, t)
    for args, kw, err in (((t.long(), t, t), {}, TypeError), ((t, t[:5], t), {}, ValueError),
                          ((t, t, t, []), {}, ValueError), ((t, t, t, [0.0, 6.0]), {}, TypeError),
                          ((t, t, t, [0, 5]), {}, ops.AcceptMoEError), ((t, t, t, [0, 4, 3, 6]), {}, ops.AcceptMoEError),
                          ((t.cpu(), t, t), {}, ValueError)):
        with pytest.raises(err):
            ops.accept(*args, **kw)
    out = ops.accept(t, t, t)
    for name, bad in (("path", out["path"][:, :5].contiguous()), ("on_path", out["on_path"][:5]),
                      ("length", out["length"].float())):
        with pytest.raises((ValueError, TypeError)):
            ops.accept(t, t, t, outputs={**out, name: bad})
