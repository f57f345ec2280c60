"""Routed-expert operators at the edges of their contracts.

Tolerances are those of test_gpu_experts.py, derived there; where a case adds to them it says so."""
import numpy as np
import pytest

import experts_ref as ref
from paper_2502_07021_b200 import binding as fs
from test_gpu_experts import ROUND, TYPES, dev, host, quantized, run_forward, scratch, t_

pytestmark = pytest.mark.gpu


# ---- product --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("first,sizes,outs,cols", [(1, [1], 16, 64), (5, [4, 0, 21], 130, 96), (37, [20, 0, 3], 70, 544),
                                                   (300, [130, 64], 200, 256), (9, [0, 0], 33, 32)])
def test_product_of_a_slice_of_the_groups(first, sizes, outs, cols):
    """offsets + 2: the rows of the groups before the slice are in none of its groups, so their results are 0."""
    import torch
    rng = np.random.default_rng(first + outs)
    groups, rows = len(sizes), first + sum(sizes) + 4
    xq, xs, xv = quantized(rng.standard_normal((rows, cols)))
    wq, ws, wv = quantized(rng.standard_normal((groups * outs, cols)))
    off = np.concatenate([[0, first // 2, first], first + np.cumsum(sizes), [rows]]).astype(np.int32)
    mine = dev(off)[2:]
    off = off[2:]
    for dtype in TYPES:
        y = torch.full((rows, outs + 1), 7.0, dtype=t_(dtype), device="cuda")
        fs.fs_mx4_product(xq, xq.stride(0), xs, xs.stride(0), rows, wq, wq.stride(0), ws, ws.stride(0), groups, mine, outs, cols, y,
                          fs.fs_dtype(y), y.stride(0), None)
        got = host(y[:, :outs])
        want, size = np.zeros((rows, outs)), np.zeros((rows, outs))
        for g in range(groups):
            a, w = xv[off[g]:off[g + 1]], wv[g * outs:(g + 1) * outs]
            want[off[g]:off[g + 1]], size[off[g]:off[g + 1]] = a @ w.T, np.abs(a) @ np.abs(w).T
        assert np.all(got[:first] == 0) and np.all(got[off[groups]:] == 0)
        assert np.all(np.abs(got - want) <= (cols / 64 + 4) * 2.0 ** -22 * size + 1.01 * ROUND[dtype] * np.abs(want) + 2.0 ** -25 * (size > 0))
        assert torch.all(y[:, outs:] == 7.0)


# ---- gradient -------------------------------------------------------------------------------------------------
def gradient_64(l, idx, k, normalize, load, d_gate, d_loss):
    """The gradient with probabilities from differences to the row's maximum, which no size of the logits hurts."""
    t, e = l.shape
    m = l.max(1, keepdims=True)
    w = np.exp(l - m)
    s = w.sum(1, keepdims=True)
    p, lse = w / s, (m + np.log(s))[:, 0]
    dw = np.zeros((t, e))
    np.put_along_axis(dw, idx, d_gate, 1)
    if normalize:
        chosen = np.zeros((t, e))
        np.put_along_axis(chosen, idx, 1.0, 1)
        z = np.where(chosen > 0, l, -np.inf)
        q = np.exp(z - z.max(1, keepdims=True))
        q /= q.sum(1, keepdims=True)
    else:
        q = p
    d = q * (dw - (q * dw).sum(1, keepdims=True))
    d += d_loss[0] * e / t * p * (load - p @ load[:, None])
    return d + d_loss[1] * 2 / t * lse[:, None] * p, p, lse


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("e", [10, 60, 256, 600])
def test_gradient_of_rows_of_large_numbers(e, dtype, normalize):
    """Rows filled with the type's lowest value share evenly (p = 1/E), and rows moved by 1e4 have the p of their differences."""
    import torch
    rng = np.random.default_rng(e)
    t, k = 300, 4
    l = rng.standard_normal((t, e)) * 1.5
    l[1::3] += 1e4
    l[2::9] -= 2e4
    x = dev(l, t_(dtype))
    x[::5] = torch.finfo(x.dtype).min
    x[5::25, e // 2] = 1.0                          # among them rows with one expert open
    l32 = x.float().cpu().numpy()
    idx = ref.select(l32, None, None, k)
    o = run_forward(x, None, None, k, normalize)
    assert np.array_equal(o["idx"].cpu().numpy(), idx)
    load = host(o["load"])
    dg = rng.standard_normal((t, k)).astype(np.float32)
    # the second loss's gradient is of the size of lse itself, so it gets a run without those rows
    for dl in (np.array([1.0, 0.0], np.float32) * t, np.array([0.5, 1e-3], np.float32) * t):
        out = torch.full((t, e), float("nan"), dtype=x.dtype, device="cuda")
        fs.fs_router_backward(x, fs.fs_dtype(x), e, t, e, None, k, 1 if normalize else 0, o["idx"], o["gate"], o["lse"], o["counts"],
                              o["load"], dev(dg), dev(dl), out, e, None)
        want, p, lse = gradient_64(l32.astype(np.float64), idx, k, normalize, load, dg.astype(np.float64), dl.astype(np.float64))
        bound = np.abs(dg).max() * k + p * (dl[0] * e / t * load.max() * 2 + dl[1] * 2 / t * np.abs(lse)[:, None])
        rows = np.ones(t, bool)
        if dl[1]:
            rows[::5] = False
        tol = 1e-5 * bound + ROUND[dtype] * 1.01 * np.abs(want) + 2.0 ** -24
        assert np.all(np.abs(host(out) - want)[rows] <= tol[rows])


# ---- choice ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("e,k", [(6, 3), (60, 4), (100, 8), (100, 12), (256, 8), (700, 32)])
def test_a_nan_reaches_every_gate_of_its_rows(e, k, normalize):
    """A NaN logit makes its row's gates NaN, a NaN in the bias those of every active row, places without an expert included;
    the choice passes over both."""
    rng = np.random.default_rng(e + k)
    l = rng.standard_normal((40, e)).astype(np.float32)
    l[1] = np.nan                                   # no score at all
    l[2, :] = -np.inf
    l[2, :2] = [np.nan, 1.0]                        # one open expert
    l[3, e - 1] = np.nan
    l[4] = -np.inf                                  # not active
    l[5, k - 1:] = -np.inf                          # fewer open than wanted
    mask = np.ones(40, np.uint8)
    mask[[6, 39]] = 0
    l[6] = np.nan
    nan_rows = [1, 2, 3]
    for bad in (False, True):
        bias = (rng.standard_normal(e) * 0.5).astype(np.float32)
        if bad:
            bias[e // 2] = np.nan
        o = run_forward(dev(l), dev(mask), dev(bias), k, normalize)
        idx, gate = o["idx"].cpu().numpy(), host(o["gate"])
        assert np.array_equal(idx, ref.select(l, mask, bias, k))
        active = np.ones(40, bool)
        active[[4, 6, 39]] = False
        assert np.all(gate[~active] == 0)
        assert np.all(np.isnan(gate[nan_rows]))
        clean = np.setdiff1d(np.flatnonzero(active), nan_rows)
        assert np.all(np.isnan(gate[clean])) if bad else np.all(np.isfinite(gate[clean]))
        if not bad:
            assert np.all(gate[5][idx[5] < 0] == 0)
        lse = host(o["lse"])                        # the bias takes no part in it
        assert np.all(np.isfinite(lse[clean])) and np.all(np.isnan(lse[nan_rows]))


@pytest.mark.parametrize("e,k", [(6, 2), (40, 5), (65, 8), (100, 8), (128, 7), (128, 16), (256, 8), (256, 16), (256, 20), (500, 8), (1000, 12)])
def test_ties_zeros_and_nan_at_every_width(e, k):
    """Equal scores go to the lower expert in every form of the choice: few ties, more ties than candidates are kept, all equal;
    -0 equals 0; a NaN is passed over."""
    rng = np.random.default_rng(e * 31 + k)
    few = rng.standard_normal((60, e))
    some = np.round(rng.standard_normal((60, e)) * 2)           # small whole numbers
    many = rng.integers(0, 2, (60, e)).astype(float)
    same = np.zeros((20, e))
    signs = np.where(rng.random((40, e)) < 0.5, -0.0, 0.0)
    signs[rng.random((40, e)) < 0.02] = 1.0
    edge = np.round(rng.standard_normal((60, e)))
    edge[rng.random((60, e)) < 0.3] = -np.inf
    edge[rng.random((60, e)) < 0.3] = np.nan
    edge[7] = np.nan
    l = np.concatenate([few, some, many, same, signs, edge])
    for dtype in TYPES:
        for bias in (None, np.round(rng.standard_normal(e)).astype(np.float32)):
            x = dev(l, t_(dtype))
            o = run_forward(x, None, None if bias is None else dev(bias), k, True)
            assert np.array_equal(o["idx"].cpu().numpy(), ref.select(x.float().cpu().numpy(), None, bias, k))


# ---- balance --------------------------------------------------------------------------------------------------
def run_duals(x, eps, iters, mask=None, start=None):
    import torch
    t, e = x.shape
    w, n = scratch(t, e, 1)
    f, g, err = torch.full((t,), 9.0, device="cuda"), torch.full((e,), 9.0, device="cuda"), torch.full((iters,), 9.0, device="cuda")
    fs.fs_router_duals(x, fs.fs_dtype(x), x.stride(0), t, e, mask, None, eps, iters, start, f, g, err, w, n, None)
    return f, g, err


def test_column_sum_of_many_powers_below_the_smallest():
    """A column whose sum comes from one row while 60000 others add powers too small to be kept: what they add, 4e-4 of it,
    counts."""
    t, eps = 60001, 1.0
    l = np.zeros((t, 3), np.float32)
    l[:, 1] = -1.0
    l[:, 2] = -87.4                                   # 2^-126.1
    l[17, 2] = -68.5                                  # 2^-98.8
    f, g, _ = run_duals(dev(l), eps, 1)
    rf, rg, _ = ref.duals(l.astype(np.float64), None, None, eps, 1)
    assert np.all(np.abs(host(g) - rg) <= 4e-6 * 2 * (1 + np.abs(rg) / 16))
    assert np.all(np.abs(host(f) - rf) <= 4e-6 * 2 * (1 + np.abs(rf) / 16))


# more sweeps over the rows than one cluster of sixteen blocks makes (eight each): the balance meets on the whole grid
GRID = [(70001, 12), (33000, 30), (17001, 40), (8500, 128), (5001, 256), (2500, 500), (2300, 1024)]


@pytest.mark.parametrize("t,e", GRID)
def test_balance_on_the_grid_with_starved_and_closed_experts(t, e):
    rng = np.random.default_rng(t)
    l = rng.standard_normal((t, e)).astype(np.float32)
    l[:, 3] -= 60.0
    l[:, 7] = -np.inf
    l[5] = -np.inf
    mask = (rng.random(t) >= 0.05).astype(np.uint8)
    l[mask == 0] = np.nan
    g0 = (rng.standard_normal(e) * 0.1).astype(np.float32)
    f, g, err = run_duals(dev(l), 0.1, 5, dev(mask), dev(g0))
    rf, rg, rerr = ref.duals(np.nan_to_num(l.astype(np.float64), nan=0.0, neginf=-np.inf), mask, None, 0.1, 5, g0.astype(np.float64))
    assert host(g)[7] == g0[7]
    # the starved column's dual is of size 60: its exponents are rounded at that size
    assert np.all(np.abs(host(g) - rg) <= 4e-6 * 6 * (1 + np.abs(rg) / 16) * 4)
    assert np.all(np.abs(host(f) - rf) <= 4e-6 * 6 * 4 * (1 + np.abs(rf) / 16))
    assert np.all(np.abs(host(err) - rerr) <= 1e-5 + 2 * 4e-6 * 6 * 4 / 0.1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,e", GRID)
def test_balance_on_the_grid_of_column_sums_of_every_size(t, e, dtype):
    """Columns from 1 down to 1e-24 of a share at the start, so that every level of the common sums is used."""
    rng = np.random.default_rng(t + 1)
    eps, iters = 0.4, 4
    l = rng.standard_normal((t, e)) * 0.3 - eps * np.log(10.0) * np.linspace(0, 24, e)
    x = dev(l, t_(dtype))
    f, g, err = run_duals(x, eps, iters)
    again = run_duals(x, eps, iters)
    assert all(np.array_equal(host(a), host(b)) for a, b in zip((f, g, err), again))
    rf, rg, rerr = ref.duals(host(x), None, None, eps, iters)
    tol = 4e-6 * (1 + iters)
    assert np.all(np.abs(host(f) - rf) <= tol * (1 + np.abs(rf) / 16))
    assert np.all(np.abs(host(g) - rg) <= tol * (1 + np.abs(rg) / 16))
    assert np.all(np.abs(host(err) - rerr) <= 1e-5 + 2 * tol / eps)


@pytest.mark.parametrize("t,e", GRID)
def test_balance_on_the_grid_with_rows_of_the_lowest_value_and_nan(t, e):
    rng = np.random.default_rng(t + 2)
    l = rng.standard_normal((t, e)).astype(np.float32)
    low = np.zeros(t, bool)
    low[::7] = True
    l[low] = np.finfo(np.float32).min
    l[3::11, 5] = np.finfo(np.float32).min
    f, g, _ = run_duals(dev(l), 0.05, 4)
    rf, rg, _ = ref.duals(l.astype(np.float64), None, None, 0.05, 4)
    assert np.all(np.abs(host(g) - rg) <= 4e-6 * 5 * (1 + np.abs(rg) / 16))
    assert np.all(np.abs(host(f) - rf)[~low] <= 4e-6 * 5 * (1 + np.abs(rf[~low]) / 16))
    assert np.allclose(host(f)[low], rf[low], rtol=1e-6)
    l[t - 1, e - 1] = np.nan                          # one active row with a NaN: nothing of the balance is a number
    f, g, err = run_duals(dev(l), 0.05, 2)
    assert np.all(np.isnan(host(g))) and np.all(np.isnan(host(err))) and np.all(np.isnan(host(f)))


# ---- the layer and the wrappers -------------------------------------------------------------------------------
def make_layer(experts, width=64, hidden=96, k=2, dtype="bfloat16", seed=3, **kw):
    import torch
    from paper_2502_07021_b200.experts import RoutedExperts
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    return RoutedExperts((r(experts, width) / width ** 0.5).to(t_(dtype)), (r(experts, hidden, width) / width ** 0.5).to(t_(dtype)),
                         (r(experts, width, hidden) / hidden ** 0.5).to(t_(dtype)), k, **kw)


def tokens_of(n, width=64, dtype="bfloat16", seed=4):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(n, width, device="cuda", generator=gen).to(t_(dtype))


def test_strided_activations_and_weights():
    import torch
    from paper_2502_07021_b200 import experts
    wide = tokens_of(70, 128)
    views = [wide[:, ::2], wide[:, 1::2], wide[:64].t()[:64], wide[:1, :64].expand(70, 64), wide[3:4, 64:], wide[:, 5:69]]
    for v in views:
        q, s = experts.quantize(v)
        q2, s2 = experts.quantize(v.clone(memory_format=torch.contiguous_format))
        assert torch.equal(q, q2) and torch.equal(s, s2)
    stack = torch.randn(3, 40, 128, device="cuda")
    for v in (stack[:, :, ::2], stack.transpose(1, 2), stack[:, ::3], stack[::2]):
        q, s = experts.quantize(v)
        q2, s2 = experts.quantize(v.contiguous())
        assert q.shape[:-1] == v.shape[:-1] and torch.equal(q, q2) and torch.equal(s, s2)
    layer = make_layer(12, k=3)
    for v in views[:4]:
        y, idx = layer(v)
        y2, idx2 = layer(v.contiguous())
        assert torch.equal(idx, idx2) and torch.equal(y, y2)


def test_wrong_types_lengths_and_devices_are_refused():
    import torch
    from paper_2502_07021_b200 import experts
    l = torch.randn(20, 8, device="cuda")
    good = torch.full((8,), 0.125, device="cuda")
    wrong = [good.bfloat16(), good.double(), good.half(), good[:7], good.repeat(2), good[None], good.cpu()]
    for v in wrong:
        for call in (lambda: experts.balance(l, 0.1, 2, share=v), lambda: experts.balance(l, 0.1, 2, start=v),
                     lambda: experts.choose(l, 2, v), lambda: experts.route(l, 2, v)):
            with pytest.raises(ValueError):
                call()
    mask = torch.ones(20, dtype=torch.bool, device="cuda")
    for m in (mask.cpu(), mask[:19], mask.int(), mask[:, None]):
        for call in (lambda: experts.balance(l, 0.1, 2, mask=m), lambda: experts.choose(l, 2, mask=m), lambda: experts.route(l, 2, mask=m)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        experts.choose(l.cpu(), 2)
    xq, xs = experts.quantize(torch.randn(10, 96, device="cuda"))
    w = experts.quantize(torch.randn(3, 40, 96, device="cuda"))
    off = torch.tensor([0, 4, 4, 10], dtype=torch.int32, device="cuda")
    args = dict(xq=xq, xs=xs, weights=w, offsets=off, cols=96, dtype=torch.float32)
    for bad in (dict(offsets=off.long()), dict(offsets=off[:3]), dict(offsets=off.cpu()), dict(offsets=off.float()), dict(xs=xs.cpu()),
                dict(xs=xs[:9]), dict(xq=xq.int()), dict(xq=xq[:, :32]), dict(xq=xq.repeat(1, 2)[:, ::2]), dict(weights=(w[0], w[1][:2])),
                dict(weights=(w[0].transpose(0, 1), w[1])), dict(weights=(w[0][0], w[1][0])),
                dict(weights=(torch.cat([w[0], w[0]])[::2], w[1]))):
        with pytest.raises(ValueError):
            experts.product(**{**args, **bad})
    layer = make_layer(12, k=3)
    for bad in (tokens_of(5).cpu(), tokens_of(5, 32), tokens_of(5)[None]):
        with pytest.raises(ValueError):
            layer(bad)


def test_strided_vectors_and_packed_matrices():
    """What the wrappers accept besides contiguous tensors gives the same results."""
    import torch
    from paper_2502_07021_b200 import experts
    l = torch.randn(50, 8, device="cuda")
    wide = torch.randn(16, device="cuda")
    mask = torch.arange(100, device="cuda") % 3 != 0
    off = torch.tensor([0, 9, 4, 9, 4, 9, 10], dtype=torch.int32, device="cuda")
    for a, b in ((wide[::2], wide[::2].contiguous()), (wide[3:11], wide[3:11].clone())):
        for p, q in zip(experts.choose(l, 3, a, mask[::2]), experts.choose(l, 3, b, mask[::2].contiguous())):
            assert torch.equal(p, q)
        for p, q in zip(experts.balance(l, 0.3, 3, mask[::2], a.abs() + 0.1, a), experts.balance(l, 0.3, 3, mask[::2], b.abs() + 0.1, b)):
            assert torch.equal(p, q)
    x = torch.randn(10, 96, device="cuda")
    for outs in (40, 1):
        w = torch.randn(3, outs, 96, device="cuda")
        xq, xs = experts.quantize(x)
        wq, ws = experts.quantize(w)
        plain = experts.product(xq, xs, (wq, ws), off[::2].contiguous(), 96, torch.float32)
        pad = lambda t, n: torch.cat([t, torch.full((*t.shape[:-1], n), 255, dtype=torch.uint8, device="cuda")], -1)[..., :t.shape[-1]]
        assert torch.equal(plain, experts.product(pad(xq, 16), pad(xs, 4), (pad(wq, 32), pad(ws, 8)), off[::2], 96, torch.float32))
        for g in range(3):                             # one group, and one row at a time
            one = experts.product(xq, xs, (wq[g:g + 1], ws[g:g + 1]), None, 96, torch.float32)
            rows = slice(int(off[2 * g]), int(off[2 * g + 2]))
            assert torch.equal(one[rows], plain[rows])
            assert torch.equal(experts.product(xq[rows][:1], xs[rows][:1], (wq[g:g + 1], ws[g:g + 1]), None, 96, torch.float32), plain[rows][:1])


def test_layer_padding_stays_zero_when_an_expert_overflows():
    """The first row of the ordered products belongs to some token; what it holds reaches that token alone."""
    import torch
    from paper_2502_07021_b200 import experts
    layer, x = make_layer(2, k=2, dtype="float16"), tokens_of(5, dtype="float16")
    layer.up = experts.quantize(torch.full((2, 96, 64), 3.0, dtype=torch.float16, device="cuda"))
    x[0] = 1000.0                                      # 64 x 3000 is beyond fp16
    x[1:] = 1.0
    mask = torch.tensor([1, 1, 0, 1, 0], dtype=torch.uint8, device="cuda")
    y, _ = layer(x, mask)
    got = host(y)
    assert not np.any(np.isfinite(got[0])) and np.all(got[[2, 4]] == 0) and np.all(np.isfinite(got[[1, 3]]))


def test_layer_with_a_token_of_nan():
    """One such token costs itself and nobody else."""
    import torch
    layer, x = make_layer(12, k=3), tokens_of(200)
    mask = torch.ones(200, dtype=torch.bool, device="cuda")
    mask[50] = False
    want, want_idx = layer(x, mask)                    # the batch without the token
    x[50, 7] = float("nan")
    y, idx = layer(x)
    rest = np.arange(200) != 50
    assert np.all(np.isnan(host(y)[50])) and np.all(idx.cpu().numpy()[50] == -1)
    assert torch.equal(idx[mask], want_idx[mask]) and np.array_equal(host(y)[rest], host(want)[rest])
    y, idx = layer(x, mask)                            # as padding it counts for nothing
    assert torch.equal(idx, want_idx) and torch.equal(y, want)


@pytest.mark.parametrize("tokens", [1, 2, 31, 63])
def test_layer_on_few_tokens_chooses_by_the_tokens_scores(tokens):
    """Fewer tokens than experts cannot be balanced among themselves: every expert's share is less than a token.  The choice is the
    token's own, or that of the duals kept from a batch."""
    layer, x = make_layer(64, k=8), tokens_of(tokens)
    logits = (x @ layer.score.T).float().cpu().numpy()
    y, idx = layer(x)
    assert np.array_equal(idx.cpu().numpy(), ref.select(logits, None, None, 8))
    kept = layer.duals(tokens_of(2000, seed=5))
    assert np.all(np.isfinite(host(kept))) and np.abs(host(kept)).max() > 0.05
    y2, idx2 = layer(x, bias=kept)
    assert np.array_equal(idx2.cpu().numpy(), ref.select(logits, None, kept.cpu().numpy(), 8))
    assert np.all(np.isfinite(host(y))) and np.all(np.isfinite(host(y2)))


def test_layer_on_a_batch_of_mostly_padding():
    import torch
    layer, x = make_layer(64, k=8), tokens_of(300)
    mask = torch.zeros(300, dtype=torch.uint8, device="cuda")
    mask[40:100] = 2                                   # 60 tokens for 64 experts; any byte but 0 is a token
    y, idx = layer(x, mask)
    logits = (x @ layer.score.T).float().cpu().numpy()
    assert np.array_equal(idx.cpu().numpy(), ref.select(logits, mask.cpu().numpy(), None, 8))
    off = mask.cpu().numpy() == 0
    assert np.all(host(y)[off] == 0)


def test_layer_with_nan_duals_returns_nan():
    import torch
    layer, x = make_layer(12, k=3), tokens_of(30)
    mask = torch.ones(30, dtype=torch.bool, device="cuda")
    mask[4] = False
    y, _ = layer(x, mask, bias=torch.full((12,), float("nan"), device="cuda"))
    on = mask.cpu().numpy()
    assert np.all(np.isnan(host(y)[on])) and np.all(host(y)[~on] == 0)


def test_no_tokens_at_all():
    import torch
    from paper_2502_07021_b200 import experts
    layer = make_layer(12, k=3)
    y, idx = layer(tokens_of(0))
    assert y.shape == (0, 64) and idx.shape == (0, 3) and torch.all(layer.duals(tokens_of(0)) == 0)
    l = torch.empty(0, 12, device="cuda", requires_grad=True)
    gate, loss, idx, counts = experts.route(l, 3)
    loss.sum().backward()
    assert l.grad.shape == (0, 12) and torch.all(loss == 0) and torch.all(counts == 0)
    f, g, err = experts.balance(l.detach(), 0.1, 2)
    assert f.shape == (0,) and torch.all(g == 0) and torch.all(err == 0)


def test_second_derivatives_and_changed_masks_are_refused():
    import torch
    from paper_2502_07021_b200 import experts
    l = torch.randn(20, 8, device="cuda", requires_grad=True)
    gate, loss, _, _ = experts.route(l, 2)
    first, = torch.autograd.grad(gate.square().sum() + loss.sum(), l, create_graph=True)
    with pytest.raises(RuntimeError):
        first.square().sum().backward()
    for mask in (torch.ones(20, dtype=torch.bool, device="cuda"), torch.ones(20, dtype=torch.uint8, device="cuda")):
        gate, loss, _, _ = experts.route(l, 2, mask=mask)
        loss.sum().backward(retain_graph=True)         # unchanged: twice gives the same
        one = l.grad.clone()
        l.grad = None
        loss.sum().backward(retain_graph=True)
        assert torch.equal(one, l.grad)
        mask[3] = 0
        with pytest.raises(RuntimeError):
            loss.sum().backward()
        l.grad = None
