"""Tokens to the experts and back, gradients, and the experts' factors, against the float64 oracle.

Tolerances, per element, u = 2^-24 (a rounding to fp32), h = half a step of the result's type (2^-8 bf16, 2^-11 fp16, u fp32), t its smallest
number over two:
  combine     K products added one after the other in fp32, one rounding to the type:  K u sum|w y| (1 + h) + h |exact| + t
  gradients   dys: a product in fp32 and a rounding to the type, (u + h) |exact| (1 + h) + t; dweights: D products, each wavefront lane D / 64 (in
              vectors of up to 8) of them one after the other, then six additions across lanes: (D / 64 + 16) u sum|dy ys|
  factors     fp32 sums of exact products in another order: 2e-5 of the Frobenius norm and of the largest entry, as for one layer
              (tests/test_parity_gpu.py); running averages one more rounding of entries of about 1: 2e-7 of the largest on top
"""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as eo
from paper_1811_12019_amd import binding as kb

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
FACTOR_TOL = 2e-5


def f64(t):
    return t.detach().double().cpu().numpy()


def guarded(shape, dtype, value, pad=64):
    """A contiguous tensor of `value` with `pad` elements of a watched value on both sides, and a check that those are untouched."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * pad,), 77, dtype=dtype, device=DEV)
    inner = whole[pad:pad + n].view(shape)
    inner.fill_(value)
    return inner, lambda: bool((whole[:pad] == 77).all() and (whole[pad + n:] == 77).all())


# ---- sort -----------------------------------------------------------------------------------------------------------
SORTS = [(1, 1, 1), (1, 8, 64), (3, 64, 5), (63, 1, 3), (64, 1, 2), (65, 2, 5), (1000, 3, 7), (4096, 2, 16), (4097, 2, 16), (8193, 1, 1), (20011, 4, 513),
         (50001, 2, 1024), (30000, 8, 256), (12345, 1, 1000), (70000, 2, 512), (1500000, 2, 37)]


def experts_of(T, K, E, how, seed):
    rng = np.random.default_rng(seed)
    if how == "one":
        return np.full((T, K), E // 2)
    if how == "none":
        return rng.choice([-1, E, 2 ** 31 - 1, -2 ** 31], (T, K))
    expert = np.minimum(rng.geometric(min(0.9, 4.0 / E), (T, K)) - 1, E - 1) if how == "skewed" else rng.integers(0, E, (T, K))
    if how == "dropped":
        expert = np.where(rng.random((T, K)) < 0.3, rng.choice([-1, E, E + 5, 2 ** 31 - 1, -2 ** 31], (T, K)), expert)
    return expert


@pytest.mark.parametrize("how", ["even", "skewed", "dropped", "one", "none"])
@pytest.mark.parametrize("T,K,E", SORTS)
def test_sort(T, K, E, how):
    expert = experts_of(T, K, E, how, T + E)
    offsets, ok0 = guarded((E + 1,), torch.int32, -9)
    order, ok1 = guarded((T * K,), torch.int32, -9)
    place, ok2 = guarded((T, K), torch.int32, -9)
    route = kb.ExpertRoute(T, K, E, offsets=offsets, order=order, place=place)
    given = torch.from_numpy(expert.astype(np.int32)).to(DEV)
    for _ in range(2):                                     # (the second call finds the first one's counts in its scratch)
        kb.kfac_expert_sort(route, given)
    flat = expert.reshape(-1)
    there = (flat >= 0) & (flat < E)
    by_expert = np.argsort(np.where(there, flat, E), kind="stable")
    rows = int(there.sum())
    want_place = np.full(T * K, -1)
    want_place[by_expert[:rows]] = np.arange(rows)
    np.testing.assert_array_equal(offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(np.bincount(flat[there].astype(np.int64), minlength=E))]))
    np.testing.assert_array_equal(place.cpu().numpy().reshape(-1), want_place)
    np.testing.assert_array_equal(order.cpu().numpy(), np.where(np.arange(T * K) < rows, by_expert, -1))
    assert ok0() and ok1() and ok2()
    if T * K < 5000:                                       # (the oracle's lists)
        for got, want in zip((offsets, order, place), eo.expert_sort(expert, E)):
            np.testing.assert_array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("E,n", [(256, 4200000), (700, 4128769), (256, 13000001), (100, 5000000)])
def test_sort_of_long_runs_to_one_expert(E, n):
    """All assignments of several runs in a row are one expert's: the most that a count of them has to hold."""
    i = torch.arange(n, device=DEV, dtype=torch.int64)
    expert = torch.where(i < n - 1000, E - 2, (i % E)).to(torch.int32)
    order, by = torch.sort(expert.long(), stable=True)
    want = torch.empty_like(by).scatter_(0, by, i)
    route = kb.ExpertRoute(n, 1, E)
    kb.kfac_expert_sort(route, expert.view(n, 1))
    torch.testing.assert_close(route.offsets.long(), torch.cat([i[:1], torch.bincount(expert.long(), minlength=E).cumsum(0)]), rtol=0, atol=0)
    assert torch.equal(route.place.view(-1).long(), want) and torch.equal(route.order.view(-1).long(), by)


def test_sort_of_no_tokens_and_without_order():
    route = kb.ExpertRoute(0, 2, 5)
    route.offsets.fill_(7)
    kb.kfac_expert_sort(route, torch.empty((0, 2), dtype=torch.int32, device=DEV))
    assert route.offsets.tolist() == [0] * 6
    expert = torch.tensor([[1, 0], [1, 1]], dtype=torch.int32, device=DEV)
    route = kb.ExpertRoute(2, 2, 2, want_order=False)
    assert kb.kfac_expert_sort(route, expert).order is None
    assert route.offsets.tolist() == [0, 1, 4] and route.place.tolist() == [[1, 0], [2, 3]]


# ---- rows -----------------------------------------------------------------------------------------------------------
def routed(T, K, E, drop, seed):
    g = torch.Generator().manual_seed(seed)
    expert = torch.randint(0, E, (T, K), generator=g, dtype=torch.int32)
    expert[torch.rand((T, K), generator=g) < drop] = -1
    route = kb.ExpertRoute(T, K, E)
    kb.kfac_expert_sort(route, expert.to(DEV))
    return route, route.place.cpu().numpy()


def rows_of(n, D, dtype, gap, seed, scale=1.0):
    """n x D, `gap` elements between rows and (odd gaps) off the 16-byte grid."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    wide = torch.randn((n, D + gap), generator=g, device=DEV).mul_(scale).to(dtype)
    return wide[:, gap // 2:gap // 2 + D] if gap else wide


ROWS = [(1, 1, 1, 1, 0, 0.0), (1, 8, 64, 2048, 0, 0.0), (3, 2, 4, 7, 0, 0.4), (5, 3, 2, 8, 0, 0.2), (17, 2, 3, 9, 3, 0.2), (33, 5, 7, 100, 0, 0.1), (70, 4, 9, 64, 8, 0.0),
        (129, 2, 8, 1001, 0, 0.1), (64, 1, 4, 4100, 12, 0.3), (9, 64, 100, 72, 0, 0.5), (40, 6, 11, 515, 1, 0.2), (2, 3, 4, 16, 0, 1.0), (700, 7, 5, 24, 0, 0.1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,E,D,gap,drop", ROWS)
def test_dispatch(T, K, E, D, gap, drop, dtype):
    route, place = routed(T, K, E, drop, D)
    x = rows_of(T, D, TYPES[dtype], gap, 1)
    whole = torch.full((T * K, D + 2 * gap + 1), 77.0, dtype=TYPES[dtype], device=DEV)
    xs = whole[:, gap:gap + D]
    kb.kfac_expert_dispatch(route, x, xs)
    np.testing.assert_array_equal(f64(xs), eo.expert_dispatch(f64(x), place, np.full((T * K, D), 77.0)))
    assert bool((whole[:, :gap] == 77).all()) and bool((whole[:, gap + D:] == 77).all())


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,E,D,gap,drop", ROWS)
def test_combine(T, K, E, D, gap, drop, dtype, weighted):
    route, place = routed(T, K, E, drop, D + 1)
    ys = rows_of(T * K, D, TYPES[dtype], gap, 2)
    ys[int(route.offsets[E]):] = float("nan")                  # rows that nothing goes to
    w = torch.rand((T, K), device=DEV) * 2 - 0.5 if weighted else None
    if weighted:
        w[route.place < 0] = float("inf")                      # ... and weights of no assignment
    whole = torch.full((T, D + gap + 1), 77.0, dtype=TYPES[dtype], device=DEV)
    y = whole[:, :D]
    kb.kfac_expert_combine(route, ys, w, y)
    np_w = None if w is None else f64(w)
    want = eo.expert_combine(f64(ys), np_w, place, D)
    size = eo.expert_combine(np.abs(f64(ys)), None if w is None else np.abs(np_w), place, D)
    t = TYPES[dtype]
    h = HALF[t]
    assert (np.abs(f64(y) - want) <= K * U * size * (1 + h) + h * np.abs(want) + TINY[t]).all()
    assert bool((whole[:, D:] == 77).all())
    again = torch.empty_like(whole)[:, :D]
    kb.kfac_expert_combine(route, ys, w, again)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,E,D,gap,drop", ROWS)
def test_combine_backward(T, K, E, D, gap, drop, dtype):
    route, place = routed(T, K, E, drop, D + 2)
    t = TYPES[dtype]
    h = HALF[t]
    ys, dy = rows_of(T * K, D, t, gap, 3), rows_of(T, D, t, gap, 4)
    ys[int(route.offsets[E]):] = float("nan")
    w = torch.rand((T, K), device=DEV) * 2 - 0.5
    w[route.place < 0] = float("nan")
    gap += 3                                                    # (dys has a stride of its own)
    whole = torch.full((T * K, D + gap), 77.0, dtype=t, device=DEV)
    dys = whole[:, gap // 2:gap // 2 + D]
    dw = torch.full((T, K), float("nan"), device=DEV)
    kb.kfac_expert_combine_backward(route, dy, ys, w, dys, dw)
    want_dys, want_dw = eo.expert_combine_backward(f64(dy), f64(ys), f64(w), place, np.full((T * K, D), 77.0))
    assert (np.abs(f64(dys) - want_dys) <= (U + h) * np.abs(want_dys) * (1 + h) + TINY[t]).all()
    _, size = eo.expert_combine_backward(np.abs(f64(dy)), np.abs(f64(ys)), np.ones((T, K)), place, np.zeros((T * K, D)))
    assert (np.abs(f64(dw) - want_dw) <= (D / 64 + 16) * U * size).all()
    assert bool((whole[:, :gap // 2] == 77).all()) and bool((whole[:, gap // 2 + D:] == 77).all())
    # without weights and without the router's gradient: the rows' copies
    alone = torch.full((T * K, D), 77.0, dtype=t, device=DEV)
    kb.kfac_expert_combine_backward(route, dy, None, None, alone)
    np.testing.assert_array_equal(f64(alone), eo.expert_dispatch(f64(dy), place, np.full((T * K, D), 77.0)))


def test_gradients_against_differences():
    """d<dy, combine(ys, w)> along random directions of ys and w, of one choice twice, in fp32: the function is linear in ys and in w, so
    that differences are exact up to roundings: 1e-5 of the sum of the terms' sizes (2 K D roundings of 2^-24 each at the most)."""
    T, K, E, D = 20, 3, 4, 50
    expert = torch.randint(0, E, (T, K), dtype=torch.int32)
    expert[:, 1] = expert[:, 0]                                # the same expert twice
    route = kb.ExpertRoute(T, K, E)
    kb.kfac_expert_sort(route, expert.to(DEV))
    ys, dy, along = rows_of(T * K, D, torch.float32, 0, 5), rows_of(T, D, torch.float32, 0, 6), rows_of(T * K, D, torch.float32, 0, 7)
    w, dirw = torch.rand((T, K), device=DEV), torch.randn((T, K), device=DEV)
    dys, dw = torch.zeros_like(ys), torch.zeros_like(w)
    kb.kfac_expert_combine_backward(route, dy, ys, w, dys, dw)

    def loss(ys, w):
        y = kb.kfac_expert_combine(route, ys, w, torch.empty((T, D), device=DEV))
        return float((y.double() * dy.double()).sum())

    for plus, minus, want in ((loss(ys + along, w), loss(ys - along, w), float((dys.double() * along.double()).sum())),
                              (loss(ys, w + dirw), loss(ys, w - dirw), float((dw.double() * dirw.double()).sum()))):
        assert abs((plus - minus) / 2 - want) <= 1e-5 * T * K * D
    # dispatch: <dxs, dispatch(x + d)> - <dxs, dispatch(x - d)> against the sum back
    x, d, dxs = rows_of(T, D, torch.float32, 0, 8), rows_of(T, D, torch.float32, 0, 9), rows_of(T * K, D, torch.float32, 0, 10)
    sent = [kb.kfac_expert_dispatch(route, v, torch.zeros_like(dxs)).double() for v in (x + d, x - d)]
    dx = kb.kfac_expert_combine(route, dxs, None, torch.empty_like(x))
    assert abs(float(((sent[0] - sent[1]) / 2 * dxs.double()).sum()) - float((dx.double() * d.double()).sum())) <= 1e-5 * T * K * D


def test_places_outside_the_rows_are_none():
    T, K, D = 4, 2, 40
    route = kb.ExpertRoute(T, K, 3)
    route.place.copy_(torch.tensor([[3, -7], [8, 0], [2 ** 31 - 1, -2 ** 31], [5, 7]], dtype=torch.int32))
    place = route.place.cpu().numpy()
    x, ys = rows_of(T, D, torch.bfloat16, 0, 1), rows_of(T * K, D, torch.bfloat16, 0, 2)
    xs, ok = guarded((T * K, D), torch.bfloat16, 5.0)
    kb.kfac_expert_dispatch(route, x, xs)
    np.testing.assert_array_equal(f64(xs), eo.expert_dispatch(f64(x), place, np.full((T * K, D), 5.0)))
    y = kb.kfac_expert_combine(route, ys, None, torch.empty_like(x))
    want = eo.expert_combine(f64(ys), None, place, D)
    assert (np.abs(f64(y) - want) <= 2 * U * 8 + 2.0 ** -8 * np.abs(want)).all() and ok()
    dw = torch.ones((T, K), device=DEV)
    kb.kfac_expert_combine_backward(route, x, ys, None, xs, dw)
    assert ok() and dw[0, 1] == 0 and dw[1, 0] == 0 and bool((dw[2] == 0).all()) and dw[0, 0] != 0


def test_rows_beyond_32_bits():
    """Rows 2^27 elements apart, 40 of them: the last one begins 10 GB in."""
    T, K, D, ld = 20, 2, 33, 1 << 27
    store = torch.empty((T * K - 1) * ld + D, dtype=torch.bfloat16, device=DEV)
    far = store.as_strided((T * K, D), (ld, 1))
    route, place = routed(T, K, 3, 0.0, 1)
    x = rows_of(T, D, torch.bfloat16, 0, 1)
    kb.kfac_expert_dispatch(route, x, far)
    want = eo.expert_dispatch(f64(x), place, np.zeros((T * K, D)))
    np.testing.assert_array_equal(f64(far), want)
    y = kb.kfac_expert_combine(route, far, None, torch.empty_like(x))
    np.testing.assert_array_equal(f64(y), 2 * f64(x))
    tokens = store.as_strided((T, D), (2 * ld, 1))
    tokens.copy_(x)
    near = torch.zeros((T * K, D), dtype=torch.bfloat16, device=DEV)
    kb.kfac_expert_dispatch(route, tokens, near)
    np.testing.assert_array_equal(f64(near), want)


# ---- factors --------------------------------------------------------------------------------------------------------
def bounds(rows, E, how, seed):
    rng = np.random.default_rng(seed)
    if how == "even":
        cut = np.linspace(0, rows, E + 1).astype(np.int64)
    elif how == "one":                                         # all rows are the last but one's
        cut = np.array([0] * (E - 1) + [rows] * 2)[-E - 1:]
    else:                                                      # some empty, some behind the last one
        cut = np.concatenate([[0], np.sort(rng.integers(0, rows + 1, E))])
        cut[E // 2:] = np.maximum(cut[E // 2:], cut[E // 2])
        cut[1:E // 2] = cut[1:E // 2] // 3
    return np.sort(cut)


def check_factor(got, want, ema=False):
    assert not np.isnan(got).any()
    for e in range(got.shape[0]):
        norm, top = np.linalg.norm(want[e]), np.abs(want[e]).max()
        extra = 2e-7 * top if ema else 0.0
        assert np.linalg.norm(got[e] - want[e]) <= FACTOR_TOL * norm + extra * got.shape[1], e
        assert np.abs(got[e] - want[e]).max() <= FACTOR_TOL * top + extra, e


FACTORS = [(1, 1, 1, False), (1, 3, 8, True), (0, 4, 16, True), (7, 2, 5, True), (33, 5, 64, False), (100, 3, 65, True), (130, 4, 128, True), (300, 7, 129, False), (512, 8, 256, True),
           (900, 19, 77, True), (1000, 300, 32, False), (1500, 2, 260, False), (2500, 3, 577, True), (5000, 1, 96, True), (9000, 3, 40, False), (12000, 2, 200, True)]


@pytest.mark.parametrize("how", ["even", "uneven", "one"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,E,dim,bias", FACTORS)
def test_factor(rows, E, dim, bias, dtype, how):
    x = rows_of(max(rows, 1), dim, TYPES[dtype], 0, rows + dim)[:rows].relu()
    cut = bounds(rows, E, how, rows)
    x[int(cut[-1]):] = float("nan")                            # rows behind the last expert's
    offsets = torch.tensor(cut, dtype=torch.int32, device=DEV)
    want = eo.expert_factor(f64(x), cut, bias)
    d = dim + int(bias)
    plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype], has_bias=bias)
    out, ok = guarded((E, d, d), torch.float32, float("nan"))
    if plan.ws is not None:
        plan.ws.fill_(255)                                     # (NaN)
    kb.kfac_expert_factor(plan, x, offsets, out=out)
    got = f64(out)
    check_factor(got, want)
    assert ok()
    assert torch.equal(out, out.transpose(1, 2))
    again = torch.empty_like(out)
    kb.kfac_expert_factor(plan, x, offsets, out=again)
    assert torch.equal(again, out)
    # the running average, bit for bit that of a stored factor, and as it was without rows
    S = torch.randn((E, d, d), device=DEV)
    S = S + S.transpose(1, 2)
    both = S.clone()
    for e in range(E):
        if cut[e + 1] > cut[e]:
            kb.kfac_ema(both[e], out[e].contiguous(), d, 0.9)
    kb.kfac_expert_factor(plan, x, offsets, running=S, decay=0.9)
    assert torch.equal(S, both)
    # the packed triangles
    tri = kb.ExpertFactors(rows, E, dim, TYPES[dtype], has_bias=bias, packed=True)
    packed, ok = guarded(tri.shape, torch.float32, float("nan"))
    kb.kfac_expert_factor(tri, x, offsets, out=packed)
    i, j = torch.triu_indices(d, d, device=DEV)
    assert torch.equal(packed, out[:, i, j]) and ok()
    # a given scale
    kb.kfac_expert_factor(plan, x, offsets, scale=0.125, out=again)
    check_factor(f64(again), eo.expert_factor(f64(x), cut, bias, scale=0.125))


@pytest.mark.parametrize("dtype,dim,gap", [("bf16", 64, 8), ("bf16", 60, 4), ("bf16", 61, 2), ("f32", 30, 2), ("f32", 29, 2), ("f16", 131, 5)])
def test_factor_of_rows_with_gaps(dtype, dim, gap):
    rows, E = 400, 3
    wide = rows_of(rows, dim + gap, TYPES[dtype], 0, dim)
    wide[:, dim:] = float("nan")
    x = wide[:, :dim]
    cut = bounds(rows, E, "uneven", 1)
    plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype], ld=dim + gap)
    out = torch.empty(plan.shape, device=DEV)
    kb.kfac_expert_factor(plan, x, torch.tensor(cut, dtype=torch.int32, device=DEV), out=out)
    check_factor(f64(out), eo.expert_factor(f64(x), cut))


@pytest.mark.parametrize("rows,E,dim,dtype", [(40000, 6, 512, "bf16"), (30000, 4, 384, "f16"), (70000, 3, 64, "bf16"), (20000, 3, 136, "f32"), (65536, 16, 768, "bf16")])
def test_factor_of_many_rows(rows, E, dim, dtype):
    """Several ranges to an expert, 256-wide tiles, and ranges by the dozen; the reference on the GPU in 64 bits."""
    x = rows_of(rows, dim, TYPES[dtype], 0, dim).relu()
    for how in ("even", "uneven", "one"):
        cut = bounds(rows, E, how, dim)
        offsets = torch.tensor(cut, dtype=torch.int32, device=DEV)
        plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype], has_bias=True)
        out = torch.full(plan.shape, float("nan"), device=DEV)
        kb.kfac_expert_factor(plan, x, offsets, out=out)
        assert torch.equal(out, out.transpose(1, 2))
        S = torch.eye(dim + 1, device=DEV).repeat(E, 1, 1)
        kb.kfac_expert_factor(plan, x, offsets, running=S, decay=0.9)
        for e in range(E):
            a = x[int(cut[e]):int(cut[e + 1])].double()
            n = a.shape[0]
            a = torch.cat([a, a.new_ones((n, 1))], 1)
            want = torch.mm(a.t().contiguous(), a) / max(n, 1)
            check_factor(f64(out[e:e + 1]), f64(want)[None])
            new = 0.9 * torch.eye(dim + 1, device=DEV).double() + 0.1 * want if n else torch.eye(dim + 1, device=DEV)
            check_factor(f64(S[e:e + 1]), f64(new)[None], ema=True)


@pytest.mark.parametrize("rows,E,dim,dtype", [(60000, 60, 768, "bf16"), (60000, 90, 640, "f16"), (30000, 90, 384, "f32"), (60000, 700, 200, "bf16"),
                                               (65536, 20, 1280, "bf16"), (40000, 14, 1536, "f16"), (65536, 70, 512, "bf16")])
def test_factor_tiles_dealt_by_work(rows, E, dim, dtype):
    """More tiles than the chip takes in two rounds, of experts of few, of many and of all the rows, one and several experts to a lane of the
    search: every expert against the reference on the GPU in 64 bits."""
    x = rows_of(rows, dim, TYPES[dtype], 0, dim).relu()
    rng = np.random.default_rng(dim)
    share = np.exp(2 * rng.standard_normal(E))
    skewed = np.concatenate([[0], np.minimum(np.round(np.cumsum(share / share.sum()) * rows), rows)]).astype(np.int64)
    for cut in (bounds(rows, E, "even", 0), bounds(rows, E, "uneven", dim), bounds(rows, E, "one", 0), skewed):
        offsets = torch.tensor(cut, dtype=torch.int32, device=DEV)
        plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype])
        out = torch.full(plan.shape, float("nan"), device=DEV)
        kb.kfac_expert_factor(plan, x, offsets, out=out)
        S = torch.eye(dim, device=DEV).repeat(E, 1, 1)
        kb.kfac_expert_factor(plan, x, offsets, running=S, decay=0.5)
        for e in range(E):
            n = int(cut[e + 1] - cut[e])
            if n == 0:
                assert not bool(out[e].any()) and torch.equal(S[e], torch.eye(dim, device=DEV))
                continue
            a = x[int(cut[e]):int(cut[e + 1])].double()
            want = torch.mm(a.t().contiguous(), a) / n
            off = out[e].double() - want
            assert float(off.norm()) <= FACTOR_TOL * float(want.norm()) and float(off.abs().max()) <= FACTOR_TOL * float(want.abs().max()), e
            new = 0.5 * torch.eye(dim, device=DEV).double() + 0.5 * want
            assert float((S[e].double() - new).abs().max()) <= (FACTOR_TOL + 2e-7) * float(new.abs().max()), e


@pytest.mark.parametrize("dtype,dim", [("bf16", 512), ("f32", 448), ("bf16", 192), ("f16", 208), ("bf16", 720)])
def test_factor_results_past_the_caches(dtype, dim):
    """Results of more than 120 MB, in rows of whole halves of cache lines (another kernel, its name says so), against fewer experts' (the same bits)."""
    E, per = (130 << 20) // (4 * dim * dim), 50
    x = rows_of(E * per, dim, TYPES[dtype], 0, dim)
    offsets = torch.arange(0, E * per + 1, per, dtype=torch.int32, device=DEV)
    S = torch.randn((E, dim, dim), device=DEV)
    S = S + S.transpose(1, 2)
    want = S.clone()
    out = torch.empty_like(S)
    plan = kb.ExpertFactors(E * per, E, dim, TYPES[dtype])
    kb.kfac_kernel_timing_enable(True)
    try:
        kb.kfac_expert_factor(plan, x, offsets, out=out)
        kb.kfac_expert_factor(plan, x, offsets, running=S, decay=0.9)
        assert any("stream>" in k for k in kb.kfac_kernel_timing_report())
    finally:
        kb.kfac_kernel_timing_enable(False)
    some = 3
    few = kb.ExpertFactors(some * per, some, dim, TYPES[dtype])
    part = torch.empty((some, dim, dim), device=DEV)
    for e in (0, E // 2, E - some):
        kb.kfac_expert_factor(few, x[e * per:(e + some) * per], offsets[:some + 1], out=part)
        assert torch.equal(out[e:e + some], part)
        kb.kfac_expert_factor(few, x[e * per:(e + some) * per], offsets[:some + 1], running=want[e:e + some], decay=0.9)
        assert torch.equal(S[e:e + some], want[e:e + some])


def test_factor_of_rows_beyond_32_bits():
    """Rows 2^17 elements apart: the last of 36,000 begins 9.4 GB in."""
    rows, E, dim, ld = 36000, 3, 48, 1 << 17
    store = torch.empty((rows - 1) * ld + dim, dtype=torch.bfloat16, device=DEV)
    far = store.as_strided((rows, dim), (ld, 1))
    near = rows_of(rows, dim, torch.bfloat16, 0, 1)
    far.copy_(near)
    offsets = torch.tensor([0, 20000, 20000, 35999], dtype=torch.int32, device=DEV)
    out, want = torch.empty((E, dim, dim), device=DEV), torch.empty((E, dim, dim), device=DEV)
    kb.kfac_expert_factor(kb.ExpertFactors(rows, E, dim, torch.bfloat16, ld=ld), far, offsets, out=out)
    kb.kfac_expert_factor(kb.ExpertFactors(rows, E, dim, torch.bfloat16), near, offsets, out=want)
    assert torch.equal(out, want)


def test_factor_offsets_are_cut_off():
    rows, E, dim = 100, 3, 24
    x = rows_of(rows, dim, torch.float32, 0, 1)
    plan = kb.ExpertFactors(rows, E, dim, torch.float32)
    got, want = torch.empty(plan.shape, device=DEV), torch.empty(plan.shape, device=DEV)
    for wild, tame in (([-5, 40, 150, 200], [0, 40, 100, 100]), ([0, 40, 40, 2 ** 31 - 1], [0, 40, 40, 100])):
        kb.kfac_expert_factor(plan, x, torch.tensor(wild, dtype=torch.int32, device=DEV), out=got)
        kb.kfac_expert_factor(plan, x, torch.tensor(tame, dtype=torch.int32, device=DEV), out=want)
        assert torch.equal(got, want)


def test_factor_of_values_that_are_not_finite():
    """They stay with their expert and their columns."""
    rows, E, dim = 64, 4, 40
    x = rows_of(rows, dim, torch.bfloat16, 0, 1)
    cut = [0, 16, 32, 48, 64]
    x[20, 3] = float("inf")
    plan = kb.ExpertFactors(rows, E, dim, torch.bfloat16)
    out = torch.empty(plan.shape, device=DEV)
    kb.kfac_expert_factor(plan, x, torch.tensor(cut, dtype=torch.int32, device=DEV), out=out)
    finite = torch.isfinite(out).cpu().numpy()
    want = np.ones((E, dim, dim), bool)
    want[1, 3, :] = want[1, :, 3] = False
    np.testing.assert_array_equal(finite, want)


# ---- use ------------------------------------------------------------------------------------------------------------
def test_bindings_refuse():
    route = kb.ExpertRoute(6, 2, 3)
    bf = torch.bfloat16
    expert = torch.zeros((6, 2), dtype=torch.int32, device=DEV)
    x, xs, w = torch.zeros((6, 16), dtype=bf, device=DEV), torch.zeros((12, 16), dtype=bf, device=DEV), torch.zeros((6, 2), device=DEV)
    plan = kb.ExpertFactors(12, 3, 16, bf)
    F = torch.zeros(plan.shape, device=DEV)
    calls = [lambda: kb.kfac_expert_sort(route, expert.long()), lambda: kb.kfac_expert_sort(route, expert.t().contiguous().t()),
             lambda: kb.kfac_expert_sort(route, expert[:5]), lambda: kb.kfac_expert_sort(route, expert.cpu()),
             lambda: kb.kfac_expert_dispatch(route, x.double(), xs), lambda: kb.kfac_expert_dispatch(route, x, xs.float()),
             lambda: kb.kfac_expert_dispatch(route, x[:5], xs), lambda: kb.kfac_expert_dispatch(route, x, xs[:11]),
             lambda: kb.kfac_expert_dispatch(route, x[:, :8], xs), lambda: kb.kfac_expert_dispatch(route, x[:1].expand(6, 16), xs),
             lambda: kb.kfac_expert_dispatch(route, x.t().contiguous().t(), xs), lambda: kb.kfac_expert_dispatch(route, x.cpu(), xs.cpu()),
             lambda: kb.kfac_expert_combine(route, xs, w.double(), x), lambda: kb.kfac_expert_combine(route, xs, w[:5], x),
             lambda: kb.kfac_expert_combine(route, xs, w.cpu(), x), lambda: kb.kfac_expert_combine_backward(route, x, None, w, xs, w),
             lambda: kb.kfac_expert_combine_backward(route, x, torch.zeros((12, 20), dtype=bf, device=DEV), w, xs, w.clone()),
             lambda: kb.kfac_expert_combine_backward(route, x, xs, w, torch.zeros((12, 16), device=DEV), w.clone()),
             lambda: kb.kfac_expert_factor(plan, xs.float(), route.offsets, out=F), lambda: kb.kfac_expert_factor(plan, xs[:11], route.offsets, out=F),
             lambda: kb.kfac_expert_factor(plan, xs, route.offsets.long(), out=F), lambda: kb.kfac_expert_factor(plan, xs, route.offsets[:3], out=F),
             lambda: kb.kfac_expert_factor(plan, xs, route.offsets), lambda: kb.kfac_expert_factor(plan, xs, route.offsets, out=F, running=F),
             lambda: kb.kfac_expert_factor(plan, xs, route.offsets, out=F[:2]), lambda: kb.kfac_expert_factor(plan, xs, route.offsets, out=F.double()),
             lambda: kb.kfac_expert_factor(plan, xs, route.offsets, running=F, decay=2.0),
             lambda: kb.ExpertRoute(6, 2, 3, place=torch.zeros((6, 2), device=DEV)), lambda: kb.ExpertRoute(-1, 2, 3),
             lambda: kb.ExpertFactors(12, 3, 16, torch.float64)]
    for k, call in enumerate(calls):
        with pytest.raises(kb.KfacError) as e:
            call()
        assert e.value.status == kb.KFAC_ERR_INVALID_ARG, k


def test_captured_and_replayed_on_another_stream():
    """Sort, dispatch, weighted sum, gradients and factors in one graph, replayed on new tokens with eager calls between, each replay against
    the same calls made eagerly; then both at once on two streams."""
    T, K, E, D = 3000, 3, 7, 200
    bf = torch.bfloat16

    def state():
        s = {"expert": torch.zeros((T, K), dtype=torch.int32, device=DEV), "x": torch.zeros((T, D), dtype=bf, device=DEV), "w": torch.zeros((T, K), device=DEV),
             "xs": torch.zeros((T * K, D), dtype=bf, device=DEV), "y": torch.zeros((T, D), dtype=bf, device=DEV),
             "dys": torch.zeros((T * K, D), dtype=bf, device=DEV), "dw": torch.zeros((T, K), device=DEV)}
        s["route"], s["plan"] = kb.ExpertRoute(T, K, E), kb.ExpertFactors(T * K, E, D, bf, has_bias=True)
        s["F"] = torch.zeros(s["plan"].shape, device=DEV)
        return s

    def fill(s, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        s["expert"].copy_(torch.randint(-1, E, (T, K), generator=g, device=DEV, dtype=torch.int32))
        s["x"].copy_(torch.randn((T, D), generator=g, device=DEV))
        s["w"].copy_(torch.rand((T, K), generator=g, device=DEV))
        s["xs"].zero_()
        s["dys"].zero_()

    def calls(s):
        r = kb.kfac_expert_sort(s["route"], s["expert"])
        kb.kfac_expert_dispatch(r, s["x"], s["xs"])
        kb.kfac_expert_combine(r, s["xs"], s["w"], s["y"])
        kb.kfac_expert_combine_backward(r, s["x"], s["xs"], s["w"], s["dys"], s["dw"])
        kb.kfac_expert_factor(s["plan"], s["xs"], r.offsets, out=s["F"])

    outs = ("xs", "y", "dys", "dw", "F")
    a, b = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fill(a, 0)
    with torch.cuda.stream(side):
        calls(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(a)
    for seed in (1, 2, 3, 4):
        fill(a, seed)
        fill(b, seed)
        graph.replay()
        calls(b)
        torch.cuda.synchronize()
        for name in outs:
            assert torch.equal(a[name], b[name]), (seed, name)
        assert torch.equal(a["route"].order, b["route"].order)
    want = {name: b[name].clone() for name in outs}
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            calls(b)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for name in outs:
        assert torch.equal(a[name], want[name]) and torch.equal(b[name], want[name]), name


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_side_by_side_in_one_buffer(dtype):
    """Tensors whose rows lie in each other's gaps, without a common element, are apart."""
    T, K, E, D = 90, 3, 4, 72
    route, _ = routed(T, K, E, 0.1, 5)
    dy, w = rows_of(T, D, TYPES[dtype], 0, 1), torch.rand((T, K), device=DEV)
    apart = [rows_of(T * K, D, TYPES[dtype], 0, 2), torch.full((T * K, D), 5.0, dtype=TYPES[dtype], device=DEV)]
    both = torch.cat(apart, 1)
    dw = [torch.zeros((T, K), device=DEV) for _ in range(2)]
    kb.kfac_expert_combine_backward(route, dy, apart[0], w, apart[1], dw[0])
    kb.kfac_expert_combine_backward(route, dy, both[:, :D], w, both[:, D:], dw[1])
    assert torch.equal(both, torch.cat(apart, 1)) and torch.equal(dw[0], dw[1])


def test_factor_of_rows_off_the_16_byte_grid():
    """Rows of whole vectors are read as they lie and have to begin on the grid: the refusal says so.  Others are copied, wherever they begin."""
    bf, rows, E = torch.bfloat16, 12, 3
    base = torch.randn(rows * 16 + 4, device=DEV).to(bf)
    offsets = torch.tensor([0, 5, 5, 12], dtype=torch.int32, device=DEV)
    plan = kb.ExpertFactors(rows, E, 16, bf)
    out = torch.empty(plan.shape, device=DEV)
    for at in (1, 4):
        with pytest.raises(kb.KfacError, match="16-byte") as e:
            kb.kfac_expert_factor(plan, base[at:at + rows * 16].view(rows, 16), offsets, out=out)
        assert e.value.status == kb.KFAC_ERR_INVALID_ARG
    kb.kfac_expert_factor(plan, base[:rows * 16].view(rows, 16), offsets, out=out)
    check_factor(f64(out), eo.expert_factor(f64(base[:rows * 16].view(rows, 16)), offsets.tolist()))
    odd = kb.ExpertFactors(rows, E, 15, bf)
    out = torch.empty(odd.shape, device=DEV)
    for at in (0, 1, 4):
        x = base[at:at + rows * 15].view(rows, 15)
        kb.kfac_expert_factor(odd, x, offsets, out=out)
        check_factor(f64(out), eo.expert_factor(f64(x), offsets.tolist()))


@pytest.mark.parametrize("rows,E,dim,dtype,name", [(64, 2, 64, "bf16", "<64, 16-bit>"), (64, 2, 48, "f32", "<64, f32>"), (1024, 8, 256, "f32", "<64, f32>"),
                                                   (20000, 200, 128, "f16", "<128, 16-bit>"), (20000, 200, 128, "f32", "<128, f32>"),
                                                   (65536, 16, 768, "bf16", "<256, 16-bit>"), (21350, 854, 192, "bf16", "<64, 16-bit, stream>")])
def test_timings_name_the_width_of_the_tiles(rows, E, dim, dtype, name):
    plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype])
    x = torch.zeros((rows, dim), dtype=TYPES[dtype], device=DEV)
    out = torch.empty(plan.shape, device=DEV)
    offsets = torch.arange(E + 1, device=DEV).mul_(rows // E).to(torch.int32)
    kb.kfac_kernel_timing_enable(True)
    try:
        kb.kfac_expert_factor(plan, x, offsets, out=out)
        assert "expert_tile_kernel" + name in kb.kfac_kernel_timing_report()
    finally:
        kb.kfac_kernel_timing_enable(False)


# ---- kernels that larger or longer calls take --------------------------------------------------------------------------
@pytest.mark.parametrize("how", ["even", "skewed", "dropped", "one", "none"])
@pytest.mark.parametrize("T,K,E", [(65536, 8, 256), (65535, 8, 256), (150000, 2, 64), (100001, 2, 700), (150001, 2, 1000), (150000, 2, 1000), (500000, 2, 37),
                                   (499999, 2, 37), (500000, 2, 300), (800000, 2, 512), (1048576, 2, 64)])
def test_sort_of_several_runs_of_several_steps(T, K, E, how):
    """Runs of many workgroups whose wavefronts hold two to eight steps of assignments in registers, whole and cut; of 256 and more experts counted
    several runs at a time."""
    test_sort(T, K, E, how)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,E,D,gap,drop", [(700, 3, 5, 1001, 0, 0.1), (600, 2, 4, 1001, 6, 0.1), (513, 5, 9, 520, 0, 0.2)])
def test_rows_of_several_vectors_to_a_lane(T, K, E, D, gap, drop, dtype):
    """More tokens than a workgroup each is taken for, rows of 65 to 255 vectors: a wavefront goes over a token's row several times."""
    test_dispatch(T, K, E, D, gap, drop, dtype)
    test_combine(T, K, E, D, gap, drop, dtype, True)
    test_combine_backward(T, K, E, D, gap, drop, dtype)


def streaming(call):
    """Runs `call` and says whether it took a kernel whose rows go past the caches."""
    kb.kfac_kernel_timing_enable(True)
    try:
        call()
        return all("stream>" in k for k in kb.kfac_kernel_timing_report())
    finally:
        kb.kfac_kernel_timing_enable(False)


PAST_THE_CACHES = [(16384, 4, 64, 2048, "bf16"), (16300, 4, 64, 2001, "f16"), (9000, 7, 30, 1031, "f32"), (70000, 4, 16, 512, "bf16"), (300000, 2, 5, 128, "f32"),
                   (430000, 4, 64, 64, "f16")]


@pytest.mark.parametrize("T,K,E,D,dtype", PAST_THE_CACHES)
def test_rows_past_the_caches(T, K, E, D, dtype):
    """Calls that move more than 256 MB, whole and odd widths, some assignments dropped, against the same in 64 bits on the GPU."""
    t = TYPES[dtype]
    h = HALF[t]
    g = torch.Generator(device=DEV).manual_seed(D)
    expert = torch.randint(0, E, (T, K), generator=g, device=DEV, dtype=torch.int32)
    expert[torch.rand((T, K), generator=g, device=DEV) < 0.05] = -1
    route = kb.ExpertRoute(T, K, E)
    kb.kfac_expert_sort(route, expert)
    rows = int(route.offsets[E])
    there, at = route.place >= 0, route.place.clamp(min=0).long()
    x, ys, dy = rows_of(T, D, t, 0, 1), rows_of(T * K, D, t, 0, 2), rows_of(T, D, t, 0, 3)
    ys[rows:] = float("nan")
    w = torch.rand((T, K), generator=g, device=DEV) * 2 - 0.5
    w[~there] = float("nan")
    token = route.order[:rows].long() // K
    xs, ok = guarded((T * K, D), t, 5.0)
    assert streaming(lambda: kb.kfac_expert_dispatch(route, x, xs))
    assert torch.equal(xs[:rows], x[token]) and bool((xs[rows:] == 5).all()) and ok()
    del xs
    for weights in (w, None):
        y, ok = guarded((T, D), t, 5.0)
        assert streaming(lambda: kb.kfac_expert_combine(route, ys, weights, y))
        want, size = torch.zeros((T, D), dtype=torch.float64, device=DEV), torch.zeros((T, D), dtype=torch.float64, device=DEV)
        for k in range(K):
            term = ys[at[:, k]].double() * (1.0 if weights is None else w[:, k:k + 1].double())
            term = torch.where(there[:, k:k + 1], term, 0.0)
            want += term
            size += term.abs()
        assert bool(((y.double() - want).abs() <= K * U * size * (1 + h) + h * want.abs() + TINY[t]).all()) and ok()
    for ask in (True, False):
        dys, ok = guarded((T * K, D), t, 5.0)
        dw = torch.full((T, K), float("nan"), device=DEV) if ask else None
        assert streaming(lambda: kb.kfac_expert_combine_backward(route, dy, ys if ask else None, w, dys, dw))
        want = dy[token].double() * w.reshape(-1)[route.order[:rows].long()].double()[:, None]
        assert bool(((dys[:rows].double() - want).abs() <= (U + h) * want.abs() * (1 + h) + TINY[t]).all())
        assert bool((dys[rows:] == 5).all()) and ok()
        for k in range(K if ask else 0):
            term = dy.double() * torch.where(there[:, k:k + 1], ys[at[:, k]].double(), 0.0)
            assert bool(((dw[:, k].double() - term.sum(1)).abs() <= (D / 64 + 16) * U * term.abs().sum(1)).all())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("rows,E,dim,gap,dtype", [(20000, 3, 60, 4, "bf16"), (20000, 3, 61, 2, "bf16"), (9000, 2, 130, 6, "f16"), (9000, 2, 300, 4, "bf16"),
                                                  (8000, 2, 30, 2, "f32"), (8000, 2, 129, 3, "f32"), (7000, 2, 29, 2, "f32")])
def test_factor_of_rows_with_gaps_in_several_ranges(rows, E, dim, gap, dtype, packed):
    """Rows with NaN between them, a bias, and several ranges to an expert: the gaps are of no influence on sums and column sums."""
    wide = rows_of(rows, dim + gap, TYPES[dtype], 0, dim)
    wide[:, dim:] = float("nan")
    x = wide[:, :dim]
    for how in ("even", "uneven", "one"):
        cut = bounds(rows, E, how, 1)
        plan = kb.ExpertFactors(rows, E, dim, TYPES[dtype], has_bias=True, packed=packed, ld=dim + gap)
        plan.ws.fill_(255)                                     # (NaN)
        out = torch.empty(plan.shape, device=DEV)
        kb.kfac_expert_factor(plan, x, torch.tensor(cut, dtype=torch.int32, device=DEV), out=out)
        want = eo.expert_factor(f64(x), cut, True)
        if packed:
            i, j = np.triu_indices(dim + 1)
            full = np.zeros_like(want)
            full[:, i, j] = f64(out)
            full[:, j, i] = f64(out)
            check_factor(full, want)
        else:
            check_factor(f64(out), want)
