"""The full-attention calls at the limits of what they take: values that are infinite or NaN under weights
that vanish, scores of -inf, the largest bf16 values in an e4m3 cache, one workspace for many batches, fp32
tokens in their rarer forms, probabilities that are all rounded one way."""
import numpy as np
import pytest

from oracle import attention as A

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2608_11231_amd import lkv  # noqa: E402
from test_gpu_attn import BF, E4, F32, Cache, _attn_paged, _check_paged, _cum, _i32, _np, _qkv  # noqa: E402

# name: h_q, h_kv, d, io, cache, context, new tokens; SPLIT: calls whose key range is split
SPLIT = {
    "one_token_8_parts": (8, 2, 128, BF, BF, 2000, 1),
    "one_token_36_parts": (8, 2, 128, BF, BF, 9000, 1),
    "drafted_e4m3": (8, 2, 64, BF, E4, 9000, 8),
    "drafted_wide": (8, 2, 256, BF, BF, 9000, 8),
    "chunk": (8, 2, 128, BF, BF, 9000, 60),
    "chunk_many_rows": (8, 2, 64, BF, E4, 9000, 300),
    "chunk_wide_e4m3": (8, 2, 256, BF, E4, 9000, 60),
    "f32_7_parts": (4, 2, 64, F32, F32, 1700, 3),
    "f32_many_parts": (4, 2, 128, F32, F32, 9000, 3),
}
WHOLE = {
    "one_token_whole": (8, 2, 128, BF, BF, 200, 1),
    "chunk_whole": (8, 2, 256, BF, BF, 200, 60),
    "f32_whole": (4, 2, 64, F32, F32, 200, 3),
}
BOTH = {**SPLIT, **WHOLE}


def _layer(name):
    hq, hkv, d, io, cache, ctx, new = BOTH[name]
    attn = lkv.make_attn(hq, hkv, d, page=16, io_dtype=io, cache_dtype=cache)
    width = -(-ctx // 16) + 1
    assert (lkv.attn_paged_workspace(attn, 1, new, width) > 0) == (name in SPLIT)
    q, k, v = _qkv(ctx, hq, hkv, d, io, 7, False)
    q = q[:new].contiguous()
    q[:, :, 0], k[:, :, 0] = 8.0, 0.0
    return attn, Cache(attn, [ctx]), q, k, v, ctx, new


def _over(attn, C, q, k, v):
    n = k.shape[0]
    lkv.kv_write(attn, C.pages, _i32([0, n]), n, k, v)
    return _attn_paged(attn, C, [0, q.shape[0]], q)


def _same_but(good, bad, channels):
    """`bad` is not finite in these channels and `good`'s bits in the others."""
    rest = [c for c in range(good.shape[-1]) if c not in channels]
    assert bool(good.isfinite().all())
    assert not bool(bad[..., channels].isfinite().any())
    assert torch.equal(good[..., rest], bad[..., rest])


@pytest.mark.parametrize("name", BOTH)
def test_values_of_vanishing_weight(name):
    """An infinite or NaN value counts however small its weight is: 0 * NaN is NaN.  One late key outweighs
    the others by 250 nats and more, past what an exponential in fp32 holds."""
    attn, C, q, k, v, ctx, new = _layer(name)
    k[ctx - new - 1, :, 0] = 512.0
    good = _over(attn, C, q, k, v)
    v[3, :, 3], v[ctx // 3, :, 7], v[ctx // 2, :, 9] = float("nan"), float("inf"), float("-inf")
    _same_but(good, _over(attn, C, q, k, v), [3, 7, 9])


@pytest.mark.parametrize("name", [x for x in BOTH if BOTH[x][4] != E4])
@pytest.mark.parametrize("seen", ["half", "none"])
def test_scores_of_minus_infinity(name, seen):
    """Keys whose scores are -inf have no weight, and a token with no other keys gives zeros; a value among
    them that is not finite counts all the same."""
    attn, C, q, k, v, ctx, new = _layer(name)
    k[:ctx // 2 if seen == "half" else ctx, :, 0] = float("-inf")
    good = _over(attn, C, q, k, v)
    if seen == "none":
        assert bool((good == 0).all())
    v[3, :, 3], v[ctx // 3, :, 7] = float("nan"), float("inf")
    _same_but(good, _over(attn, C, q, k, v), [3, 7])


@pytest.mark.parametrize("n", [70, 1100])
@pytest.mark.parametrize("hq,d,io", [(2, 64, BF), (2, 128, BF), (2, 256, BF), (2, 128, F32)])
def test_prefill_scores_of_minus_infinity(n, hq, d, io):
    attn = lkv.make_attn(hq, 1, d, io_dtype=io)
    q, k, v = _qkv(n, hq, 1, d, io, 5, False)
    q[:, :, 0], k[:, :, 0] = 1.0, float("-inf")
    outs = []
    for _ in range(2):
        o = torch.full_like(q, 7.0)
        lkv.attn_prefill(attn, _i32([0, n]), n, q, k, v, o)
        outs.append(o)
        v[20, :, 3] = float("nan")
    torch.cuda.synchronize()
    assert bool((outs[0] == 0).all()) and torch.equal(outs[0][:20], outs[1][:20])
    _same_but(outs[0][20:], outs[1][20:], [3])


def test_a_token_without_keys_beside_values_not_finite():
    """Tokens before the context's start give zeros, whatever their request's values hold."""
    for new, io in ((5, BF), (60, BF), (5, F32)):
        attn = lkv.make_attn(8, 2, 64, page=16, io_dtype=io)
        C = Cache(attn, [3])
        q, k, v = _qkv(new, 8, 2, 64, io, 7, False)
        v[0] = float("nan")
        o = torch.full_like(q, 7.0)
        lkv.kv_write(attn, C.pages, _i32([0, 3]), 3, k, v)
        ws = torch.empty(lkv.attn_paged_workspace(attn, 1, new, 2), dtype=torch.uint8, device="cuda")
        lkv.attn_paged(attn, C.pages, _i32([0, new]), new, q, o, ws)
        torch.cuda.synchronize()
        assert bool((o[:new - 3] == 0).all()) and bool(o[new - 3:].isnan().all())


# ---------------------------------------------------------------- cache
@pytest.mark.parametrize("hkv,d", [(1, 64), (4, 128), (8, 128)])
def test_largest_values_in_e4m3(hkv, d):
    """The largest finite bf16 values stay finite in an e4m3 cache."""
    top = torch.finfo(BF).max
    rows = [[top, -top, 1.0], [248 * 2.0 ** 120, -248 * 2.0 ** 120, 247 * 2.0 ** 120], [240 * 2.0 ** 120, 3e38, -3e38],
            [top, float("inf"), float("nan")], [224 * 2.0 ** 120, 225 * 2.0 ** 120, 2.0 ** 127], [2.0 ** 127, top, 0.0]]
    n = len(rows)
    x = torch.zeros((n, hkv, d), dtype=BF)
    x[:, :, :3] = torch.tensor(rows, dtype=torch.float64).to(BF)[:, None]
    k, v = x.cuda(), x.flip(0).cuda()
    attn = lkv.make_attn(hkv, hkv, d, page=16, cache_dtype=E4)
    C = Cache(attn, [n])
    lkv.kv_write(attn, C.pages, _i32([0, n]), n, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    lkv.kv_read(attn, C.pages, _i32([0, n]), n, ko, vo)
    torch.cuda.synchronize()
    for a, b in ((k, ko), (v, vo)):
        want = A.e4m3_values(*A.e4m3_rows(_np(a)))
        assert np.array_equal(_np(b), want, equal_nan=True)
        assert bool((b.isfinite() == a.isfinite()).all())


# ---------------------------------------------------------------- workspace
def test_one_workspace_for_every_batch():
    """A workspace by the bound of the largest batch serves the smaller ones, which need more of it."""
    attn = lkv.make_attn(8, 2, 128, page=16)
    rng = np.random.default_rng(5)
    C = Cache(attn, [int(c) for c in rng.integers(1, 4000, 600)])
    C.fill()
    width = C.table.shape[1]
    ws = torch.empty(lkv.attn_paged_workspace_bound(attn, 600, width), dtype=torch.uint8, device="cuda")
    assert lkv.attn_paged_workspace(attn, 600, 600, width) < lkv.attn_paged_workspace(attn, 7, 420, width) <= ws.numel()
    for n_req, m in ((600, 1), (40, 5), (7, 60), (1, 600), (1, 1)):
        q = _qkv(n_req * m, 8, 1, 128, BF, n_req)[0]
        cu = np.arange(n_req + 1) * m
        want = _attn_paged(attn, C, cu, q)
        o, ws[:] = torch.full_like(want, 7.0), 255
        lkv.attn_paged(attn, C.pages, _i32(cu), n_req * m, q, o, ws)
        torch.cuda.synchronize()
        assert torch.equal(o, want)


@pytest.mark.parametrize("hkv,d,page", [(3, 128, 32), (9, 64, 16), (5, 128, 1024)])
def test_write_and_read_of_many_fp32_heads(hkv, d, page):
    """Tokens that a whole wave moves, in more than one round of its lanes among them."""
    attn = lkv.make_attn(hkv, hkv, d, page=page, io_dtype=F32)
    ctx, new = [300, 0, 90, 1], [130, 0, 90, 1]
    C = Cache(attn, ctx)
    rng = np.random.default_rng(3)
    pos = np.concatenate([rng.choice(c, m, replace=False) for c, m in zip(ctx, new)]).astype(np.int32)
    pos[[4, 140]] = [300, -1]
    n = sum(new)
    _, k, v = _qkv(n + 2, 1, hkv, d, F32, 4)
    ko, vo = (torch.full((n + 2, hkv, d), 7.0, device="cuda") for _ in range(2))
    at = _i32(np.append(pos, [0, 0]))
    lkv.kv_write(attn, C.pages, _i32(_cum(new)), n + 2, k, v, at)
    lkv.kv_read(attn, C.pages, _i32(_cum(new)), n + 2, ko, vo, at)
    torch.cuda.synchronize()
    for x, o in ((k, ko), (v, vo)):
        want = _np(x)
        want[[4, 140]] = np.nan
        want[n:] = 7.0
        assert np.array_equal(_np(o), want, equal_nan=True)
    assert int((~C.k.isnan()).all(-1).all(1).sum()) == n - 2


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("ctx,new", [([9000], [1]), ([12000, 5, 3000], [3, 7, 1])], ids=str)
def test_fp32_over_many_parts(hq, hkv, d, ctx, new):
    """Few fp32 rows over more than eight parts of the key range, rows that see nothing among them."""
    attn = lkv.make_attn(hq, hkv, d, page=64, io_dtype=F32)
    C = Cache(attn, ctx)
    size = lkv.attn_paged_workspace(attn, len(ctx), sum(new) + 1, C.table.shape[1])
    assert size > 8 * (sum(new) + 1) * hq * (4 * d + 8) + 256 and (sum(new) + 1) * hq < 1024
    C.fill()
    q = _qkv(sum(new) + 1, hq, 1, d, F32, 6)[0]
    o = _attn_paged(attn, C, _cum(new), q)
    _check_paged(attn, C, new, q, o)
    assert bool((o[sum(new):] == 7.0).all())


def _one_way_keys(n_one, n_down):
    """Keys of scores s (q = 1, 1, 0 ..): exp(s) = 1, then just below 1 + 2^-8, which bf16 rounds down to 1,
    and a last one just above, rounded up to 1 + 2^-7."""
    tie = np.log1p(2.0 ** -8)
    s = np.concatenate([np.zeros(n_one), np.full(n_down, tie - 2e-6), [tie + 2e-6]])
    hi = torch.from_numpy(s).to(BF)
    lo = (torch.from_numpy(s) - hi.double()).to(BF)
    k = torch.zeros((len(s), 1, 64), dtype=BF)
    k[:, 0, 0], k[:, 0, 1] = hi, lo
    return k


@pytest.mark.parametrize("call,n_req,m", [("prefill", 1, 6257), ("one_token", 2048, 1), ("chunk", 350, 130)])
def test_probabilities_rounded_one_way(call, n_req, m):
    """Tolerance: a probability is off by 2^-8 of itself at most, and so is their sum (which is of the rounded
    ones, so that weights add up to 1): 2 * 2^-8 of A = sum_j p_j |v_j| for the weights, 2^-8 for the
    output, and 2^-10 for products of these and all that is fp32.  Here the roundings add up: nearly all
    probabilities are rounded down, and that of the one key with a value, up.  The requests share their
    pages and are as many as leave the key range whole."""
    k = _one_way_keys(256, 6000).cuda()
    n = k.shape[0]
    v = torch.zeros((n, 1, 64), dtype=BF, device="cuda")
    v[-1, 0] = torch.linspace(1, 2, 65)[:64].to(BF).cuda()
    q = torch.zeros((n_req * m, 2, 64), dtype=BF, device="cuda")
    q[:, :, :2] = 1.0
    attn = lkv.make_attn(2, 1, 64, scale=1.0, page=64)
    o = torch.full_like(q, 7.0)
    if call == "prefill":
        lkv.attn_prefill(attn, _i32([0, n]), n, q, k, v, o)
    else:
        C = Cache(attn, [n])
        lkv.kv_write(attn, C.pages, _i32([0, n]), n, k, v)
        pages = lkv.make_pages(attn, C.k, C.v, _i32(np.repeat(C.table, n_req, 0)), _i32([n] * n_req))
        assert lkv.attn_paged_workspace(attn, n_req, n_req * m, C.table.shape[1]) == 0
        lkv.attn_paged(attn, pages, _i32(np.arange(n_req + 1) * m), n_req * m, q, o, None)
    torch.cuda.synchronize()
    ref, mag, _ = A.attention(_np(q[-1:]), _np(k), _np(v), [n - 1], 1.0)
    last = o.view(n_req, m, 2, 64)[:, -1]
    assert bool((last == last[:1]).all()) and bool((o.view(n_req, m, 2, 64)[:, :-1] == 0).all())
    assert np.max(np.abs(_np(last[:1]) - ref) / mag) <= 3 * 2.0 ** -8 + 2.0 ** -10
