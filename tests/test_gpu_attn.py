"""GPU parity of the full-attention layers' calls against the fp64 oracle.

Tolerances, per element, with A = sum_j p_j |v_j| (the oracle gives it): with bf16 tokens every
probability is rounded to bf16 once (relative 2^-8 at most) and the output once (2^-8 of |o| <=
A); the fp32 scores, exponentials and sums add less than 2^-10 of A.  With fp32 tokens a score is
off by at most d 2^-24 sum |q_e k_e| scale, which enters p and its normalisation once each, and
sums of n terms by n 2^-24."""
import numpy as np
import pytest

from oracle import attention as A

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2608_11231_amd import lkv  # noqa: E402

BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def _close(got, ref, f32=False, n=1, d=1):
    o, mag, dot = ref
    if f32:
        tol = (2 * d * dot[..., None] + 2 * n + 16) * 2.0 ** -24 * mag
    else:
        tol = (2 * 2.0 ** -8 + 2.0 ** -10) * mag
    err = np.abs(got.double().cpu().numpy() - o)
    worst = np.max(err - tol) if err.size else -1.0
    assert not np.isnan(err).any() and worst <= 1e-30, (worst, np.max(err))


def _np(t):
    return t.double().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _cum(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _qkv(n, hq, hkv, d, io, seed=0, fused=True):
    """q, k, v of n tokens, views of one projection's output or apart; fused rows carry a NaN tail
    that no call may touch."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, (hq + 2 * hkv) * d), generator=g).to(io)
    if fused:
        y = torch.full((n, (hq + 2 * hkv) * d + 8), float("nan"), dtype=io)
        y[:, :-8] = x
        y = y.cuda()
    else:
        y = x.cuda()
    out = [y[:, a * d:b * d].view(n, b - a, d) if fused else y[:, a * d:b * d].reshape(n, b - a, d).contiguous()
           for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
    return out


class Cache:
    """A paged cache on the GPU whose slots hold NaN until written, and its requests."""

    def __init__(self, attn, ctx, seed=0, spare=2, pad=1):
        rng = np.random.default_rng(seed)
        need = [-(-c // attn.page) for c in ctx]
        n_page, wide = sum(need) + spare, max(need + [0]) + pad
        perm = list(rng.permutation(n_page))
        self.table = np.full((len(ctx), wide), -7, np.int32)
        for r, m in enumerate(need):
            self.table[r, :m] = [perm.pop() for _ in range(m)]
        self.ctx, self.attn = list(ctx), attn
        shape = (n_page, attn.h_kv, attn.page, attn.d)
        self.k, self.v = (torch.full(shape, float("nan"), device="cuda").to(attn._cache) for _ in range(2))
        e = attn.cache_dtype == lkv.E4M3
        self.ke, self.ve = (torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda") if e else None for _ in range(2))
        self.table_dev, self.len_dev = _i32(self.table), _i32(ctx)
        self.pages = lkv.make_pages(attn, self.k, self.v, self.table_dev, self.len_dev, self.ke, self.ve)

    def fill(self, seed=1):
        """Write every context whole; returns nothing, rows() tells what is stored."""
        a, n = self.attn, sum(self.ctx)
        _, k, v = _qkv(n, 1, a.h_kv, a.d, a._io, seed)
        lkv.kv_write(a, self.pages, _i32(_cum(self.ctx)), n, k, v)
        torch.cuda.synchronize()
        return k, v

    def rows(self, r):
        """Request r's keys and values [c, h_kv, d] as the stored bytes stand for."""
        a, c = self.attn, self.ctx[r]
        ids = self.table[r, :-(-c // a.page)] if c else np.zeros(0, int)
        out = []
        for x, e in ((self.k, self.ke), (self.v, self.ve)):
            if e is not None:
                y = A.e4m3_values(x.view(torch.uint8).cpu().numpy()[ids], e.cpu().numpy()[ids])
            else:
                y = _np(x)[ids]
            out.append(np.swapaxes(y, 1, 2).reshape(-1, a.h_kv, a.d)[:c])
        return out


def _attn_paged(attn, cache, cu, q, pos=None, n_tok=None):
    n_tok = q.shape[0] if n_tok is None else n_tok
    size = lkv.attn_paged_workspace(attn, len(cu) - 1, n_tok, cache.table.shape[1])
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # NaN
    o = torch.full(tuple(q.shape), 7.0, dtype=attn._io, device="cuda")
    lkv.attn_paged(attn, cache.pages, _i32(cu), n_tok, q, o, ws, None if pos is None else _i32(pos))
    torch.cuda.synchronize()
    return o


# ---------------------------------------------------------------- prefill
LENS = [(1,), (0, 2, 0, 1, 33, 0), (31, 32, 33), (63, 64, 65, 17), (127, 128, 129), (255, 300, 5), (700,)]
HEADS = [(8, 2, 128), (4, 4, 64), (6, 1, 64), (8, 8, 128), (16, 2, 256), (15, 5, 128), (3, 3, 256)]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("io", [BF, F32], ids=["bf16", "f32"])
def test_prefill(heads, lens, io):
    hq, hkv, d = heads
    if io == F32 and d == 256:
        pytest.skip("fp32 tokens are taken up to d = 128")
    attn = lkv.make_attn(hq, hkv, d, io_dtype=io)
    cu, n = _cum(lens), sum(lens)
    q, k, v = _qkv(n + 3, hq, hkv, d, io, seed=n, fused=n % 2 == 1)
    o = torch.full((n + 3, hq, d), 7.0, dtype=io, device="cuda")
    lkv.attn_prefill(attn, _i32(cu), n + 3, q, k, v, o)
    torch.cuda.synchronize()
    for a, b in zip(cu[:-1], cu[1:]):
        ref = A.attention(_np(q[a:b]), _np(k[a:b]), _np(v[a:b]), np.arange(b - a), attn.scale)
        _close(o[a:b], ref, io == F32, b - a, d)
    assert bool((o[n:] == 7.0).all())  # behind the last sequence


def test_prefill_scale_and_large_scores():
    """Scores in the hundreds, where one key wins, and a running maximum that keeps growing."""
    attn = lkv.make_attn(4, 1, 64, scale=1.75)
    q, k, v = _qkv(400, 4, 1, 64, BF, 3, False)
    k *= torch.linspace(0.1, 4, 400, device="cuda").to(BF)[:, None, None]
    o = torch.empty_like(q)
    lkv.attn_prefill(attn, _i32([0, 400]), 400, q, k, v, o)
    torch.cuda.synchronize()
    _close(o, A.attention(_np(q), _np(k), _np(v), np.arange(400), 1.75))


@pytest.mark.parametrize("lens", [(1024,), (1025, 1087), (1100,), (1153, 1, 2000), (2049,)], ids=str)
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (4, 1, 128), (4, 2, 256)])
def test_prefill_of_few_long_sequences(hq, hkv, d, lens):
    """Launches of few workgroups, with an odd and an even number of key tiles; NaN and infinities
    behind a token change nothing of it, bit for bit."""
    attn = lkv.make_attn(hq, hkv, d)
    cu, n = _cum(lens), sum(lens)
    q, k, v = _qkv(n + 2, hq, hkv, d, BF, seed=n)
    o, o2 = (torch.full((n + 2, hq, d), 7.0, dtype=BF, device="cuda") for _ in range(2))
    lkv.attn_prefill(attn, _i32(cu), n + 2, q, k, v, o)
    k2, v2 = k.clone(), v.clone()
    first = [b - 1 - (b - a) // 3 for a, b in zip(cu[:-1], cu[1:])]
    for x in first:
        k2[x] = float("inf")
        v2[x] = float("nan")
    lkv.attn_prefill(attn, _i32(cu), n + 2, q, k2, v2, o2)
    torch.cuda.synchronize()
    for a, b, x in zip(cu[:-1], cu[1:], first):
        rows = np.unique(np.r_[a:min(a + 3, b), np.arange(a, b, 29), max(a, b - 140):b])
        ref = A.attention(_np(q[rows]), _np(k[a:b]), _np(v[a:b]), rows - a, attn.scale)
        _close(o[torch.from_numpy(rows).cuda()], ref, False, b - a, d)
        assert torch.equal(o[a:x], o2[a:x]) and not bool(o2[x:b].isfinite().any())
    assert bool((o[n:] == 7.0).all()) and bool((o2[n:] == 7.0).all())


@pytest.mark.parametrize("io", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (2, 2, 128)])
def test_unseen_keys_do_not_matter(hq, hkv, d, io):
    """NaN and infinities in keys and values change only the tokens that see them, bit for bit."""
    attn = lkv.make_attn(hq, hkv, d, io_dtype=io)
    n, cu = 333, _i32([0, 100, 333])
    q, k, v = _qkv(n, hq, hkv, d, io, 5, False)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    lkv.attn_prefill(attn, cu, n, q, k, v, o)
    k2, v2 = k.clone(), v.clone()
    k2[50], v2[60], v2[170, :, 3], v2[171, :, 3] = float("nan"), float("inf"), float("inf"), float("-inf")
    v2[250, 0, 7] = float("nan")
    k2[332] = float("inf")
    lkv.attn_prefill(attn, cu, n, q, k2, v2, o2)
    torch.cuda.synchronize()
    assert torch.equal(o2[:50], o[:50]) and torch.equal(o2[100:170], o[100:170])
    assert bool(o2[50:100].isnan().all())
    ch = [c for c in range(d) if c != 3]
    assert torch.equal(o2[170:250][..., ch], o[170:250][..., ch])
    assert not bool(o2[170:, :, 3].isfinite().any())
    assert bool(o2[250:, 0, 7].isnan().all())
    assert torch.equal(o2[250:332, hq - 1, 9:], o[250:332, hq - 1, 9:])


def test_prefill_scores_of_minus_infinity():
    """A token all of whose scores are -inf gives zeros; one that also sees a finite one ignores them."""
    attn = lkv.make_attn(1, 1, 64)
    q, k, v = (torch.ones((70, 1, 64), dtype=BF, device="cuda") for _ in range(3))
    k[:20] = float("-inf")
    o = torch.empty_like(q)
    lkv.attn_prefill(attn, _i32([0, 70]), 70, q, k, v, o)
    torch.cuda.synchronize()
    assert bool((o[:20] == 0).all()) and bool((o[20:] == 1).all())


# ---------------------------------------------------------------- cache
@pytest.mark.parametrize("page,hkv,d,cache,io", [(16, 2, 128, E4, BF), (64, 1, 64, E4, BF), (32, 3, 256, E4, BF),
                                                 (256, 9, 64, BF, BF), (16, 2, 128, F32, F32), (1024, 8, 128, E4, BF)])
@pytest.mark.parametrize("select", [False, True])
def test_write_and_read(page, hkv, d, cache, io, select):
    attn = lkv.make_attn(hkv, hkv, d, page=page, io_dtype=io, cache_dtype=cache)
    ctx, new = [70, 0, 5, 300, 129], [33, 0, 5, 120, 1]
    C = Cache(attn, ctx)
    rng = np.random.default_rng(2)
    pos = np.concatenate([np.sort(rng.choice(c, m, replace=False)) if select else np.arange(c - m, c)
                          for c, m in zip(ctx, new)]).astype(np.int32)
    n = sum(new)
    _, k, v = _qkv(n, 1, hkv, d, io, 4)
    if io == BF:
        k *= torch.exp(8 * torch.randn((n, hkv, 1), generator=torch.Generator().manual_seed(1))).cuda().to(BF)
        k[3], k[4, 0, :5] = 0.0, torch.tensor([float("inf"), float("-inf"), float("nan"), 3e38, -1.0])
        v[5, 0, :3] = torch.tensor([2.0 ** -126, 2.0 ** -133, -(2.0 ** -120)])
        v[5, 0, 3:] = 0.0
    before = [x.clone().view(torch.uint8) for x in (C.k, C.v)]
    lkv.kv_write(attn, C.pages, _i32(_cum(new)), n, k, v, _i32(pos) if select else None)
    ko, vo = torch.empty((n, hkv, d), dtype=io, device="cuda"), torch.empty((n, hkv, d), dtype=io, device="cuda")
    lkv.kv_read(attn, C.pages, _i32(_cum(new)), n, ko, vo, _i32(pos) if select else None)
    torch.cuda.synchronize()
    r = np.repeat(np.arange(5), new)
    pid, slot = C.table[r, pos // page], pos % page
    for x, exps, new_rows, out, old in ((C.k, C.ke, k, ko, before[0]), (C.v, C.ve, v, vo, before[1])):
        stored = x.view(torch.uint8).cpu().numpy()[pid, :, slot]
        if cache == E4:
            codes, byte = A.e4m3_rows(_np(new_rows))
            nan = codes & 0x7f == 0x7f
            assert np.array_equal(exps.cpu().numpy()[pid, :, slot], byte)
            assert np.array_equal(stored[~nan], codes[~nan]) and (stored[nan] & 0x7f == 0x7f).all()
            want = A.e4m3_values(codes, byte)
        else:
            want = _np(new_rows)
        assert np.array_equal(_np(out), want, equal_nan=True)
        # nothing else was written
        untouched = np.ones((x.shape[0], page), bool)
        untouched[pid, slot] = False
        same = (x.view(torch.uint8) == old).all(dim=-1).all(dim=1).cpu().numpy()
        assert same[untouched].all()


@pytest.mark.parametrize("cache,hkv,d", [(E4, 3, 128), (BF, 9, 128), (E4, 2, 256)])
def test_write_and_read_many(cache, hkv, d):
    """Thousands of tokens of ragged requests, spread over their contexts, some outside them."""
    attn = lkv.make_attn(hkv, hkv, d, page=32, cache_dtype=cache)
    rng = np.random.default_rng(4)
    ctx = [5000, 1, 0, 7000] + [int(x) for x in rng.integers(1, 60, 90)]
    new = [4001, 1, 0, 6002] + [int(rng.integers(0, c + 1)) for c in ctx[4:]]
    C = Cache(attn, ctx)
    pos = np.concatenate([np.sort(rng.choice(c, m, replace=False)) if m else np.zeros(0, int) for c, m in zip(ctx, new)])
    out = np.array([7, 2000, 4001, len(pos) - 1])
    pos[out] = [-1, 5000, 1, 10 ** 6]
    n = len(pos)
    _, k, v = _qkv(n + 3, 1, hkv, d, BF, 4)
    ko, vo = (torch.full((n + 3, hkv, d), 7.0, dtype=BF, device="cuda") for _ in range(2))
    lkv.kv_write(attn, C.pages, _i32(_cum(new)), n + 3, k, v, _i32(np.append(pos, [0, 0, 0])))
    lkv.kv_read(attn, C.pages, _i32(_cum(new)), n + 3, ko, vo, _i32(np.append(pos, [0, 0, 0])))
    torch.cuda.synchronize()
    for x, o in ((k, ko), (v, vo)):
        want = _np(x[:n])
        if cache == E4:
            e = np.exp2(np.clip(np.ceil(np.log2(np.abs(want).max(-1) / 448)), -100, 120))[..., None]
            want = A.e4m3_values(A.e4m3_codes(want / e), np.log2(e[..., 0]) + 127)
        want[out] = np.nan  # position 1 of the context of one token among them
        assert np.array_equal(_np(o[:n]), want, equal_nan=True) and bool((o[n:] == 7.0).all())


@pytest.mark.parametrize("cache,hkv,d", [(E4, 1, 128), (E4, 1, 64), (BF, 2, 64), (BF, 2, 256)])
def test_write_and_read_many_of_few_heads(cache, hkv, d):
    test_write_and_read_many(cache, hkv, d)


def test_write_drops_and_duplicates():
    """Positions outside the context and pages outside the pool are dropped, and read as NaN; of
    neighbours with one position the last is written; rows behind the batch stay."""
    attn = lkv.make_attn(2, 2, 64, page=16)
    C = Cache(attn, [40, 20])
    C.table[1, 1] = 10 ** 6  # positions 16.. of request 1
    C.pages = lkv.make_pages(attn, C.k, C.v, _i32(C.table), C.len_dev)
    pos = np.array([-1, 3, 3, 3, 39, 40, 0, 15, 16, 10 ** 9], np.int32)
    _, k, v = _qkv(12, 1, 2, 64, BF, 9)
    cu = _i32([0, 6, 10])
    lkv.kv_write(attn, C.pages, cu, 12, k, v, _i32(np.append(pos, [1, 2])))
    ko, vo = (torch.full((12, 2, 64), 7.0, dtype=BF, device="cuda") for _ in range(2))
    lkv.kv_read(attn, C.pages, cu, 12, ko, vo, _i32(np.append(pos, [1, 2])))
    torch.cuda.synchronize()
    for x, o in ((k, ko), (v, vo)):
        want = x.clone()
        want[1] = want[2] = x[3]
        for i in (0, 5, 8, 9):
            want[i] = float("nan")
        want[10:] = 7.0
        assert np.array_equal(_np(o), _np(want), equal_nan=True)
    assert int((~C.k.isnan()).any(-1).any(1).sum()) == 4  # slots 3, 39 and 0, 15


# ---------------------------------------------------------------- attention over the cache
def _check_paged(attn, C, new, q, o, pos=None):
    cu = _cum(new)
    for r, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
        if a == b:
            continue
        k, v = C.rows(r)
        p = np.asarray(pos[a:b]) if pos is not None else C.ctx[r] - (b - a) + np.arange(b - a)
        ok = (p >= 0) & (p < C.ctx[r]) if pos is not None else np.ones(b - a, bool)
        assert bool(o[a:b][torch.from_numpy(~ok).cuda()].isnan().all())
        sel = torch.from_numpy(ok).cuda()
        _close(o[a:b][sel], A.attention(_np(q[a:b][sel]), k, v, p[ok], attn.scale), attn._io == F32, C.ctx[r], attn.d)


PAGED = [  # h_q, h_kv, d, page, cache, io
    (8, 2, 128, 16, BF, BF), (8, 2, 128, 64, E4, BF), (4, 4, 64, 32, E4, BF), (6, 1, 64, 128, BF, BF),
    (16, 2, 256, 64, BF, BF), (16, 2, 256, 16, E4, BF), (4, 2, 128, 16, F32, F32), (3, 3, 64, 256, F32, F32)]


@pytest.mark.parametrize("geo", PAGED, ids=lambda g: "-".join(str(x).replace("torch.", "") for x in g))
@pytest.mark.parametrize("ctx,new", [([1], [1]), ([0, 5, 64, 65, 200], [0, 1, 1, 1, 1]), ([300, 17, 1, 129], [1, 4, 1, 3]),
                                     ([100, 260], [100, 60]), ([2, 40, 0], [5, 40, 3]), ([700], [301])], ids=str)
def test_paged_last_tokens(geo, ctx, new):
    hq, hkv, d, page, cache, io = geo
    attn = lkv.make_attn(hq, hkv, d, page=page, io_dtype=io, cache_dtype=cache)
    C = Cache(attn, ctx)
    C.fill()
    n = sum(new)
    q = _qkv(n + 2, hq, 1, d, io, 6)[0]
    o = _attn_paged(attn, C, _cum(new), q)
    _check_paged(attn, C, new, q, o)
    assert bool((o[n:] == 7.0).all())


@pytest.mark.parametrize("geo", PAGED, ids=lambda g: "-".join(str(x).replace("torch.", "") for x in g))
@pytest.mark.parametrize("order", ["ascending", "any"])
def test_paged_at_positions(geo, order):
    """Tokens at positions inside their contexts, in any order, some outside (NaN rows)."""
    hq, hkv, d, page, cache, io = geo
    attn = lkv.make_attn(hq, hkv, d, page=page, io_dtype=io, cache_dtype=cache)
    ctx, new = [513, 90, 0, 260], [130, 7, 1, 1]
    C = Cache(attn, ctx)
    C.fill()
    rng = np.random.default_rng(3)
    pos = [rng.choice(c, m, replace=False) if c else np.zeros(m, int) for c, m in zip(ctx, new)]
    pos = np.concatenate([np.sort(p) if order == "ascending" else p for p in pos]).astype(np.int32)
    pos[[4, 131]] = [513, -1]
    q = _qkv(sum(new), hq, 1, d, io, 6)[0]
    _check_paged(attn, C, new, q, _attn_paged(attn, C, _cum(new), q, pos), pos)


@pytest.mark.parametrize("cache", [BF, E4], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("ctx,new", [([20000], [1]), ([9000, 12000, 1], [1, 3, 1]), ([30000], [9])], ids=str)
def test_paged_long_contexts(cache, ctx, new):
    attn = lkv.make_attn(8, 2, 128, page=64, cache_dtype=cache)
    C = Cache(attn, ctx)
    C.fill()
    q = _qkv(sum(new), 8, 1, 128, BF, 6)[0]
    _check_paged(attn, C, new, q, _attn_paged(attn, C, _cum(new), q))


@pytest.mark.parametrize("new", [(1, 1), (40, 40)])
@pytest.mark.parametrize("ctx", [(200, 100), (9000, 100)])
def test_paged_invalid_page(ctx, new):
    """An invalid page makes NaN of the tokens that see it and leaves other requests alone; a length
    past the table's width is clamped to it."""
    attn = lkv.make_attn(4, 2, 64, page=16)
    C = Cache(attn, ctx, pad=0)
    C.fill()
    q = _qkv(sum(new), 4, 1, 64, BF, 6)[0]
    good = _attn_paged(attn, C, _cum(new), q)
    last = (ctx[0] - 1) // 16
    C.table[0, last] = C.k.shape[0]
    C.pages = lkv.make_pages(attn, C.k, C.v, _i32(C.table), C.len_dev)
    bad = _attn_paged(attn, C, _cum(new), q)
    assert bool(bad[new[0] - 1].isnan().all()) and torch.equal(bad[new[0]:], good[new[0]:])
    C2 = Cache(attn, (128, 64), pad=0)
    C2.fill()
    q = _qkv(2, 4, 1, 64, BF, 6)[0]
    good = _attn_paged(attn, C2, [0, 1, 2], q)
    C2.len_dev[0] = 10 ** 9
    assert torch.equal(_attn_paged(attn, C2, [0, 1, 2], q), good)


@pytest.mark.parametrize("cache", [BF, E4], ids=["bf16", "e4m3"])
def test_paged_values_not_seen(cache):
    """NaN in later values of the context (drafted tokens that will be thrown away) stays out."""
    attn = lkv.make_attn(4, 2, 128, page=16, cache_dtype=cache)
    C = Cache(attn, [150])
    k, v = C.fill()
    q = _qkv(6, 4, 1, 128, BF, 6)[0]
    pos = [10, 100, 120, 121, 130, 149]
    good = _attn_paged(attn, C, [0, 6], q, pos)
    v = v.clone()
    v[121:] = float("nan")
    lkv.kv_write(attn, C.pages, _i32([0, 150]), 150, k, v)
    bad = _attn_paged(attn, C, [0, 6], q, pos)
    assert torch.equal(bad[:3], good[:3]) and bool(bad[3:].isnan().all())


@pytest.mark.parametrize("hq,hkv,d,cache", [(8, 2, 128, BF), (8, 1, 64, E4), (16, 2, 256, E4)])
def test_paged_mixed_batch(hq, hkv, d, cache):
    """Decoding requests beside chunks, empty requests among them: every request is taken once."""
    attn = lkv.make_attn(hq, hkv, d, page=16, cache_dtype=cache)
    new = [1, 130, 0, 1, 4, 8, 9, 33, 1, 0, 2]
    ctx = [40, 300, 10, 1, 4, 700, 90, 33, 2000, 0, 64]
    C = Cache(attn, ctx)
    C.fill()
    q = _qkv(sum(new) + 1, hq, 1, d, BF, 6)[0]
    _check_paged(attn, C, new, q, _attn_paged(attn, C, _cum(new), q))


@pytest.mark.parametrize("hq,hkv,d,cache,io", [(8, 2, 128, BF, BF), (8, 2, 64, E4, BF), (16, 2, 256, BF, BF), (8, 2, 128, F32, F32)])
def test_paged_chunks_in_many_parts(hq, hkv, d, cache, io):
    """Chunks over split contexts, a thousand rows and more to join, rows that see nothing among them."""
    attn = lkv.make_attn(hq, hkv, d, page=64, io_dtype=io, cache_dtype=cache)
    ctx, new = [9000, 5, 3000], [130, 8, 40]
    C = Cache(attn, ctx)
    C.fill()
    q = _qkv(sum(new) + 1, hq, 1, d, io, 6)[0]
    o = _attn_paged(attn, C, _cum(new), q)
    _check_paged(attn, C, new, q, o)
    assert bool((o[sum(new):] == 7.0).all()) and bool((o[130:133] == 0).all())


@pytest.mark.parametrize("n_req", [4, 70])
@pytest.mark.parametrize("hq,hkv,d,cache", [(8, 2, 64, BF), (8, 2, 128, E4), (16, 2, 256, BF), (16, 2, 256, E4)])
def test_paged_drafted_tokens(n_req, hq, hkv, d, cache):
    """Small and large batches of a few tokens each, 17 to 32 rows of a group on average, one chunk among
    them in the large one, one long context whose keys are split."""
    attn = lkv.make_attn(hq, hkv, d, page=16, cache_dtype=cache)
    g = hq // hkv
    new = [(17, 40, 24, 30)[i % 4] // g for i in range(n_req)]
    ctx = [new[i] + 13 * i % 90 for i in range(n_req)]
    ctx[1] += 2500
    if n_req > 4:
        new[9] = ctx[9] = 120 // g
    assert 16 * n_req < g * sum(new) <= 32 * n_req
    C = Cache(attn, ctx)
    C.fill()
    q = _qkv(sum(new) + 1, hq, 1, d, BF, 6)[0]
    o = _attn_paged(attn, C, _cum(new), q)
    _check_paged(attn, C, new, q, o)
    assert bool((o[sum(new):] == 7.0).all())


def test_far_offsets():
    """Rows and pages whose byte offsets pass 32 bits."""
    n, far = 530, 1 << 22  # 530 rows 2^22 elements apart: 4.4 GB
    x = torch.empty(n * far, dtype=BF, device="cuda")
    small = _qkv(n, 2, 1, 64, BF, 3, False)
    views, at = [], 0
    for t in small:
        y = x.as_strided((n, t.shape[1], 64), (far, 64, 1), at)
        y.copy_(t)
        views.append(y)
        at += t.shape[1] * 64
    attn = lkv.make_attn(2, 1, 64, page=16)
    o, o2 = torch.empty_like(small[0]), torch.empty_like(small[0])
    cu = _i32([0, 200, n])
    lkv.attn_prefill(attn, cu, n, *small, o)
    lkv.attn_prefill(attn, cu, n, *views, o2)
    assert torch.equal(o, o2)
    del x, views, y
    pool = (1 << 32) // (16 * 64) // 2 + 200  # pages of 2 KB: past 4 GB
    k, v = (torch.empty((pool, 1, 16, 64), dtype=BF, device="cuda") for _ in range(2))
    ids = np.arange(pool - 40, pool, dtype=np.int32).reshape(1, 40)
    P = lkv.make_pages(attn, k, v, _i32(ids), _i32([n]))
    lkv.kv_write(attn, P, _i32([0, n]), n, small[1], small[2])
    back = [torch.empty_like(t) for t in small[1:]]
    lkv.kv_read(attn, P, _i32([0, n]), n, *back)
    torch.cuda.synchronize()
    assert torch.equal(back[0], small[1]) and torch.equal(back[1], small[2])
    for m in (1, 60):
        q = small[0][:m].contiguous()
        ws = torch.empty(lkv.attn_paged_workspace(attn, 1, m, 40), dtype=torch.uint8, device="cuda")
        om = torch.empty_like(q)
        lkv.attn_paged(attn, P, _i32([0, m]), m, q, om, ws)
        _close(om, A.attention(_np(q), _np(small[1]), _np(small[2]), np.arange(n - m, n), attn.scale))


@pytest.mark.parametrize("call", ["prefill", "paged"])
def test_rows_are_independent(call):
    """A large score of one token leaves the sums of the others, in the same tile of rows, as they are:
    their results are the same bits."""
    h, d, c, n_seq, m, x = 32, 128, 300, 40, 8, 295
    attn = lkv.make_attn(h, h, d, page=16)
    q, k, v = _qkv(n_seq * c, h, h, d, BF, 11, False)
    outs, at = [], torch.arange(n_seq, device="cuda") * c + x
    C = Cache(attn, [c] * n_seq)
    for _ in range(2):
        if call == "prefill":
            o = torch.empty_like(q)
            lkv.attn_prefill(attn, _i32(np.arange(n_seq + 1) * c), n_seq * c, q, k, v, o)
            outs.append(o.view(n_seq, c, h, d)[:, :x])
        else:
            lkv.kv_write(attn, C.pages, _i32(np.arange(n_seq + 1) * c), n_seq * c, k, v)
            last = q.view(n_seq, c, h, d)[:, c - m:].reshape(n_seq * m, h, d)
            o = _attn_paged(attn, C, np.arange(n_seq + 1) * m, last)
            outs.append(o.view(n_seq, m, h, d)[:, :x - (c - m)])
        k[at] *= 30
    torch.cuda.synchronize()
    assert torch.equal(*outs)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("cache", [BF, E4], ids=["bf16", "e4m3"])
def test_reuse_flow(cache):
    """A hybrid model's reuse of cached blocks in one layer: blocks attended to and written each on its
    own, concatenated by their pages, overwritten at U, U's queries attended, then decoding."""
    hq, hkv, d, page = 8, 2, 128, 16
    attn = lkv.make_attn(hq, hkv, d, page=page, cache_dtype=cache)
    blocks = [48, 64, 33]  # the last block of a context may end inside a page
    ctx = sum(blocks)
    q, k, v = _qkv(ctx, hq, hkv, d, BF, 1)
    cu = _i32(_cum(blocks))
    o = torch.empty((ctx, hq, d), dtype=BF, device="cuda")
    lkv.attn_prefill(attn, cu, ctx, q, k, v, o)
    C = Cache(attn, [ctx + 3])
    first = np.cumsum([0] + [b // page for b in blocks[:-1]])
    wide = max(-(-b // page) for b in blocks)
    by_block = np.full((3, wide), -1, np.int32)
    for i, b in enumerate(blocks):
        m = -(-b // page)
        by_block[i, :m] = C.table[0, first[i]:first[i] + m]
    block_pages = lkv.make_pages(attn, C.k, C.v, _i32(by_block), _i32(blocks), C.ke, C.ve)
    lkv.kv_write(attn, block_pages, cu, ctx, k, v)
    torch.cuda.synchronize()
    for a, b in zip(_cum(blocks)[:-1], _cum(blocks)[1:]):
        _close(o[a:b], A.attention(_np(q[a:b]), _np(k[a:b]), _np(v[a:b]), np.arange(b - a), attn.scale))
    # U: a window around the seams, in context order
    pos = np.array([46, 47, 48, 49, 110, 111, 112, 113], np.int32)
    qU, kU, vU = _qkv(len(pos), hq, hkv, d, BF, 2)
    C.len_dev.fill_(ctx)
    C.ctx = [ctx]
    lkv.kv_write(attn, C.pages, _i32([0, len(pos)]), len(pos), kU, vU, _i32(pos))
    oU = _attn_paged(attn, C, [0, len(pos)], qU, pos)
    rows = C.rows(0)
    kept = np.setdiff1d(np.arange(ctx), pos)
    if cache == BF:
        assert np.array_equal(rows[0][kept], _np(k)[kept]) and np.array_equal(rows[1][pos], _np(vU))
    _check_paged(attn, C, [len(pos)], qU, oU, pos)
    for step in range(3):
        C.ctx[0] += 1
        C.len_dev += 1
        q1, k1, v1 = _qkv(1, hq, hkv, d, BF, 10 + step)
        lkv.kv_write(attn, C.pages, _i32([0, 1]), 1, k1, v1)
        _check_paged(attn, C, [1], q1, _attn_paged(attn, C, [0, 1], q1))


@pytest.mark.parametrize("ctx", [(70, 40), (6000, 2500)])
def test_captured_decode(ctx):
    """A captured decoding step (write, attention) replayed while the contexts grow, with eager work
    between the replays: each replay bit for bit the eager step."""
    attn = lkv.make_attn(8, 2, 128, page=16, cache_dtype=E4)
    C = Cache(attn, [c + 8 for c in ctx])
    C.fill()
    C.len_dev.copy_(_i32(ctx))
    cu, n = _i32([0, 1, 2]), 2
    q, k, v = _qkv(n, 8, 2, 128, BF, 3)
    size = lkv.attn_paged_workspace(attn, 2, 2, C.table.shape[1])
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    o = torch.empty((n, 8, 128), dtype=BF, device="cuda")

    def step(out, work):
        lkv.kv_write(attn, C.pages, cu, n, k, v)
        lkv.attn_paged(attn, C.pages, cu, n, q, out, work)

    step(o, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.len_dev.add_(1)
        step(o, ws)
    for i in range(5):
        x = _qkv(n, 8, 2, 128, BF, 20 + i)
        for a, b in zip((q, k, v), x):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want, ws2 = torch.empty_like(o), torch.empty_like(ws)
        step(want, ws2)  # writes the same rows again
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        C.ctx = [c + 1 + i for c in ctx]
        _check_paged(attn, C, [1, 1], q, o)


def test_other_stream_and_repeat():
    """The calls run on the current stream, and twice give the same bits."""
    attn = lkv.make_attn(8, 2, 128, page=64)
    C = Cache(attn, [5000, 300])
    C.fill()
    q = _qkv(6, 8, 1, 128, BF, 2)[0]
    want = _attn_paged(attn, C, [0, 5, 6], q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _attn_paged(attn, C, [0, 5, 6], q)
    side.synchronize()
    assert torch.equal(got, want)
    qk = _qkv(300, 8, 2, 128, BF, 3)
    o = [torch.empty((300, 8, 128), dtype=BF, device="cuda") for _ in range(2)]
    for x in o:
        lkv.attn_prefill(attn, _i32([0, 100, 300]), 300, *qk, x)
    torch.cuda.synchronize()
    assert torch.equal(o[0], o[1])


def test_no_tokens_and_empty_pool():
    attn = lkv.make_attn(4, 2, 64, page=16)
    x = torch.empty((0, 4, 64), dtype=BF, device="cuda")
    kv = torch.empty((0, 2, 64), dtype=BF, device="cuda")
    lkv.attn_prefill(attn, _i32([0, 0]), 0, x, kv, kv, x)
    pool = torch.empty((0, 2, 16, 64), dtype=BF, device="cuda")
    pages = lkv.make_pages(attn, pool, pool, _i32(np.zeros((1, 3))), _i32([40]))
    q = torch.ones((2, 4, 64), dtype=BF, device="cuda")
    o = torch.full((2, 4, 64), 7.0, dtype=BF, device="cuda")
    ws = torch.empty(lkv.attn_paged_workspace(attn, 1, 2, 3), dtype=torch.uint8, device="cuda")
    lkv.attn_paged(attn, pages, _i32([0, 2]), 2, q, o, ws)
    torch.cuda.synchronize()
    assert bool((o == 0).all())
