"""Performance cases of a hybrid model's full-attention layers: what the serving program calls
there beside the recurrent layers' calls.

 - ``prefill``: causal attention with grouped heads over packed sequences: the cached blocks,
   each on its own, or whole prompts.
 - ``cache``: new tokens' keys and values written into the paged cache (in bf16, fp32, or e4m3
   with one power-of-two scale per token and head) and read back.
 - ``paged``: attention of new tokens over the paged cache: the recomputed tokens at their
   positions inside the context, the last tokens of a prompt, drafted tokens, single tokens.

Every function takes the plain form where ``own`` is false: elementary torch operations in fp32.
``exact`` evaluates the same definitions in fp64.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases
def _case(name, op, **kw):
    # n_req requests of q_lo..q_hi new tokens; cache and paged: contexts of c_lo..c_hi tokens, the new
    # ones included, in pages of `page` tokens; select: the new tokens' positions are spread over the
    # context (else they are its last); fused: q, k and v are views of one projection's output
    c = dict(name=name, op=op, n_req=1, hq=32, hkv=8, d=128, io="bf16", cache="bf16", page=64, q_lo=1, q_hi=1,
             c_lo=0, c_hi=0, select=False, fused=True, layout=1)
    c.update(kw)
    return c


def listed():
    return [
        # one short prompt: a call that is all latency
        _case("prefill_short", "prefill", hq=16, hkv=2, d=256, q_lo=77, q_hi=77),
        # the cached blocks of one 32K context, each on its own
        _case("prefill_blocks", "prefill", n_req=32, q_lo=512, q_hi=1536),
        # one 8K prompt of a layer with few wide heads
        _case("prefill_8k", "prefill", hq=16, hkv=2, d=256, q_lo=8192, q_hi=8192),
        # one 32K prompt without reuse: the largest call
        _case("prefill_32k", "prefill", q_lo=32768, q_hi=32768),
        # fp32 tokens, as numerics checks run them: short ragged sequences, no grouping
        _case("prefill_f32", "prefill", n_req=4, hq=8, hkv=8, d=64, io="f32", cache="f32", q_lo=100, q_hi=700,
              fused=False),
        # one decoding step's tokens into an e4m3 cache: latency
        _case("cache_step", "cache", n_req=64, cache="e4m3", c_lo=1024, c_hi=8192),
        # the recomputed tokens of four 32K contexts overwritten in an e4m3 cache
        _case("cache_recompute", "cache", n_req=4, cache="e4m3", q_lo=4096, q_hi=4096, c_lo=32768, c_hi=32768,
              select=True),
        # a whole prompt into a bf16 cache of small pages
        _case("cache_prompt", "cache", page=16, q_lo=32768, q_hi=32768, c_lo=32768, c_hi=32768),
        # decoding for four requests: latency, few heads to spread
        _case("paged_decode_4", "paged", n_req=4, c_lo=8192, c_hi=8192),
        # decoding at a serving batch of ragged contexts from an e4m3 cache: cache traffic
        _case("paged_decode_128", "paged", n_req=128, cache="e4m3", c_lo=1024, c_hi=8192),
        # the last chunk of two long prompts, few wide heads, e4m3 cache
        _case("paged_chunk", "paged", n_req=2, hq=16, hkv=2, d=256, cache="e4m3", page=32, q_lo=512, q_hi=512,
              c_lo=8192, c_hi=16384),
        # the recomputed tokens of four 32K contexts, at their own positions
        _case("paged_recompute", "paged", n_req=4, q_lo=4096, q_hi=4096, c_lo=32768, c_hi=32768, select=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (0.8e15 if case["io"] == "bf16" else 0.06e15)


def _held(case):
    """Elements that a prepared case holds."""
    ctx = case["n_req"] * case["c_hi"] * 2 * case["hkv"] * case["d"]
    return ctx + case["n_req"] * case["q_hi"] * (2 * case["hq"] + 2 * case["hkv"]) * case["d"]


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= 0.7 * most and _held(c) <= 1.5e9:
            return c


def _draw(rng):
    kind = rng.choice(["prompt", "blocks", "cache", "decode", "decode", "draft", "chunk", "recompute"])
    hq, hkv = rng.choice([(16, 2), (32, 8), (32, 4), (8, 8), (24, 8), (15, 5), (64, 8), (6, 1)])
    geo = dict(hq=hq, hkv=hkv, d=rng.choice([64, 128, 128, 256]), layout=rng.randrange(1, 1 << 20),
               fused=rng.random() < 0.7, page=rng.choice([16, 32, 64, 64, 128, 256]),
               cache=rng.choice(["bf16", "bf16", "e4m3", "e4m3"]))
    if rng.random() < 0.1:
        geo.update(io="f32", cache="f32", d=rng.choice([64, 128]))
    if kind == "prompt":
        n = _log_int(rng, 1, 24000)
        return _case("", "prefill", n_req=1, q_lo=n, q_hi=n, **geo)
    if kind == "blocks":
        n_req, hi = _log_int(rng, 2, 48), _log_int(rng, 16, 4096)
        return _case("", "prefill", n_req=n_req, q_lo=max(1, hi // rng.choice([1, 2, 6, 20])), q_hi=hi, **geo)
    n_req, hi = _log_int(rng, 1, 160), _log_int(rng, 50, 32768)
    ctx = dict(c_lo=max(1, hi // rng.choice([1, 2, 8])), c_hi=hi)
    if kind == "decode":
        return _case("", "paged", n_req=n_req, **ctx, **geo)
    if kind == "draft":
        return _case("", "paged", n_req=n_req, q_lo=1, q_hi=rng.randint(2, 16), **ctx, **geo)
    n_req = _log_int(rng, 1, 16)
    q = _log_int(rng, 8, max(9, hi // 2))
    sel = kind == "recompute" or (kind == "cache" and rng.random() < 0.5)
    return _case("", "cache" if kind == "cache" else "paged", n_req=n_req, q_lo=max(1, q // rng.choice([1, 2, 5])), q_hi=q,
                 select=sel, **ctx, **geo)


# ---------------------------------------------------------------- layout (from the case alone)
def _lens(case):
    """New tokens and context lengths of the requests."""
    rng = random.Random("lengths %d" % case["layout"])
    q = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["n_req"])]
    if case["op"] == "prefill":
        return q, list(q)
    c = [rng.randint(case["c_lo"], case["c_hi"]) for _ in range(case["n_req"])]
    return [min(a, b) for a, b in zip(q, c)], c


def _cum(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return out


def _positions(case):
    """Positions of every request's new tokens inside its context, ascending."""
    rng = random.Random("positions %d" % case["layout"])
    q, c = _lens(case)
    if not case["select"]:
        return [list(range(n - m, n)) for m, n in zip(q, c)]
    return [sorted(rng.sample(range(n), m)) for m, n in zip(q, c)]


# ---------------------------------------------------------------- inputs
def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tokens(case, gen, n):
    """q, k and v of n tokens.  Keys have loud and quiet channels, as projections give them."""
    hq, hkv, d, io = case["hq"], case["hkv"], case["d"], _DT[case["io"]]
    gain = torch.exp(0.5 * torch.randn((hkv, d), device="cuda", generator=gen))
    if case["fused"]:
        x = torch.empty((n, (hq + 2 * hkv) * d), dtype=io, device="cuda")
        q, k, v = (x[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    else:
        q, k, v = (torch.empty((n, h, d), dtype=io, device="cuda") for h in (hq, hkv, hkv))
    step = max(1, (1 << 27) // ((hq + 2 * hkv) * d))
    for a in range(0, n, step):
        b = min(n, a + step)
        q[a:b] = torch.randn((b - a, hq, d), device="cuda", generator=gen).to(io)
        k[a:b] = (torch.randn((b - a, hkv, d), device="cuda", generator=gen) * gain).to(io)
        v[a:b] = torch.randn((b - a, hkv, d), device="cuda", generator=gen).to(io)
    return q, k, v


def _cache(case, gen, n_page):
    """Pages as earlier writes left them: e4m3 codes fill their range, with a scale byte per row."""
    hkv, d, page = case["hkv"], case["d"], case["page"]
    shape = (n_page, hkv, page, d)
    gain = torch.exp(0.5 * torch.randn((hkv, 1, d), device="cuda", generator=gen))
    out = {}
    for name in ("k", "v"):
        g = gain if name == "k" else 1.0
        if case["cache"] == "e4m3":
            x = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
            out[name + "_exp"] = torch.randint(119, 122, shape[:3], device="cuda", generator=gen, dtype=torch.int32).to(
                torch.uint8)
            g = g * 96.0
        else:
            x = torch.empty(shape, dtype=_DT[case["cache"]], device="cuda")
        step = max(1, (1 << 27) // (hkv * page * d))
        for a in range(0, n_page, step):
            b = min(n_page, a + step)
            y = torch.randn((b - a,) + shape[1:], device="cuda", generator=gen) * g
            x[a:b] = (y.clamp_(-448.0, 448.0) if case["cache"] == "e4m3" else y).to(x.dtype)
        out[name] = x
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    hq, hkv, d, io = case["hq"], case["hkv"], case["d"], _DT[case["io"]]
    nq, nc = _lens(case)
    n = sum(nq)
    s = dict(case=case, n=n, cu=_i32(_cum(nq)), scale=d ** -0.5)
    s["q"], s["k"], s["v"] = _tokens(case, gen, n)
    s["o"] = torch.empty((n, hq, d), dtype=io, device="cuda")
    if case["op"] == "prefill":
        if own:
            from paper_2608_11231_amd import lkv
            s["attn"] = lkv.make_attn(hq, hkv, d, io_dtype=io)
        return s
    page = case["page"]
    need = [-(-c // page) for c in nc]
    n_page = sum(need) + 3
    perm = torch.randperm(n_page, generator=gen, device="cuda").cpu().tolist()
    wide, at, table = max(need) + 1, 0, []
    for m in need:
        table.append(perm[at:at + m] + [-1] * (wide - m))
        at += m
    c = _cache(case, gen, n_page)
    s["k_pages"], s["v_pages"] = c.pop("k"), c.pop("v")
    s.update(c)
    if case["op"] == "cache":
        s["k_out"], s["v_out"] = (torch.empty((n, hkv, d), dtype=io, device="cuda") for _ in range(2))
    else:
        del s["k"], s["v"]  # the new tokens' rows are in the cache already
    s["table"], s["len"] = _i32(table), _i32(nc)
    s["pos"] = _i32([p for r in _positions(case) for p in r]) if case["select"] else None
    if own:
        from paper_2608_11231_amd import lkv
        s["attn"] = lkv.make_attn(hq, hkv, d, io_dtype=io, cache_dtype=s["k_pages"].dtype, page=page)
        s["pages"] = lkv.make_pages(s["attn"], s["k_pages"], s["v_pages"], s["table"], s["len"], s.get("k_exp"),
                                    s.get("v_exp"))
        if case["op"] == "paged":
            size = lkv.attn_paged_workspace(s["attn"], case["n_req"], n, wide)
            s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if not own:
        return _plain(s)
    from paper_2608_11231_amd import lkv
    if op == "prefill":
        lkv.attn_prefill(s["attn"], s["cu"], s["n"], s["q"], s["k"], s["v"], s["o"])
        return s["o"]
    if op == "cache":
        lkv.kv_write(s["attn"], s["pages"], s["cu"], s["n"], s["k"], s["v"], s["pos"])
        lkv.kv_read(s["attn"], s["pages"], s["cu"], s["n"], s["k_out"], s["v_out"], s["pos"])
        return s["k_out"], s["v_out"]
    lkv.attn_paged(s["attn"], s["pages"], s["cu"], s["n"], s["q"], s["o"], s["ws"], s["pos"])
    return s["o"]


def _plain(s):
    case = s["case"]
    nq, nc = _lens(case)
    cu, page = _cum(nq), case["page"]
    if case["op"] == "prefill":
        for r in range(case["n_req"]):
            a, b = cu[r], cu[r + 1]
            pos = torch.arange(b - a, device="cuda")
            _plain_attention(s["q"][a:b], s["k"][a:b].transpose(0, 1).float(), s["v"][a:b].transpose(0, 1).float(), pos,
                             s["scale"], s["o"][a:b])
        return s["o"]
    tok_pos = s["pos"].long() if s["pos"] is not None else None
    for r in range(case["n_req"]):
        a, b = cu[r], cu[r + 1]
        pos = tok_pos[a:b] if tok_pos is not None else torch.arange(nc[r] - nq[r], nc[r], device="cuda")
        ids = s["table"][r, :-(-nc[r] // page)].long()
        if case["op"] == "cache":
            pid, slot = ids[pos // page], pos % page
            for x in ("k", "v"):
                pages, new = s[x + "_pages"], s[x][a:b]
                if case["cache"] == "e4m3":
                    code, exp = _plain_e4m3(new.float())
                    pages.view(torch.uint8)[pid, :, slot] = code.view(torch.uint8)
                    s[x + "_exp"][pid, :, slot] = exp
                else:
                    pages[pid, :, slot] = new
                s[x + "_out"][a:b] = _plain_values(s, x, (pid, slice(None), slot))
            continue
        kv = []
        for x in ("k", "v"):
            y = _plain_values(s, x, ids)
            kv.append(y.transpose(0, 1).reshape(case["hkv"], -1, case["d"])[:, :nc[r]])
        _plain_attention(s["q"][a:b], kv[0], kv[1], pos, s["scale"], s["o"][a:b])
    return (s["k_out"], s["v_out"]) if case["op"] == "cache" else s["o"]


def _plain_e4m3(x):
    """Codes and scale bytes of rows of fp32 values: the least power of two that brings the row into
    e4m3's range."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), torch.full_like(e, -100)).clamp(-100, 120)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _plain_values(s, x, at):
    """The values that the cache rows at an index stand for."""
    pages = s[x + "_pages"]
    if x + "_exp" not in s:
        return pages[at].float()
    code = pages.view(torch.uint8)[at].view(pages.dtype)
    return torch.ldexp(code.float(), (s[x + "_exp"][at].int() - 127)[..., None])


def _plain_attention(q, k, v, pos, scale, o):
    """o [n, hq, d] <- attention of q [n, hq, d] at positions pos [n] over k, v [hkv, c, d] in fp32."""
    n, hq, d = q.shape
    hkv, c = k.shape[0], k.shape[1]
    g = hq // hkv
    kt = k.transpose(1, 2).contiguous()
    v = v.contiguous()
    j = torch.arange(c, device="cuda")
    step = max(1, (1 << 28) // (hq * c))
    for a in range(0, n, step):
        b = min(n, a + step)
        x = q[a:b].view(b - a, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * (b - a), d).float()
        s = torch.bmm(x, kt).mul_(scale).view(hkv, g, b - a, c)
        s.masked_fill_(j[None, :] > pos[a:b, None], -math.inf)
        s = s.sub_(s.amax(-1, keepdim=True)).exp_()
        total = s.sum(-1, keepdim=True)
        y = torch.bmm(s.view(hkv, g * (b - a), c), v).view(hkv, g, b - a, d) / total
        o[a:b] = y.permute(2, 0, 1, 3).reshape(b - a, hq, d).to(o.dtype)


# ---------------------------------------------------------------- the definition in fp64
def exact(case, seed):
    x = prepare(case, seed)
    nq, nc = _lens(case)
    cu, page, where = _cum(nq), case["page"], _positions(case)
    if case["op"] == "cache":
        return _exact_stored(x["k"], case), _exact_stored(x["v"], case)
    out = torch.empty((sum(nq), case["hq"], case["d"]), dtype=torch.float64, device="cuda")
    group = case["hq"] // case["hkv"]
    for r in range(case["n_req"]):
        rows, p = slice(cu[r], cu[r + 1]), torch.tensor(where[r], device="cuda")
        for h in range(case["hkv"]):
            if case["op"] == "prefill":
                K, V = x["k"][rows, h].double(), x["v"][rows, h].double()
            else:
                ids = x["table"][r, :-(-nc[r] // page)].long()
                K, V = (_exact_read(x, a, ids, h)[:nc[r]] for a in ("k", "v"))
            Q = x["q"][rows, h * group:(h + 1) * group].double()
            for a in range(0, nq[r], max(1, (1 << 26) // (group * nc[r]))):
                b = min(nq[r], a + max(1, (1 << 26) // (group * nc[r])))
                seen = torch.arange(nc[r], device="cuda")[None, None] <= p[a:b, None, None]
                w = (Q[a:b].reshape(-1, case["d"]) @ K.T).view(b - a, group, nc[r]) * x["scale"]
                w = torch.where(seen, w, -math.inf)
                w = torch.exp(w - w.max(dim=-1, keepdim=True).values)
                w = w / w.sum(dim=-1, keepdim=True)
                out[cu[r] + a:cu[r] + b, h * group:(h + 1) * group] = (w.view(-1, nc[r]) @ V).view(b - a, group, case["d"])
    return out


def _exact_read(x, a, ids, h):
    pages = x[a + "_pages"]
    if a + "_exp" not in x:
        y = pages[ids, h].double()
    else:
        y = pages.view(torch.uint8)[ids, h].view(pages.dtype).double()
        y = y * torch.pow(2.0, x[a + "_exp"][ids, h].double() - 127.0)[..., None]
    return y.reshape(-1, y.shape[-1])


def _exact_stored(x, case):
    """What a row written to the cache stands for afterwards."""
    y = x.double()
    if case["cache"] != "e4m3":
        return y
    scale = torch.exp2(torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True) / 448.0)).clamp(-100, 120))
    y = y / scale
    # e4m3: three bits behind the leading one, and a least exponent of -6
    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(y / ulp) * ulp * scale


# ---------------------------------------------------------------- work
def work(case):
    """Every input read once, every output written once.  A cache is read up to the last position
    that the request's tokens see."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    io = 2 if case["io"] == "bf16" else 4
    row = hkv * {"bf16": 2 * d, "f32": 4 * d, "e4m3": d + 1}[case["cache"]]  # of k or of v in the cache
    nq, nc = _lens(case)
    n = sum(nq)
    if case["op"] == "prefill":
        return {"bytes": n * (2 * hq + 2 * hkv) * d * io, "flops": 4 * d * hq * sum(m * (m + 1) // 2 for m in nq)}
    if case["op"] == "cache":
        return {"bytes": n * 2 * (2 * hkv * d * io + 2 * row), "flops": 0}
    pos = _positions(case)
    return {"bytes": n * 2 * hq * d * io + sum((p[-1] + 1) * 2 * row for p in pos if p),
            "flops": 4 * d * hq * sum(x + 1 for p in pos for x in p)}
