"""The paged-cache operators: block tables and slot maps, the rotating append, and attention of a chunk of new tokens over the
pages, plain and with capped scores, a distance bias, a window or a prefix.

`listed()` names the cases, `draw()` samples more from the same ranges, `prepare()` builds what a server holds before the call,
`run()` is one pass (in elementary torch operations, or through the library where `own` is set), `work()` what a pass cannot do
without, `exact()` the same results in 64 bits.

A cache is two pools: keys [page][kv head][position][feature], values [page][kv head][position / 8][feature][position % 8].
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases

def _plan(name, batch, new, cached, ragged, page, short=False):
    """Step planning for `batch` requests with up to `new` new tokens behind up to `cached` cached ones; short: the free list
    holds too few pages for the last requests."""
    return {"name": name, "kind": "plan", "batch": batch, "new": new, "cached": cached, "ragged": ragged, "page": page, "short": short}


def _append(name, batch, new, cached, ragged, heads, kv_heads, dim, page, dtype):
    return {"name": name, "kind": "append", "batch": batch, "new": new, "cached": cached, "ragged": ragged, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype}


def _attend(name, batch, new, cached, ragged, heads, kv_heads, dim, page, dtype, softcap=0.0, window=0, slopes=False, prefix=0):
    return {"name": name, "kind": "attend", "batch": batch, "new": new, "cached": cached, "ragged": ragged, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "softcap": softcap, "window": window, "slopes": slopes,
            "prefix": prefix}


def listed():
    return [
        # a small server's next round: sixteen streams with six drafted tokens each
        _plan("plan_b16_k6", 16, 6, 2048, False, 16),
        # a large mixed step: single tokens, drafted blocks and prompts' chunks of many streams
        _plan("plan_b512_mixed", 512, 256, 8192, True, 64),
        # one stream's drafted block: latency
        _append("append_b1_k4", 1, 4, 512, False, 32, 8, 128, 16, "bf16"),
        # a step of prompts, beginning and ending anywhere in their pages
        _append("append_b8_prompts", 8, 1999, 1000, True, 32, 8, 128, 32, "bf16"),
        # the tiny fp32 target: a prompt
        _append("append_f32_b3", 3, 700, 60, True, 4, 4, 64, 16, "f32"),
        # one stream's drafted block over a short cache: latency
        _attend("attend_b1_k4_l512", 1, 4, 512, False, 32, 8, 128, 16, "bf16"),
        # a busy server: 64 streams' drafted blocks over long caches (2.1 GB of keys and values)
        _attend("attend_b64_k8_l8192", 64, 8, 8184, False, 32, 8, 128, 64, "bf16"),
        # prompts: two chunks of 2048 tokens behind 6144 cached ones
        _attend("attend_b2_prompts", 2, 2048, 6144, False, 32, 8, 128, 32, "bf16"),
        # the tiny fp32 target: a ragged batch
        _attend("attend_f32_b5", 5, 37, 300, True, 4, 4, 64, 16, "f32"),
        # single tokens with capped scores inside a sliding window, wide heads
        _attend("capped_b37_tokens", 37, 1, 6000, True, 16, 8, 256, 32, "bf16", softcap=50.0, window=4096),
        # ragged prompts with a distance bias behind a prefix that every token sees, seven query heads per kv head
        _attend("biased_b6_prompts", 6, 777, 900, True, 28, 4, 64, 16, "bf16", slopes=True, prefix=96),
        # one stream's single token over a very long cache, capped scores
        _attend("capped_b1_l131072", 1, 1, 131071, False, 32, 8, 128, 256, "bf16", softcap=30.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128, 256])
    ragged = rng.random() < 0.6
    if kind == "plan":
        c = _plan("", _log(rng, 1, 512), _log(rng, 1, 256), _log(rng, 1, 8192), ragged, page, rng.random() < 0.25)
    else:
        kv_heads, rep, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8]), rng.choice([32, 64, 64, 128, 128, 128, 256])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        batch, new = _log(rng, 1, 64), _log(rng, 1, 2048)
        if kind == "append":
            while batch * new * (rep + 2) * kv_heads * dim * (2 if dtype == "f32" else 1) > 8 * 1999 * 48 * 128:
                batch, new = max(1, batch // 2), max(1, new * 2 // 3)
            c = _append("", batch, new, _log(rng, 1, 4000), ragged, kv_heads * rep, kv_heads, dim, page, dtype)
        else:
            cached = _log(rng, 1, 65536)
            while (batch * new * (new + cached) * kv_heads * rep > 2 * 2048 * 8192 * 32 or
                   batch * new * (new + cached) * kv_heads * rep * dim > 2 * 2048 * 8192 * 32 * 128 or
                   batch * (new + cached) * kv_heads * dim > 64 * 8192 * 8 * 128 / (2 if dtype == "f32" else 1)):
                batch, new, cached = max(1, batch * 3 // 4), max(1, new * 3 // 4), max(1, cached * 3 // 4)
            softcap = rng.choice([0.0, 0.0, 30.0, 50.0])
            window = rng.choice([0, 0, _log(rng, 16, 4096)])
            c = _attend("", batch, new, cached, ragged, kv_heads * rep, kv_heads, dim, page, dtype, softcap, window,
                        rng.random() < 0.25, rng.choice([0, 0, _log(rng, 1, 500)]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """(cached, new) of every request, by the case alone: the largest first; ragged batches hold single tokens, idle requests
    and everything between."""
    b, new, cached = case["batch"], case["new"], case["cached"]
    if not case["ragged"]:
        return [cached] * b, [new] * b
    rng = random.Random(b * 1000003 + new * 8191 + cached)
    cs = [cached] + [_log(rng, 1, cached) - 1 for _ in range(b - 1)]
    ns = [new] + [0 if rng.random() < 0.05 else _log(rng, 1, new) for _ in range(b - 1)]
    return cs, ns


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + tag * 7919 + 12345) % (1 << 62))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pages(n, page):
    return -(-n // page)


def _tables(case, seed, lengths):
    """A table of distinct pages for requests of these lengths, scattered over a pool that is a little larger, and the pages
    of the pool that no request holds."""
    page = case["page"]
    counts = torch.tensor([_pages(n, page) for n in lengths], device=DEV)
    total, width = sum(_pages(n, page) for n in lengths), max(1, max(_pages(n, page) for n in lengths))
    pool = total + 7
    perm = torch.randperm(pool, generator=_gen(seed, 1), device=DEV).to(torch.int32)
    col = torch.arange(width, device=DEV)[None, :]
    at = (torch.cumsum(counts, 0) - counts)[:, None] + col
    table = torch.where(col < counts[:, None], perm[at.clamp(max=pool - 1)], torch.full_like(perm[:1], -1))
    return table.contiguous(), pool, perm[total:]


def _normal(seed, tag, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=_gen(seed, tag))


def prepare(case, seed):
    cs, ns = _lengths(case)
    b, page, kind = case["batch"], case["page"], case["kind"]
    if kind == "plan":
        table, pool, _ = _tables(case, seed, cs)
        need = sum(_pages(c + n, page) - _pages(c, page) for c, n in zip(cs, ns))
        n_free = max(1, need * 3 // 4 if case["short"] else need + 5)
        free = (pool + torch.randperm(n_free, generator=_gen(seed, 2), device=DEV)).to(torch.int32)
        width = max(_pages(c + n, page) for c, n in zip(cs, ns))
        rows = torch.full((b, width), -1, dtype=torch.int32, device=DEV)
        rows[:, :table.shape[1]] = table
        # the step's token buffers are a little longer than its tokens
        return {"case": case, "cached": _ints(cs), "new": _ints(ns), "free": free, "table": rows, "tokens": sum(ns) + 5}
    h, g, d, dt = case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    t = sum(ns)
    lens = [c + n for c, n in zip(cs, ns)]
    table, pool, _ = _tables(case, seed, lens)
    s = {"case": case, "table": table, "k_pages": _normal(seed, 3, (pool, g, page, d), dt),
         "v_pages": _normal(seed, 4, (pool, g, page // 8, d, 8), dt)}
    starts = [0]
    for n in ns:
        starts.append(starts[-1] + n)
    if kind == "append":
        # one packed row per token, as a QKV product leaves it
        s["qkv"] = _normal(seed, 5, (t, h + 2 * g, d), dt)
        pos = torch.cat([torch.arange(c, c + n, device=DEV) for c, n in zip(cs, ns)])
        req = torch.repeat_interleave(torch.arange(b, device=DEV), torch.tensor(ns, device=DEV))
        s["positions"] = pos.to(torch.int32)
        s["slots"] = (table[req, pos // page].long() * page + pos % page).to(torch.int32)
        freq = 500000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEV) / d)
        ang = torch.arange(max(lens), dtype=torch.float64, device=DEV)[:, None] * freq[None, :]
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        return s
    s["q"] = _normal(seed, 5, (t, h, d), dt, 2.0)     # peaked attention: scores of deviation 2
    s["q_start"], s["kv_len"], s["max_new"], s["max_len"] = _ints(starts), _ints(lens), max(ns), max(lens)
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, h + 1, dtype=torch.float32, device=DEV) / h) if case["slopes"] else None
    pre = torch.randint(0, case["prefix"] + 1, (b,), generator=_gen(seed, 6), device=DEV)
    s["prefix"] = pre.to(torch.int32) if case["prefix"] else None
    return s


# ------------------------------------------------------------------------------------------------ one pass

_ctx = None


def _context():
    """The handle a server keeps: a context of the library (its own small target plays no part here)."""
    global _ctx
    if _ctx is None:
        from types import SimpleNamespace

        from paper_2604_17701_amd import binding
        m = SimpleNamespace(n_layers=1, d_model=64, n_heads=1, n_kv_heads=1, head_dim=64, d_ff=64, vocab=64, dtype="f32",
                            rms_eps=1e-5, rope_theta=10000.0, d_draft=8, d_csi=1, d_head_hidden=8, head_act=0)
        z = lambda *shape: torch.zeros(shape, device=DEV)  # noqa: E731
        w = {"embed": z(64, 64), "lm_head": z(64, 64), "final_norm": z(64), "head_w1": z(8, 73), "head_b1": z(8),
             "head_w2": z(8), "head_b2": z(1)}
        for n in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
            w[n] = [z(64, 64)]
        w["attn_norm"], w["ffn_norm"] = [z(64)], [z(64)]
        _ctx = binding.Context(m, w, 1, 32, 1)
    return _ctx


def run(s):
    return {"plan": _run_plan, "append": _run_append, "attend": _run_attend}[s["case"]["kind"]](s)


def _run_plan(s):
    page, tokens = s["case"]["page"], s["tokens"]
    if own:
        return tuple(_context().wisv_paged_plan(s["cached"], s["new"], s["free"], s["table"], page, tokens)) + (s["table"],)
    cached, new, free, table = s["cached"].long(), s["new"].long(), s["free"], s["table"]
    total = cached + new
    have = (cached + page - 1) // page
    need = (total + page - 1) // page - have
    q_end = new.cumsum(0)
    too_long, over = total > table.shape[1] * page, q_end > tokens
    need = torch.where(too_long | over, torch.zeros_like(need), need)
    last = need.cumsum(0)
    short = (need > 0) & (last > free.numel())
    served = ~(too_long | over | short)
    status = short.int() + 2 * too_long.int() + 4 * over.int()
    used = torch.where(served & (need > 0), last, torch.zeros_like(last)).amax().int().reshape(1)
    q_end = q_end.clamp(max=tokens)
    q_start = torch.cat([torch.zeros_like(q_end[:1]), q_end])
    kv_len = torch.where(served, total, cached)
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    first = last - need
    fresh = served[:, None] & (col >= have[:, None]) & (col < (have + need)[:, None])
    table = torch.where(fresh, free[(first[:, None] + col - have[:, None]).clamp(0, free.numel() - 1)], table)
    t = torch.arange(tokens, device=DEV)
    r = torch.searchsorted(q_end, t, right=True).clamp(max=cached.numel() - 1)
    live = t < q_end[-1]
    pos = torch.where(live, cached[r] + t - q_start[r], torch.zeros_like(t))
    pages = table[r, (pos // page).clamp(max=table.shape[1] - 1)].long()
    slots = torch.where(live & served[r] & (pages >= 0), pages * page + pos % page, torch.full_like(t, -1))
    return q_start.int(), kv_len.int(), pos.int(), slots.int(), used, status, table


def _rotate(x, c, s):
    """Pairs (i, i + dim / 2) turned by the angle of their row."""
    a, b = x.float().chunk(2, -1)
    c, s = c[:, None, :], s[:, None, :]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _run_append(s):
    h, g, page = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["page"]
    q, k, v = s["qkv"][:, :h], s["qkv"][:, h:h + g], s["qkv"][:, h + g:]
    kp, vp = s["k_pages"], s["v_pages"]
    if own:
        return _context().wisv_paged_append(q, k, v, s["positions"], s["slots"], kp, vp, cos=s["cos"], sin=s["sin"]), kp, vp
    pos, slot = s["positions"].long(), s["slots"].long()
    c, sn = s["cos"][pos], s["sin"][pos]
    at, off = slot // page, slot % page
    kp[at, :, off] = _rotate(k, c, sn).to(kp.dtype)
    vp[at, :, off // 8, :, off % 8] = v
    return _rotate(q, c, sn).to(q.dtype), kp, vp


def _run_attend(s):
    case = s["case"]
    if own:
        return _context().wisv_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["q_start"], s["kv_len"],
                                               max_new=s["max_new"], max_len=s["max_len"], softcap=case["softcap"],
                                               window=case["window"], slopes=s["slopes"], prefix_len=s["prefix"])
    h, g, d, b = case["heads"], case["kv_heads"], case["dim"], case["batch"]
    rep, n, t = h // g, s["max_new"], s["q"].shape[0]
    table = s["table"].long().clamp(min=0)
    L = table.shape[1] * case["page"]
    k = s["k_pages"][table].permute(0, 2, 1, 3, 4).reshape(b, g, L, d).float()
    v = s["v_pages"][table].permute(0, 2, 1, 3, 5, 4).reshape(b, g, L, d).float()
    start, length = s["q_start"].long(), s["kv_len"].long()
    i = torch.arange(n, device=DEV)
    q = s["q"][(start[:-1, None] + i).clamp(max=t - 1)].float()                                       # [b, n, h, d]
    q = q.reshape(b, n, g, rep, d).permute(0, 2, 3, 1, 4).reshape(b, g, rep * n, d)
    x = torch.matmul(q, k.transpose(2, 3)).reshape(b, g, rep, n, L).mul_(1.0 / math.sqrt(d))
    if case["softcap"]:
        x = x.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    p = (length - (start[1:] - start[:-1]))[:, None] + i                                              # [b, n] positions
    j = torch.arange(L, device=DEV)
    if s["slopes"] is not None:
        x += s["slopes"].reshape(1, g, rep, 1, 1) * (j - p[:, :, None]).float()[:, None, None]
    sees = j <= p[:, :, None]
    if case["window"]:
        sees &= j > p[:, :, None] - case["window"]
    if s["prefix"] is not None:
        sees |= j < s["prefix"].long()[:, None, None]
    sees &= j < length[:, None, None]
    x.masked_fill_(~sees[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top > float("-inf"), top, torch.zeros_like(top))).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(b, g, rep * n, L), v).reshape(b, g, rep, n, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(b, n, h, d)
    row = torch.arange(t, device=DEV)
    r = torch.searchsorted(start[1:], row, right=True)
    return o[r, row - start[r]].to(s["q"].dtype)


# ------------------------------------------------------------------------------------------------ required work

def work(case):
    cs, ns = _lengths(case)
    page, t = case["page"], sum(ns)
    pages = sum(_pages(c + n, page) for c, n in zip(cs, ns))
    if case["kind"] == "plan":
        fresh = pages - sum(_pages(c, page) for c in cs)
        return {"bytes": 4 * (len(cs) * 5 + 2 * fresh + 2 * t + len([n for n in ns if n])), "flops": 0}
    h, g, d, e = case["heads"], case["kv_heads"], case["dim"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "append":
        rows = max(c + n for c, n in zip(cs, ns))
        return {"bytes": 2 * t * (h + 2 * g) * d * e + 8 * t + 4 * d * min(t, rows), "flops": 3 * t * (h + g) * d}
    pairs = keys = 0
    w, pre = case["window"], case["prefix"] // 2
    for c, n in zip(cs, ns):
        if not n:
            continue
        lo = max(0, c - w + 1) if w else 0                    # the first key that the first query's window holds
        keys += c + n - lo + min(pre, lo)
        if w:
            ramp = max(0, min(n, w - c))                      # queries whose window still holds everything before them
            pairs += ramp * c + ramp * (ramp + 1) // 2 + (n - ramp) * w
        else:
            pairs += n * c + n * (n + 1) // 2
    return {"bytes": 2 * keys * g * d * e + 2 * t * h * d * e + 4 * pages, "flops": 4 * d * h * pairs}


# ------------------------------------------------------------------------------------------------ 64-bit results

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return None
    h, g, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    if case["kind"] == "append":
        x = s["qkv"].double()
        half = d // 2
        z = torch.complex(x[:, :h + g, :half].contiguous(), x[:, :h + g, half:].contiguous())
        turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()]
        z = z * turn[:, None, :]
        rot = torch.cat([z.real, z.imag], -1)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        slot = s["slots"].long()
        flat = kp.transpose(1, 2).reshape(-1, g, d)
        flat[slot] = rot[:, h:]
        kp = flat.reshape(-1, page, g, d).transpose(1, 2).contiguous()
        flat = vp.permute(0, 2, 4, 1, 3).reshape(-1, g, d)
        flat[slot] = x[:, h + g:]
        vp = flat.reshape(-1, page // 8, 8, g, d).permute(0, 3, 1, 4, 2).contiguous()
        return rot[:, :h], kp, vp
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    starts, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    prefix = s["prefix"].tolist() if s["prefix"] is not None else [0] * len(lens)
    rep = h // g
    for b, length in enumerate(lens):
        n = starts[b + 1] - starts[b]
        if not n:
            continue
        ids = s["table"][b, :_pages(length, page)].long()
        keep = torch.arange(length, device=DEV)
        at = torch.arange(length - n, length, device=DEV)
        far = at[:, None] - keep[None, :]
        hidden = far < 0
        if case["window"]:
            hidden = hidden | (far >= case["window"])
        hidden = hidden & (keep >= prefix[b])[None, :]
        for gh in range(g):
            k = s["k_pages"][ids, gh].reshape(-1, d)[:length].double()
            v = s["v_pages"][ids, gh].transpose(2, 3).reshape(-1, d)[:length].double()
            for r in range(rep):
                head = gh * rep + r
                z = s["q"][starts[b]:starts[b + 1], head].double() @ k.t() / math.sqrt(d)
                if case["softcap"]:
                    z = case["softcap"] * torch.tanh(z / case["softcap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][head].double() * far
                z = z.masked_fill(hidden, float("-inf"))
                out[starts[b]:starts[b + 1], head] = torch.softmax(z, -1) @ v
    return out
