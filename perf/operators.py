"""The prompt side of the library as cases that can be timed: what a serving program does between a layer's projections
and the compression of its cache.

Four operators.  `rope`: per-head norms of queries and keys and the position rotation in one pass, keys and values into
the cache.  `attn`: attention of a chunk of new tokens over the cache, which the chunk's own rows are part of.  `mass`:
the attention weight that each cached token receives from the last queries, summed over the query heads of its KV head.
`evict`: the tokens that are kept when a cache is cut down by that weight, and the cache cut down to them.

The cache is contiguous ([B, Hkv, max_len, 128]) or, with `page` > 0, a pool of pages ([pages, Hkv, page, 128]) with a
page table per sequence.  Head counts are those of sik_workloads.py and the tests.

Keys of a case: op; batch, n_kv_heads, n_q_heads; dtype ("bf16" | "fp16"); n (new tokens per sequence), past (tokens in the
cache before them), ragged (unequal sequences: past and n fall from these values), page; and by operator
  rope   to ("cache" | "rows": a decode step's rows, which sik_decode_step appends itself), fused (q, k and v are views of
         one projection), norm, rotary (rotated channels), interleaved (pairs of neighbours instead of halves)
  mass   n_obs (queries of each sequence that count), add (the weights join those of earlier calls)
  evict  past (tokens of the longest sequence), n_keep, n_sink, n_recent, rows (False: the list of kept tokens only)
"""
import math
import random

import torch

own = False

D = 128
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 1 << 27  # logits that the plain forms hold at a time


def _case(op, batch, n_kv_heads, n_q_heads, n, past, **more):
    c = dict(op=op, batch=batch, n_kv_heads=n_kv_heads, n_q_heads=n_q_heads, n=n, past=past, dtype="bf16", ragged=False,
             page=0)
    c.update({"rope": dict(to="cache", fused=True, norm=True, rotary=D, interleaved=False),
              "attn": dict(), "mass": dict(n_obs=min(n, 64), add=False),
              "evict": dict(n_keep=64, n_sink=0, n_recent=0, rows=True)}[op])
    c.update(more)
    return c


def listed():
    return [
        # one token of one user: the rows that the decode step takes, latency only
        dict(_case("rope", 1, 8, 32, 1, 32768, to="rows"), name="rope-token"),
        # an ordinary prompt chunk of a small batch, from a fused projection into contiguous caches
        dict(_case("rope", 4, 8, 32, 2048, 2048), name="rope-4x2048"),
        # unequal prompts into a paged cache, part of the channels rotated in neighbouring pairs, 5 heads to a KV head
        dict(_case("rope", 7, 8, 40, 777, 1500, dtype="fp16", ragged=True, page=64, rotary=64, interleaved=True, norm=False),
             name="rope-paged-ragged-gqa5"),
        # one token over a 32K context in full: what a layer without selection does at each step
        dict(_case("attn", 1, 8, 32, 1, 32767), name="attn-token-32k"),
        # a whole prompt at once, no history
        dict(_case("attn", 1, 8, 32, 8192, 0), name="attn-prompt-8k"),
        # a server's ordinary moment: unequal chunks and histories over pages, 5 query heads to a KV head
        dict(_case("attn", 6, 8, 40, 333, 9000, dtype="fp16", ragged=True, page=16), name="attn-paged-ragged-gqa5"),
        # the last chunk of a 128K prompt over pages: the most arithmetic there is in one call
        dict(_case("attn", 1, 8, 32, 2048, 129024, page=64), name="attn-chunk-128k-paged"),
        # after a 32K prompt: the weight that its tokens get from the last 64 queries
        dict(_case("mass", 1, 8, 32, 2048, 30720, n_obs=64), name="mass-last64-32k"),
        # a batch that generates: one token's weights join the sums of the tokens before
        dict(_case("mass", 8, 8, 64, 1, 16383, add=True, page=64, n_obs=1), name="mass-token-8x16k-paged"),
        # the 64 full-precision sink tokens of a batch of long prompts: the list only
        dict(_case("evict", 4, 8, 32, 1, 65536, rows=False), name="evict-sinks-4x64k"),
        # a full batch cut down to an eighth, first and last tokens kept in any case
        dict(_case("evict", 32, 8, 32, 1, 16384, n_keep=2048, n_sink=4, n_recent=64), name="evict-32x16k"),
        # short unequal sequences out of pages, some of them shorter than what is kept
        dict(_case("evict", 5, 2, 6, 1, 1777, n_keep=500, n_recent=33, ragged=True, page=32, dtype="fp16"),
             name="evict-ragged-paged"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["rope", "rope", "attn", "attn", "attn", "mass", "mass", "evict", "evict"])
    n_kv, n_q = rng.choice([(8, 32), (8, 32), (8, 40), (8, 64), (4, 28), (2, 6), (8, 8), (1, 4)])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([0, 0, 16, 32, 64, 128])
    batch = _log_uniform(rng, 1, 32)
    ragged = batch > 1 and rng.random() < 0.5
    common = dict(dtype=dtype, page=page, ragged=ragged)
    if op == "rope":
        n = max(1, min(_log_uniform(rng, 1, 8192), 8192 * 48 // (batch * (n_q + 2 * n_kv))))
        past = _log_uniform(rng, 1, max(2, min(32768, (1 << 21) // (batch * n_kv))))
        return _case(op, batch, n_kv, n_q, n, past, to=rng.choice(["cache", "cache", "rows"]), fused=rng.random() < 0.7,
                     norm=rng.random() < 0.7, rotary=rng.choice([128, 128, 64, 96, 32]), interleaved=rng.random() < 0.3,
                     **common)
    if op == "attn":
        past = _log_uniform(rng, 1, max(2, min(131072, (1 << 22) // (batch * n_kv))))
        n = rng.choice([1, _log_uniform(rng, 2, 64), _log_uniform(rng, 64, 8192)])
        # no more logits than the last chunk of the 128K prompt
        n = max(1, min(n, 32 * 2048 * 130000 // (2 * batch * n_q * (past + n))))
        return _case(op, batch, n_kv, n_q, n, past, **common)
    if op == "mass":
        past = _log_uniform(rng, 64, max(128, min(131072, (1 << 22) // (batch * n_kv))))
        n_obs = rng.choice([1, _log_uniform(rng, 2, 32), _log_uniform(rng, 32, 256)])
        n_obs = max(1, min(n_obs, (1 << 32) // (batch * n_q * past)))
        n = n_obs if rng.random() < 0.5 else _log_uniform(rng, n_obs, 2 * n_obs + 64)
        return _case(op, batch, n_kv, n_q, n, past, n_obs=n_obs, add=rng.random() < 0.4, **common)
    past = _log_uniform(rng, 512, max(1024, min(131072, (1 << 22) // (batch * n_kv))))
    n_keep = _log_uniform(rng, 16, min(past, 8192))
    n_sink, n_recent = rng.choice([(0, 0), (4, n_keep // 4), (0, n_keep // 2), (min(64, n_keep // 3), 1)])
    return _case(op, batch, n_kv, n_q, 1, past, n_keep=n_keep, n_sink=n_sink, n_recent=n_recent, rows=rng.random() < 0.7,
                 **common)


def _lengths(case):
    """(tokens before the chunk, tokens of the chunk) of each sequence."""
    B, past, n = case["batch"], case["past"], case["n"]
    if not case["ragged"]:
        return [past] * B, [n] * B
    pasts = [past - (3 * past // 4) * b // (B - 1) for b in range(B)]
    news = [n - (n // 2) * ((b * 5) % B) // (B - 1) for b in range(B)]
    return pasts, news


def _capacity(case):
    """Tokens that a sequence's cache holds: the longest sequence and a little room, whole pages of them."""
    most = case["past"] + (case["n"] if case["op"] != "evict" else 0)
    unit = case["page"] or 8
    return (most + 8 + unit - 1) // unit * unit


def _table(case, gen):
    """Page table of a paged case (a random order of the pool's pages) and the number of pages, else (None, 0)."""
    if not case["page"]:
        return None, 0
    per = _capacity(case) // case["page"]
    pages = case["batch"] * per + 3
    return torch.randperm(pages, generator=gen, device="cuda")[:case["batch"] * per].view(case["batch"], per).int(), pages


def _rows(shape, gen, dtype, channels=False):
    x = torch.randn(shape, generator=gen, device="cuda")
    if channels:  # keys and values: channels of unequal spread, a few of them far larger
        s = torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))
        s[torch.randperm(D, generator=gen, device="cuda")[:2]] *= 8.0
        x *= s
    return x.to(TORCH[dtype])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, Hkv, Hq, n, op = case["batch"], case["n_kv_heads"], case["n_q_heads"], case["n"], case["op"]
    pasts, news = _lengths(case)
    cap, dt = _capacity(case), case["dtype"]
    table, pages = _table(case, gen)
    shape = (pages, Hkv, case["page"], D) if case["page"] else (B, Hkv, cap, D)
    st = dict(case=case, pasts=pasts, news=news, table=table, cap=cap,
              seq_len=torch.tensor(pasts, dtype=torch.int32, device="cuda"),
              n_new=torch.tensor(news, dtype=torch.int32, device="cuda") if case["ragged"] else None)
    if op == "rope":
        if case["fused"]:
            qkv = _rows((B, n, (Hq + 2 * Hkv) * D), gen, dt)
            st["q"] = qkv[:, :, :Hq * D].unflatten(2, (Hq, D))
            st["k"] = qkv[:, :, Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
            st["v"] = qkv[:, :, (Hq + Hkv) * D:].unflatten(2, (Hkv, D))
        else:
            st["q"], st["k"], st["v"] = (_rows((B, n, h, D), gen, dt) for h in (Hq, Hkv, Hkv))
        st["qw"] = 1.0 + 0.2 * torch.randn(D, generator=gen, device="cuda") if case["norm"] else None
        st["kw"] = 1.0 + 0.2 * torch.randn(D, generator=gen, device="cuda") if case["norm"] else None
        r = case["rotary"]
        st["inv_freq"] = (500000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)).float()
        st["q_out"] = torch.zeros(B, n, Hq, D, dtype=TORCH[dt], device="cuda")
        if case["to"] == "rows":
            st["k_out"] = torch.zeros(B, n, Hkv, D, dtype=TORCH[dt], device="cuda")
        else:
            st["K"], st["V"] = (torch.zeros(shape, dtype=TORCH[dt], device="cuda") for _ in range(2))
    else:
        if op != "evict" or case["rows"]:
            st["K"] = _rows(shape, gen, dt, channels=True)
        if op == "attn" or (op == "evict" and case["rows"]):
            st["V"] = _rows(shape, gen, dt, channels=True)
    if op in ("attn", "mass"):
        st["q"] = _rows((B, n, Hq, D), gen, dt)
    if op == "attn":
        st["out"] = torch.zeros(B, n, Hq, D, dtype=TORCH[dt], device="cuda")
        st["lse"] = torch.zeros(B, n, Hq, device="cuda")
    if op == "mass":
        st["lse"] = _lse_of_last(st, case["n_obs"])
        st["before"] = torch.rand(B, Hkv, cap, generator=gen, device="cuda") if case["add"] else None
        st["mass"] = torch.zeros(B, Hkv, cap, device="cuda")
    if op == "evict":
        w = torch.exp(2.0 * torch.randn(B, Hkv, cap, generator=gen, device="cuda"))
        # weights so small that they vanished in the sums: equal masses, of which the first tokens go first
        st["mass"] = torch.where(torch.rand(B, Hkv, cap, generator=gen, device="cuda") < 0.3, 0.0, w)
        st["keep"] = torch.zeros(B, Hkv, case["n_keep"], dtype=torch.int32, device="cuda")
        st["new_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        if case["rows"]:
            st["K_out"], st["V_out"] = (torch.zeros(B, Hkv, case["n_keep"] + 8, D, dtype=TORCH[dt], device="cuda")
                                        for _ in range(2))
            st["mass_out"] = torch.zeros(B, Hkv, case["n_keep"] + 8, device="cuda")
    if own:
        import paper_2603_14224_amd as sik
        st["layout"] = sik.make_layout(B, Hkv, Hq, D, cap, TORCH[dt])
        st["pages"] = sik.make_pages(table, case["page"], pages) if case["page"] else None
        st["chunk"] = sik.make_chunk(n, st["seq_len"], n_new=st["n_new"], pages=st["pages"])
        if op in ("attn", "evict"):
            st["ws"] = sik.alloc_chunk_workspace(st["layout"], n)
    return st


def _cached(st, which, b, h, length):
    """Rows 0 .. length of one KV head of one sequence, in their 16-bit type."""
    x = st[which]
    if st["table"] is None:
        return x[b, h, :length]
    page = st["case"]["page"]
    return x[st["table"][b, :(length + page - 1) // page].long(), h].flatten(0, 1)[:length]


def _lse_of_last(st, n_obs):
    """Logarithms of the softmax sums of the last n_obs queries of each sequence (elsewhere zero), from 64-bit sums."""
    B, n, Hq, _ = st["q"].shape
    R = Hq // st["case"]["n_kv_heads"]
    lse = torch.zeros(B, n, Hq, device="cuda")
    for b, (past, new) in enumerate(zip(st["pasts"], st["news"])):
        t0 = max(0, new - n_obs)
        for h in range(Hq // R):
            k = _cached(st, "K", b, h, past + new).double()
            for t in range(t0, new, 64):
                t1 = min(new, t + 64)
                s = st["q"][b, t:t1, h * R:(h + 1) * R].double() @ k.T / math.sqrt(D)
                unseen = torch.arange(past + new, device="cuda") > past + torch.arange(t, t1, device="cuda")[:, None]
                lse[b, t:t1, h * R:(h + 1) * R] = s.masked_fill_(unseen[:, None], -math.inf).logsumexp(-1).float()
    return lse


# ------------------------------------------------------------------------------------------------- the plain forms, 32 bits

def _norm_rotate(x, weight, angle, interleaved):
    """x [n, heads, D] -> its norm times the weight, the first channels rotated by angle [n, pairs]."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    half = angle.shape[-1]
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat([torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2), rest], -1)
    a, b = head[..., :half], head[..., half:]
    return torch.cat([a * c - b * s, a * s + b * c, rest], -1)


def _rope_plain(st):
    case = st["case"]
    for b, (past, new) in enumerate(zip(st["pasts"], st["news"])):
        at = torch.arange(past, past + new, device="cuda")
        angle = at[:, None].double() * st["inv_freq"].double()  # far positions need 64 bits
        q = _norm_rotate(st["q"][b, :new], st["qw"], angle, case["interleaved"])
        k = _norm_rotate(st["k"][b, :new], st["kw"], angle, case["interleaved"])
        st["q_out"][b, :new] = q.to(st["q_out"].dtype)
        if case["to"] == "rows":
            st["k_out"][b, :new] = k.to(st["k_out"].dtype)
        elif st["table"] is None:
            st["K"][b, :, past:past + new] = k.transpose(0, 1).to(st["K"].dtype)
            st["V"][b, :, past:past + new] = st["v"][b, :new].transpose(0, 1)
        else:
            page, row = st["table"][b, at // case["page"]].long(), at % case["page"]
            st["K"][page, :, row] = k.to(st["K"].dtype)
            st["V"][page, :, row] = st["v"][b, :new]
    return _rope_outputs(st)


def _rope_outputs(st):
    return [st["q_out"], st["k_out"]] if st["case"]["to"] == "rows" else [st["q_out"], st["K"], st["V"]]


def _attn_plain(st):
    _, _, Hq, _ = st["q"].shape
    R = Hq // st["case"]["n_kv_heads"]
    for b, (past, new) in enumerate(zip(st["pasts"], st["news"])):
        for h in range(Hq // R):
            k = _cached(st, "K", b, h, past + new).float()
            v = _cached(st, "V", b, h, past + new).float()
            step = max(1, BLOCK // (R * (past + new)))
            for t in range(0, new, step):
                t1 = min(new, t + step)
                seen = past + t1
                s = (st["q"][b, t:t1, h * R:(h + 1) * R].float() @ k[:seen].T) * (1.0 / math.sqrt(D))
                unseen = torch.arange(seen, device="cuda") > past + torch.arange(t, t1, device="cuda")[:, None]
                s = s.masked_fill_(unseen[:, None], -math.inf)
                m = s.amax(-1, keepdim=True)
                p = torch.exp(s.sub_(m))
                l = p.sum(-1, keepdim=True)
                st["out"][b, t:t1, h * R:(h + 1) * R] = ((p @ v[:seen]) / l).to(st["out"].dtype)
                st["lse"][b, t:t1, h * R:(h + 1) * R] = (m + torch.log(l))[..., 0]
    return [st["out"], st["lse"]]


def _mass_plain(st):
    _, _, Hq, _ = st["q"].shape
    R, n_obs = Hq // st["case"]["n_kv_heads"], st["case"]["n_obs"]
    for b, (past, new) in enumerate(zip(st["pasts"], st["news"])):
        t0 = max(0, new - n_obs)
        for h in range(Hq // R):
            k = _cached(st, "K", b, h, past + new).float()
            got = st["before"][b, h, :past + new].clone() if st["before"] is not None else \
                torch.zeros(past + new, device="cuda")
            step = max(1, BLOCK // (R * (past + new)))
            for t in range(t0, new, step):
                t1 = min(new, t + step)
                s = (st["q"][b, t:t1, h * R:(h + 1) * R].float() @ k.T) * (1.0 / math.sqrt(D))
                p = torch.exp(s - st["lse"][b, t:t1, h * R:(h + 1) * R, None])
                unseen = torch.arange(past + new, device="cuda") > past + torch.arange(t, t1, device="cuda")[:, None]
                got += p.masked_fill_(unseen[:, None], 0.0).sum((0, 1))
            st["mass"][b, h, :past + new] = got
    return [st["mass"]]


def _evict_plain(st):
    case = st["case"]
    n_keep, n_sink, n_recent = case["n_keep"], case["n_sink"], case["n_recent"]
    for b, length in enumerate(st["pasts"]):
        kept = min(length, n_keep)
        st["new_len"][b] = kept
        mass = st["mass"][b, :, :length]
        if length <= n_keep:
            order = torch.arange(length, device="cuda").expand(mass.shape[0], -1)
        else:
            middle = mass[:, n_sink:length - n_recent]
            best = torch.sort(middle, dim=-1, descending=True, stable=True)[1][:, :n_keep - n_sink - n_recent] + n_sink
            first = torch.arange(n_sink, device="cuda").expand(mass.shape[0], -1)
            last = torch.arange(length - n_recent, length, device="cuda").expand(mass.shape[0], -1)
            order = torch.cat([first, torch.sort(best, dim=-1)[0], last], -1)
        st["keep"][b, :, :kept] = order.int()
        st["keep"][b, :, kept:] = -1
        if case["rows"]:
            for h in range(mass.shape[0]):
                st["K_out"][b, h, :kept] = _cached(st, "K", b, h, length)[order[h]]
                st["V_out"][b, h, :kept] = _cached(st, "V", b, h, length)[order[h]]
            st["mass_out"][b, :, :kept] = torch.gather(mass, 1, order)
    return _evict_outputs(st)


def _evict_outputs(st):
    more = [st["K_out"], st["V_out"], st["mass_out"]] if st["case"]["rows"] else []
    return [st["keep"], st["new_len"], *more]


# ------------------------------------------------------------------------------------------------- the framework's calls

def run(st):
    case, op = st["case"], st["case"]["op"]
    if not own:
        return {"rope": _rope_plain, "attn": _attn_plain, "mass": _mass_plain, "evict": _evict_plain}[op](st)
    import paper_2603_14224_amd as sik
    if op == "rope":
        rows = case["to"] == "rows"
        sik.sik_rope_append(st["layout"], st["chunk"], st["q"], st["k"], st["q_out"], v=None if rows else st["v"],
                            k_out=st["k_out"] if rows else None, K=None if rows else st["K"],
                            V=None if rows else st["V"], q_weight=st["qw"], k_weight=st["kw"], eps=1e-6,
                            inv_freq=st["inv_freq"], interleaved=case["interleaved"])
        return _rope_outputs(st)
    if op == "attn":
        sik.sik_chunk_attn(st["layout"], st["chunk"], st["q"], st["K"], st["V"], 0.0, st["out"], st["lse"], st["ws"])
        return [st["out"], st["lse"]]
    if op == "mass":
        sik.sik_attn_mass(st["layout"], st["chunk"], st["q"], st["K"], 0.0, st["lse"], case["n_obs"], st["before"],
                          st["mass"])
        return [st["mass"]]
    rows = case["rows"]
    sik.sik_evict(st["layout"], st["mass"], st["seq_len"], case["n_keep"], st["keep"], st["ws"], n_sink=case["n_sink"],
                  n_recent=case["n_recent"], new_len=st["new_len"], pages=st["pages"] if rows else None,
                  K=st["K"] if rows else None, V=st["V"] if rows else None, K_out=st["K_out"] if rows else None,
                  V_out=st["V_out"] if rows else None, mass_out=st["mass_out"] if rows else None)
    return _evict_outputs(st)


def work(case):
    """Bytes that have to be read and written, and the multiplications and additions of the products."""
    pasts, news = _lengths(case)
    Hkv, Hq, op = case["n_kv_heads"], case["n_q_heads"], case["op"]
    tokens = sum(news)
    seen = sum(p + n for p, n in zip(pasts, news))
    if op == "rope":
        heads = Hq + Hkv + (Hkv if case["to"] == "cache" else 0)
        return {"bytes": tokens * heads * D * 2 * 2, "flops": tokens * (Hq + Hkv) * D * 7}
    if op == "attn":
        pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(pasts, news))
        return {"bytes": seen * Hkv * D * 4 + tokens * Hq * (D * 4 + 4), "flops": pairs * Hq * D * 4}
    if op == "mass":
        obs = [min(n, case["n_obs"]) for n in news]
        pairs = sum(o * (p + n) - o * (o - 1) // 2 for p, n, o in zip(pasts, news, obs))
        sums = seen * Hkv * 4 * (2 if case["add"] else 1)
        return {"bytes": seen * Hkv * D * 2 + sum(obs) * Hq * (D * 2 + 4) + sums, "flops": pairs * Hq * D * 2}
    kept = sum(min(p, case["n_keep"]) for p in pasts)
    rows = kept * Hkv * (D * 8 + 4) if case["rows"] else 0
    return {"bytes": sum(pasts) * Hkv * 4 + case["batch"] * Hkv * case["n_keep"] * 4 + rows, "flops": sum(pasts) * Hkv}


# ------------------------------------------------------------------------------------------------- the definitions, 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    B, Hkv, Hq = case["batch"], case["n_kv_heads"], case["n_q_heads"]
    R, op, dev, f64 = Hq // Hkv, case["op"], "cuda", torch.float64

    def slots(b, tokens):  # where a sequence's tokens lie in the cache seen as [places, Hkv, D]
        if st["table"] is None:
            return b * st["cap"] + tokens
        return st["table"][b].long()[tokens // case["page"]] * case["page"] + tokens % case["page"]

    def flat(x):  # the cache with the places in front
        return x.transpose(1, 2).flatten(0, 1)

    def unflat(x, like):
        return x.unflatten(0, (like.shape[0], like.shape[2])).transpose(1, 2).contiguous()

    if op == "rope":
        rot = case["rotary"]
        first = torch.arange(rot // 2, device=dev) * (2 if case["interleaved"] else 1)
        second = first + (1 if case["interleaved"] else rot // 2)

        def turned(x, weight, phase):
            y = x.to(f64)
            if weight is not None:
                y = y / torch.sqrt(torch.sum(y ** 2, -1, keepdim=True) / D + 1e-6) * weight.to(f64)
            z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(phase), phase)[:, None]
            y[..., first], y[..., second] = z.real, z.imag
            return y

        q_ref = torch.zeros(st["q_out"].shape, dtype=f64, device=dev)
        rows = case["to"] == "rows"
        k_ref = torch.zeros(st["k_out"].shape if rows else flat(st["K"]).shape, dtype=f64, device=dev)
        v_ref = None if rows else torch.zeros_like(k_ref)
        for b in range(B):
            new, at = st["news"][b], st["pasts"][b] + torch.arange(st["news"][b], device=dev)
            phase = at.to(f64)[:, None] * st["inv_freq"].to(f64)[None]
            q_ref[b, :new] = turned(st["q"][b, :new].clone(), st["qw"], phase)
            k = turned(st["k"][b, :new].clone(), st["kw"], phase)
            if rows:
                k_ref[b, :new] = k
            else:
                k_ref[slots(b, at)] = k
                v_ref[slots(b, at)] = st["v"][b, :new].to(f64)
        return [q_ref, k_ref] if rows else [q_ref, unflat(k_ref, st["K"]), unflat(v_ref, st["V"])]

    if op == "evict":
        keep = torch.full(st["keep"].shape, -1, dtype=torch.int32, device=dev)
        mass = st["mass"].cpu().tolist()
        picks = []
        for b in range(B):
            length = st["pasts"][b]
            lo, hi = case["n_sink"], length - case["n_recent"]
            for h in range(Hkv):
                if length <= case["n_keep"]:
                    chosen = list(range(length))
                else:
                    m = mass[b][h]
                    best = sorted(range(lo, hi), key=lambda i: -m[i])[:case["n_keep"] - lo - case["n_recent"]]
                    chosen = sorted([*range(lo), *best, *range(hi, length)])
                keep[b, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
                picks.append(torch.tensor(chosen, device=dev))
        new_len = torch.tensor([min(p, case["n_keep"]) for p in st["pasts"]], dtype=torch.int32, device=dev)
        if not case["rows"]:
            return [keep, new_len]
        outs = [torch.zeros(st[x].shape, dtype=f64, device=dev) for x in ("K_out", "V_out", "mass_out")]
        for i, pick in enumerate(picks):
            b, h = divmod(i, Hkv)
            at = slots(b, pick)
            outs[0][b, h, :len(pick)] = flat(st["K"])[at, h].to(f64)
            outs[1][b, h, :len(pick)] = flat(st["V"])[at, h].to(f64)
            outs[2][b, h, :len(pick)] = st["mass"][b, h, pick].to(f64)
        return [keep, new_len, *outs]

    n = case["n"]
    out = torch.zeros(B, n, Hq, D, dtype=f64, device=dev)
    lse = torch.zeros(B, n, Hq, dtype=f64, device=dev)
    total = torch.zeros(B, Hkv, st["cap"], dtype=f64, device=dev)
    for b in range(B):
        past, new = st["pasts"][b], st["news"][b]
        at = slots(b, torch.arange(past + new, device=dev))
        for hq in range(Hq):
            k = flat(st["K"])[at, hq // R].to(f64)
            v = flat(st["V"])[at, hq // R].to(f64) if op == "attn" else None
            start = 0 if op == "attn" else max(0, new - case["n_obs"])
            size = max(1, (1 << 26) // (past + new))
            for t in range(start, new, size):
                rows = torch.arange(t, min(new, t + size), device=dev)
                e = torch.matmul(st["q"][b, rows, hq].to(f64), k.T) / math.sqrt(D)
                allowed = torch.arange(past + new, device=dev)[None] <= past + rows[:, None]
                if op == "attn":
                    top = torch.where(allowed, e, -math.inf).max(1, keepdim=True)[0]
                    w = torch.where(allowed, torch.exp(e - top), 0.0)
                    norm = w.sum(1, keepdim=True)
                    out[b, rows, hq] = torch.matmul(w / norm, v)
                    lse[b, rows, hq] = (top + norm.log())[:, 0]
                else:
                    w = torch.where(allowed, torch.exp(e - st["lse"][b, rows, hq].to(f64)[:, None]), 0.0)
                    total[b, hq // R, :past + new] += w.sum(0)
        if op == "mass" and st["before"] is not None:
            total[b, :, :past + new] += st["before"][b, :, :past + new].to(f64)
    return [out, lse] if op == "attn" else [total]
