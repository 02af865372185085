"""Measured cases of the attention side of a decode step: the block tables and slot maps of a step (moe_kv_assign), the
norm and rotation of queries and keys with the write into the paged cache (moe_qk_norm_rope), and the attention of single
tokens over that cache (moe_attn_decode).  `run` computes an operator in elementary torch operations, or with `own` through the
library's entry points; `exact` states the definitions again in 64 bits.

The cache is two tensors [pages, key/value heads, tokens of a page, head size]; token t of a request is in page
block_table[request, t // tokens] at place t % tokens, and slot = page * tokens + place.  Pages sit at shuffled places, as in a
pool that has been in use."""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
THETA = 1e6                                      # base of the rotation frequencies


def listed():
    return [
        # the tables of a decode step: one new token for each request of a micro-batch, one seat of it vacant
        _assign("assign_decode_b36", 36, 60, 700, 1, 1, 16, empty=1),
        # prompts of 77 tokens on average and 418 at most go into an empty cache: 128 requests of one prefill micro-batch
        _assign("assign_prefill_b128", 128, 0, 0, 30, 418, 16),
        # a large mixed step of chunked prompts and single tokens, more of them than there are pages, rows padded to a fixed number
        _assign("assign_mixed_b4000", 4000, 1, 30000, 1, 900, 64, short=True, pad=777),
        # single precision, a handful of tokens: launches and latency
        _rope("rope_tiny_f32_t5", 5, 4, 2, 64, 16, dtype="f32", x="f32", far=600),
        # a decode micro-batch of 256 tokens of the 8x7B shape, projection in float32, norms of both
        _rope("rope_decode_t256", 256, 32, 8, 128, 16, far=32000),
        # a prefill micro-batch of the 8x22B shape, no norms, ragged number of rows with padding rows behind
        _rope("rope_prefill_t9857", 9857, 48, 8, 128, 16, norm=False, far=64000, pad=31),
        # single precision, pages of 7 tokens, a few short requests
        _attn("attn_tiny_f32_b3", 3, 1, 130, 4, 2, 64, 7, dtype="f32"),
        # decode of the micro-batch of the tables above: the smallest calls in which bandwidth counts
        _attn("attn_decode_b36", 36, 60, 700, 32, 8, 128, 16, empty=1),
        # prompts, every token a row of its own that sees the tokens up to itself
        _attn("attn_prompts_n6", 6, 30, 418, 32, 8, 128, 16, prompt=True),
        # one very long request: the split along the cache and the join
        _attn("attn_long_b1", 1, 131001, 131001, 48, 8, 128, 64),
        # a window of 1000 tokens over long caches, one head per key/value head, head size 96
        _attn("attn_window_b61", 61, 300, 9000, 20, 20, 96, 32, window=1000),
        # a full decode batch: 256 requests of 500 to 5000 tokens
        _attn("attn_decode_b256", 256, 500, 5000, 32, 8, 128, 16),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _assign(name, B, lo, hi, new_lo, new_hi, page, short=False, pad=0, empty=0):
    return _named(name, {"op": "assign", "B": B, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "page": page, "short": short, "pad": pad, "empty": empty})


def _rope(name, T, n_q, n_kv, D, page, dtype="bf16", x="f32", norm=True, pairs=False, rot=None, far=4000, pad=0):
    return _named(name, {"op": "rope", "T": T, "n_q": n_q, "n_kv": n_kv, "D": D, "page": page, "dtype": dtype, "x": x, "norm": norm, "pairs": pairs,
                         "rot": D if rot is None else rot, "far": far, "pad": pad})


def _attn(name, B, lo, hi, n_q, n_kv, D, page, dtype="bf16", window=0, prompt=False, empty=0):
    return _named(name, {"op": "attn", "B": B, "lo": lo, "hi": hi, "n_q": n_q, "n_kv": n_kv, "D": D, "page": page, "dtype": dtype, "window": window,
                         "prompt": prompt, "empty": empty})


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    n_kv = rng.choice([1, 2, 4, 8, 8, 8, 20])
    return n_kv * rng.choice([1, 3, 4, 4, 5, 6, 7] if n_kv > 1 else [1, 4, 7, 16, 24]), n_kv


def draw(rng):
    op = rng.choice(["assign", "rope", "rope", "attn", "attn", "attn"])
    page = rng.choice([1, 5, 7, 16, 16, 32, 64, 100, 256])
    if op == "assign":
        if rng.random() < 0.5:                   # decode
            lo = _log_uniform(rng, 1, 3000)
            return _assign("", _log_uniform(rng, 1, 4000), lo, lo * rng.randint(1, 9), 1, 1, page, empty=rng.randint(0, 1))
        new = _log_uniform(rng, 4, 2000)
        return _assign("", min(4000, max(1, _log_uniform(rng, 1, 400000) // new)), 1, _log_uniform(rng, 2, 20000), 1, new, page, short=rng.random() < 0.3, pad=rng.choice([0, 9, 500]))
    n_q, n_kv = _heads(rng)
    D, dtype = rng.choice([64, 96, 128, 128, 128, 256]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "rope":
        T = _log_uniform(rng, 1, max(2, 80_000_000 // ((n_q + 2 * n_kv) * D)))
        return _rope("", T, n_q, n_kv, D, page, dtype, rng.choice(["f32", "f32", "bf16"]) if dtype == "bf16" else "f32", rng.random() < 0.5, rng.random() < 0.3,
                     rng.choice([D, D, D // 2]), _log_uniform(rng, 100, 1000000), rng.choice([0, 0, 3]) if T > 8 else 0)
    if rng.random() < 0.25:
        hi = _log_uniform(rng, 20, 900)
        return _attn("", max(1, _log_uniform(rng, 20, 1500) // hi), max(1, hi // 4), hi, n_q, n_kv, D, page, dtype, prompt=True)
    hi = _log_uniform(rng, 10, 100000)
    lo = max(1, int(hi * rng.choice([0.02, 0.3, 1.0])))
    token_bytes = 2 * n_kv * D * (2 if dtype == "bf16" else 4)
    most = max(1, min(600, 1_200_000_000 // (hi * token_bytes)))     # the plain form pads every request to the longest
    return _attn("", _log_uniform(rng, 1, most), lo, hi, n_q, n_kv, D, page, dtype, rng.choice([0, 0, 0, 17, 500, 4096]), empty=rng.choice([0, 0, 1]))


def _spread(n, lo, hi, empty=0):
    """n whole numbers from lo to hi, even on a logarithmic scale (lo 0: all zero unless hi is more); the last `empty` of more than one are 0."""
    if hi <= 0:
        return [0] * n
    lo = max(lo, 1)
    v = [min(hi, int(round(lo * (hi / lo) ** (((i + 1) * 0.6180339887498949) % 1.0)))) for i in range(n)]
    return v[:n - empty] + [0] * empty if n > empty else v


def _shuffled(v, rng):
    return np.asarray(v, dtype=np.int64)[rng.permutation(len(v))]


def _pages_of(lens, page):
    return -(-np.asarray(lens, dtype=np.int64) // page)


def _assign_sizes(case):
    cached = _spread(case["B"], case["lo"], case["hi"])
    fresh = _spread(case["B"], case["new_lo"], case["new_hi"], case["empty"])
    return cached, fresh


def _rows(case):
    """(lengths the rows attend to, their requests, the requests' lengths) in the order of the case, before the seed's permutation."""
    lens = _spread(case["B"], case["lo"], case["hi"], case["empty"])
    if not case["prompt"]:
        return lens, list(range(case["B"])), lens
    return [t + 1 for n in lens for t in range(n)], [b for b, n in enumerate(lens) for _ in range(n)], lens


def _table(held, width, pages, rng):
    """Block table [len(held), width] with held[b] of the shuffled pages in row b and -1 behind, and the pages that are left over."""
    order = rng.permutation(pages).astype(np.int32)
    held = np.asarray(held, dtype=np.int64)
    table = np.full((len(held), width), -1, dtype=np.int32)
    row, place = np.repeat(np.arange(len(held)), held), np.arange(held.sum()) - np.repeat(np.cumsum(held) - held, held)
    table[row, place] = order[:held.sum()]
    return table, order[held.sum():]


def _cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    P = case["page"]
    st = dict(case)
    if case["op"] == "assign":
        a, f = _assign_sizes(case)
        cached, fresh = _shuffled(a, rng), _shuffled(f, rng)
        held = _pages_of(cached, P)
        need = int((_pages_of(cached + fresh, P) - held).sum())
        taken, spare = 3, 5                      # free pages that went to earlier steps, and that stay
        table, free = _table(held, int(_pages_of(cached.max() + fresh.max(), P)) + 1, int(held.sum()) + taken + need + spare, rng)
        if case["short"]:
            free = free[:taken + need * 3 // 4]
        st.update(rows=int(fresh.sum()) + case["pad"], pool=int(held.sum()) + taken + need + spare, cached=_cuda(cached), fresh=_cuda(fresh), table=_cuda(table),
                  free=_cuda(free), head=_cuda([taken]))
        if own:
            import paper_2411_11217_amd as M
            st["M"], st["kv"] = M, M.make_kv_shape(1, 1, 64, P, table.shape[1], st["pool"], "bf16")
            st["step"] = M.KvStep(st["kv"], case["B"], st["rows"])
        return st

    n_q, n_kv, D, dt = case["n_q"], case["n_kv"], case["D"], DTYPES[case["dtype"]]
    if case["op"] == "rope":
        T = case["T"]
        pages = -(-T // P) + 4
        slots = rng.permutation(pages * P)[:T]
        slots[T - case["pad"]:] = -1
        st.update(x_in=normal((T, (n_q + 2 * n_kv) * D), 1.5, DTYPES[case["x"]]), slots=_cuda(slots), positions=_cuda(rng.integers(0, case["far"], T)),
                  inv_freq=torch.tensor([THETA ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)], dtype=torch.float64).cuda(),
                  q_gamma=1.0 + normal((D,), 0.1, torch.float32) if case["norm"] else None, k_gamma=1.0 + normal((D,), 0.1, torch.float32) if case["norm"] else None,
                  k_cache=normal((pages, n_kv, P, D), 1.0, dt), v_cache=normal((pages, n_kv, P, D), 1.0, dt))
        if own:
            import paper_2411_11217_amd as M
            st["M"], st["kv"] = M, M.make_kv_shape(n_q, n_kv, D, P, 1, pages, case["dtype"])
            st["q"] = torch.empty((T, n_q, D), dtype=dt, device="cuda")
        return st

    lens, request, per_request = _rows(case)
    order = rng.permutation(len(lens)) if not case["prompt"] else np.arange(len(lens))
    lens = np.asarray(lens)[order]
    if not case["prompt"]:
        per_request = lens
    held = _pages_of(per_request, P)
    pages = int(held.sum()) + 3
    table, _ = _table(held, max(1, int(held.max())), pages, rng)
    st.update(q=normal((len(lens), n_q, D), 2.5, dt), lens=_cuda(lens), table=_cuda(table), k_cache=normal((pages, n_kv, P, D), 1.0, dt),
              v_cache=normal((pages, n_kv, P, D), 1.0, dt), request=_cuda(request) if case["prompt"] else None, longest=int(lens.max()))
    if own:
        import paper_2411_11217_amd as M
        st["M"], st["kv"] = M, M.make_kv_shape(n_q, n_kv, D, P, table.shape[1], pages, case["dtype"])
        st["ws"] = M.AttnWorkspace(st["kv"], len(lens))
        st["out"] = torch.empty((len(lens), n_q, D), dtype=dt, device="cuda")
    return st


def run(st):
    if own:
        M = st["M"]
        if st["op"] == "assign":
            s = M.moe_kv_assign(st["kv"], st["cached"], st["fresh"], st["free"], st["head"], st["table"], step=st["step"])
            return {"seq_len": s.seq_len, "row_start": s.row_start, "positions": s.positions, "slots": s.slots, "request": s.request, "free_head": s.free_head,
                    "table": st["table"]}
        if st["op"] == "rope":
            q = M.moe_qk_norm_rope(st["kv"], st["x_in"], st["inv_freq"], st["positions"], st["slots"], st["k_cache"], st["v_cache"], q_gamma=st["q_gamma"],
                                   k_gamma=st["k_gamma"], eps=EPS, pairs=st["pairs"], q=st["q"])
            return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
        out, _ = M.moe_attn_decode(st["kv"], st["q"], st["lens"], st["table"], st["k_cache"], st["v_cache"], window=st["window"], table_row=st["request"], out=st["out"],
                                   workspace=st["ws"])
        return {"out": out}
    return {"assign": _plain_assign, "rope": _plain_rope, "attn": _plain_attn}[st["op"]](st)


def _plain_assign(st):
    P, B, T, table = st["page"], st["B"], st["rows"], st["table"]
    cached, fresh = st["cached"].long(), st["fresh"].long()
    ends = fresh.cumsum(0)
    held = (cached + P - 1) // P
    need = (cached + fresh + P - 1) // P - held
    fits = (ends <= T) & (held + need <= table.shape[1])
    need = torch.where(fits, need, 0)
    upto = need.cumsum(0)
    left = st["free"].numel() - st["head"].long()
    served = fits & ((need == 0) | (upto <= left))
    page = torch.arange(int(table.shape[1]), device="cuda")[None]
    new = served[:, None] & (page >= held[:, None]) & (page < (held + need)[:, None])
    which = st["head"].long() + (upto - need)[:, None] + page - held[:, None]
    table.copy_(torch.where(new, st["free"][which.clamp(0, st["free"].numel() - 1)], table))
    r = torch.arange(T, device="cuda")
    b = torch.searchsorted(ends, r, right=True)
    live = b < B
    b = b.clamp(max=B - 1)
    start = ends - fresh
    pos = torch.where(live, cached[b] + r - start[b], 0)
    slot = torch.where(live & served[b], table[b, (pos // P).clamp(max=table.shape[1] - 1)].long() * P + pos % P, -1)
    used = torch.where(served & (need > 0), upto, 0).amax()
    i32 = torch.int32
    return {"seq_len": torch.where(served, cached + fresh, cached).to(i32), "row_start": torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=T).to(i32),
            "positions": pos.to(i32), "slots": slot.to(i32), "request": torch.where(live, b, -1).to(i32), "free_head": (st["head"] + used).to(i32), "table": table}


def _rotated(x, cos, sin, rot, pairs):
    """x [T, heads, D] float32; cos and sin [T, 1, rot / 2]."""
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        both = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        both = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([both, x[..., rot:]], dim=-1)


def _plain_rope(st):
    n_q, n_kv, D, P, T = st["n_q"], st["n_kv"], st["D"], st["page"], st["T"]
    x = st["x_in"].float().view(T, n_q + 2 * n_kv, D)
    angle = st["positions"].double()[:, None] * st["inv_freq"][None]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def head(v, gamma):
        if gamma is not None:
            v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * gamma
        return _rotated(v, cos, sin, st["rot"], st["pairs"])

    dt = st["k_cache"].dtype
    q = head(x[:, :n_q], st["q_gamma"]).to(dt)
    k = head(x[:, n_q:n_q + n_kv], st["k_gamma"]).to(dt)
    v = x[:, n_q + n_kv:].to(dt)
    slot = st["slots"].long()
    stays = slot >= 0                            # a row without a slot writes what the first row with one writes
    src = torch.where(stays, torch.arange(T, device="cuda"), stays.int().argmax())
    slot = slot[src]
    st["k_cache"][slot // P, :, slot % P] = k[src]
    st["v_cache"][slot // P, :, slot % P] = v[src]
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _plain_attn(st):
    n_q, n_kv, D, P = st["n_q"], st["n_kv"], st["D"], st["page"]
    lens = st["lens"].long()[:, None]
    whole = st["request"] is not None            # every request's keys once for all of its rows
    first = (lens - st["window"]).clamp(min=0) if st["window"] and not whole else torch.zeros_like(lens)
    span = min(st["longest"], st["window"]) if st["window"] and not whole else st["longest"]
    t = torch.arange(span, device="cuda")[None] + (first if not whole else 0)
    table = st["table"].clamp(min=0).long()
    page = torch.gather(table, 1, (t // P).clamp(max=table.shape[1] - 1).expand(table.shape[0], span))

    def gathered(cache):                         # [requests, key/value heads, tokens, D]
        return cache[page, :, (t % P).expand_as(page)].permute(0, 2, 1, 3).float().contiguous()

    k, v = gathered(st["k_cache"]), gathered(st["v_cache"])
    q = st["q"].float().view(-1, n_kv, n_q // n_kv, D)
    seen = t < lens
    if st["window"]:
        seen = seen & (t >= lens - st["window"])

    def attend(q, k, v, seen):
        s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D)
        s = torch.where(seen[:, None, None], s, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
        total = p.sum(-1, keepdim=True)
        return torch.matmul(p, v) / torch.where(total > 0, total, 1.0)

    if st["request"] is None:
        out = attend(q, k, v, seen)
    else:                                        # rows of one request against its keys together: they are consecutive, in the requests' order
        lens_of, at, parts = _spread(st["B"], st["lo"], st["hi"], st["empty"]), 0, []
        for b, n in enumerate(lens_of):
            parts.append(attend(q[at:at + n].permute(1, 2, 0, 3).reshape(1, n_kv, -1, D), k[b:b + 1, :, :n], v[b:b + 1, :, :n],
                                seen[at:at + n, :n].repeat(n_q // n_kv, 1)[None, None]).view(n_kv, n_q // n_kv, n, D).permute(2, 0, 1, 3)
                         if n else q[:0])
            at += n
        out = torch.cat(parts)
    return {"out": out.reshape(-1, n_q, D).to(st["q"].dtype)}


def work(case):
    P = case["page"]
    if case["op"] == "assign":
        cached, fresh = _assign_sizes(case)
        c, f = np.asarray(cached), np.asarray(fresh)
        T, B = int(f.sum()) + case["pad"], case["B"]
        # which length meets which number of new tokens is the seed's: the pages of an average pairing
        need = float(f.sum()) / P + float((f > 0).sum()) * (P - 1) / P / (2 if case["hi"] else 1) if P > 1 else float(f.sum())
        return {"bytes": 4 * (2 * B + B + 2 * need + 2 * B + 1 + 3 * T), "flops": 3 * T}
    n_q, n_kv, D = case["n_q"], case["n_kv"], case["D"]
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rope":
        n = case["T"] * (n_q + 2 * n_kv) * D
        live = case["T"] * n_q * D + (case["T"] - case["pad"]) * 2 * n_kv * D
        return {"bytes": n * (4 if case["x"] == "f32" else 2) + live * b + 8 * case["T"], "flops": 8 * n}
    lens, _, per_request = _rows(case)
    w = case["window"] or 1 << 40
    seen = sum(min(n, w) for n in lens)
    tokens = sum(min(n, w) for n in per_request)
    return {"bytes": 2 * tokens * n_kv * D * b + 2 * len(lens) * n_q * D * b + 4 * len(lens) + 4 * tokens / P, "flops": 4 * seen * n_q * D}


def exact(case, seed):
    st = prepare(case, seed)
    return {"assign": _exact_assign, "rope": _exact_rope, "attn": _exact_attn}[case["op"]](st)


def _exact_assign(st):
    """Request by request, token by token, as the definition reads."""
    P, T = st["page"], st["rows"]
    cached, fresh, free = (st[n].cpu().numpy() for n in ("cached", "fresh", "free"))
    table = st["table"].cpu().numpy().copy()
    head, width = int(st["head"].item()), table.shape[1]
    positions, slots, request = np.zeros(T, np.int32), np.full(T, -1, np.int32), np.full(T, -1, np.int32)
    seq_len, row_start = cached.copy(), np.zeros(len(cached) + 1, np.int32)
    row, wanted = 0, 0
    used = head
    for b, (c, n) in enumerate(zip(cached.tolist(), fresh.tolist())):
        total = math.ceil((c + n) / P)
        need = total - math.ceil(c / P)
        good = row + n <= T and total <= width
        if good:
            wanted += need
            good = need == 0 or head + wanted <= len(free)
            if good:
                for i in range(need):
                    table[b, total - need + i] = free[head + wanted - need + i]
                seq_len[b] = c + n
                used = head + wanted if need else used
        for i in range(n):
            if row + i < T:
                p = c + i
                positions[row + i], request[row + i] = p, b
                slots[row + i] = table[b, p // P] * P + p % P if good else -1
        row += n
        row_start[b + 1] = min(row, T)
    out = {"seq_len": seq_len, "row_start": row_start, "positions": positions, "slots": slots, "request": request, "free_head": np.asarray([used], np.int32), "table": table}
    return {k: torch.from_numpy(v) for k, v in out.items()}


def _exact_rope(st):
    n_q, n_kv, D, P, T, rot = st["n_q"], st["n_kv"], st["D"], st["page"], st["T"], st["rot"]
    x = st["x_in"].double().view(T, n_q + 2 * n_kv, D)
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * st["inv_freq"])[:, None]

    def head(v, gamma):
        if gamma is not None:
            v = v / torch.sqrt(v.square().sum(-1, keepdim=True) / D + EPS) * gamma.double()
        turned = v.clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if st["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        w = torch.complex(v[..., first].contiguous(), v[..., second].contiguous()) * z
        turned[..., first], turned[..., second] = w.real, w.imag
        return turned

    k, v = head(x[:, n_q:n_q + n_kv], st["k_gamma"]), x[:, n_q + n_kv:]
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    rows = torch.nonzero(st["slots"] >= 0)[:, 0]
    slot = st["slots"].long()[rows]
    kc[slot // P, :, slot % P], vc[slot // P, :, slot % P] = k[rows], v[rows]
    return {"q": head(x[:, :n_q], st["q_gamma"]), "k_cache": kc, "v_cache": vc}


def _exact_attn(st):
    n_q, n_kv, D, P = st["n_q"], st["n_kv"], st["D"], st["page"]
    G = n_q // n_kv
    lens = st["lens"].tolist()
    rows = st["request"].tolist() if st["request"] is not None else list(range(len(lens)))
    out = torch.zeros((len(lens), n_q, D), dtype=torch.float64, device="cuda")
    held, k, v = -1, None, None
    for r, (b, n) in enumerate(zip(rows, lens)):
        if n <= 0:
            continue
        first = max(0, n - st["window"]) if st["window"] else 0
        if st["request"] is None or b != held:   # rows of one request are next to each other
            most = n if st["request"] is None else max(m for m, c in zip(lens, rows) if c == b)
            t = torch.arange(0 if st["request"] is not None else first, most, device="cuda")
            page, place = st["table"][b].long()[t // P], t % P
            k, v, held, base = st["k_cache"][page, :, place].double(), st["v_cache"][page, :, place].double(), b, int(t[0])
        for h in range(n_kv):
            s = (k[first - base:n - base, h] @ st["q"][r, h * G:(h + 1) * G].double().T) / math.sqrt(D)
            out[r, h * G:(h + 1) * G] = torch.softmax(s, 0).T @ v[first - base:n - base, h]
    return {"out": out}
