"""Measured cases of the layer in 8-bit integers: rows quantised with a scale each (moe_quantize_i8), the residual and RMS norm with 8-bit
rows (moe_add_rmsnorm_i8), the dense linear map (moe_linear_i8) and the experts' SwiGLU network (moe_expert_ffn_i8) as products of
8-bit integers with a scale for each token and each output channel.  `run` computes an operator in elementary torch operations, or
with `own` through the library's entry points; `exact` states the definitions again in 64 bits.

Quantisation of a row v: scale = max |v| / 127, q = the whole number next to v * (127 / max |v|), ties to even; q * scale stands for v.
A product's output is the sum of the products of whole numbers, times the scales of its row and of its column.  Rows held in 8 bits come back
as the values that they stand for, in bf16."""
import math

import torch

own = False

KIB, MIB = 1 << 10, 1 << 20
EPS = 1e-5

# hidden size, expert FFN size, experts, experts per token, page size
SHAPES = {
    "8x7b": (4096, 14336, 8, 2, 2 * MIB),        # the repository's Mixtral-8x7B shape
    "fine": (2048, 1024, 64, 8, 1 * MIB),        # as many experts as the library takes, each of them small
    "mid": (2048, 4096, 8, 2, 2 * MIB),          # a layer of a smaller model
    "tiny": (256, 512, 8, 2, 64 * KIB),          # the repository's smallest workload
    "small": (1024, 2816, 8, 2, 512 * KIB),      # odd numbers of tiles
    "few": (1280, 768, 5, 3, 64 * KIB),          # odd numbers of experts and tiles
}


def listed():
    return [
        # the attention's output of a decode micro-batch, before the O projection: launch and latency
        _quantize("quantize_attention_t36", 36, 4096),
        # float32 rows out of a wider matrix, neither length a power of two
        _quantize("quantize_strided_f32_t777", 777, 2820, "f32", extra=12),
        # a weight matrix of the 8x7B shape's experts, its rows the channels
        _quantize("quantize_weight_n14336", 14336, 4096),
        # a handful of tokens of the smallest shape, first layer (no residual yet)
        _norm("norm_tiny_t5", 5, 256, hidden=False),
        # the norm before the MoE layer in a decode step of 256 requests: the router takes the bf16 rows, the experts the others
        _norm("norm_decode_t256", 256, 4096),
        # the norm before the QKV projection in a prefill micro-batch of the 8x22B shape: nobody needs bf16 rows
        _norm("norm_prefill_t9857", 9857, 6144, x=False),
        # QKV projection in a decode step of 36 requests: the weights' way from memory
        _linear("linear_decode_t36", 36, 4096, 6144),
        # O projection of a full decode micro-batch
        _linear("linear_decode_t256", 256, 4096, 4096),
        # QKV projection of a prefill micro-batch of the 8x22B shape, ragged number of rows
        _linear("linear_prefill_t9857", 9857, 6144, 8192),
        # the smallest workload: launches and latency
        _ffn("experts_tiny_t64", "tiny", 64),
        # decode: every expert's weights once for some 64 rows
        _ffn("experts_decode_8x7b_t256", "8x7b", 256),
        # the benchmark's number of tokens, two fifths of the rows on one expert, one expert with hardly any
        _ffn("experts_batch_8x7b_t4096", "8x7b", 4096, skew=True),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _quantize(name, T, N, dtype="bf16", extra=0):
    return _named(name, {"op": "quantize", "T": T, "N": N, "dtype": dtype, "extra": extra})


def _norm(name, T, H, hidden=True, x=True):
    return _named(name, {"op": "norm", "T": T, "H": H, "hidden": hidden, "x": x})


def _linear(name, T, K, N, page=64 * KIB):
    return _named(name, {"op": "linear", "T": T, "K": K, "N": N, "page": page})


def _ffn(name, shape, T, skew=False):
    return _named(name, {"op": "ffn", "shape": shape, "T": T, "skew": skew})


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "norm", "linear", "linear", "ffn", "ffn"])
    if op == "quantize":
        N = 4 * _log_uniform(rng, 1, 7000)
        return _quantize("", _log_uniform(rng, 1, max(1, min(60000, 58_000_000 // N))), N, rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 0, 4, 128]))
    if op == "norm":
        H = rng.choice([256, 512, 1024, 2048, 2880, 4096, 5120, 6144, 8192, 4 * rng.randint(1, 2048)])
        return _norm("", _log_uniform(rng, 1, max(1, min(60000, 60_000_000 // H))), H, rng.random() < 0.8, rng.random() < 0.6)
    if op == "linear":
        K, N = 256 * _log_uniform(rng, 1, 56), 128 * _log_uniform(rng, 1, 128)
        return _linear("", _log_uniform(rng, 1, max(2, min(12000, 490_000_000_000 // (K * N)))), K, N, rng.choice([16 * KIB, 64 * KIB, 2 * MIB]))
    shape = rng.choice(["8x7b", "fine", "mid", "mid", "small", "few", "tiny"])
    return _ffn("", shape, _log_uniform(rng, 1, 4096), rng.random() < 0.4)


def _whole_numbers(shape, g, std=30.0):
    """8-bit integers as quantised rows have them: normal values, the largest of a row some four deviations out."""
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).round_().clamp_(-127, 127).to(torch.int8)


def _scales(shape, g, about):
    """Scales of rows or channels, within a factor of three of each other."""
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(0.5 * about, 1.5 * about, generator=g)


def _shuffled_table(shape, slots, g):
    return torch.randperm(slots, generator=g, device="cuda")[:math.prod(shape)].to(torch.int32).view(shape)


def _routing(st, g):
    """The experts of every token, the rows sorted by expert in the order of the tokens, and what the library's permutation gives."""
    T, E, k = st["T"], st["E"], st["k"]
    logits = torch.empty((T, E), dtype=torch.float32, device="cuda").normal_(generator=g)
    if st["skew"]:
        logits[:, 0] += 2.5
        logits[:, E - 1] -= 1.9
    best, ids = logits.topk(k, dim=1)
    flat = ids.flatten()
    row_src = torch.sort(flat, stable=True).indices
    counts = torch.bincount(flat, minlength=E)
    st.update(offsets=torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32), row_src=row_src.to(torch.int32),
              row_w=torch.softmax(best, 1).flatten()[row_src].contiguous(), most=int(counts.max()))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case)

    def normal(shape, std, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    if own:
        import paper_2411_11217_amd as M
        st["M"] = M
    if case["op"] == "quantize":
        T, N = case["T"], case["N"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        st["v"] = normal((T, N + case["extra"]), 1.3, dt)[:, :N]
        st["q"], st["scale"] = torch.empty((T, N), dtype=torch.int8, device="cuda"), torch.empty(T, dtype=torch.float32, device="cuda")
    elif case["op"] == "norm":
        T, H = case["T"], case["H"]
        st.update(h_in=normal((T, H), 2.0) if case["hidden"] else None, delta=normal((T, H), 0.7), gamma=1.0 + normal((H,), 0.1))
    elif case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        st.update(q=_whole_numbers((T, K), g), scale=_scales(T, g, 0.03), W=_whole_numbers((N, K), g), w_scale=_scales(N, g, 7e-4))
        if own:
            st["ls"] = M.make_linear_shape(T, K, N, case["page"], "i8")
            pages = M.linear_pages_required(st["ls"])
            st["table"] = _shuffled_table((pages,), pages + 3, g)
            host = torch.zeros((pages + 3, case["page"]), dtype=torch.uint8)
            M.linear_pack(st["ls"], st.pop("W").cpu(), st["table"].cpu(), host)
            st["pool"] = host.cuda()
    else:
        H, F, E, k, page = SHAPES[case["shape"]]
        st.update(H=H, F=F, E=E, k=k, page=page)
        st.update(q=_whole_numbers((case["T"], H), g), scale=_scales(case["T"], g, 0.03), W1=_whole_numbers((E, F, H), g), W3=_whole_numbers((E, F, H), g),
                  W2=_whole_numbers((E, H, F), g), s1=_scales((E, F), g, 7e-4), s3=_scales((E, F), g, 7e-4), s2=_scales((E, H), g, 7e-4))
        _routing(st, g)
        if own:
            st["s"] = M.make_shape(case["T"], H, F, E, k, "i8", page)
            paged = M.PagedWeights(st["s"], *(st.pop(n).cpu() for n in ("W1", "W3", "W2")), order=torch.Generator().manual_seed(seed), extra_pages=3).to_device()
            st["pool"], st["table"] = paged.pages_dev, paged.table_dev
            st["scales"] = M.ExpertScales(st["s1"], st["s3"], st["s2"])
    return st


def run(st):
    if not own:
        return {"quantize": _plain_quantize, "norm": _plain_norm, "linear": _plain_linear, "ffn": _plain_ffn}[st["op"]](st)
    M = st["M"]
    if st["op"] == "quantize":
        q, scale = M.moe_quantize_i8(st["v"], x_q=st["q"], x_scale=st["scale"])
        return {"values": _values(q, scale), "scale": scale}
    if st["op"] == "norm":
        hidden, x, q, scale = M.moe_add_rmsnorm_i8(st["h_in"], st["delta"], st["gamma"], EPS, want_x=st["x"])
        return {"hidden": hidden, "x": x, "values": _values(q, scale), "scale": scale}
    if st["op"] == "linear":
        return {"out": M.moe_linear_i8(st["ls"], st["q"], st["scale"], st["table"], st["pool"], st["w_scale"])}
    _, _, out = M.moe_expert_ffn_i8(st["s"], st["q"], st["scale"], st["offsets"], st["table"], st["pool"], st["scales"], row_src=st["row_src"], row_w=st["row_w"])
    return {"out": out}


def _values(q, scale):
    """What rows held in 8 bits stand for, in one pass."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))


def _quantized(v):
    """float32 rows -> (whole numbers as float32, scales)."""
    most = v.abs().amax(-1, keepdim=True)
    scale = (most / torch.full_like(most, 127.0)).clamp(min=2.0 ** -126)
    inverse = torch.where(most > 0, 127.0 / most.clamp(min=2.0 ** -119), 0.0)
    return torch.round(v * inverse), scale


def _plain_quantize(st):
    q, scale = _quantized(st["v"].float())
    return {"values": (q * scale).to(torch.bfloat16), "scale": scale[:, 0]}


def _plain_norm(st):
    s = st["delta"] if st["h_in"] is None else st["h_in"] + st["delta"]
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + EPS) * st["gamma"]
    q, scale = _quantized(y)
    return {"hidden": s, "x": y.to(torch.bfloat16) if st["x"] else None, "values": (q * scale).to(torch.bfloat16), "scale": scale[:, 0]}


def _plain_linear(st):
    return {"out": torch.matmul(st["q"].float(), st["W"].float().T) * st["scale"][:, None] * st["w_scale"]}


def _plain_ffn(st):
    E, most = st["E"], st["most"]
    start = st["offsets"][:-1, None].long()
    row = start + torch.arange(most, device="cuda")                # [E, most]: every expert's rows, the missing ones another's
    here = row < st["offsets"][1:, None]
    row = row.clamp(max=st["row_src"].numel() - 1)
    token = (st["row_src"].long() // st["k"])[row]
    x, scale = st["q"].float()[token], st["scale"][token][..., None]

    def times(a, W, per_channel):
        return torch.matmul(a, W.float().transpose(1, 2)) * per_channel[:, None]

    gate, up = times(x, st["W1"], st["s1"]) * scale, times(x, st["W3"], st["s3"]) * scale
    h = (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16).float()
    q, h_scale = _quantized(h)
    out = times(q, st["W2"], st["s2"]) * h_scale * st["row_w"][row][..., None]
    return {"out": out[here].to(torch.bfloat16)}


def work(case):
    if case["op"] == "quantize":
        n = case["T"] * case["N"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + n + 4 * case["T"], "flops": 3 * n}
    if case["op"] == "norm":
        n = case["T"] * case["H"]
        return {"bytes": n * (4 + 4 * case["hidden"] + 4 + 2 * case["x"] + 1) + 4 * case["T"] + 4 * case["H"], "flops": 7 * n}
    if case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        return {"bytes": T * K + N * K + 4 * T * N + 4 * (T + N), "flops": 2 * T * K * N}
    H, F, E, k, _ = SHAPES[case["shape"]]
    T = case["T"]
    chosen = E * (1.0 - (1.0 - k / E) ** T)      # experts with rows, of an average routing
    return {"bytes": chosen * (3 * H * F + 4 * (2 * F + H)) + T * (H + 4) + T * k * (2 * H + 8), "flops": 6 * T * k * H * F}


def exact(case, seed):
    st = prepare(case, seed)
    return {"quantize": _exact_quantize, "norm": _exact_norm, "linear": _exact_linear, "ffn": _exact_ffn}[case["op"]](st)


def _exact_rows(v):
    """The nearest multiples of a 127th of each row's largest magnitude, and that step."""
    step = torch.linalg.vector_norm(v, ord=math.inf, dim=1) / 127
    return torch.where(step > 0, torch.div(v.T, step).round() * step, 0.0).T.contiguous(), step


def _exact_quantize(st):
    values, step = _exact_rows(st["v"].double())
    return {"values": values, "scale": step}


def _exact_norm(st):
    s = st["delta"].double()
    if st["h_in"] is not None:
        s = s + st["h_in"].double()
    y = s * torch.rsqrt(s.square().sum(1) / s.shape[1] + EPS)[:, None] * st["gamma"].double()
    values, step = _exact_rows(y)
    return {"hidden": s, "x": y if st["x"] else None, "values": values, "scale": step}


def _exact_linear(st):
    return {"out": (st["q"].double() * st["scale"].double()[:, None]) @ (st["W"].double() * st["w_scale"].double()[:, None]).T}


def _exact_ffn(st):
    bounds, parts = st["offsets"].tolist(), []
    for e, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        if a == b:
            continue
        token = torch.div(st["row_src"][a:b].long(), st["k"], rounding_mode="floor")
        x = st["q"][token].double() * st["scale"][token].double()[:, None]
        g = x @ (st["W1"][e].double() * st["s1"][e].double()[:, None]).T
        h = torch.nn.functional.silu(g) * (x @ (st["W3"][e].double() * st["s3"][e].double()[:, None]).T)
        values, _ = _exact_rows(h.bfloat16().double())               # rounded to bf16 before the 8 bits: part of the definition
        parts.append(values @ (st["W2"][e].double() * st["s2"][e].double()[:, None]).T * st["row_w"][a:b].double()[:, None])
    return {"out": torch.cat(parts)}
