"""What the operators around a prompt and the cache's pages are measured on: queries and keys normed per head and rotated by their
positions, causal attention over whole prompts in 16 bits, and the block tables, lengths, positions and slots of a step with the free
pages behind them.

A case is one layer's pass (for the pages: one step of all sequences, there and back, so that it can be repeated).  What a serving
program keeps (plans, weights, pools, output buffers) is made once (`prepare`).
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
DIM = 128
EPS = 1e-6
MOST_PAIRS = 64 * 32768 * 32768          # query heads x tokens^2 of the largest listed attention; draws stay below it
MOST_ROWS = 72 * 32768                   # rows of heads of the largest listed rotation
PIECE = 1 << 28                          # scores that the plain attention has at once

DEFAULTS = {
    "kind": "attend",                    # attend | rotate | pages
    "kv_heads": 8, "per_kv": 4,          # query heads per KV head; head_dim is 128
    "dtype": "f16",
    "sequences": 1, "lengths": 0,        # seed of the sequences' lengths (the same for all inputs of a case)
    "past_lo": 0, "past_hi": 0,          # tokens before the new ones: positions of a rotation, pages held
    "new_lo": 1, "new_hi": 1,            # new tokens (the prompt) of a sequence
    "fused": False,                      # q, k, v are parts of one tensor [rows, all heads, 128], as one projection leaves them
    # rotate
    "norm": True, "rotary_dim": 128, "pairs": False, "base": 500000.0, "scaling": "none", "factor": 1.0, "low": 1.0, "high": 4.0,
    "original": 8192, "amplitude": 1.0,
    # pages
    "block_tokens": 16, "leaving": 0,    # sequences that end in this step, the others being new ones; on the way back it is the other way round
}


def _case(name=None, **fields):
    case = dict(DEFAULTS, **fields)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # a question of 37 tokens, 64 query heads on 8 KV heads (Llama-3.1-70B shape): latency
        _case("attend_37", per_kv=8, new_lo=37, new_hi=37),
        # 48 short requests packed into one call, as many query heads as KV heads, q, k, v in one tensor
        _case("attend_short48", kv_heads=10, per_kv=1, dtype="bf16", sequences=48, new_lo=17, new_hi=400, lengths=3, fused=True),
        # a prompt of 8k tokens, Llama-3.1-8B shape
        _case("attend_8k", dtype="bf16", new_lo=8192, new_hi=8192),
        # a batch of ragged prompts, odd lengths, Qwen3-235B shape
        _case("attend_ragged6", kv_heads=4, per_kv=16, dtype="bf16", sequences=6, new_lo=601, new_hi=6011, lengths=5, fused=True),
        # the longest: 32k tokens, Llama-3.1-70B shape
        _case("attend_32k", per_kv=8, new_lo=32768, new_hi=32768),
        # one new token of one sequence, 8B shape, plain rotation, no norm: latency
        _case("rotate_one", kind="rotate", norm=False, dtype="bf16", past_lo=1023, past_hi=1023),
        # one step of 32 sequences far into their contexts, heads normed, frequencies in bands for long contexts
        _case("rotate_step32", kind="rotate", per_kv=8, sequences=32, past_lo=500, past_hi=131000, lengths=7, scaling="bands", factor=8.0),
        # ragged prompts, half of each head rotated in neighbouring pairs, positions far out, one tensor for q, k, v
        _case("rotate_pairs", kind="rotate", kv_heads=4, per_kv=16, dtype="bf16", norm=False, rotary_dim=64, pairs=True, base=10000.0,
              scaling="ramp", factor=4.0, low=1.0, high=32.0, amplitude=1.1386, sequences=5, past_lo=0, past_hi=900000, new_lo=301,
              new_hi=2003, lengths=9, fused=True),
        # a prompt of 32k tokens, 70B shape, heads normed
        _case("rotate_32k", kind="rotate", per_kv=8, dtype="bf16", new_lo=32768, new_hi=32768, base=1000000.0),
        # one step of 32 sequences: a page now and then
        _case("pages_step32", kind="pages", sequences=32, past_lo=511, past_hi=2047, lengths=11),
        # trees of drafts for 256 sequences, larger pages
        _case("pages_drafts256", kind="pages", sequences=256, past_lo=100, past_hi=9000, new_lo=5, new_hi=64, block_tokens=32, lengths=13),
        # 24 sequences end and prompts of up to 32k tokens take their places
        _case("pages_turnover", kind="pages", sequences=40, leaving=24, past_lo=900, past_hi=40000, new_lo=33, new_hi=32768, lengths=15),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: any operator, heads, lengths, type, layout, scaling, page size."""
    kind = rng.choice(["attend", "attend", "rotate", "rotate", "pages"])
    kv_heads, per_kv = rng.choice([(8, 8), (8, 4), (4, 16), (10, 1), (2, 5), (1, 8)])
    heads = kv_heads * per_kv
    fields = dict(kind=kind, kv_heads=kv_heads, per_kv=per_kv, dtype=rng.choice(["f16", "bf16"]), lengths=rng.randrange(1 << 20),
                  fused=rng.random() < 0.5)
    if kind == "attend":
        sequences, new = rng.choice([1, 1, 2, 5, 16, 48]), _log_int(rng, 1, 32768)
        while sequences * heads * new * new > MOST_PAIRS // 2 or sequences * new > 65536:
            new = new * 2 // 3
        return _case(sequences=sequences, new_lo=(new + 3) // 4 if sequences > 1 else new, new_hi=new, **fields)
    if kind == "rotate":
        sequences, new = rng.choice([1, 3, 32, 200]), _log_int(rng, 1, 32768)
        while sequences * new * (heads + kv_heads) > MOST_ROWS:
            new = max(new * 2 // 3, 1)
        past = _log_int(rng, 1, 1000000)
        pairs, scaling = rng.random() < 0.5, rng.choice(["none", "linear", "base", "bands", "ramp"])
        return _case(sequences=sequences, past_lo=past // 4, past_hi=past, new_lo=(new + 1) // 2, new_hi=new, norm=rng.random() < 0.6,
                     rotary_dim=rng.choice([128, 128, 96, 64, 32]), pairs=pairs, base=rng.choice([10000.0, 500000.0, 1000000.0]),
                     scaling=scaling, factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0), high=32.0 if scaling == "ramp" else 4.0,
                     amplitude=rng.uniform(1.0, 1.3) if scaling == "ramp" else 1.0, **fields)
    sequences, past, new = _log_int(rng, 1, 400), _log_int(rng, 16, 40000), _log_int(rng, 1, 32768)
    while sequences * (past + new) > 1 << 20:
        past, new = (past + 1) // 2, (new + 1) // 2
    return _case(sequences=sequences, leaving=rng.choice([0, 0, sequences // 2]), past_lo=past // 4, past_hi=past, new_lo=(new + 1) // 2,
                 new_hi=new, block_tokens=rng.choice([16, 32, 64, 128]), **fields)


# ---- inputs -----------------------------------------------------------------------------------------

def _lengths(case):
    """(tokens before the new ones, new tokens) of every sequence; the first has the most of both."""
    g = torch.Generator().manual_seed(case["lengths"] * 2 + 1)
    n = case["sequences"]
    past = torch.randint(case["past_lo"], case["past_hi"] + 1, (n,), generator=g)
    new = torch.randint(case["new_lo"], case["new_hi"] + 1, (n,), generator=g)
    past[0], new[0] = case["past_hi"], case["new_hi"]
    return past.tolist(), new.tolist()


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _heads(case, rows, seed):
    """Queries, keys and values: normal values, keys with channels of different size; one tensor, or three."""
    kv, heads, dtype = case["kv_heads"], case["kv_heads"] * case["per_kv"], DTYPES[case["dtype"]]
    g = torch.Generator(device=DEVICE).manual_seed(seed * 4 + 1)
    x = torch.empty(rows, heads + 2 * kv, DIM, dtype=dtype, device=DEVICE)
    for a in range(0, rows, 4096):
        x[a: a + 4096] = torch.randn(x[a: a + 4096].shape, generator=g, device=DEVICE).to(dtype)
    size = torch.exp(0.5 * torch.randn(kv, DIM, generator=g, device=DEVICE))
    x[:, heads: heads + kv] = (x[:, heads: heads + kv].float() * size).to(dtype)
    parts = x[:, :heads], x[:, heads: heads + kv], x[:, heads + kv:]
    return parts if case["fused"] else tuple(p.contiguous() for p in parts)


def _page_inputs(case, seed):
    """A pool in use: what the sequences hold, which pages are free, and the two steps (there and back) in tokens kept and new."""
    past, new = _lengths(case)
    n, bt, leaving = case["sequences"], case["block_tokens"], case["leaving"]
    go = torch.zeros(n, dtype=torch.bool)
    go[torch.randperm(n, generator=torch.Generator().manual_seed(case["lengths"]))[:leaving]] = True
    go = go.tolist()
    held = [p if gone or not leaving else 0 for p, gone in zip(past, go)]
    kept = [0 if gone else h for h, gone in zip(held, go)]
    fresh = [0 if gone else t for t, gone in zip(new, go)]
    back = [p if gone else 0 for p, gone in zip(past, go)]
    need = [(h + bt - 1) // bt for h in held]
    most = max(max(h, k + f) for h, k, f in zip(held, kept, fresh))
    extra = sum((k + f + bt - 1) // bt for k, f in zip(kept, fresh))
    pages = sum(need) + extra + 5
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed * 7 + 3)).to(torch.int32)
    table = torch.full((n, (most + bt - 1) // bt), -1, dtype=torch.int32)
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = order[at: at + c]
        at += c
    return {"held": held, "kept": kept, "fresh": fresh, "kept_back": kept, "fresh_back": back, "pages": pages, "most": most,
            "table": table, "free": order[at:]}


def prepare(case, seed):
    past, new = _lengths(case)
    kv, heads, dtype = case["kv_heads"], case["kv_heads"] * case["per_kv"], DTYPES[case["dtype"]]
    rows = sum(new)
    state = {"case": case}
    if own:
        from paper_2605_13734_amd import kvc
        own_type = kvc.F16 if case["dtype"] == "f16" else kvc.BF16
    if case["kind"] == "pages":
        x = _page_inputs(case, seed)
        n = case["sequences"]
        state.update(x=x, kept=_i32(x["kept"]) if case["leaving"] else None, fresh=_i32(x["fresh"]), kept_back=_i32(x["kept_back"]),
                     fresh_back=_i32(x["fresh_back"]) if case["leaving"] else None, rows=sum(x["fresh"]), rows_back=sum(x["fresh_back"]))
        state["out"] = [_i32([0] * (n + 1)), _i32([0] * n), _i32([0] * state["rows"]),
                        torch.zeros(state["rows"], dtype=torch.int64, device=DEVICE), _i32([0] * (n + 1)), _i32([0] * n)]
        if own:
            plan = kvc.CachePlan(own_type, kv, heads, DIM, block_tokens=case["block_tokens"], max_batch=n, max_tokens=x["most"])
            pages = kvc.CachePages(plan, x["pages"], n, DEVICE)
            pages.held.copy_(_i32(x["held"]))
            pages.table.copy_(x["table"])
            pages.set_free(x["free"])
            state["pages"] = pages
        else:
            free = torch.zeros(x["pages"], dtype=torch.int32)
            free[: len(x["free"])] = x["free"]
            state.update(held=_i32(x["held"]), table=x["table"].to(DEVICE), free=free.to(DEVICE), count=_i32([len(x["free"])]))
        return state
    state["q"], state["k"], state["v"] = _heads(case, rows, seed)
    if case["kind"] == "attend":
        state.update(scale=1 / math.sqrt(DIM), start=_starts(new))
        if own:
            state["prompt"] = kvc.Prompt(kvc.PromptPlan(own_type, kv, heads, DIM, max_batch=len(new)), DEVICE)
            state["batch"] = kvc.PromptBatch(_i32(state["start"]), max(new))
            state["out"] = torch.empty(rows, heads, DIM, dtype=dtype, device=DEVICE)
            state["lse"] = torch.empty(rows, heads, dtype=torch.float32, device=DEVICE)
        return state
    g = torch.Generator(device=DEVICE).manual_seed(seed * 4 + 2)
    state["positions"] = _i32([p + i for p, t in zip(past, new) for i in range(t)])
    state["q_weight"], state["k_weight"] = ((1 + 0.2 * torch.randn(DIM, generator=g, device=DEVICE)).to(dtype) for _ in "qk")
    if own:
        scalings = {"none": kvc.SCALE_NONE, "linear": kvc.SCALE_LINEAR, "base": kvc.SCALE_BASE, "bands": kvc.SCALE_BANDS, "ramp": kvc.SCALE_RAMP}
        frequencies = kvc.rotary_frequencies(case["rotary_dim"], case["base"], scalings[case["scaling"]], case["factor"], case["low"],
                                             case["high"], case["original"])
        plan = kvc.PromptPlan(own_type, kv, heads, DIM, rotary_dim=case["rotary_dim"], frequencies=frequencies,
                              layout=kvc.ROTARY_PAIRS if case["pairs"] else kvc.ROTARY_HALVES, amplitude=case["amplitude"],
                              eps=EPS if case["norm"] else None)
        state["prompt"] = kvc.Prompt(plan, DEVICE)
        state["q_out"] = torch.empty(rows, heads, DIM, dtype=dtype, device=DEVICE)
        state["k_out"] = torch.empty(rows, kv, DIM, dtype=dtype, device=DEVICE)
    else:
        state["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEVICE)
    return state


def _frequencies(case):
    """Radians per position of every pair of channels, scaled for long contexts."""
    R, base, factor = case["rotary_dim"], case["base"], case["factor"]
    if case["scaling"] == "base":
        base = base * factor ** (R / (R - 2))
    f = [base ** (-2 * i / R) for i in range(R // 2)]
    if case["scaling"] == "linear":
        return [x / factor for x in f]
    if case["scaling"] == "bands":                 # by the turns that a pair makes in the original context
        out = []
        for x in f:
            turns = case["original"] * x / (2 * math.pi)
            t = min(max((turns - case["low"]) / (case["high"] - case["low"]), 0.0), 1.0)
            out.append(t * x + (1 - t) * x / factor)
        return out
    if case["scaling"] == "ramp":                  # along the pairs, between those that make `high` and `low` turns
        at = lambda turns: R * math.log(case["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))       # noqa: E731
        first, last = max(math.floor(at(case["high"])), 0), min(math.ceil(at(case["low"])), R - 1)
        out = []
        for i, x in enumerate(f):
            t = min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
            out.append(t * x / factor + (1 - t) * x)
        return out
    return f


# ---- the plain forms --------------------------------------------------------------------------------

def _attention(case, q, k, v, start, scale, real):
    """Causal attention of every sequence in numbers of type `real`, a block of rows at a time."""
    kv, per = case["kv_heads"], case["per_kv"]
    out, lse = [], []
    for a, b in zip(start, start[1:]):
        keys, values = k[a:b].to(real).transpose(0, 1).contiguous(), v[a:b].to(real).transpose(0, 1).contiguous()
        piece = max(PIECE // (kv * per * (b - a)), 1)
        for lo in range(a, b, piece):
            hi = min(lo + piece, b)
            rows = q[lo:hi].to(real).reshape(hi - lo, kv, per, DIM).permute(1, 2, 0, 3).reshape(kv, per * (hi - lo), DIM)
            s = torch.matmul(rows, keys[:, : hi - a].transpose(1, 2)).mul_(scale).reshape(kv, per, hi - lo, hi - a)
            later = torch.arange(hi - a, device=DEVICE)[None, :] > torch.arange(lo - a, hi - a, device=DEVICE)[:, None]
            s.masked_fill_(later, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = s.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.reshape(kv, per * (hi - lo), hi - a), values[:, : hi - a]).reshape(kv, per, hi - lo, DIM) / total
            out.append(o.permute(2, 0, 1, 3).reshape(hi - lo, kv * per, DIM).to(q.dtype if real == torch.float32 else real))
            lse.append((top + total.log()).reshape(kv * per, hi - lo).transpose(0, 1))
            del s, p
    return torch.cat(out), torch.cat(lse)


def _rotated(case, x, weight, cos, sin):
    """One tensor's rows normed and rotated in 32 bits."""
    y = x.float()
    if case["norm"]:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
    R = case["rotary_dim"]
    turned, rest = y[..., :R], y[..., R:]
    if case["pairs"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).reshape(turned.shape)
    else:
        a, b = turned[..., : R // 2], turned[..., R // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _advance(state, kept, fresh, rows, out):
    """One step: pages that are no longer needed become free, the next ones are taken.  The i-th page taken is the i-th given back, and
    after those the top of the stack downwards; what is left of the given ones goes onto the stack, the first given on top."""
    bt, table, free = state["case"]["block_tokens"], state["table"], state["free"]
    held = state["held"].long()
    kept = held if kept is None else kept.long()
    fresh = torch.zeros_like(held) if fresh is None else fresh.long()
    n, places = table.shape
    pages_of = lambda t: torch.div(t + bt - 1, bt, rounding_mode="floor")                  # noqa: E731
    before, after = pages_of(held), pages_of(kept + fresh)
    start = torch.cat([torch.zeros_like(held[:1]), fresh.cumsum(0)])
    place = torch.arange(places, device=DEVICE)[None, :]
    take, give = (place >= before[:, None]) & (place < after[:, None]), (place >= after[:, None]) & (place < before[:, None])
    takes, gives = take.sum(), give.sum()
    count = state["count"][0].long()
    rank_take = (take.flatten().cumsum(0) - 1).reshape(n, places)
    rank_give = (give.flatten().cumsum(0) - 1).reshape(n, places)
    size = n * places
    # the given pages by their rank (others go to a place behind all)
    given = torch.zeros(size + 1, dtype=torch.int32, device=DEVICE)
    given.scatter_(0, torch.where(give, rank_give, size).flatten(), table.flatten())
    from_stack = free[(count - 1 - (rank_take - gives)).clamp(0, free.shape[0] - 1)]
    taken = torch.where(rank_take < gives, given[rank_take.clamp(0, size)], from_stack)
    table.copy_(torch.where(take, taken, table))
    j = torch.arange(free.shape[0], device=DEVICE)
    rank = gives - 1 - (j - count)                                 # of the page that comes to place j of the stack
    free.copy_(torch.where((j >= count) & (rank >= takes), given[rank.clamp(0, size)], free))
    state["count"].copy_((count + gives - takes).to(torch.int32).reshape(1))
    state["held"].copy_((kept + fresh).to(torch.int32))
    out[0].copy_(start.to(torch.int32))
    out[1].copy_((kept + fresh).to(torch.int32))
    if rows:
        r = torch.arange(rows, device=DEVICE)
        s = torch.searchsorted(start, r, right=True) - 1
        position = kept[s] + r - start[s]
        page = table[s, torch.div(position, bt, rounding_mode="floor")].long()
        out[2].copy_(position.to(torch.int32))
        out[3].copy_(page * bt + position % bt)


def run(state):
    case = state["case"]
    if case["kind"] == "attend":
        if own:
            stream = torch.cuda.current_stream().cuda_stream
            state["prompt"].attend(state["batch"], state["q"], state["k"], state["v"], state["out"], state["scale"], state["lse"], stream)
            return state["out"], state["lse"]
        return _attention(case, state["q"], state["k"], state["v"], state["start"], state["scale"], torch.float32)
    if case["kind"] == "rotate":
        if own:
            stream = torch.cuda.current_stream().cuda_stream
            weights = (state["q_weight"], state["k_weight"]) if case["norm"] else (None, None)
            state["prompt"].rotate(state["q"], state["k"], state["positions"], state["q_out"], state["k_out"], *weights, stream=stream)
            return state["q_out"], state["k_out"]
        angle = state["positions"].double()[:, None] * state["frequencies"]
        cos, sin = (angle.cos() * case["amplitude"]).float()[:, None], (angle.sin() * case["amplitude"]).float()[:, None]
        return (_rotated(case, state["q"], state["q_weight"], cos, sin), _rotated(case, state["k"], state["k_weight"], cos, sin))
    x, out = state["x"], state["out"]
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        pages = state["pages"]
        pages.advance(out[0], out[1], kept=state["kept"], fresh=state["fresh"], max_new=max(x["fresh"]), max_tokens=x["most"],
                      positions=out[2], slots=out[3], stream=stream)
        pages.advance(out[4], out[5], kept=state["kept_back"], fresh=state["fresh_back"], max_new=max(x["fresh_back"]),
                      max_tokens=x["most"], rows=state["rows_back"], stream=stream)
        return [*out, pages.table, pages.held, pages.free_count, pages.free_pages[: len(x["free"])]]
    _advance(state, state["kept"], state["fresh"], state["rows"], out)
    _advance(state, state["kept_back"], state["fresh_back"], 0, out[4:])
    return [*out, state["table"], state["held"], state["count"], state["free"][: len(x["free"])]]


# ---- from the definitions, in 64 bits ---------------------------------------------------------------

def _exact_attention(case, seed):
    _, new = _lengths(case)
    q, k, v = _heads(case, sum(new), seed)
    per, start = case["per_kv"], _starts(new)
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEVICE)
    step = 2048
    for a, b in zip(start, start[1:]):
        for h in range(q.shape[1]):
            key, value = k[a:b, h // per].double(), v[a:b, h // per].double()
            for i in range(a, b, step):
                e = min(i + step, b)
                s = q[i:e, h].double() @ key[: e - a].T / math.sqrt(DIM)
                s = torch.where(torch.ones_like(s, dtype=torch.bool).tril(i - a), s, -math.inf)
                lse[i:e, h] = torch.logsumexp(s, -1)
                out[i:e, h] = torch.exp(s - lse[i:e, h, None]) @ value[: e - a]
    return out, lse


def _exact_rotation(case, seed):
    past, new = _lengths(case)
    q, k, _ = _heads(case, sum(new), seed)
    g = torch.Generator(device=DEVICE).manual_seed(seed * 4 + 2)
    weights = [(1 + 0.2 * torch.randn(DIM, generator=g, device=DEVICE)).to(q.dtype).double() for _ in "qk"]
    R, f = case["rotary_dim"], _frequencies(case)
    at = torch.cat([torch.arange(p, p + t, device=DEVICE, dtype=torch.float64) for p, t in zip(past, new)])
    done = []
    for x, w in zip((q, k), weights):
        y = torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
        for lo in range(0, x.shape[0], 4096):
            z = x[lo: lo + 4096].double()
            if case["norm"]:
                z = z / torch.sqrt(z.pow(2).mean(-1, keepdim=True) + EPS) * w
            y[lo: lo + 4096] = z
            for i in range(R // 2):
                m, o = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + R // 2)
                turn = torch.polar(torch.full_like(at[lo: lo + 4096], case["amplitude"]), at[lo: lo + 4096] * f[i])
                point = torch.complex(z[..., m].contiguous(), z[..., o].contiguous()) * turn[:, None]
                y[lo: lo + 4096, :, m], y[lo: lo + 4096, :, o] = point.real, point.imag
        done.append(y)
    return tuple(done)


def _exact_pages(case, seed):
    x = _page_inputs(case, seed)
    bt, stack = case["block_tokens"], x["free"].tolist()
    tables = [[p for p in row if p >= 0] for row in x["table"].tolist()]
    held, result = list(x["held"]), []
    for kept, fresh in ((x["kept"], x["fresh"]), (x["kept_back"], x["fresh_back"])):
        kept = held if kept is None else kept
        now = [a + b for a, b in zip(kept, fresh)]
        result += [_starts(fresh), now]
        given = [p for t, m in zip(tables, now) for p in t[(m + bt - 1) // bt:]]
        stack += given[::-1]
        for i, m in enumerate(now):
            need = (m + bt - 1) // bt
            del tables[i][need:]
            while len(tables[i]) < need:
                tables[i].append(stack.pop())
        if len(result) == 2:
            position = [k + i for k, f in zip(kept, fresh) for i in range(f)]
            seq = [s for s, f in enumerate(fresh) for _ in range(f)]
            result += [position, [tables[s][p // bt] * bt + p % bt for s, p in zip(seq, position)]]
            widest = [list(t) for t in tables]
        held = now
    # what a table holds behind a sequence's pages is what was there before
    table = x["table"].clone()
    for rows in (widest, tables):
        for i, t in enumerate(rows):
            table[i, : len(t)] = torch.tensor(t, dtype=torch.int32)
    types = [torch.int32] * 3 + [torch.int64] + [torch.int32] * 2
    out = [torch.tensor(r, dtype=t, device=DEVICE) for r, t in zip(result, types)]
    return [*out, table.to(DEVICE), _i32(held), _i32([len(stack)]), _i32(stack)]


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    return {"attend": _exact_attention, "rotate": _exact_rotation, "pages": _exact_pages}[case["kind"]](case, seed)


def work(case):
    """Bytes that a pass reads and writes at least once, and its arithmetic: two products of 128 per pair of a query head's row and a
    token that it sees, or some 14 operations per element of a rotation."""
    past, new = _lengths(case)
    kv, heads, rows = case["kv_heads"], case["kv_heads"] * case["per_kv"], sum(new)
    if case["kind"] == "attend":
        return {"bytes": rows * ((2 * heads + 2 * kv) * DIM * 2 + heads * 4),
                "flops": 4 * DIM * heads * sum(t * (t + 1) // 2 for t in new)}
    if case["kind"] == "rotate":
        return {"bytes": rows * ((heads + kv) * DIM * 4 + 4), "flops": 14 * rows * (heads + kv) * DIM}
    x = _page_inputs(case, 0)
    n, bt = case["sequences"], case["block_tokens"]
    pages = sum(abs((k + f + bt - 1) // bt - (h + bt - 1) // bt) for h, k, f in zip(x["held"], x["kept"], x["fresh"]))
    return {"bytes": 2 * (n * 24 + 2 * pages * 4) + sum(x["fresh"]) * 12, "flops": 2 * n}
