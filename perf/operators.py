"""What the operators of the quantised cache are measured on: rows quantised into pages as they are written, rows read back,
attention of new or drafted tokens over the pages, and the accepted drafts of a tree moved together.

A case is one pass over one layer.  Its plan, pages, block tables and index arrays are made once (`prepare`), as a serving
program keeps them; a pass (`run`) is the calls of one step.  The plain form keeps the same cache as separate tensors (one byte
per code, scales and zeros in fp16): the framework's pages are filled and read by its own calls only.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
DIM = 128
TOP = 65504.0                 # stored values are limited to the range of the scales' and zeros' type
MOST_SCORES = 1 << 30         # query rows x tokens of the largest listed case (heads included); draws stay below it
MOST_CODES = 1 << 27          # codes of K (and of V) of the largest listed case

DEFAULTS = {
    "kind": "attend",                    # attend | verify (store, attend, keep, load) | write (store, load) | read (load)
    "kv_heads": 8, "per_kv": 4,          # query heads per KV head; head_dim is 128
    "dtype": "f16", "bits_k": 4, "bits_v": 4, "group": 32, "transform": 0, "block_tokens": 16,
    "sequences": 1, "lengths": 0,        # seed of the sequences' lengths (the same for all inputs of a case)
    "past_lo": 0, "past_hi": 0,          # tokens in the cache before the new ones
    "new_lo": 1, "new_hi": 1,            # new tokens of a sequence
    "tree": False,                       # the new tokens are a tree of drafts (a mask), not consecutive tokens
}


def _case(name=None, **fields):
    case = dict(DEFAULTS, **fields)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the smallest step: one sequence, one token, 1024 tokens of context, 64 query heads on 8 KV heads (Llama-3.1-70B shape)
        _case("attend_one_1k", per_kv=8, past_lo=1023, past_hi=1023),
        # continuous batching: 32 short sequences of odd lengths, one token each, Llama-3.1-8B shape, bf16
        _case("attend_batch32_short", dtype="bf16", group=64, sequences=32, past_lo=511, past_hi=2047, lengths=5),
        # one long-context request, one token over 128k tokens, Llama-3.1-8B shape
        _case("attend_long_128k", past_lo=131071, past_hi=131071),
        # four ragged long requests, 64 query heads on 4 KV heads (Qwen3-235B shape), K at 8 bits and V at 4, pages of 64 tokens
        _case("attend_ragged4_k8v4", kv_heads=4, per_kv=16, dtype="bf16", bits_k=8, group=128, block_tokens=64,
              sequences=4, past_lo=16383, past_hi=32767, lengths=3),
        # speculative decoding: trees of 64 drafts over 8k tokens of context, K rotated
        _case("attend_tree64_8k", per_kv=8, transform=1, sequences=8, past_lo=8191, past_hi=8191, new_lo=64, new_hi=64, tree=True),
        # a chunk of a long prompt: 512 tokens over the 32k before them, both tensors at 8 bits
        _case("attend_chunk512_32k", per_kv=8, dtype="bf16", bits_k=8, bits_v=8, group=64, past_lo=32256, past_hi=32256,
              new_lo=512, new_hi=512),
        # a whole verification step of one request: 15 drafts written, attended, the accepted ones moved together and read back
        _case("verify_one_1k", kind="verify", past_lo=1000, past_hi=1000, new_lo=15, new_hi=15, tree=True),
        # the same for 32 short sequences with up to 32 drafts each
        _case("verify_batch32", kind="verify", per_kv=8, dtype="bf16", group=64, block_tokens=32, sequences=32, past_lo=511, past_hi=2047,
              new_lo=17, new_hi=32, lengths=9, tree=True),
        # the rows of one decoding step of 32 sequences, written and read back (a copy for a replica)
        _case("write_step32", kind="write", sequences=32, past_lo=511, past_hi=2047, lengths=7),
        # a prompt of 32k tokens as one layer has it, K rotated, written and read back for a 16-bit attention over the prompt
        _case("write_prompt_32k", kind="write", transform=1, new_lo=32768, new_hi=32768),
        # a short prefix read back
        _case("read_1k", kind="read", dtype="bf16", new_lo=1024, new_hi=1024),
        # four ragged long caches read back for a transfer, odd lengths
        _case("read_ragged4_k8v4", kind="read", kv_heads=4, per_kv=16, dtype="bf16", bits_k=8, group=64, block_tokens=64,
              sequences=4, new_lo=16384, new_hi=32768, lengths=11),
    ]


def draw(rng):
    """One more case of the same ranges: any kind, shape, length, type, width, group, page size and mask."""
    kind = rng.choice(["attend", "attend", "attend", "verify", "write", "read"])
    kv_heads, per_kv = rng.choice([(8, 8), (8, 4), (4, 16), (8, 1), (2, 5), (1, 8)])
    sequences = rng.choice([1, 1, 2, 4, 7, 32])
    past = int(round(2 ** rng.uniform(4, 17)))
    tree = kind == "verify" or rng.random() < 0.3
    new = 1
    if kind == "attend" and not tree and rng.random() < 0.3:
        new = int(round(2 ** rng.uniform(4, 9)))
    elif kind in ("attend", "verify") and tree:
        new = int(round(2 ** rng.uniform(2, 6)))
    elif kind == "read" or (kind == "write" and rng.random() < 0.6):
        new, past = past, 0
    while sequences > 1 and sequences * (past + new) * kv_heads * DIM > MOST_CODES // 2:
        sequences -= 1
    while (past + new) * sequences * kv_heads * DIM > MOST_CODES:
        past, new = past // 2, new if past else new // 2
    while past > 16 and sequences * kv_heads * per_kv * new * (past + new) > MOST_SCORES // 2 and kind in ("attend", "verify"):
        past = past * 2 // 3
    ragged = sequences > 1
    return _case(kind=kind, kv_heads=kv_heads, per_kv=per_kv, dtype=rng.choice(["f16", "bf16"]), bits_k=rng.choice([4, 4, 8]),
                 bits_v=rng.choice([4, 4, 8]), group=rng.choice([32, 64, 128]), transform=int(rng.random() < 0.25),
                 block_tokens=rng.choice([16, 16, 32, 64, 128]), sequences=sequences, lengths=rng.randrange(1 << 20),
                 past_lo=past // 2 if ragged else past, past_hi=past, new_lo=(new + 1) // 2 if ragged else new, new_hi=new, tree=tree)


# ---- inputs -----------------------------------------------------------------------------------------

def _lengths(case):
    """(tokens before the new ones, new tokens) of every sequence; the first has the longest of both."""
    g = torch.Generator().manual_seed(case["lengths"] * 2 + 1)
    n = case["sequences"]
    past = torch.randint(case["past_lo"], case["past_hi"] + 1, (n,), generator=g)
    new = torch.randint(case["new_lo"], case["new_hi"] + 1, (n,), generator=g)
    past[0], new[0] = case["past_hi"], case["new_hi"]
    return past.tolist(), new.tolist()


def _tree(new, g):
    """(parent of every draft, -1 = the context; the accepted path, ascending) of one tree."""
    parent = [int(torch.randint(-1 if i < 3 else max(-1, i - 9), i, (1,), generator=g)) if i else -1 for i in range(new)]
    node, path = new - 1, []
    while node >= 0:
        path.append(node)
        node = parent[node]
    return parent, path[::-1]


def _masks(case, new):
    """Bit masks (a row of 64-bit words per new token: itself and its ancestors) and the accepted paths; the trees, like the lengths,
    are those of the case."""
    words = (max(new) + 63) // 64
    g = torch.Generator().manual_seed(case["lengths"] * 31 + 5)
    rows, start, kept = [], [0], []
    for n in new:
        parent, path = _tree(n, g)
        sets = []
        for i, p in enumerate(parent):
            bits = (1 << i) | (sets[p] if p >= 0 else 0)
            sets.append(bits)
            word = [(bits >> (64 * w)) & ((1 << 64) - 1) for w in range(words)]
            rows.append([w - (1 << 64) if w >> 63 else w for w in word])
        kept += path
        start.append(len(kept))
    i32 = dict(dtype=torch.int32, device=DEVICE)
    return (torch.tensor(rows, dtype=torch.int64, device=DEVICE), torch.tensor(start, **i32), torch.tensor(kept, **i32))


def _rows(shape, seed, spread, dtype):
    """Rows of K, V or q: normal values, for K with a factor per (head, channel) and a few channels far above the others."""
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    x = torch.randn(shape, generator=g, device=DEVICE)
    if spread:
        f = torch.exp(0.5 * torch.randn(shape[1:], generator=g, device=DEVICE))
        at = torch.randint(0, DIM, (shape[1], 3), generator=g, device=DEVICE)
        x = x * f.scatter(1, at, 6.0)
    return x.to(dtype)


def _start(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _place(past, new):
    """Positions and sequence numbers of all new rows, in the order of the rows."""
    lens = torch.tensor(new)
    seq = torch.repeat_interleave(torch.arange(len(new)), lens)
    first = torch.tensor(_start(new)[:-1])
    pos = torch.arange(sum(new)) - first[seq] + torch.tensor(past)[seq]
    return pos.to(DEVICE), seq.to(DEVICE)


def _hadamard():
    h = torch.ones(1, 1, device=DEVICE)
    while h.shape[0] < DIM:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h


def _inputs(case, seed):
    """What both sides and the 64-bit values start from: the sequences' rows of K and V (past and new), queries, tables, masks."""
    dtype = DTYPES[case["dtype"]]
    past, new = _lengths(case)
    n, bt, H = case["sequences"], case["block_tokens"], case["kv_heads"]
    total = [p + t for p, t in zip(past, new)]
    need = [(t + bt - 1) // bt for t in total]
    g = torch.Generator().manual_seed(seed * 7 + 3)
    order = torch.randperm(sum(need) + 3, generator=g)
    table = torch.zeros(n, max(need), dtype=torch.int32)
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = order[at: at + c]
        at += c
    i32 = dict(dtype=torch.int32, device=DEVICE)
    x = {"past": past, "new": new, "pages": sum(need) + 3, "table": table.to(DEVICE),
         "tokens": torch.tensor(total, **i32), "new_start": torch.tensor(_start(new), **i32),
         "tokens_past": torch.tensor(past, **i32), "past_start": torch.tensor(_start(past), **i32),
         "k_past": _rows((sum(past), H, DIM), seed * 8 + 1, True, dtype), "v_past": _rows((sum(past), H, DIM), seed * 8 + 2, False, dtype),
         "mask": None, "keep_start": None, "keep": None, "scale": 1 / math.sqrt(DIM)}
    x["k"], x["v"] = _rows((sum(new), H, DIM), seed * 8 + 3, True, dtype), _rows((sum(new), H, DIM), seed * 8 + 4, False, dtype)
    if case["kind"] in ("attend", "verify"):
        x["q"] = _rows((sum(new), H * case["per_kv"], DIM), seed * 8 + 5, False, dtype)
        if case["tree"]:
            x["mask"], x["keep_start"], x["keep"] = _masks(case, new)
    return x


def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    x = _inputs(case, seed)
    past, new, H = x["past"], x["new"], case["kv_heads"]
    state = {"case": case, "x": x, "kind": case["kind"]}
    rows = sum(new)
    if case["kind"] == "verify":
        kept = [int(v) for v in x["keep_start"].tolist()]
        kept = [b - a for a, b in zip(kept, kept[1:])]
        x["tokens_kept"] = torch.tensor([p + c for p, c in zip(past, kept)], dtype=torch.int32, device=DEVICE)
        rows, x["kept"] = sum(kept), kept
    # the cache as the steps before left it: the past rows, and for calls that write nothing the new ones
    writes = case["kind"] in ("write", "verify")
    if own:
        from paper_2605_13734_amd import kvc
        plan = kvc.CachePlan(kvc.F16 if case["dtype"] == "f16" else kvc.BF16, H, H * case["per_kv"], DIM, case["bits_k"],
                             case["bits_v"], case["group"], case["block_tokens"], case["transform"],
                             max_batch=case["sequences"], max_tokens=max(p + t for p, t in zip(past, new)), max_new=max(new))
        cache = kvc.Cache(plan, x["pages"], DEVICE)
        stream = torch.cuda.current_stream().cuda_stream
        most = max(p + t for p, t in zip(past, new))
        if sum(past):
            cache.store(kvc.CacheBatch(x["past_start"], x["tokens_past"], x["table"], max(past), max(past), x["pages"]),
                        x["k_past"], x["v_past"], stream)
        batch = kvc.CacheBatch(x["new_start"], x["tokens"], x["table"], max(new), most, x["pages"], x["mask"])
        if not writes:
            cache.store(batch, x["k"], x["v"], stream)
        state.update(cache=cache, batch=batch)
        if case["kind"] == "verify":
            state["batch_kept"] = kvc.CacheBatch(x["keep_start"], x["tokens_kept"], x["table"], max(x["kept"]), most, x["pages"])
        if case["kind"] in ("attend", "verify"):
            state["out"] = torch.empty_like(x["q"])
        if case["kind"] != "attend":
            state["k_back"] = torch.empty(rows, H, DIM, dtype=dtype, device=DEVICE)
            state["v_back"] = torch.empty(rows, H, DIM, dtype=dtype, device=DEVICE)
    else:
        slots, groups = x["pages"] * case["block_tokens"], DIM // case["group"]
        store = {w: {"codes": torch.zeros(slots, H, DIM, dtype=torch.uint8, device=DEVICE),
                     "scale": torch.zeros(slots, H, groups, dtype=torch.float16, device=DEVICE),
                     "zero": torch.zeros(slots, H, groups, dtype=torch.float16, device=DEVICE)} for w in "kv"}
        state.update(store=store, hadamard=_hadamard())
        state["at_new"], state["seq_new"] = _place(past, new)
        if sum(past):
            at, seq = _place([0] * len(past), past)
            _plain_store(state, at, seq, x["k_past"], x["v_past"])
        if not writes:
            _plain_store(state, state["at_new"], state["seq_new"], x["k"], x["v"])
        if case["kind"] == "verify":
            state["at_kept"], state["seq_kept"] = _place(past, x["kept"])
    torch.cuda.synchronize()
    return state


# ---- the plain form ---------------------------------------------------------------------------------

def _slots(state, at, seq):
    bt = state["case"]["block_tokens"]
    page = state["x"]["table"][seq, torch.div(at, bt, rounding_mode="floor")].long()
    return page * bt + at % bt


def _rotate_in(x):
    """y = H x / 8 as the fast transform of order 128: sums and differences at strides 1, 2, ..., 64, one rounding to 32 bits each;
    limited to the type's range and rounded to the type."""
    y = (x.float() * 0.125).reshape(-1, DIM // 2, 2, 1)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, DIM // 4, 2, 2)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, DIM // 8, 2, 4)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, DIM // 16, 2, 8)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, DIM // 32, 2, 16)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, DIM // 64, 2, 32)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(-1, 1, 2, 64)
    y = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2).reshape(x.shape)
    top = torch.finfo(x.dtype).max
    return y.clamp(-top, top).to(x.dtype)


def _quantise(x, bits, group):
    """Codes, scales and zeros of rows [..., 128] in groups of channels."""
    v = torch.nan_to_num(x.float(), nan=0.0).clamp(-TOP, TOP).reshape(*x.shape[:-1], DIM // group, group)
    lo, hi = v.amin(-1, keepdim=True) + 0.0, v.amax(-1, keepdim=True) + 0.0
    zero = lo.half()
    scale = ((hi - lo) / (2 ** bits - 1)).half()
    inv = torch.where(scale > 0, 1.0 / scale.float(), torch.zeros_like(lo))
    codes = torch.round((v - zero.float()) * inv).clamp(0, 2 ** bits - 1)
    return codes.to(torch.uint8).reshape(x.shape), scale.squeeze(-1), zero.squeeze(-1)


def _plain_store(state, at, seq, k, v):
    case, to = state["case"], _slots(state, at, seq)
    if case["transform"]:
        k = _rotate_in(k)
    ck, sk, zk = _quantise(k, case["bits_k"], case["group"])
    cv, sv, zv = _quantise(v, case["bits_v"], case["group"])
    K, V = state["store"]["k"], state["store"]["v"]
    K["codes"][to], K["scale"][to], K["zero"][to] = ck, sk, zk
    V["codes"][to], V["scale"][to], V["zero"][to] = cv, sv, zv


def _values(tensor, at):
    """The values in 32 bits that the slots `at` hold."""
    codes, scale, zero = tensor["codes"][at].float(), tensor["scale"][at].float(), tensor["zero"][at].float()
    shape = codes.shape
    x = codes.reshape(*shape[:-1], scale.shape[-1], -1) * scale.unsqueeze(-1) + zero.unsqueeze(-1)
    return x.reshape(shape)


def _rounded(x, dtype):
    top = min(TOP, torch.finfo(dtype).max)
    return x.clamp(-top, top).to(dtype)


def _plain_load(state, at, seq):
    case, slots = state["case"], _slots(state, at, seq)
    k, v = _values(state["store"]["k"], slots), _values(state["store"]["v"], slots)
    if case["transform"]:
        k = torch.matmul(k, state["hadamard"]) * 0.0625
    dtype = DTYPES[case["dtype"]]
    return _rounded(k, dtype), _rounded(v, dtype)


def _visible(x, most_new, most, device=DEVICE):
    """[sequences, new, tokens]: which tokens a new token sees."""
    n = x["table"].shape[0]
    past = x["tokens_past"].reshape(n, 1, 1)
    t = torch.arange(most, device=device).reshape(1, 1, most)
    i = torch.arange(most_new, device=device).reshape(1, most_new, 1)
    j = t - past                                       # the token's number among the new ones
    if x["mask"] is None:
        return (j <= i) & (t < x["tokens"].reshape(n, 1, 1))
    row = (x["new_start"][:-1].reshape(n, 1) + torch.arange(most_new, device=device)).clamp(max=x["mask"].shape[0] - 1)
    words = x["mask"][row.long()]                      # [sequences, new, words]
    jj = j.clamp(0, 64 * words.shape[-1] - 1).expand(n, most_new, most)
    bit = (torch.gather(words, 2, jj >> 6) >> (jj & 63)) & 1
    return ((j < 0) | (bit == 1)) & (t < x["tokens"].reshape(n, 1, 1))


def _plain_attend(state):
    case, x = state["case"], state["x"]
    n, H, G = case["sequences"], case["kv_heads"], case["per_kv"]
    most_new, most = max(x["new"]), max(p + t for p, t in zip(x["past"], x["new"]))
    t = torch.arange(most, device=DEVICE).expand(n, most)
    s = torch.arange(n, device=DEVICE).reshape(n, 1).expand(n, most)
    at = _slots(state, t, s)
    k, v = _values(state["store"]["k"], at), _values(state["store"]["v"], at)        # [n, tokens, H, 128]
    row = (x["new_start"][:-1].reshape(n, 1) + torch.arange(most_new, device=DEVICE)).clamp(max=x["q"].shape[0] - 1).long()
    q = x["q"].float()
    if case["transform"]:
        q = torch.matmul(q, state["hadamard"]) * 0.0625
    q = q[row].reshape(n, most_new, H, G, DIM).permute(0, 2, 1, 3, 4).reshape(n, H, most_new * G, DIM)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).mul_(x["scale"]).reshape(n, H, most_new, G, most)
    del k
    seen = _visible(x, most_new, most).reshape(n, 1, most_new, 1, most)
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    w = scores.sub_(top).exp_()
    norm = w.sum(-1, keepdim=True)
    o = torch.matmul(w.reshape(n, H, most_new * G, most), v.permute(0, 2, 1, 3).contiguous()).reshape(n, H, most_new, G, DIM)
    o = torch.where(norm > 0, o / norm, torch.zeros_like(o))
    o = o.permute(0, 2, 1, 3, 4).reshape(n, most_new, H * G, DIM)
    return o[state["seq_new"], state["at_new"] - x["tokens_past"][state["seq_new"]]].to(x["q"].dtype)


def _plain_keep(state):
    x = state["x"]
    past = x["tokens_past"][state["seq_kept"]]
    src = _slots(state, past + x["keep"], state["seq_kept"])
    dst = _slots(state, state["at_kept"], state["seq_kept"])
    K, V = state["store"]["k"], state["store"]["v"]
    K["codes"][dst], K["scale"][dst], K["zero"][dst] = K["codes"][src], K["scale"][src], K["zero"][src]
    V["codes"][dst], V["scale"][dst], V["zero"][dst] = V["codes"][src], V["scale"][src], V["zero"][src]


def _run_plain(state):
    x, kind = state["x"], state["kind"]
    out = {}
    if kind in ("write", "verify"):
        _plain_store(state, state["at_new"], state["seq_new"], x["k"], x["v"])
    if kind in ("attend", "verify"):
        out["out"] = _plain_attend(state)
    if kind == "verify":
        _plain_keep(state)
        out["k"], out["v"] = _plain_load(state, state["at_kept"], state["seq_kept"])
    elif kind in ("write", "read"):
        out["k"], out["v"] = _plain_load(state, state["at_new"], state["seq_new"])
    return out


def run(state):
    if not own:
        return _run_plain(state)
    x, kind, cache, batch = state["x"], state["kind"], state["cache"], state["batch"]
    stream = torch.cuda.current_stream().cuda_stream
    out = {}
    if kind in ("write", "verify"):
        cache.store(batch, x["k"], x["v"], stream)
    if kind in ("attend", "verify"):
        cache.attend(batch, x["q"], state["out"], x["scale"], stream=stream)
        out["out"] = state["out"]
    if kind == "verify":
        cache.keep(batch, x["keep_start"], x["keep"], stream)
        batch = state["batch_kept"]
    if kind != "attend":
        cache.load(batch, state["k_back"], state["v_back"], stream)
        out["k"], out["v"] = state["k_back"], state["v_back"]
    return out


def work(case):
    """Bytes: 16-bit rows once, codes and parameters once per operator that needs them.  Operations: two multiply-adds per channel,
    query row and visible token, and the quantiser's five or three per value."""
    past, new = _lengths(case)
    H, G = case["kv_heads"], case["per_kv"]
    held = H * (16 * (case["bits_k"] + case["bits_v"]) + 8 * (DIM // case["group"]))        # bytes of a token in the cache
    row = H * DIM * 2
    rows, bytes_, flops = sum(new), 0, 0
    kept = rows
    if case["kind"] == "verify":
        g = torch.Generator().manual_seed(case["lengths"] * 31 + 5)
        kept = sum(len(_tree(t, g)[1]) for t in new)
        bytes_ += 2 * kept * held
    if case["kind"] in ("write", "verify"):
        bytes_ += rows * (2 * row + held)
        flops += rows * H * 2 * DIM * 5
    if case["kind"] != "attend":
        bytes_ += kept * (2 * row + held)
        flops += kept * H * 2 * DIM * 3
    if case["kind"] in ("attend", "verify"):
        bytes_ += sum(p + t for p, t in zip(past, new)) * held + 2 * rows * row * G
        flops += sum(t * p + (t * 4 if case["tree"] else t * (t + 1) // 2) for p, t in zip(past, new)) * H * G * 4 * DIM
    return {"bytes": bytes_, "flops": flops}


# ---- the values in 64 bits --------------------------------------------------------------------------

def _exact_rows(x, bits, group, rotate):
    """What the cache holds for rows [..., 128], in 64 bits: the codes are decisions taken on 32-bit differences and 16-bit scales
    and zeros, the rest is exact.  Rows that went through the rotation come back rotated."""
    if rotate:
        h = _hadamard().double()
        y = x.double() @ h / 8
        x = y.clamp(-torch.finfo(x.dtype).max, torch.finfo(x.dtype).max).to(x.dtype)
    parts = x.float().unflatten(-1, (DIM // group, group)).nan_to_num(nan=0.0).clip(-TOP, TOP)
    lowest = parts.min(-1, keepdim=True).values + 0.0
    step = ((parts.max(-1, keepdim=True).values - lowest) / float(2 ** bits - 1)).to(torch.float16).double()
    base = lowest.to(torch.float16).double()
    inverse = torch.where(step > 0, (1 / step).float(), torch.zeros_like(lowest))
    number = ((parts - base.float()) * inverse).round().clip(0, 2 ** bits - 1).double()
    return (number * step + base).flatten(-2)


def exact(case, seed):
    x = _inputs(case, seed)
    past, new = x["past"], x["new"]
    G, limit = case["per_kv"], TOP
    rotate = bool(case["transform"])
    h = _hadamard().double()
    at_past, at_new = _start(past), _start(new)
    outs, ks, vs = [], [], []
    for s in range(len(new)):
        k = torch.cat([x["k_past"][at_past[s]: at_past[s + 1]], x["k"][at_new[s]: at_new[s + 1]]])
        v = torch.cat([x["v_past"][at_past[s]: at_past[s + 1]], x["v"][at_new[s]: at_new[s + 1]]])
        k = _exact_rows(k, case["bits_k"], case["group"], rotate)
        v = _exact_rows(v, case["bits_v"], case["group"], False)
        if case["kind"] in ("attend", "verify"):
            q = x["q"][at_new[s]: at_new[s + 1]].double()
            if rotate:
                q = q @ h / 16
            seen = torch.ones(new[s], past[s] + new[s], dtype=torch.bool, device=DEVICE)
            if x["mask"] is None:
                seen[:, past[s]:] = torch.ones(new[s], new[s], device=DEVICE).tril().bool()
            else:
                words = x["mask"][at_new[s]: at_new[s + 1]]
                for j in range(new[s]):
                    seen[:, past[s] + j] = (words[:, j // 64] >> (j % 64)) & 1 == 1
            o = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
            for head in range(case["kv_heads"]):
                for one in range(head * G, (head + 1) * G):
                    logits = (q[:, one] @ k[:, head].T) * x["scale"]
                    weights = torch.softmax(logits.masked_fill(~seen, -math.inf), -1)
                    o[:, one] = weights @ v[:, head]
            outs.append(o)
        if case["kind"] != "attend":
            rows = torch.arange(past[s], past[s] + new[s], device=DEVICE)
            if case["kind"] == "verify":
                a, b = x["keep_start"][s: s + 2].tolist()
                rows = past[s] + x["keep"][a:b].long()
            back = k[rows]
            ks.append((back @ h / 16 if rotate else back).clip(-limit, limit))
            vs.append(v[rows].clip(-limit, limit))
    result = {}
    if outs:
        result["out"] = torch.cat(outs)
    if ks:
        result["k"], result["v"] = torch.cat(ks), torch.cat(vs)
    return result
