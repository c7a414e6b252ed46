"""64-bit definitions of the calls on prompts and of the pages' tables, and what the results may be off by."""
import numpy as np
import torch

from paper_2605_13734_amd import kvc

DIM = 128
DEVICE = "cuda"


def typed(bf16):
    return torch.bfloat16 if bf16 else torch.float16


def own_type(bf16):
    return kvc.BF16 if bf16 else kvc.F16


def half_step(bf16):
    return 2.0 ** (-8 if bf16 else -11)


def smallest(bf16):
    """Half of the smallest number above zero."""
    return 2.0 ** (-134 if bf16 else -25)


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def heads(rows, kv_heads, per_kv, bf16, seed=0, fused=False, spread=1.0):
    """q, k, v on the GPU: normal values, keys with channels of different size."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, kv_heads * (per_kv + 2), DIM, generator=g)
    x[:, kv_heads * per_kv: kv_heads * (per_kv + 1)] *= torch.exp(0.5 * torch.randn(kv_heads, DIM, generator=g)) * spread
    x = x.to(typed(bf16)).to(DEVICE)
    parts = x[:, : kv_heads * per_kv], x[:, kv_heads * per_kv: kv_heads * (per_kv + 1)], x[:, kv_heads * (per_kv + 1):]
    return parts if fused else tuple(p.contiguous() for p in parts)


def attention(q, k, v, scale, rows=None):
    """One sequence in 64 bits (`rows`: of these query rows only).  Returns out, lse, and for the tolerances sum of weight * |value| and the largest
    sum of |products| of a row."""
    per, n = q.shape[1] // k.shape[1], k.shape[0]
    rows = torch.arange(n, device=q.device) if rows is None else rows
    out, size, lse, reach = [], [], [], []
    for h in range(q.shape[1]):
        x, key, value = q[rows, h].double(), k[:, h // per].double(), v[:, h // per].double()
        see = torch.arange(n, device=q.device)[None, :] <= rows[:, None]
        s = torch.where(see, x @ key.T * scale, -torch.inf)
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - top)
        total = w.sum(1, keepdim=True)
        w = w / total
        out.append(w @ value)
        size.append(w @ value.abs())
        lse.append((top + total.log())[:, 0])
        reach.append(torch.where(see, x.abs() @ key.abs().T * abs(scale), 0.0).amax(1))
    return torch.stack(out, 1), torch.stack(lse, 1), torch.stack(size, 1), torch.stack(reach, 1)


def check_attention(out, lse, q, k, v, scale, bf16, rows=None):
    """Errors: a weight is rounded to the type (half a step; below 2^-22 of the largest of its row by 2^-33 of it), a score comes from sums of 128
    products in 32 bits and one multiplication (2^-19 of the sum of magnitudes allows for some 30 roundings; both the weights and
    their sum have it), the exponential and the sums in 32 bits (2^-20 allows for the 16 roundings that matter in sums of positive numbers taken
    by four lanes, their own among them), the result is rounded to its type."""
    want, want_lse, size, reach = attention(q, k, v, scale, rows)
    score = reach * 2.0 ** -19
    unit, most = half_step(bf16), v.double().abs().max().item()
    tol = want.abs() * unit * 1.01 + size * (unit * 1.01 + 2 * score[:, :, None] + 2.0 ** -18) + k.shape[0] * 2.0 ** -33 * most + smallest(bf16)
    got = out if rows is None else out[rows]
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])
    if lse is not None:
        got_lse = lse if rows is None else lse[rows]
        off = (got_lse.double() - want_lse).abs()
        assert (off <= score + want_lse.abs() * 2.0 ** -20 + 2.0 ** -18).all(), off.max()


def frequencies_of(plan_args):
    f = plan_args.get("frequencies")
    return kvc.rotary_frequencies(plan_args.get("rotary_dim", DIM)) if f is None and plan_args.get("rotary_dim", DIM) else f


def rotation(x, weight, positions, frequencies, pairs, amplitude, eps):
    """Rows [rows, heads, 128] in 64 bits (angles in the host's long numbers); returns y and the sum of magnitudes of the terms of each element."""
    x = x.double().cpu().numpy()
    if eps is not None:
        # (as 64-bit numbers: squares of the largest bf16 numbers fit)
        with np.errstate(invalid="ignore"):
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.double().cpu().numpy()
    y, size, R = x.copy(), np.abs(x), 2 * len(frequencies)
    if R:
        angle = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(frequencies, dtype=np.longdouble)
        c, s = (np.asarray(f(angle), dtype=np.float64)[:, None] * amplitude for f in (np.cos, np.sin))
        first = slice(0, R, 2) if pairs else slice(0, R // 2)
        second = slice(1, R, 2) if pairs else slice(R // 2, R)
        a, b = x[..., first], x[..., second]
        y[..., first], y[..., second] = a * c - b * s, a * s + b * c
        size[..., first] = size[..., second] = (np.abs(a) + np.abs(b)) * amplitude
    return y, size


def check_rotation(got, x, weight, positions, frequencies, pairs, amplitude, eps, bf16):
    """Errors: 2^-19 of the terms allows for the roundings of the mean (a sum of 128, 10 in a row), the root, weights, cosines (2^-21) and products
    in 32 bits; then the type's rounding."""
    y, size = rotation(x, weight, positions, frequencies, pairs, amplitude, eps)
    tol = np.abs(y) * half_step(bf16) * 1.01 + size * 2.0 ** -19 + smallest(bf16)
    got, some = got.double().cpu().numpy(), np.isfinite(y)
    assert not np.isfinite(got[~some]).any()             # (inputs beyond the type's range)
    off, tol = np.abs(got - y)[some], tol[some]
    assert np.all(off <= tol), (np.argwhere(~(off <= tol))[:4], (off / tol).max())


class Pages:
    """A step of the sequences by its definition: lists of pages, one after the other."""

    def __init__(self, n, num_pages, block_tokens, max_tokens, free):
        self.bt, self.most, self.num_pages = block_tokens, max_tokens, num_pages
        self.held, self.stack, self.pages = [0] * n, list(free), [[] for _ in range(n)]

    def need(self, tokens):
        return (tokens + self.bt - 1) // self.bt

    def advance(self, kept, fresh, max_new, rows, max_tokens=None):
        """Returns new_start, tokens, positions, slots, status."""
        n, most = len(self.held), self.most if max_tokens is None else max_tokens
        kept = list(self.held) if kept is None else kept
        fresh = [0] * n if fresh is None else fresh
        count = [f if 0 <= f <= max_new else 0 for f in fresh]
        start = np.concatenate([[0], np.cumsum(count)]).tolist()
        status, ok = [0] * n, [False] * n
        for s in range(n):
            ok[s] = 0 <= kept[s] <= self.held[s] <= most and 0 <= fresh[s] <= max_new and kept[s] + fresh[s] <= most and start[s + 1] <= rows
            if not ok[s]:
                status[s] |= kvc.DEV_BAD_ROW
        given = []
        for s in range(n):
            if ok[s]:
                given += self.pages[s][self.need(kept[s] + fresh[s]):]
        room, wanted = len(self.stack) + len(given), 0
        for s in range(n):
            if ok[s]:
                more = self.need(kept[s] + fresh[s]) - len(self.pages[s])
                if more > 0:
                    wanted += more
                    if wanted > room:
                        status[s] |= kvc.DEV_NO_PAGE
                        ok[s] = False
        self.stack += given[::-1]
        for s in range(n):
            if ok[s]:
                need = self.need(kept[s] + fresh[s])
                del self.pages[s][need:]
                while len(self.pages[s]) < need:
                    self.pages[s].append(self.stack.pop())
                self.held[s] = kept[s] + fresh[s]
        tokens = [self.held[s] if ok[s] else -1 for s in range(n)]
        positions, slots = [-1] * rows, [-1] * rows
        for s in range(n):
            if ok[s]:
                for i in range(count[s]):
                    p = kept[s] + i
                    positions[start[s] + i] = p
                    slots[start[s] + i] = self.pages[s][p // self.bt] * self.bt + p % self.bt
        return start, tokens, positions, slots, status
