"""The operators of a steered conversation over a paged key/value cache, as measured cases.

A serving program that highlights parts of its prompts keeps the edited keys in a cache of pages.  Per chunk of new
tokens (a part of a prompt, or the one token of a generation step) and layer it

  rotary     turns queries and keys to their positions                       seka_rotary
  append     does that and writes the chunk's keys and values to their pages  seka_cache_append
  attention  lets the chunk's queries attend to the pages                     seka_attention_chunk
  weights    adds up how much attention every cached token gets               seka_attention_weights
  evict      keeps the tokens with the most of it, and the last ones          seka_cache_evict

Tensors: new tokens are packed, [tokens, heads, D]; request b owns rows cu[b] .. cu[b + 1] - 1.  Pages are
[pages, page_size, Hkv, D] and, for the accumulated weights, [pages, Hkv, page_size].  Token j of request b lies in page
table[b, j // page_size].  lens[b] counts the tokens of request b with those of the chunk, which are its last ones.
"""
import math

import numpy as np
import torch

own = False


def listed():
    return [
        # one generation step of 48 conversations at far positions: latency
        dict(name="rotary_step", kind="rotary", dtype="bf16", T=48, Hq=32, Hkv=8, D=128, dim=128, interleaved=False, base=500000.0, stretch=1.0, far=120000),
        # packed prompts, half of every head turned, neighbouring pairs, frequencies stretched for a long context
        dict(name="rotary_prompt", kind="rotary", dtype="bf16", T=16381, Hq=32, Hkv=8, D=128, dim=64, interleaved=True, base=10000.0, stretch=8.0, far=60000),
        # the new token of 64 conversations into pages of 16
        dict(name="append_step", kind="append", dtype="bf16", B=64, n=1, S=4096, Hq=32, Hkv=8, D=128, ps=16, dim=128, interleaved=False, highlight=0.0),
        # chunks of five prompts, with highlighted tokens, in fp32
        dict(name="append_chunk_f32", kind="append", dtype="f32", B=5, n=2047, S=9000, Hq=32, Hkv=8, D=128, ps=64, dim=128, interleaved=False, highlight=0.12),
        # generation step of one short conversation on the fp32 path: latency
        dict(name="attention_one_f32", kind="attention", dtype="f32", B=1, n=1, S=777, Hq=8, Hkv=2, D=64, ps=16, lse=True),
        # generation step of a batch at mixed positions
        dict(name="attention_step", kind="attention", dtype="bf16", B=24, n=1, S=8192, Hq=32, Hkv=8, D=128, ps=16, lse=True),
        # chunks of prompts and single tokens together, seven query heads to a key head
        dict(name="attention_mixed", kind="attention", dtype="bf16", B=9, n=700, S=6001, Hq=28, Hkv=4, D=128, ps=64, lse=False),
        # one long prompt, a chunk of 2048 tokens near its end
        dict(name="attention_chunk", kind="attention", dtype="bf16", B=1, n=2048, S=31111, Hq=32, Hkv=8, D=128, ps=32, lse=False),
        # what a generation step of a batch adds to its tokens' weights
        dict(name="weights_step", kind="weights", dtype="bf16", B=24, n=1, S=8192, Hq=32, Hkv=8, D=128, ps=16, window=1, decay=1.0),
        # what two chunks add
        dict(name="weights_chunk", kind="weights", dtype="bf16", B=2, n=1000, S=8192, Hq=32, Hkv=8, D=128, ps=64, window=1000, decay=0.95),
        # one fp32 conversation is cut to half its length: latency
        dict(name="evict_one_f32", kind="evict", dtype="f32", B=1, S=4097, Hkv=8, D=64, ps=16, budget=2048, recent=256),
        # a batch is cut to 4096 tokens each
        dict(name="evict_batch", kind="evict", dtype="bf16", B=16, S=16384, Hkv=8, D=128, ps=16, budget=4096, recent=512),
    ]


# ---- drawn cases: the same kinds over their ranges -----------------------------------------------------------------

_HEADS = [(32, 8), (32, 8), (28, 4), (24, 8), (32, 32), (32, 4), (16, 8), (8, 2), (6, 2), (5, 5)]
_MOST_FLOPS = 9e11
_MOST_CACHE = 1 << 18         # tokens of all requests together


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attention", "attention", "attention", "weights", "evict"])
    Hq, Hkv = rng.choice(_HEADS)
    D = rng.choice([64, 128, 128])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), Hq=Hq, Hkv=Hkv, D=D)
    rot = dict(dim=rng.choice([D, D, D // 2, D // 4 * 3, 20]), interleaved=rng.random() < 0.5)
    if kind == "rotary":
        return dict(c, T=_log(rng, 1, 16381), base=rng.choice([1e4, 5e5, 1e6]), stretch=rng.choice([1.0, 2.0, 8.0, 32.0]),
                    far=_log(rng, 100, 1000000), **rot)
    c["ps"] = rng.choice([8, 16, 16, 32, 64, 128, 256])
    S = _log(rng, 32, 32768)
    if kind == "evict":
        c.pop("Hq")
        B = _log(rng, 1, max(1, min(32, _MOST_CACHE // S)))
        budget = max(1, int(S * rng.uniform(0.1, 0.95)))
        return dict(c, B=B, S=S, budget=budget, recent=int(budget * rng.uniform(0.0, 0.5)))
    B = _log(rng, 1, max(1, min(64, _MOST_CACHE // S)))
    n = 1 if rng.random() < 0.4 else min(S, _log(rng, 2, 2048))
    if kind == "append":
        n = max(1, min(n, 16384 // B))
        return dict(c, B=B, n=n, S=S, highlight=rng.choice([0.0, 0.1]), **rot)
    pairs = _MOST_FLOPS * (0.05 if c["dtype"] == "f32" else 1.0) / (4.0 * Hq * D)
    n = max(1, min(n, int(pairs / (B * S))))
    if kind == "weights":
        return dict(c, B=B, n=n, S=S, window=max(1, n // rng.choice([1, 1, 4])), decay=rng.choice([0.0, 0.9, 1.0]))
    return dict(c, B=B, n=n, S=S, lse=n == 1)


# ---- inputs --------------------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ragged(case):
    """Chunk lengths and cached lengths of the requests.  They belong to the case, not to the seed: every pass is the same
    amount of work.  The longest cache has S tokens and the longest chunk n; others are spread down to a sixteenth by ratio,
    and where the longest chunk is longer than one token, one request in three is at a generation step."""
    B, S, n = case["B"], case["S"], case.get("n", 1)
    g = np.random.Generator(np.random.Philox(key=[1000 * B + n, S]))
    spread = lambda top: np.maximum(1, np.exp(g.uniform(math.log(max(1.0, top / 16)), math.log(top), size=B)).astype(np.int64))  # noqa: E731
    lens, new = spread(S), spread(n)
    lens[int(g.integers(B))] = S
    new[g.random(B) < 1 / 3] = 1
    new[int(np.argmax(lens))] = n
    return [int(min(a, b)) for a, b in zip(new, lens)], [int(x) for x in lens]


def _frequencies(dim, base, stretch, original=4096, fast=32.0, slow=1.0):
    """Radians per position of the dim / 2 pairs.  Stretched for contexts `stretch` times the original: pairs that turn more than
    `fast` times over the original context keep their frequency, those of less than `slow` turns are divided by the stretch,
    with a linear ramp over the pair's index between the two."""
    freq = [base ** (-2.0 * i / dim) for i in range(dim // 2)]
    if stretch == 1.0:
        return freq
    at = lambda turns: dim * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), dim - 1)
    ramp = [min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3))) for i in range(dim // 2)]
    return [f * (1 - r) + f / stretch * r for f, r in zip(freq, ramp)]


class State:
    """Plain attributes: what the calls of one pass take."""


def _table(B, pages, g):
    """A page table of a pool in use: pages in no order.  Entries behind a request's last page name page 0, which no request owns."""
    most = max(pages)
    order = torch.randperm(sum(pages), generator=g, device="cuda", dtype=torch.int32) + 1
    table = torch.zeros((B, most), dtype=torch.int32, device="cuda")
    first = 0
    for b, k in enumerate(pages):
        table[b, :k] = order[first:first + k]
        first += k
    return table


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + 17)
    s = State()
    s.case, t, Hkv, D = case, _TYPES[case["dtype"]], case["Hkv"], case["D"]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(t)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    if case["kind"] == "rotary":
        T = case["T"]
        s.freq = _frequencies(case["dim"], case["base"], case["stretch"])
        s.positions = torch.randint(0, case["far"] + 1, (1, T), generator=g, device="cuda", dtype=torch.int32)
        s.factor = 0.1 * math.log(case["stretch"]) + 1.0
        s.Q, s.K = normal(1, T, case["Hq"], D), normal(1, T, Hkv, D)
        s.Q_out, s.K_out = torch.empty_like(s.Q), torch.empty_like(s.K)
        return s
    B, S, ps = case["B"], case["S"], case["ps"]
    new, lens = _ragged(case)
    s.lens = ints(lens)
    pages = [-(-n // ps) for n in lens]
    s.table = _table(B, pages, g)
    s.K, s.V = normal(sum(pages) + 1, ps, Hkv, D), normal(sum(pages) + 1, ps, Hkv, D)
    if case["kind"] == "evict":
        # accumulated weights of a long conversation: a few tokens have most of it, many the same; highlighted ones are held with inf
        w = torch.rand((sum(pages) + 1, Hkv, ps), generator=g, device="cuda")
        s.W = torch.where(w < 0.02, math.inf, torch.where(w < 0.3, 0.0, torch.exp(8.0 * w - 8.0)))
        kept = [-(-min(n, case["budget"]) // ps) for n in lens]
        s.table_to = _table(B, kept, g)
        s.K_to, s.V_to, s.W_to = normal(sum(kept) + 1, ps, Hkv, D), normal(sum(kept) + 1, ps, Hkv, D), torch.zeros((sum(kept) + 1, Hkv, ps), device="cuda")
        s.lens_to = torch.zeros_like(s.lens)
        s.kept = torch.zeros((B, Hkv, case["budget"]), dtype=torch.int32, device="cuda")
        return s
    s.cu = ints([0] + [int(x) for x in np.cumsum(new)])
    s.max_q, total = max(new), sum(new)
    s.Q = normal(total, case["Hq"], D)
    if case["kind"] == "append":
        s.freq = _frequencies(case["dim"], 500000.0, 1.0)
        # conversations that were shortened before: positions run ahead of the places in the cache
        ahead = torch.randint(0, 5000, (B,), generator=g, device="cuda")
        req, i = _place(s, total)
        s.positions = (s.lens.long()[req] - (s.cu[1:] - s.cu[:-1]).long()[req] + i + ahead[req]).to(torch.int32)
        s.K_new, s.V_new, s.Q_out = normal(total, Hkv, D), normal(total, Hkv, D), torch.empty_like(s.Q)
        s.mask = (torch.rand(total, generator=g, device="cuda") < case["highlight"]).to(torch.uint8)
        s.W = torch.rand((sum(pages) + 1, Hkv, ps), generator=g, device="cuda")
    elif case["kind"] == "attention":
        s.O = torch.empty_like(s.Q)
        s.lse = torch.empty((case["Hq"], total), dtype=torch.float32, device="cuda") if case["lse"] else None
    else:
        # the softmax denominators that the attention of the same chunk gave
        s.lse = _plain_attention(s)[1]
        s.W = torch.rand((sum(pages) + 1, Hkv, ps), generator=g, device="cuda")
        s.W_to = torch.zeros_like(s.W)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _turn(x, positions, freq, interleaved, factor):
    """x [..., heads, D] turned to its positions [...]: angles in 64 bits."""
    dim = 2 * len(freq)
    angle = positions.double()[..., None, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    c, s = (factor * torch.cos(angle)).float(), (factor * torch.sin(angle)).float()
    r = x[..., :dim].float()
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = r[..., :dim // 2], r[..., dim // 2:]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((turned.to(x.dtype), x[..., dim:]), -1)


def _place(s, total):
    """Request and index within its chunk of every packed token."""
    t = torch.arange(total, device="cuda")
    req = torch.searchsorted(s.cu[1:].long(), t, right=True)
    return req, t - s.cu.long()[req]


def _rows(s, S):
    """Page and slot of token j < S of every request: [B, S]."""
    ps = s.case["ps"]
    j = torch.arange(S, device="cuda")
    return s.table.long()[:, (j // ps).clamp(max=s.table.shape[1] - 1)], j % ps


def _scores(s):
    """Scores of the padded chunks [B, Hkv, G, max_q, S] in units of the logits, and which of them exist."""
    case, total = s.case, s.Q.shape[0]
    B, S, Hq, Hkv, D = case["B"], case["S"], case["Hq"], case["Hkv"], case["D"]
    page, slot = _rows(s, S)
    K = s.K[page, slot].float()                                              # [B, S, Hkv, D]
    i = torch.arange(s.max_q, device="cuda")
    n = (s.cu[1:] - s.cu[:-1]).long()
    q = s.Q[(s.cu[:-1].long()[:, None] + i).clamp(max=total - 1)].float()     # [B, max_q, Hq, D]
    q = q.reshape(B, s.max_q, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    x = torch.matmul(q, K.permute(0, 2, 3, 1).contiguous()) * (1.0 / math.sqrt(D))
    x = x.reshape(B, Hkv, Hq // Hkv, s.max_q, S)
    last = s.lens.long()[:, None] - n[:, None] + i                           # the last key that row i sees
    there = (torch.arange(S, device="cuda") <= last[..., None]) & (i < n[:, None])[..., None]
    return x, there[:, None, None], page, slot


def _plain_attention(s):
    case, total = s.case, s.Q.shape[0]
    B, Hq, D = case["B"], case["Hq"], case["D"]
    x, there, page, slot = _scores(s)
    x = torch.where(there, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total_p = p.sum(-1, keepdim=True)
    V = s.V[page, slot].float().permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.flatten(2, 3), V).reshape(*p.shape[:4], D) / torch.where(total_p > 0, total_p, 1.0)
    lse = (top + torch.log(total_p))[..., 0]
    req, i = _place(s, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, s.max_q, Hq, D)[req, i]
    return o.to(s.Q.dtype), lse.permute(0, 3, 1, 2).reshape(B, s.max_q, Hq)[req, i].t().contiguous()


def _plain_append(s):
    case, total = s.case, s.Q.shape[0]
    req, i = _place(s, total)
    n = (s.cu[1:] - s.cu[:-1]).long()
    j = s.lens.long()[req] - n[req] + i
    page, slot = s.table.long()[req, j // case["ps"]], j % case["ps"]
    q = _turn(s.Q, s.positions, s.freq, case["interleaved"], 1.0)
    s.K[page, slot] = _turn(s.K_new, s.positions, s.freq, case["interleaved"], 1.0)
    s.V[page, slot] = s.V_new
    s.W[page, :, slot] = torch.where(s.mask[:, None] != 0, math.inf, 0.0)
    return q, s.K, s.V, s.W


def _plain_weights(s):
    case, total = s.case, s.Q.shape[0]
    x, there, page, slot = _scores(s)
    i = torch.arange(s.max_q, device="cuda")
    n = (s.cu[1:] - s.cu[:-1]).long()
    counts = (i >= n[:, None] - case["window"])[:, None, None, :, None] & there
    lse = s.lse.t()[(s.cu[:-1].long()[:, None] + i).clamp(max=total - 1)]     # [B, max_q, Hq]
    lse = lse.reshape(case["B"], s.max_q, case["Hkv"], -1).permute(0, 2, 3, 1)[..., None]
    got = torch.where(counts, torch.exp(x - lse), 0.0).sum((2, 3))            # [B, Hkv, S]
    held = (torch.arange(case["S"], device="cuda") < s.lens[:, None])[..., None]
    slot = slot.expand_as(page)
    new = got.permute(0, 2, 1) + (case["decay"] * s.W[page, :, slot] if case["decay"] else 0.0)
    s.W_to[page, :, slot] = torch.where(held, new, s.W_to[page, :, slot])
    return s.W_to


def _plain_evict(s):
    case = s.case
    B, S, Hkv, ps, budget, recent = (case[k] for k in ("B", "S", "Hkv", "ps", "budget", "recent"))
    page, slot = _rows(s, S)
    j = torch.arange(S, device="cuda")
    n = s.lens.long()[:, None]
    w = s.W[page, :, slot.expand_as(page)].permute(0, 2, 1)                   # [B, Hkv, S]
    by_weight = torch.sort(w, dim=-1, descending=True, stable=True).indices
    # the last `recent` tokens before the others, and those that do not exist behind them
    group = torch.where(j < n, torch.where((j >= n - recent) | (n <= budget), 2, 1), 0)[:, None].expand(B, Hkv, S)
    by_group = torch.sort(group.gather(-1, by_weight), dim=-1, descending=True, stable=True).indices
    kept = by_weight.gather(-1, by_group)[..., :budget]
    m = torch.clamp(n, max=budget)
    k = torch.arange(min(budget, S), device="cuda")
    there = (k < m)[:, None]
    kept = torch.sort(torch.where(there, kept, S), dim=-1).values
    src = kept.clamp(max=S - 1)
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hkv, device="cuda")[:, None]
    to_page = s.table_to.long()[:, (k // ps).clamp(max=s.table_to.shape[1] - 1)][:, None].expand(B, Hkv, k.numel())
    to = (to_page, (k % ps).expand_as(to_page), h.expand_as(to_page))
    from_page = s.table.long()[b, src // ps]
    for a, c in ((s.K, s.K_to), (s.V, s.V_to)):
        c[to] = torch.where(there[..., None], a[from_page, src % ps, h], c[to])
    to = (to[0], to[2], to[1])
    s.W_to[to] = torch.where(there, s.W[from_page, h, src % ps], s.W_to[to])
    s.kept.fill_(-1)
    s.kept[..., :k.numel()] = torch.where(there, kept, -1).to(torch.int32)
    return s.K_to, s.V_to, s.W_to, m[:, 0].to(torch.int32), s.kept


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _descriptors(s, seka):
    """The descriptions of rotation and pages that a program makes once and hands to every call (pointers and frequencies, no
    work of a pass)."""
    case, kind = s.case, s.case["kind"]
    s.cache = None
    if kind in ("rotary", "append"):
        s.rope = seka.rope(s.freq, interleaved=case["interleaved"], factor=s.factor if kind == "rotary" else 1.0)
    if kind != "rotary":
        W = {"append": "W", "weights": "W_to", "evict": "W"}.get(kind)
        s.cache = seka.paged_cache(s.K, s.V, s.table, s.lens, W=getattr(s, W) if W else None)
    if kind == "evict":
        s.cache_to = seka.paged_cache(s.K_to, s.V_to, s.table_to, s.lens_to, W=s.W_to)


def run(state):
    s, case = state, state.case
    kind = case["kind"]
    if own:
        from paper_2603_01281_amd import binding as seka
        if not hasattr(s, "cache"):
            _descriptors(s, seka)
        if kind == "rotary":
            seka.seka_rotary(s.Q, s.Q_out, s.rope, K=s.K, K_out=s.K_out, positions=s.positions)
            return s.Q_out, s.K_out
        if kind == "append":
            seka.seka_cache_append(s.K_new, s.V_new, s.cache, s.cu, s.max_q, rope=s.rope, positions=s.positions, Q=s.Q, Q_out=s.Q_out, mask=s.mask)
            return s.Q_out, s.K, s.V, s.W
        if kind == "attention":
            seka.seka_attention_chunk(s.Q, s.O, s.cache, s.cu, s.max_q, max_len=case["S"], lse=s.lse)
            return (s.O, s.lse) if case["lse"] else s.O
        if kind == "weights":
            seka.seka_attention_weights(s.Q, s.lse, s.cache, s.cu, s.max_q, max_len=case["S"], window=case["window"], W_in=s.W, decay=case["decay"])
            return s.W_to
        seka.seka_cache_evict(s.cache, s.cache_to, s.kept, case["recent"], max_len=case["S"])
        return s.K_to, s.V_to, s.W_to, s.lens_to, s.kept
    if kind == "rotary":
        return tuple(_turn(x, s.positions, s.freq, case["interleaved"], s.factor) for x in (s.Q, s.K))
    if kind == "attention":
        o, lse = _plain_attention(s)
        return (o, lse) if case["lse"] else o
    return {"append": _plain_append, "weights": _plain_weights, "evict": _plain_evict}[kind](s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    Hkv, D = case["Hkv"], case["D"]
    if case["kind"] == "rotary":
        rows = case["T"] * (case["Hq"] + Hkv)
        return dict(bytes=2 * rows * D * e + 4 * case["T"], flops=3 * rows * case["dim"])
    new, lens = _ragged(case)
    total = sum(new)
    if case["kind"] == "append":
        rows = total * (case["Hq"] + Hkv)
        return dict(bytes=2 * (rows + total * Hkv) * D * e + total * (5 + 4 * Hkv), flops=3 * rows * case["dim"])
    if case["kind"] == "evict":
        moved = sum(min(n, case["budget"]) for n in lens)
        # every weight is read; the rows that stay are read and written
        return dict(bytes=4 * Hkv * sum(lens) + moved * Hkv * (4 * D * e + 8), flops=0)
    rows = [min(n, case.get("window", n)) for n in new]                       # queries that count
    pairs = sum(r * (n - r) + r * (r + 1) / 2 for r, n in zip(rows, lens))
    queries = sum(rows) * case["Hq"]
    if case["kind"] == "weights":
        held = sum(lens) * Hkv
        return dict(bytes=held * D * e + queries * (D * e + 4) + held * (8 if case["decay"] else 4), flops=2 * D * case["Hq"] * pairs)
    return dict(bytes=2 * sum(lens) * Hkv * D * e + queries * (2 * D * e + (4 if case["lse"] else 0)), flops=4 * D * case["Hq"] * pairs)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _exact_turn(x, positions, freq, interleaved, factor):
    """Every pair as a complex number, multiplied by factor * exp(i angle)."""
    half = len(freq)
    x = x.double()
    turn = torch.polar(torch.full((1,), factor, dtype=torch.float64, device=x.device),
                       positions.double().reshape(-1, 1) * torch.tensor(freq, dtype=torch.float64, device=x.device))[:, None]
    y = x.clone().reshape(-1, *x.shape[-2:])
    first = [2 * i for i in range(half)] if interleaved else list(range(half))
    second = [2 * i + 1 for i in range(half)] if interleaved else [half + i for i in range(half)]
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y.reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hkv, D = case["kind"], case["Hkv"], case["D"]
    if kind == "rotary":
        return tuple(_exact_turn(x, s.positions, s.freq, case["interleaved"], s.factor) for x in (s.Q, s.K))
    ps = case["ps"]
    new, lens = _ragged(case)
    cu = [0] + [int(x) for x in np.cumsum(new)]
    home = lambda table, b, j: (table[b].long()[j // ps], j % ps)  # noqa: E731
    if kind == "append":
        K, V, W = s.K.double(), s.V.double(), s.W.double()
        turned = _exact_turn(s.K_new, s.positions, s.freq, case["interleaved"], 1.0)
        for b, n in enumerate(new):
            page, slot = home(s.table, b, torch.arange(lens[b] - n, lens[b], device="cuda"))
            K[page, slot], V[page, slot] = turned[cu[b]:cu[b + 1]], s.V_new[cu[b]:cu[b + 1]].double()
            W[page, :, slot] = torch.where(s.mask[cu[b]:cu[b + 1], None] != 0, math.inf, 0.0).double().expand(n, Hkv)
        return _exact_turn(s.Q, s.positions, s.freq, case["interleaved"], 1.0), K, V, W
    if kind == "evict":
        K, V, W = s.K_to.double(), s.V_to.double(), s.W_to.double()
        for b, n in enumerate(lens):
            weights = s.W[home(s.table, b, torch.arange(n, device="cuda"))[0], :, torch.arange(n, device="cuda") % ps].cpu().numpy()
            for h in range(Hkv):
                keep = np.arange(n)
                if n > case["budget"]:
                    old = n - case["recent"]
                    ranked = np.lexsort((np.arange(old), -weights[:old, h]))[:case["budget"] - case["recent"]]
                    keep = np.concatenate([np.sort(ranked), np.arange(old, n)])
                at = torch.from_numpy(keep).cuda()
                (a, i), (c, k) = home(s.table, b, at), home(s.table_to, b, torch.arange(len(keep), device="cuda"))
                K[c, k, h], V[c, k, h], W[c, h, k] = s.K[a, i, h].double(), s.V[a, i, h].double(), s.W[a, h, i].double()
        return K, V, W, None, None
    G = case["Hq"] // Hkv
    O, L = torch.zeros(s.Q.shape, dtype=torch.float64, device="cuda"), torch.full((case["Hq"], cu[-1]), -math.inf, dtype=torch.float64, device="cuda")
    W = s.W_to.double() if kind == "weights" else None
    for b, n in enumerate(new):
        page, slot = home(s.table, b, torch.arange(lens[b], device="cuda"))
        hidden = torch.ones((n, lens[b]), dtype=torch.bool, device="cuda").triu(lens[b] - n + 1)
        for h in range(Hkv):
            k, v = s.K[page, slot, h].double(), s.V[page, slot, h].double()
            for hq in range(h * G, h * G + G):
                logits = (s.Q[cu[b]:cu[b + 1], hq].double() @ k.t().contiguous()) / math.sqrt(D)
                logits.masked_fill_(hidden, -math.inf)
                if kind == "attention":
                    O[cu[b]:cu[b + 1], hq] = torch.softmax(logits, -1) @ v
                    L[hq, cu[b]:cu[b + 1]] = torch.logsumexp(logits, -1)
                else:
                    share = torch.exp(logits - s.lse[hq, cu[b]:cu[b + 1]].double()[:, None])[-case["window"]:].sum(0)
                    if hq == h * G:
                        W[page, h, slot] = case["decay"] * s.W[page, h, slot].double()
                    W[page, h, slot] += share
    if kind == "weights":
        return W
    return (O, L) if case["lse"] else O
