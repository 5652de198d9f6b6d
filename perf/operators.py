"""The operators of the paged KV cache as measured cases: rows written, read back and attended to.

A server holds the keys and values of its sequences in pages of `ps` rows.  A sequence has two page tables, one for the
rows of its text tokens and one for those of its summary tokens; pages of text that have left every window are given back
(entry -1).  A call takes a batch of sequences, each with `cached` rows (text and summaries interleaved, Eq. 1) before the
call and a run of new ones:

  append  the new rows' K and V into their pages, as bf16 or as e4m3 with one power-of-two scale a row and head
  attn    the new rows' queries over everything they may see (Eq. 3; a summary: its own chunk)
  gather  a run of rows back out of the pages, as bf16

Layouts and heads are those of the repository's workloads (P: chunks of 8 with a summary, window of 128; G: chunks of 64
with 8 summaries, window of 16; F: the plain causal layers; 32/8, 32/4, 16/16 and 4/4 heads).  A case is a flat dict;
`ctx` and `new` list, sequence by sequence, the rows cached before the call and the rows of the call.
"""
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
LAYOUTS = {"P": (8, 1, 128), "G": (64, 8, 16), "F": (8, 0, 1 << 20)}        # k, m, C


def listed():
    return [
        # Interactive decoding: one sequence, one token. Latency of the call.
        dict(name="attn_one", op="attn", layout="P", ctx="9219", new="1", pad=0, hq=32, hkv=8, d=128, ps=64, fmt="bf16"),
        # A serving batch, one token each, contexts from hundreds of tokens to 131,072, in a call padded to a fixed size.
        dict(name="attn_tokens", op="attn", layout="P", pad=3, hq=32, hkv=4, d=128, ps=64, fmt="e4m3", new=",".join(["1"] * 29),
             ctx="147455,1203,88213,52007,131071,147001,9219,60111,30017,146313,700,101009,73728,36866,18433,120113,"
                 "140007,95003,4609,66671,110521,27649,143369,82945,129031,14001,57347,117649,40013"),
        # Drafted tokens: five rows a sequence, to be accepted or not.
        dict(name="attn_drafts", op="attn", layout="P", pad=0, hq=32, hkv=8, d=128, ps=32, fmt="bf16", new=",".join(["5"] * 16),
             ctx="36860,9221,4095,20003,33333,811,15555,28001,36001,12345,7777,30303,2048,25252,18181,35353"),
        # A prompt in pieces: the next 1,024 tokens over 32,768.
        dict(name="attn_chunk", op="attn", layout="P", ctx="36864", new="1152", pad=0, hq=32, hkv=8, d=128, ps=64, fmt="bf16"),
        # The same at the longest context, cache in 8 bits: the last 4,096 of 131,072 tokens.
        dict(name="attn_chunk_128k", op="attn", layout="P", ctx="142848", new="4608", pad=0, hq=32, hkv=4, d=128, ps=128, fmt="e4m3"),
        # Decoding and prompts in one call, long chunks, small heads and pages.
        dict(name="attn_mixed", op="attn", layout="G", ctx="20011,3,0,31007,777,12013,0,28888", new="1,1,577,1,1,301,72,1", pad=0, hq=32, hkv=8, d=64, ps=16, fmt="e4m3"),
        # A plain causal layer of the hybrid model.
        dict(name="attn_full_layer", op="attn", layout="F", ctx="16001,7168", new="1000,1024", pad=0, hq=16, hkv=16, d=128, ps=64, fmt="bf16"),
        # One token a sequence into the cache.
        dict(name="append_tokens", op="append", layout="P", pad=0, hq=32, hkv=4, d=128, ps=64, fmt="e4m3", new=",".join(["1"] * 32),
             ctx=",".join(str(271 * i * i % 36001) for i in range(32))),
        # A piece of a prompt, quantised on the way.
        dict(name="append_chunk", op="append", layout="P", ctx="36864", new="9216", pad=0, hq=32, hkv=8, d=128, ps=64, fmt="e4m3"),
        # The prompts that are waiting, in one call, kept as they are.
        dict(name="append_prompts", op="append", layout="P", ctx="0,0,0,0,5", new="581,3376,1451,6757,20011", pad=0, hq=16, hkv=16, d=128, ps=16, fmt="bf16"),
        # A whole sequence back, to go on with it elsewhere.
        dict(name="gather_128k", op="gather", layout="P", ctx="0", new="147456", pad=0, hq=32, hkv=4, d=128, ps=64, fmt="e4m3"),
        # Parts of several sequences, small heads.
        dict(name="gather_parts", op="gather", layout="G", ctx="0,31,4097,200", new="577,1,3001,2250", pad=5, hq=4, hkv=4, d=64, ps=32, fmt="bf16"),
    ]


def draw(rng: random.Random):
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    op = rng.choice(["attn", "attn", "attn", "append", "gather"])
    hq, hkv, d = rng.choice([(32, 8, 128), (32, 8, 128), (32, 4, 128), (16, 16, 128), (4, 4, 64), (32, 8, 64), (12, 4, 128), (10, 2, 64)])
    layout = rng.choice(["P", "P", "P", "G", "F"])
    k, m, C = LAYOUTS[layout]
    s = k + m
    most = 16384 if layout == "F" else 131072 * s // k
    if op == "attn":
        kind = rng.choice(["one", "tokens", "drafts", "chunk", "chunk", "mixed"])
        B = {"one": 1, "tokens": log(2, 32), "drafts": log(1, 16), "chunk": rng.choice([1, 1, 2, 3]), "mixed": log(2, 10)}[kind]
        ctx = [log(1, most) - 1 for _ in range(B)]
        if kind in ("one", "tokens"):
            new = [1] * B
        elif kind == "drafts":
            new = [rng.randint(2, 9) for _ in range(B)]
        elif kind == "chunk":
            new = [log(17, 4096 // B if layout == "F" else 4608 // B) for _ in range(B)]
        else:
            new = [log(8, 500) if rng.random() < 0.3 else 1 for _ in range(B)]
        # the plain form pads the batch: no more than the largest listed case's scores
        keys = max(c + n if layout == "F" else min(c + n, C * k + n + 2 * k) + (c + n) // s * m for c, n in zip(ctx, new))
        while B * max(new) * keys * hq > 4608 * 21000 * 32:
            new = [max(1, n // 2) for n in new]
    else:
        B = rng.choice([1, 2, 5, log(1, 32)])
        one = op == "append" and rng.random() < 0.3
        new = [1 if one else log(1, 18432 // B if op == "append" else 36864 // B) for _ in range(B)]
        ctx = [rng.choice([0, log(1, 36864)]) for _ in range(B)]
    if B > 1 and rng.random() < 0.3:
        new[rng.randrange(B)] = 0                                  # a sequence that sits this call out
        if not any(new):
            new[0] = 1
    return dict(op=op, layout=layout, ctx=",".join(map(str, ctx)), new=",".join(map(str, new)), pad=rng.choice([0, 0, 7]),
                hq=hq, hkv=hkv, d=d, ps=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["bf16", "e4m3"]))


def _ints(text):
    return [int(x) for x in text.split(",")]


def _split(a, k, m):
    """Text and summary rows among the first `a` rows of a sequence (Eq. 1)."""
    c, r = divmod(a, k + m)
    return c * k + min(r, k), c * m + max(0, r - k)


def _spans(case):
    """Per sequence: (first row, rows, text range of the call's rows, summary range, first text row anyone may see)."""
    k, m, C = LAYOUTS[case["layout"]]
    spans = []
    for a0, n in zip(_ints(case["ctx"]), _ints(case["new"])):
        (t0, s0), (t1, s1) = _split(a0, k, m), _split(a0 + n, k, m)
        first = 0 if case["op"] != "attn" else max(0, a0 // (k + m) - C) * k
        spans.append((a0, n, t0, t1, s0, s1, first))
    return spans


def _normal(shape, gen):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    return out


def _kv_rows(shape, gen):
    """Rows of K or V: normal, 1 % of the rows four times larger, a few channels twice as large."""
    x = _normal(shape, gen)
    x[torch.rand(shape[0], generator=gen, device=DEV) < 0.01] *= 4.0
    x[..., ::37] *= 2.0
    return x


_CONTEXT = []


def _context(ksa):
    """The library's handle on the device: one a process, as a server opens it, however many caches it has."""
    if not _CONTEXT:
        _CONTEXT.append(ksa.Context(0))
    return _CONTEXT[0]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    k, m, C = LAYOUTS[case["layout"]]
    hq, hkv, d, ps, op = case["hq"], case["hkv"], case["d"], case["ps"], case["op"]
    spans = _spans(case)
    B = len(spans)
    rows = sum(sp[1] for sp in spans)
    total = rows + case["pad"]
    # page tables: the pages of text that someone may still see, all of the summaries', in any order of the pool
    text_cols = max(1, max(-(-sp[3] // ps) for sp in spans))
    summ_cols = max(1, max(-(-sp[5] // ps) for sp in spans))
    text = np.full((B, text_cols), -1, dtype=np.int32)
    summ = np.full((B, summ_cols), -1, dtype=np.int32)
    need = sum(-(-sp[3] // ps) - sp[6] // ps + -(-sp[5] // ps) for sp in spans)
    num_pages = need + 3
    order = np.random.RandomState(seed % (1 << 31)).permutation(num_pages)
    used = 0
    for b, (a0, n, t0, t1, s0, s1, first) in enumerate(spans):
        lo, hi, hs = first // ps, -(-t1 // ps), -(-s1 // ps)
        text[b, lo:hi] = order[used:used + hi - lo]
        used += hi - lo
        summ[b, :hs] = order[used:used + hs]
        used += hs
    put = lambda x, t=torch.int32: torch.as_tensor(x, dtype=t, device=DEV)
    st = dict(case=case, B=B, total=total, rows=rows, spans=spans, text=put(text), summ=put(summ),
              cached=put([sp[0] for sp in spans]), cu=put(np.cumsum([0] + [sp[1] for sp in spans])))
    if op == "append":                                             # pages as an allocator gives them
        dt = torch.bfloat16 if case["fmt"] == "bf16" else torch.float8_e4m3fn
        st["kp"], st["vp"] = (torch.zeros((num_pages, hkv, ps, d), dtype=dt, device=DEV) for _ in range(2))
        st["ke"], st["ve"] = (torch.zeros((num_pages, hkv, ps), dtype=torch.uint8, device=DEV) for _ in range(2))
        st["k"], st["v"] = _kv_rows((total, hkv, d), gen), _kv_rows((total, hkv, d), gen)
    else:                                                          # pages as earlier calls left them
        for p, e in (("kp", "ke"), ("vp", "ve")):
            x = _kv_rows((num_pages * hkv * ps, d), gen)
            if case["fmt"] == "bf16":
                st[p], st[e] = x.view(num_pages, hkv, ps, d), None
            else:
                y, z = _quantise(x)
                st[p], st[e] = y.view(num_pages, hkv, ps, d), z.view(num_pages, hkv, ps)
    if op == "attn":
        st["q"] = _normal((total, hq, d), gen)
        st["scale"] = float(np.float32(d ** -0.5))
        st["out"] = torch.zeros((total, hq, d), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.zeros((hq, total), dtype=torch.float32, device=DEV)
        # what a batch's padded form needs: where each row stands, how many keys of each kind there are at most
        at = np.concatenate([b * max(sp[1] for sp in spans) + np.arange(sp[1]) for b, sp in enumerate(spans)])
        st["at"] = put(at, torch.int64)
        st["longest"] = max(sp[1] for sp in spans)
        st["text_from"] = put([sp[6] for sp in spans], torch.int64)
        st["text_most"] = max(1, max(sp[3] - sp[6] for sp in spans))
        st["summ_most"] = max(sp[5] for sp in spans)
    if op == "gather":
        st["k"], st["v"] = (torch.zeros((total, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if own:
        from paper_2604_24432_b200 import binding as ksa
        spec = ksa.PagedSpec(k, m, C, hq, hkv, d, float(np.float32(d ** -0.5)), ps, num_pages, case["fmt"])
        st["cache"] = ksa.PagedCache(_context(ksa), spec, st["kp"], st["vp"], st["ke"] if case["fmt"] == "e4m3" else None, st["ve"] if case["fmt"] == "e4m3" else None)
        st["batch"] = ksa.PagedBatch(st["cached"], st["cu"], st["text"], st["summ"])
    return st


def run(st):
    op = st["case"]["op"]
    if own:
        cache, batch = st["cache"], st["batch"]
        if op == "append":
            cache.append(batch, st["k"], st["v"])
            return [st["kp"], st["vp"], st["ke"], st["ve"]]
        if op == "gather":
            cache.gather(batch, st["k"], st["v"])
            return [st["k"], st["v"]]
        cache.attn(batch, st["q"], st["out"], st["lse"])
        return [st["out"], st["lse"]]
    return {"append": _append, "gather": _gather, "attn": _attn}[op](st)


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _quantise(x):
    """Rows as e4m3 and one scale 2^(e - 127) a row: the smallest power of two, from 2^-110 up, at which the row's largest
    value is within 448. A row that holds an infinity or a NaN: zeros and e = 255, which stands for NaN."""
    x = x.float()
    top = x.abs().amax(-1)
    fine = torch.isfinite(top)
    mant, exp = torch.frexp(torch.where(fine, top, 0.0))           # top = mant 2^exp, mant in [1/2, 1); 448 = 0.875 * 2^9
    e = torch.where(mant > 0.875, exp - 8, exp - 9)
    e = torch.where(mant == 0, -110, e).clamp(min=-110)
    y = torch.where(fine[..., None], torch.ldexp(x, -e[..., None]), 0.0).to(torch.float8_e4m3fn)
    return y, torch.where(fine, e + 127, 255).to(torch.uint8)


def _rows(st):
    """For the packed rows of the call: page and row in the page (page -1: none)."""
    k, m, _ = LAYOUTS[st["case"]["layout"]]
    ps = st["case"]["ps"]
    i = torch.arange(st["rows"], device=DEV)
    cu = st["cu"].long()
    b = torch.bucketize(i, cu[1:], right=True)
    a = st["cached"].long()[b] + i - cu[b]
    c, r = a // (k + m), a % (k + m)
    is_text = r < k
    x = torch.where(is_text, c * k + r, c * m + r - k)
    tp = st["text"][b, torch.where(is_text, x // ps, 0)]
    sp = st["summ"][b, torch.where(is_text, 0, x // ps)]
    return torch.where(is_text, tp, sp).long(), x % ps


def _append(st):
    page, slot = _rows(st)
    n = st["rows"]
    for name, p, e in (("k", "kp", "ke"), ("v", "vp", "ve")):
        x = st[name][:n]
        if st["case"]["fmt"] == "e4m3":
            x, z = _quantise(x)
            st[e][page, :, slot] = z
        st[p].view(torch.uint8 if x.dtype == torch.float8_e4m3fn else x.dtype)[page, :, slot] = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    return [st["kp"], st["vp"], st["ke"], st["ve"]]


def _values(p, e, page, *where):
    """Rows of the pool as fp32 (page -1: zeros)."""
    x = p.view(torch.uint8)[(page.clamp(min=0),) + where].view(p.dtype).float() if p.dtype == torch.float8_e4m3fn else p[(page.clamp(min=0),) + where].float()
    if e is not None:
        z = e[(page.clamp(min=0),) + where].int()
        x = x * torch.where(z == 255, float("nan"), torch.ldexp(torch.ones_like(z, dtype=torch.float32), z - 127))[..., None]
    return torch.where((page >= 0).view(page.shape + (1,) * (x.dim() - page.dim())), x, 0.0)


def _gather(st):
    page, slot = _rows(st)
    for name, p, e in (("k", "kp", "ke"), ("v", "vp", "ve")):
        st[name][:st["rows"]] = _values(st[p], st[e], page, slice(None), slot).to(torch.bfloat16)
    return [st["k"], st["v"]]


def _attn(st):
    case = st["case"]
    k, m, C = LAYOUTS[case["layout"]]
    hq, hkv, d, ps, B, N = case["hq"], case["hkv"], case["d"], case["ps"], st["B"], st["longest"]
    G = hq // hkv
    cu, cached = st["cu"].long(), st["cached"].long()
    # queries, padded to the longest run of the batch, with the ranges of text and of summaries that each may see
    q = torch.zeros((B * N, hq, d), device=DEV)
    q[st["at"]] = st["q"][:st["rows"]].float() * st["scale"]
    q = q.view(B, N, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, G * N, d)
    a = cached[:, None] + torch.arange(N, device=DEV)
    c, r = a // (k + m), a % (k + m)
    is_text = r < k
    far = (c - C).clamp(min=0)
    t_lo, t_hi = torch.where(is_text, far * k, c * k), torch.where(is_text, c * k + r + 1, (c + 1) * k)
    s_lo, s_hi = torch.where(is_text, 0, c * m), torch.where(is_text, far * m, c * m + r - k + 1)
    # keys: the batch's text from its first visible row, then its summaries
    ti = st["text_from"][:, None] + torch.arange(st["text_most"], device=DEV)
    si = torch.arange(st["summ_most"], device=DEV).expand(B, -1)
    bi = torch.arange(B, device=DEV)[:, None]
    t_page = st["text"][bi, (ti // ps).clamp(max=st["text"].shape[1] - 1)].long()
    s_page = st["summ"][bi, si // ps].long()
    page, slot = torch.cat([t_page, s_page], 1), torch.cat([ti, si], 1) % ps
    see = torch.cat([(ti[:, None] >= t_lo[..., None]) & (ti[:, None] < t_hi[..., None]), (si[:, None] >= s_lo[..., None]) & (si[:, None] < s_hi[..., None])], 2)
    see = see & ((t_lo < t_hi) & (torch.arange(N, device=DEV) < (cu[1:] - cu[:-1])[:, None]))[..., None]
    hide = ~see[:, None, None]
    key = _values(st["kp"], st["ke"], page, slice(None), slot).transpose(1, 2)
    s = (q @ key.transpose(2, 3)).view(B, hkv, G, N, -1)
    del key
    s.masked_fill_(hide, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s = s.sub_(top).exp_()
    l = s.sum(-1, keepdim=True)
    val = _values(st["vp"], st["ve"], page, slice(None), slot).transpose(1, 2)
    val = torch.where(see.any(1)[:, None, :, None], val, 0.0)
    o = (s.view(B, hkv, G * N, -1) @ val).view(B, hkv, G, N, d) / l
    lse = (top + l.log()).squeeze(-1)
    st["out"][:st["rows"]] = o.permute(0, 3, 1, 2, 4).reshape(B * N, hq, d)[st["at"]].to(torch.bfloat16)
    st["lse"][:, :st["rows"]] = lse.permute(1, 2, 0, 3).reshape(hq, B * N)[:, st["at"]]
    return [st["out"], st["lse"]]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    k, m, C = LAYOUTS[case["layout"]]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    row = 2 * d * hkv * 2 if case["fmt"] == "bf16" else 2 * (d + 1) * hkv      # K and V of a cached row
    n = sum(_ints(case["new"]))
    if case["op"] != "attn":
        return {"bytes": n * (row + 4 * d * hkv), "flops": 0}
    keys = pairs = 0
    for a0, cnt, t0, t1, s0, s1, first in _spans(case):
        if cnt == 0:
            continue
        i = np.arange(t0, t1, dtype=np.int64)                      # text rows
        far = np.maximum(0, i // k - C)
        pairs += int((i + 1 - far * k + far * m).sum())
        j = np.arange(s0, s1, dtype=np.int64)                      # summaries
        pairs += int((k + j % m + 1).sum()) if m else 0
        tk, sk = np.zeros(t1 + k, dtype=bool), np.zeros(s1 + 1, dtype=bool)     # rows that someone sees
        if i.size:
            tk[far[0] * k:t1] = True
            sk[:far[-1] * m] = True
        if j.size:
            tk[s0 // m * k:((s1 - 1) // m + 1) * k] = True
            sk[s0 // m * m:s1] = True
        keys += int(tk.sum() + sk.sum())
    return {"bytes": keys * row + n * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------------------
def _exact_row(st, p, e, pages, slots):
    """[rows, heads, d] in 64 bits."""
    raw = st[p].view(torch.uint8) if st[p].dtype == torch.float8_e4m3fn else st[p]
    x = raw[pages, :, slots]
    if st[e] is None:
        return x.double()
    code = x.long()
    mag, expo = (code & 7).double(), (code >> 3) & 15
    val = torch.where(expo == 0, mag * 2.0 ** -9, (8 + mag) * torch.exp2((expo - 10).double()))
    return torch.where(code >= 128, -val, val) * torch.exp2(st[e][pages, :, slots].double() - 127)[..., None]


def _exact_places(st):
    """(stream, index, page, slot) of each row of the call, row by row."""
    case = st["case"]
    k, m, _ = LAYOUTS[case["layout"]]
    text, summ, pages, slots = st["text"].cpu().numpy(), st["summ"].cpu().numpy(), [], []
    for b, (a0, n, *_r) in enumerate(st["spans"]):
        a = np.arange(a0, a0 + n)
        chunk = a // (k + m)
        rest = a - chunk * (k + m)
        ix = np.where(rest < k, a - chunk * m, a - (chunk + 1) * k)
        pages.append(np.where(rest < k, text[b][np.minimum(ix // case["ps"], text.shape[1] - 1)], summ[b][np.minimum(ix // case["ps"], summ.shape[1] - 1)]))
        slots.append(ix % case["ps"])
    return torch.as_tensor(np.concatenate(pages), device=DEV).long(), torch.as_tensor(np.concatenate(slots), device=DEV).long()


def _exact_e4m3(x):
    """Nearest e4m3 value (ties to even) of values within 448, in 64 bits."""
    _, ex = torch.frexp(x)
    step = torch.exp2((ex - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    k, m, C = LAYOUTS[case["layout"]]
    op, n = case["op"], st["rows"]
    if op == "gather":
        page, slot = _exact_places(st)
        outs = []
        for name, p, e in (("k", "kp", "ke"), ("v", "vp", "ve")):
            o = st[name].double()
            o[:n] = _exact_row(st, p, e, page.clamp(min=0), slot) * (page >= 0)[:, None, None]
            outs.append(o)
        return outs
    if op == "append":
        page, slot = _exact_places(st)
        vals, exps = [], []
        for name, p, e in (("k", "kp", "ke"), ("v", "vp", "ve")):
            x, pool, ze = st[name][:n].double(), st[p].double(), st[e].clone()
            if case["fmt"] == "e4m3":
                top = x.abs().amax(-1)
                z = torch.full(top.shape, -110, device=DEV)
                for _ in range(240):                               # up, a power at a time, until the row fits
                    z = torch.where(top > 448 * torch.exp2(z.double()), z + 1, z)
                x = _exact_e4m3(x * torch.exp2(-z.double())[..., None])
                ze[page, :, slot] = (z + 127).to(torch.uint8)
            pool[page, :, slot] = x
            vals.append(pool)
            exps.append(ze)
        return vals + exps
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["ps"]
    G = hq // hkv
    out, lse = st["out"].double(), st["lse"].double()
    row0 = 0
    for b, (a0, cnt, t0, t1, s0, s1, first) in enumerate(st["spans"]):
        if cnt == 0:
            continue
        ti, si = torch.arange(first, t1, device=DEV), torch.arange(0, s1, device=DEV)
        pages = torch.cat([st["text"][b][ti // ps], st["summ"][b][si // ps]]).long()
        slots = torch.cat([ti, si]) % ps
        chunk = torch.cat([ti // k, si // max(m, 1)])              # of each key
        kind = torch.cat([torch.zeros_like(ti), torch.ones_like(si)])
        pos = torch.cat([ti + ti // k * m, si + (si // max(m, 1) + 1) * k])     # rows of the keys in the sequence (Eq. 1)
        key, val = _exact_row(st, "kp", "ke", pages, slots), _exact_row(st, "vp", "ve", pages, slots)
        step = max(1, (1 << 28) // (pos.numel() * G))
        for i in range(0, cnt, step):
            a = torch.arange(a0 + i, a0 + min(cnt, i + step), device=DEV)[:, None]
            qc, q_text = a // (k + m), a % (k + m) < k
            near = (kind == 0) & (chunk >= qc - C) & (pos <= a)
            away = (kind == 1) & (chunk < qc - C)
            mine = (chunk == qc) & (pos <= a)
            see = torch.where(q_text, near | away, mine)
            for h in range(hkv):
                q = st["q"][row0 + i:row0 + i + a.shape[0], h * G:(h + 1) * G].double() * st["scale"]
                x = torch.einsum("ngd,kd->gnk", q, key[:, h])
                x.masked_fill_(~see, float("-inf"))
                z = torch.logsumexp(x, -1)
                x = x.sub_(z[..., None]).exp_()
                out[row0 + i:row0 + i + a.shape[0], h * G:(h + 1) * G] = torch.einsum("gnk,kd->ngd", x, torch.where(see.any(0)[:, None], val[:, h], 0.0))
                lse[h * G:(h + 1) * G, row0 + i:row0 + i + a.shape[0]] = z
        row0 += cnt
    return [out, lse]
