"""Paged KV cache on the GPU: rows written, read back and attended to against the definitions in 64 bits (paged_ref.py, whose
`check` derives the bounds).  Pools start as NaN, so that nothing unwritten may reach a result; pages stand in random order."""
import numpy as np
import pytest
import torch

from paper_2604_24432_b200 import binding as ksa
from paper_2604_24432_b200 import build as ksa_build
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# the kernel as the call takes it, and held to the one for many query rows
BY_RULE, MANY, FEW = 0, ksa.KSA_FLAG_PAGED_TCGEN05, ksa.KSA_FLAG_PAGED_MMA_SYNC


@pytest.fixture(scope="module")
def ctx():
    ksa_build.build()
    c = ksa.Context(0)
    yield c
    c.close()


def _i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32, device=DEV)


def _texts(k, m, a):
    c, r = divmod(a, k + m)
    return c * k + min(r, k)


class Server:
    """Sequences with all their rows on the host, and a cache with the pages they need."""

    def __init__(self, ctx, k, m, C, Hq, Hkv, D, ps, fmt, lens, flags=0, seed=0, spare=2, pools=None, qkv_scale=1.0):
        self.ctx, self.k, self.m, self.C, self.Hq, self.Hkv, self.D, self.ps, self.fmt, self.flags = ctx, k, m, C, Hq, Hkv, D, ps, fmt, flags
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.lens = lens
        norm = lambda n, H: (torch.randn((n, H, D), generator=g) * qkv_scale).bfloat16()
        self.q, self.key, self.val = [norm(n, Hq) for n in lens], [norm(n, Hkv) for n in lens], [norm(n, Hkv) for n in lens]
        cols_t = max(1, max(-(-_texts(k, m, n) // ps) for n in lens))
        cols_s = max(1, max(-(-(n - _texts(k, m, n)) // ps) for n in lens))
        of_summ = len(lens) * cols_s if m else 0
        pages = rng.permutation(len(lens) * cols_t + of_summ + spare)
        self.text = pages[:len(lens) * cols_t].reshape(len(lens), cols_t).copy()
        self.summ = pages[len(lens) * cols_t:len(lens) * cols_t + of_summ].reshape(len(lens), -1).copy() if m else np.full((len(lens), 1), -1)
        self.scale = float(np.float32(D ** -0.5))
        spec = ksa.PagedSpec(k, m, C, Hq, Hkv, D, self.scale, ps, len(pages), fmt, flags)
        self.cache = ksa.PagedCache(ctx, spec, *(pools(len(pages)) if pools else ()))
        self.poison()

    def poison(self):
        c = self.cache
        for t in (c.kpages, c.vpages):
            t.copy_(torch.full(t.shape, float("nan"), device=DEV).to(t.dtype))
        for t in (c.kscale, c.vscale):
            if t is not None:
                t.fill_(255)

    def batch(self, spans):
        """spans: (first row, rows) of every sequence."""
        return ksa.PagedBatch(_i32([a for a, _ in spans]), _i32(np.cumsum([0] + [n for _, n in spans])), _i32(self.text), _i32(self.summ))

    def rows(self, what, spans, pad=0):
        x = torch.cat([t[a:a + n] for t, (a, n) in zip(what, spans)] + [torch.zeros((pad,) + what[0].shape[1:], dtype=what[0].dtype)])
        return x.to(DEV)

    def append(self, spans, pad=0):
        self.cache.append(self.batch(spans), self.rows(self.key, spans, pad), self.rows(self.val, spans, pad))

    def fill(self, spans):
        """Everything before the spans' rows, and those, in one call."""
        self.append([(0, a + n) for a, n in spans])

    def attn(self, spans, pad=0, batch=None, q=None, **how):
        q = self.rows(self.q, spans, pad) if q is None else q
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((self.Hq, q.shape[0]), -1.0, device=DEV)
        self.ctx.clear_device_status()
        self.cache.attn(batch or self.batch(spans), q, out, lse, **how)
        torch.cuda.synchronize()
        assert self.ctx.device_status() == 0
        return out, lse

    def cached_values(self, rows):
        """What the cache stands for, in 64 bits: bf16 rows as they are, e4m3 rows rounded by the reference."""
        if self.fmt == "bf16":
            return rows.double().numpy()
        x = rows.double().numpy().reshape(-1, self.D)
        return np.stack([ref.values(*ref.quantise_row(r)) for r in x]).reshape(rows.shape)

    def check(self, out, lse, spans, sample=None):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy().T
        row0 = 0
        for b, (a, n) in enumerate(spans):
            if n:
                key, val = self.cached_values(self.key[b][:a + n]), self.cached_values(self.val[b][:a + n])
                picks = range(n) if sample is None or n <= sample else sorted(set([0, n - 1, *np.random.default_rng(b).integers(0, n, sample)]))
                for i in picks:
                    r = ref.attention(self.q[b][a + i:a + i + 1].double().numpy(), key[:a + i + 1], val[:a + i + 1], self.k, self.m, self.C, a + i, self.scale, bool(self.flags & ksa.KSA_FLAG_SUMMARY_TEXT_ONLY))
                    ref.check(out[row0 + i:row0 + i + 1], lse[row0 + i:row0 + i + 1], r, self.D)
            row0 += n
        assert (out[row0:] == 7.0).all() and (lse[row0:] == -1.0).all()      # rows behind the last sequence


# ---- writing and reading back ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("k,m,Hkv,D,ps,spans,pad", [
    (8, 1, 2, 128, 64, [(0, 1)], 0),
    (8, 1, 3, 64, 16, [(5, 40), (0, 0), (17, 1), (100, 333)], 3),
    (3, 2, 1, 128, 32, [(0, 0), (7, 129)], 0),
    (64, 8, 4, 64, 128, [(70, 500), (0, 3)], 1),
    (8, 0, 2, 128, 16, [(31, 2), (0, 65)], 0),
    (1, 1, 2, 64, 16, [(0, 50)] * 33, 2),                      # more than 32 sequences
    (8, 1, 1, 128, 16, [(9 * i, i % 3) for i in range(32)], 0),
])
def test_append_and_gather(ctx, fmt, k, m, Hkv, D, ps, spans, pad):
    s = Server(ctx, k, m, 4, Hkv, Hkv, D, ps, fmt, [a + n + 1 for a, n in spans], seed=3)
    c = s.cache
    before = [t.clone() if t is not None else None for t in (c.kpages, c.vpages, c.kscale, c.vscale)]
    ctx.clear_device_status()
    s.append(spans, pad)
    got = [s.rows(s.key, spans, pad).fill_(7.0) for _ in range(2)]
    c.gather(s.batch(spans), *got)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    raw = lambda t: None if t is None else t.view(torch.uint8 if t.element_size() == 1 else torch.int16).cpu().numpy()
    want = [raw(t).copy() if t is not None else None for t in before]
    expect = [[], []]
    for b, (a, n) in enumerate(spans):
        where = ref.places(k, m, a + n)[a:]
        for i, (is_summ, x) in enumerate(where):
            page, slot = (s.summ if is_summ else s.text)[b][x // ps], x % ps
            for j, rows in enumerate((s.key, s.val)):
                for h in range(Hkv):
                    r = rows[b][a + i, h]
                    if fmt == "bf16":
                        want[j][page, h, slot] = r.view(torch.int16).numpy()
                        expect[j].append(r.double().numpy())
                    else:
                        codes, byte = ref.quantise_row(r.double().numpy())
                        want[j][page, h, slot], want[2 + j][page, h, slot] = codes, byte
                        expect[j].append(ref.values(codes, byte))
    for t, w in zip((c.kpages, c.vpages, c.kscale, c.vscale), want):     # every byte of the pools: the rows, and nothing else
        assert t is None or (raw(t) == w).all()
    rows = sum(n for _, n in spans)
    for j in range(2):
        g = got[j].double().cpu().numpy()
        assert (g[:rows].reshape(-1, D) == np.array(expect[j]).reshape(-1, D)).all() and (g[rows:] == 7.0).all()


def test_quantisation_edges(ctx):
    """Zeros, values near the ends of bf16, scale borders, ties, infinities and NaN, each a row of its own."""
    D = 64
    rows = []
    for top in (0.0, 448.0, 449.0, 450.0, 446.0, 2.0 ** -118, 2.0 ** -126, 1e-38, 3.3e38, 2.0 ** -101, 448 * 2.0 ** -110, 452 * 2.0 ** -110, 1.0, 0.875, 0.8750001):
        r = np.linspace(-1.0, 1.0, D) * top
        rows.append(r)
    rows.append(np.concatenate([[448.0], (ref.E4M3[1:64] + ref.E4M3[:63]) / 2]))       # ties (exact in bf16)
    rows.append(np.concatenate([[-448.0], -(ref.E4M3[64:126] + ref.E4M3[63:125]) / 2, [0.0]]))
    for bad in (np.inf, -np.inf, np.nan):
        r = np.ones(D); r[D // 3] = bad
        rows.append(r)
    x = torch.tensor(np.array(rows)).bfloat16()
    n = len(rows)
    s = Server(ctx, 8, 0, 4, 1, 1, D, 16, "e4m3", [n], seed=1)
    s.key, s.val = [x.view(n, 1, D)], [x.flip(0).reshape(n, 1, D)]
    s.append([(0, n)])
    got = [torch.empty((n, 1, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    s.cache.gather(s.batch([(0, n)]), *got)
    for g, rows_ in zip(got, (x, x.flip(0))):
        want = np.stack([ref.values(*ref.quantise_row(r)) for r in rows_.double().numpy()])
        np.testing.assert_array_equal(g.view(n, D).double().cpu().numpy(), want)


def test_gather_of_pages_given_back(ctx):
    s = Server(ctx, 8, 1, 1, 2, 2, 64, 16, "e4m3", [100])
    s.append([(0, 100)])
    s.text[0, 1] = -1
    got = [torch.full((100, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ctx.clear_device_status()
    s.cache.gather(s.batch([(0, 100)]), *got)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    gone = torch.tensor([not w[0] and 16 <= w[1] < 32 for w in ref.places(8, 1, 100)])
    for g, rows in zip(got, (s.key, s.val)):
        assert (g.cpu()[gone] == 0).all()
        assert (g.double().cpu().numpy()[~gone.numpy()] == s.cached_values(rows[0])[~gone.numpy()]).all()


# ---- attention ---------------------------------------------------------------------------------------------------------------
SHAPES = [
    # k, m, C, Hq, Hkv, D, ps, flags, spans, pad
    (8, 1, 3, 4, 1, 128, 64, 0, [(0, 1)], 0),                                         # the first token of a sequence
    (8, 1, 3, 8, 2, 128, 16, 0, [(7, 1), (8, 1), (9, 1), (100, 1), (332, 1)], 2),     # text and summary rows alone
    (8, 1, 128, 8, 1, 64, 32, 0, [(700, 1), (3, 1), (1500, 1)], 0),                   # window wider than the sequence
    (8, 1, 4, 16, 16, 64, 16, 0, [(61, 5), (0, 5), (200, 5)], 0),                     # multi-head, drafts
    (8, 1, 4, 32, 4, 128, 64, 0, [(130, 7), (0, 0), (1, 2), (0, 0), (77, 12)], 5),    # sequences without rows
    (8, 1, 2, 10, 2, 64, 32, 0, [(37, 50)], 0),                                       # group of 5
    (8, 1, 2, 6, 2, 128, 16, 0, [(0, 40), (99, 3)], 0),                               # group of 3
    (8, 1, 2, 32, 1, 64, 64, 0, [(90, 3), (20, 1)], 0),                               # one KV head for 32
    (8, 1, 2, 64, 1, 128, 16, 0, [(45, 2)], 0),
    (8, 1, 2, 17, 1, 64, 16, 0, [(45, 20)], 1),
    (64, 8, 1, 8, 2, 128, 128, 0, [(60, 90), (500, 1)], 0),                           # several summaries a chunk
    (64, 8, 1, 8, 2, 64, 16, ksa.KSA_FLAG_SUMMARY_TEXT_ONLY, [(60, 90), (135, 1)], 0),
    (8, 1, 0, 4, 2, 64, 16, 0, [(0, 100)], 0),                                        # no window: summaries and the own chunk
    (1, 1, 3, 4, 2, 64, 16, 0, [(10, 60)], 0),
    (3, 2, 2, 4, 4, 128, 16, 0, [(0, 70), (64, 9)], 3),
    (200, 3, 1, 4, 2, 64, 64, 0, [(190, 30), (400, 2)], 0),
    (8, 0, 1 << 20, 8, 2, 128, 64, 0, [(0, 200), (333, 70)], 0),                      # plain causal
    (8, 0, 3, 4, 4, 64, 32, 0, [(100, 150)], 0),                                      # sliding chunks alone (Eq. 2)
    (8, 1, 5, 8, 2, 128, 64, 0, [(0, 580)], 0),                                       # a whole prompt
    (8, 1, 16, 4, 4, 128, 128, 0, [(290, 400), (0, 129), (63, 64)], 0),
]


@pytest.mark.parametrize("kernel", [BY_RULE, MANY, FEW])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("k,m,C,Hq,Hkv,D,ps,flags,spans,pad", SHAPES)
def test_attention(ctx, kernel, fmt, k, m, C, Hq, Hkv, D, ps, flags, spans, pad):
    s = Server(ctx, k, m, C, Hq, Hkv, D, ps, fmt, [max(1, a + n) for a, n in spans], flags | kernel, seed=11)
    s.fill(spans)
    out, lse = s.attn(spans, pad)
    s.check(out, lse, spans, sample=60)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,n", [(8, 2, 128, 1), (8, 2, 128, 300), (4, 4, 64, 40)])
def test_long_context_with_released_pages(ctx, kernel, fmt, Hq, Hkv, D, n):
    """Text that has left every window is given back (and its pages poisoned); rows behind the sequence are NaN."""
    k, m, C, ps = 8, 1, 9, 16
    a = 6007
    s = Server(ctx, k, m, C, Hq, Hkv, D, ps, fmt, [a + n + 40, 33], seed=5, flags=kernel)
    spans = [(a, n), (20, 3)]
    s.fill(spans)
    first = max(0, a // 9 - C) * k // ps
    gone = s.text[0, :first].copy()
    s.text[0, :first] = -1
    s.cache.kpages[torch.from_numpy(gone).to(DEV)] = float("nan")
    s.cache.vpages[torch.from_numpy(gone).to(DEV)] = float("nan")
    if fmt == "e4m3":
        s.cache.kscale[torch.from_numpy(gone).to(DEV)] = 255
        s.cache.vscale[torch.from_numpy(gone).to(DEV)] = 255
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=25)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt,k,m,D,ctx_rows,n", [
    ("bf16", 8, 0, 128, 4300, 40), ("e4m3", 8, 0, 64, 4300, 70), ("bf16", 8, 1, 64, 4200, 90),     # six CTAs a query tile
    ("bf16", 8, 0, 64, 2200, 600), ("e4m3", 8, 0, 128, 2200, 150),                                # four
    ("bf16", 8, 0, 64, 1200, 1000), ("e4m3", 8, 0, 64, 1200, 1000),                               # three
])
def test_long_views_on_several_ctas(ctx, kernel, fmt, k, m, D, ctx_rows, n):
    s = Server(ctx, k, m, 1 << 20, 8, 2, D, 64, fmt, [ctx_rows + n], seed=n, flags=kernel)
    spans = [(ctx_rows, n)]
    s.fill(spans)
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=40)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt,B,most", [("bf16", 65, 1), ("e4m3", 65, 3), ("bf16", 1100, 1), ("e4m3", 1100, 2), ("bf16", 2049, 2),   # single tokens' kernel
                                        ("bf16", 33, 30), ("bf16", 800, 11), ("e4m3", 90, 40), ("bf16", 1537, 11)])                  # the other
def test_many_sequences(ctx, kernel, fmt, B, most):
    """Tens to thousands of sequences, some without rows, in whole groups too, of lengths from nothing to a few pages."""
    rng = np.random.default_rng(B + most)
    spans = [(int(a), int(n)) for a, n in zip(rng.integers(0, 60, B), rng.integers(0 if most > 1 else 1, most + 1, B))]
    for b in range(32, min(B, 64)):
        spans[b] = (spans[b][0], 0)
    spans[B - 1] = (37, most)
    s = Server(ctx, 8, 1, 3, 4, 1, 64, 16, fmt, [max(1, a + n) for a, n in spans], seed=B, flags=kernel)
    s.fill(spans)
    out, lse = s.attn(spans, pad=3)
    s.check(out, lse, spans, sample=2)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 150])
def test_peaked_and_spread_scores(ctx, kernel, fmt, n):
    """Scores up to hundreds: the running maximum moves often, and rows differ by orders of magnitude."""
    s = Server(ctx, 8, 1, 40, 8, 2, 128, 32, fmt, [1000], seed=8, qkv_scale=4.0, flags=kernel)
    for b in (s.key, s.val):
        b[0][::97] *= 16.0
        b[0][5::41] *= 2.0 ** -20
    spans = [(1000 - n, n)]
    s.fill(spans)
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=25)


@pytest.mark.parametrize("kernel", [MANY])
@pytest.mark.parametrize("k,m,C,Hq,Hkv,D,ps,flags,spans,pad", [
    (8, 1, 9, 16, 4, 128, 64, 0, [(2003, 700)], 0),
    (8, 1, 9, 8, 1, 64, 16, 0, [(77, 800), (0, 0), (1500, 300)], 3),
    (64, 8, 1, 16, 4, 128, 32, ksa.KSA_FLAG_SUMMARY_TEXT_ONLY, [(500, 530)], 0),
    (64, 8, 2, 16, 2, 64, 128, 0, [(66, 330), (70, 300)], 0),
    (8, 0, 1 << 20, 16, 4, 128, 64, 0, [(300, 520)], 0),
    (8, 1, 0, 32, 4, 128, 16, 0, [(9, 300)], 0),
    (8, 1, 5, 16, 2, 128, 32, 0, [(900, 1), (13, 1400), (0, 0), (300, 2), (44, 17)], 2),      # single tokens among them
])
def test_long_runs_over_e4m3(ctx, kernel, k, m, C, Hq, Hkv, D, ps, flags, spans, pad):
    """With the workspace (the rows in view as bf16 pages) and without: each against the reference.  Pages before every window are
    given back, and whatever nobody sees is NaN; so is the workspace."""
    s = Server(ctx, k, m, C, Hq, Hkv, D, ps, "e4m3", [a + n + 7 for a, n in spans], flags | kernel, seed=19)
    s.fill(spans)
    for b, (a, n) in enumerate(spans):
        s.text[b, :max(0, a // (k + m) - C) * k // ps] = -1
    batch = s.batch(spans)
    p = s.cache._params(batch, sum(n for _, n in spans) + pad, (0, 0), (0, 0), (0, 0), (0, 0))
    ws = s.cache._workspace(p, None)
    assert ws is not None
    ws.fill_(255)                                             # (as bf16: NaN)
    before = ctx.launch_count()
    for how, launches in ((dict(workspace=ws), 2), (dict(workspace=ws[:256]), 1), (dict(), 2)):
        launches += len(spans) >= 4                           # the kernel for sequences of few rows, beside the other
        out, lse = s.attn(spans, pad, **how)
        assert ctx.launch_count() == before + launches
        before += launches
        s.check(out, lse, spans, sample=24)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 150, 700])
@pytest.mark.parametrize("what", ["all V", "some V", "all K", "tiny V", "huge V"])
def test_rows_of_zeros_and_of_extreme_size(ctx, kernel, fmt, n, what):
    """Rows of zeros have the least scale: their keys count in the sums all the same.  V of 1e-15 or 1e30 scales the output."""
    s = Server(ctx, 8, 1, 100, 8, 2, 128, 32, fmt, [1100], seed=9, flags=kernel)
    rows = (s.val if "V" in what else s.key)[0]
    if what.startswith("all"):
        rows.zero_()
    elif what == "some V":
        rows[::3] = 0
        s.q[0] *= 3.0                                          # scores far apart: zero rows dominate some sums, not others
    else:
        rows.copy_((rows.float() * (1e-15 if what == "tiny V" else 1e30)).bfloat16())
    spans = [(1100 - n, n)]
    s.fill(spans)
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=12)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
def test_one_page_and_one_head_of_any_stride(ctx, kernel):
    """Strides of a dimension of one are not looked at."""
    D = 64
    base = torch.empty(5 * 128 * D + 3 * D, dtype=torch.bfloat16, device=DEV)
    pools = lambda n: tuple(torch.as_strided(base, (1, 1, 128, D), (3, 5, D, 1), off) for off in (0, 128 * D + 2 * D))
    for n in (1, 90):
        s = Server(ctx, 8, 0, 100, 4, 1, D, 128, "bf16", [100], seed=2, spare=0, pools=pools, flags=kernel)
        spans = [(100 - n, n)]
        s.fill(spans)
        out, lse = s.attn(spans)
        s.check(out, lse, spans, sample=20)


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
def test_strided_pools_and_rows(ctx, kernel):
    """Pages as [page, row, head, d] and padded heads; q a slice of a fused projection; out a slice of a wider tensor."""
    k, m, C, Hq, Hkv, D, ps = 8, 1, 3, 8, 2, 128, 32
    pools = lambda n: tuple(torch.empty((n, ps, Hkv + 1, D), dtype=torch.bfloat16, device=DEV)[:, :, :Hkv].transpose(1, 2) for _ in range(2))
    for n in (1, 200):
        spans = [(150, n), (31, 2)]
        s = Server(ctx, k, m, C, Hq, Hkv, D, ps, "bf16", [a + c for a, c in spans], pools=pools, seed=4, flags=kernel)
        total = n + 2
        fused = torch.zeros((a_ := sum(a + c for a, c in spans), Hkv * 2 + 1, D), dtype=torch.bfloat16, device=DEV)
        full = [(0, a + c) for a, c in spans]
        fused[:, :Hkv], fused[:, Hkv + 1:] = s.rows(s.key, full), s.rows(s.val, full)
        s.cache.append(s.batch(full), fused[:, :Hkv], fused[:, Hkv + 1:])
        qkv = torch.randn((total, Hq + 3, D), device=DEV).bfloat16()
        qkv[:, 2:2 + Hq] = s.rows(s.q, spans)
        wide = torch.full((total, Hq, 2 * D), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((Hq, total), -1.0, device=DEV)
        s.cache.attn(s.batch(spans), qkv[:, 2:2 + Hq], wide[..., :D], lse)
        torch.cuda.synchronize()
        s.check(wide[..., :D], lse, spans, sample=30)
        assert (wide[..., D:] == 7.0).all()
        back = torch.full((total, Hkv, 3 * D), 7.0, dtype=torch.bfloat16, device=DEV)
        s.cache.gather(s.batch(spans), back[..., :D], back[..., D:2 * D])
        assert torch.equal(back[..., :D].cpu(), s.rows(s.key, spans).cpu()) and torch.equal(back[..., D:2 * D].cpu(), s.rows(s.val, spans).cpu())
        assert (back[..., 2 * D:] == 7.0).all()


def test_shared_prefix_pages(ctx):
    """Two sequences read the same pages for a common prefix."""
    s = Server(ctx, 8, 1, 4, 4, 2, 64, 16, "bf16", [150, 150], seed=6)
    for x in (s.key, s.val):
        x[1][:72] = x[0][:72]
    s.text[1, :4] = s.text[0, :4]
    s.append([(0, 72), (0, 0)])
    s.append([(72, 78), (72, 78)])                        # (rows 72 .. share no page: 64 text tokens before them; summaries differ)
    s.append([(0, 0), (64, 8)])                           # the second sequence's own summary page, rows of chunk 7 once more
    for c in range(8):
        s.append([(0, 0), (c * 9 + 8, 1)])
    spans = [(72, 78), (72, 78)]
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=40)


def test_bad_pages_and_lengths_are_reported(ctx):
    """Entries that are no pages, columns past the table, lengths that are none: a status, nothing else touched, and the context
    goes on.  (That no such entry becomes an address is shown on the host: test_paged.py, test_entries_and_lengths.)"""
    for n in (1, 130):
        s = Server(ctx, 8, 1, 4, 4, 2, 64, 16, "bf16", [400, 200], seed=6)
        spans = [(60, n), (60, n)]
        s.fill(spans)
        good = s.batch(spans)
        q = s.rows(s.q, spans)
        out, lse = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), torch.full((4, 2 * n), -1.0, device=DEV)
        pools = [s.cache.kpages.clone(), s.cache.vpages.clone()]

        def status(batch, call):
            ctx.clear_device_status()
            call(batch)
            torch.cuda.synchronize()
            got = ctx.device_status()
            ctx.clear_device_status()
            return got
        attn = lambda b: s.cache.attn(b, q, out, lse)
        append = lambda b: s.cache.append(b, s.rows(s.key, spans), s.rows(s.val, spans))
        gather = lambda b: s.cache.gather(b, torch.empty((2 * n, 2, 64), dtype=torch.bfloat16, device=DEV), torch.empty((2 * n, 2, 64), dtype=torch.bfloat16, device=DEV))
        for entry in (-1, -7, s.cache.spec.num_pages, 2**31 - 1):
            t = good.text_table.clone()
            t[1, (60 * 8 // 9) // 16] = entry
            b = ksa.PagedBatch(good.cached, good.cu_rows, t, good.summ_table)
            assert status(b, attn) == ksa.KSA_PAGED_STATUS_BAD_PAGE and status(b, append) == ksa.KSA_PAGED_STATUS_BAD_PAGE
            assert status(b, gather) == (0 if entry == -1 else ksa.KSA_PAGED_STATUS_BAD_PAGE)
        short = ksa.PagedBatch(good.cached, good.cu_rows, good.text_table[:, :3].contiguous(), good.summ_table)
        assert status(short, attn) == status(short, append) == status(short, gather) == ksa.KSA_PAGED_STATUS_BAD_PAGE
        same = lambda x, y: torch.equal(x.view(torch.int16), y.view(torch.int16))
        for cached, cu in (([60, -1], [0, n, 2 * n]), ([60, 60], [0, n, 2 * n + 1]), ([60, 2**30], [0, n, 2 * n]), ([60, 60], [-1, n, 2 * n]), ([60, 60], [0, 2 * n, n])):
            b = ksa.PagedBatch(_i32(cached), _i32(cu), good.text_table, good.summ_table)
            assert status(b, attn) == status(b, append) == status(b, gather) == ksa.KSA_PAGED_STATUS_BAD_ROWS
            if cu[1] == n:                                     # (the last pair gives the first sequence 2 n rows of its own)
                unwritten = same(s.cache.kpages, pools[0]) and same(s.cache.vpages, pools[1])
                assert unwritten, (cached, cu)
        out, lse = s.attn(spans)
        s.check(out, lse, spans, sample=20)


# ---- the operators together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_prompt_in_pieces_then_tokens_then_drafts(ctx, fmt):
    """A prompt in uneven pieces beside another sequence that decodes, drafts of which some are thrown away and written again."""
    s = Server(ctx, 8, 1, 6, 8, 2, 128, 16, fmt, [700, 400], seed=21)
    steps = [[(0, 300), (0, 1)], [(300, 211), (1, 1)], [(511, 0), (2, 90)], [(511, 1), (92, 1)], [(512, 1), (93, 5)], [(513, 6), (95, 4)], [(516, 160), (99, 301)]]
    for spans in steps:
        s.append(spans, pad=2)
        out, lse = s.attn(spans, pad=2)
        s.check(out, lse, spans, sample=20)


def test_pieces_equal_the_forward_pass_and_go_on_in_the_contiguous_cache(ctx):
    """One sequence: pieces over the paged cache against ksa_attn_fwd of the whole; read back, it fills the Summary KV cache, whose
    next step equals the paged one.  Two computations of the same numbers: each within its own bounds of the reference."""
    k, m, C, Hq, Hkv, D, n_text = 8, 1, 10, 8, 2, 128, 500
    L = ksa.aug_len(n_text, k, m)
    s = Server(ctx, k, m, C, Hq, Hkv, D, 32, "bf16", [L + 1], seed=13)
    outs, lses = [], []
    for a, n in ((0, 100), (100, 17), (117, L - 117)):
        s.append([(a, n)])
        out, lse = s.attn([(a, n)])
        outs.append(out); lses.append(lse)
    out, lse = torch.cat(outs), torch.cat(lses, 1)
    prob = ksa.Problem([n_text], k, m, C, Hq, Hkv, D, s.scale)
    fwd, fwd_lse = ksa.attn_fwd(ctx, prob, s.q[0][:L].to(DEV), s.key[0][:L].to(DEV), s.val[0][:L].to(DEV))
    s.check(out, lse, [(0, L)], sample=40)
    s.check(fwd, fwd_lse, [(0, L)], sample=40)
    kk, vv = (torch.empty((L, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s.cache.gather(s.batch([(0, L)]), kk, vv)
    spec = ksa.CacheSpec(1, k, C, n_text // k + 8, Hq, Hkv, D, s.scale)
    dec = ksa.DecodeCache(ctx, spec)
    dec.fill_from_prefill(prob, kk, vv)
    step_out, step_lse = torch.empty((1, Hq, D), dtype=torch.bfloat16, device=DEV), torch.empty((1, Hq), device=DEV)
    dec.decode_text(s.q[0][L:].to(DEV), s.key[0][L:].to(DEV), s.val[0][L:].to(DEV), step_out, step_lse)
    s.append([(L, 1)])
    out, lse = s.attn([(L, 1)])
    s.check(out, lse, [(L, 1)])
    s.check(step_out, step_lse.t().contiguous(), [(L, 1)])


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (16, 1, 64), (16, 2, 64), (20, 1, 128)])
def test_tokens_and_prompts_in_one_call(ctx, kernel, fmt, Hq, Hkv, D):
    """Sequences of one row to hundreds in a call, more than 32 of them, in and out of order: every row by the kernel it falls to.  Many
    calls after another, each appending what the next attends to."""
    lens = [700, 40, 300, 33, 1, 9, 150] + [20 + 7 * i for i in range(30)]
    s = Server(ctx, 8, 1, 4, Hq, Hkv, D, 16, fmt, lens, seed=23, flags=kernel)
    at = [n // 2 for n in lens]
    s.append([(0, n) for n in at])
    for step in range(3):
        spans = [(a, min(lens[b] - a, [1, 130, 3, 0, 60, 2, 17][(b + step) % 7] if b < 7 else 1)) for b, a in enumerate(at)]
        s.append(spans, pad=step)
        out, lse = s.attn(spans, pad=step)
        s.check(out, lse, spans, sample=6)
        at = [a + n for a, n in spans]


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 40])
def test_captured_calls_follow_lengths_and_tables(ctx, kernel, fmt, n):
    """append + attn in a graph, replayed with other lengths, tables and rows; two graphs of the same cache; on a side stream."""
    s = Server(ctx, 8, 1, 5, 8, 2, 128, 16, fmt, [600, 600], seed=31, flags=kernel)
    rows = 2 * n
    batch = s.batch([(0, n), (0, n)])
    q = torch.zeros((rows, 8, 128), dtype=torch.bfloat16, device=DEV)
    kk, vv = (torch.zeros((rows, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    outs = [torch.full((rows, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    lses = [torch.full((8, rows), -1.0, device=DEV) for _ in range(2)]
    side = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.cache.append(batch, kk, vv); s.cache.attn(batch, q, outs[0], lses[0])      # once before capture
        torch.cuda.synchronize()
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                s.cache.append(batch, kk, vv)
                s.cache.attn(batch, q, outs[i], lses[i])
            graphs.append(g)
    torch.cuda.synchronize()
    s.poison()
    for step, spans in enumerate([[(0, n), (250, n)], [(n, n), (250 + n, n - 1)], [(2 * n, 0), (249 + 2 * n, n)]]):
        full = [(0, a) for a, _ in spans]
        if step == 0:
            s.append(full)
        if step == 2:                                       # a sequence moves to other pages
            s.text[1] = s.text[1][::-1].copy()
            s.append([(0, 0), full[1]])
        nb = s.batch(spans)
        batch.cached.copy_(nb.cached); batch.cu_rows.copy_(nb.cu_rows); batch.text_table.copy_(nb.text_table)
        have = sum(c for _, c in spans)
        q[:have], kk[:have], vv[:have] = s.rows(s.q, spans), s.rows(s.key, spans), s.rows(s.val, spans)
        for i, g in enumerate(graphs):
            outs[i].fill_(7.0); lses[i].fill_(-1.0)
            g.replay()
            torch.cuda.synchronize()
            s.check(outs[i], lses[i], spans, sample=12)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_many_calls_in_a_row_in_a_graph(ctx, kernel, fmt):
    """Eight steps of append and attn, one after another without a pause, kernels beside one another: as each step alone, twice."""
    lens = [500, 60, 340, 90, 340, 700]
    s = Server(ctx, 8, 1, 5, 16, 2, 128, 16, fmt, lens, seed=41, flags=kernel)
    start = [n // 2 for n in lens]
    steps = [[(start[b] + (i if b % 2 else 20 * i), 1 if b % 2 else 20) for b in range(len(lens))] for i in range(8)]
    s.append([(0, n) for n in start])
    pools = [t.clone() for t in (s.cache.kpages, s.cache.vpages)] + [t.clone() for t in (s.cache.kscale, s.cache.vscale) if t is not None]
    calls, want = [], []
    for spans in steps:
        b, q, k, v = s.batch(spans), s.rows(s.q, spans), s.rows(s.key, spans), s.rows(s.val, spans)
        out, lse = torch.empty_like(q), torch.empty((16, q.shape[0]), device=DEV)
        s.cache.append(b, k, v)
        torch.cuda.synchronize()
        s.cache.attn(b, q, out, lse)
        torch.cuda.synchronize()
        s.check(out, lse, spans, sample=3)
        want.append((out.clone(), lse.clone()))
        calls.append((b, q, k, v, out, lse))
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        for b, q, k, v, out, lse in calls:
            s.cache.append(b, k, v)
            s.cache.attn(b, q, out, lse)
    for _ in range(3):
        for t, p in zip([s.cache.kpages, s.cache.vpages, s.cache.kscale, s.cache.vscale], pools):
            t.copy_(p)
        for c in calls:
            c[4].fill_(7.0); c[5].fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        for c, (out, lse) in zip(calls, want):
            assert torch.equal(c[4], out) and torch.equal(c[5], lse)
    assert ctx.device_status() == 0


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
def test_two_streams_and_repeated_calls_agree(ctx, kernel):
    """The same calls on two streams at once, and again: bit for bit the same (sums are in a fixed order)."""
    for n in (1, 5, 200):
        s = Server(ctx, 8, 1, 20, 32, 4, 128, 64, "e4m3", [900, 700, 300], seed=17, flags=kernel)
        spans = [(700, n), (500, n), (100, n)]
        s.fill(spans)
        want = s.attn(spans)
        batch, q = s.batch(spans), s.rows(s.q, spans)
        got = []
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(4):
            for st in streams:
                out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
                torch.cuda.synchronize() if not got else None
                s.cache.attn(batch, q, out, lse, stream=st.cuda_stream)
                got.append((out, lse))
        torch.cuda.synchronize()
        for out, lse in got:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_nothing_to_do(ctx):
    s = Server(ctx, 8, 1, 4, 4, 2, 64, 16, "bf16", [50])
    before = ctx.launch_count()
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    s.cache.append(s.batch([(10, 0)]), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV))
    assert torch.isnan(s.cache.kpages).all() and ctx.launch_count() == before + 1
    s.attn([(10, 0)], pad=4)
    before = ctx.launch_count()
    s.cache.append(s.batch([(10, 0)]), empty, empty)
    s.cache.gather(s.batch([(10, 0)]), empty, empty)
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    s.cache.attn(s.batch([(10, 0)]), none, none, torch.empty((4, 0), device=DEV))
    assert ctx.launch_count() == before


def test_refusals_of_tensors(ctx):
    s = Server(ctx, 8, 1, 4, 4, 2, 64, 16, "bf16", [50])
    b = s.batch([(0, 3)])
    x = lambda *shape, **kw: torch.zeros(shape, **{**dict(dtype=torch.bfloat16, device=DEV), **kw})
    for k, v in ((x(3, 2, 128), x(3, 2, 64)), (x(3, 1, 64), x(3, 2, 64)), (x(3, 2, 64), x(4, 2, 64)), (x(3, 2, 64, dtype=torch.float16), x(3, 2, 64)),
                 (x(3, 2, 64, device="cpu"), x(3, 2, 64)), (x(3, 64, 2).transpose(1, 2), x(3, 2, 64))):
        with pytest.raises(ValueError):
            s.cache.append(b, k, v)
    for lse in (x(3, 4, dtype=torch.float32), x(4, 3), x(4, 4, dtype=torch.float32), x(3, 4, dtype=torch.float32).t()):
        with pytest.raises(ValueError):
            s.cache.attn(b, x(3, 4, 64), x(3, 4, 64), lse)
    with pytest.raises(ksa.KsaError):                          # not 16-byte aligned
        s.cache.attn(b, x(3 * 4 * 64 + 4)[4:].view(3, 4, 64), x(3, 4, 64), x(4, 3, dtype=torch.float32))
    cpu = ksa.PagedBatch(*(t.cpu() for t in (b.cached, b.cu_rows, b.text_table, b.summ_table)))
    with pytest.raises(ValueError):
        s.cache.append(cpu, x(3, 2, 64), x(3, 2, 64))


def test_written_rows_have_places_of_their_own(ctx):
    """Read tensors may repeat rows or heads (strides of 0); written ones may not."""
    s = Server(ctx, 8, 1, 3, 4, 2, 64, 16, "bf16", [20])
    s.key[0], s.val[0] = s.key[0][:1, :1].expand(20, 2, 64), s.val[0][:, :1].expand(20, 2, 64)
    spans = [(0, 20)]
    dev = lambda t: t.to(DEV)
    s.cache.append(s.batch(spans), dev(s.key[0][:1, :1].contiguous()).expand(20, 2, 64), dev(s.val[0][:, :1].contiguous()).expand(20, 2, 64))
    s.q[0] = s.q[0][:1].expand(20, 4, 64)
    q = dev(s.q[0][:1].contiguous()).expand(20, 4, 64)
    out, lse = torch.empty((20, 4, 64), dtype=torch.bfloat16, device=DEV), torch.empty((4, 20), device=DEV)
    s.cache.attn(s.batch(spans), q, out, lse)
    s.check(out, lse, spans)
    rows = torch.empty((20, 2, 64), dtype=torch.bfloat16, device=DEV)
    q = torch.zeros((20, 4, 64), dtype=torch.bfloat16, device=DEV)
    for bad in (rows[:1].expand(20, 2, 64), rows[:, :1].expand(20, 2, 64)):
        with pytest.raises(ksa.KsaError):
            s.cache.gather(s.batch(spans), bad, rows)
        with pytest.raises(ksa.KsaError):
            s.cache.gather(s.batch(spans), rows, bad)
    for bad in (q[:1].expand(20, 4, 64), q[:, :1].expand(20, 4, 64)):
        with pytest.raises(ksa.KsaError):
            s.cache.attn(s.batch(spans), q, bad, torch.empty((4, 20), device=DEV))


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
@pytest.mark.parametrize("fmt,n", [("bf16", 1), ("bf16", 90), ("e4m3", 1), ("e4m3", 90), ("e4m3", 700)])
def test_pools_past_32_bits(ctx, kernel, fmt, n):
    """Pages 2^28 elements apart, the last of them past 2^32 elements."""
    D, ps, far = 64, 128, 1 << 28
    base = []

    def pools(pages):
        base.append(torch.empty((pages - 1) * far + 4 * ps * D, dtype=torch.bfloat16 if fmt == "bf16" else torch.float8_e4m3fn, device=DEV))
        return tuple(torch.as_strided(base[0], (pages, 2, ps, D), (far, ps * D, D, 1), off) for off in (0, 2 * ps * D))

    s = Server(ctx, 8, 1, 4, 8, 2, D, ps, fmt, [1000, 900], seed=n, pools=pools, flags=kernel)
    assert s.cache.spec.num_pages > 16
    spans = [(1000 - n, n), (900 - n // 3, n // 3)]
    s.fill(spans)
    out, lse = s.attn(spans)
    s.check(out, lse, spans, sample=20)
    got = [torch.empty((1000, 2, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    s.cache.gather(s.batch([(0, 1000), (0, 0)]), *got)
    for g, rows in zip(got, (s.key, s.val)):
        assert (g.double().cpu().numpy() == s.cached_values(rows[0])).all()


@pytest.mark.parametrize("kernel", [BY_RULE, MANY])
def test_two_captured_calls_with_workspaces_run_at_once(ctx, kernel):
    """Long runs over e4m3 pages (which the calls copy to workspaces of their own), captured twice and replayed on two streams."""
    k, n = 8, 700
    s = Server(ctx, k, 1, 12, 16, 2, 128, 32, "e4m3", [1500, 1200], seed=3, flags=kernel)
    calls = []
    for spans in ([(800, n), (500, n)], [(400, n), (450, n)]):
        s.fill(spans)
        want = s.attn(spans)
        s.check(*want, spans, sample=8)
        calls.append((s.batch(spans), s.rows(s.q, spans), torch.zeros_like(want[0]), torch.zeros_like(want[1]), want))
    s.append([(0, 1500), (0, 1200)])
    streams, graphs = [torch.cuda.Stream() for _ in calls], []
    for st, (b, q, out, lse, _) in zip(streams, calls):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.cache.attn(b, q, out, lse)
        graphs.append(g)
    for _ in range(5):
        for c in calls:
            c[2].fill_(7.0); c[3].fill_(7.0)
        torch.cuda.synchronize()
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay(); g.replay()
        torch.cuda.synchronize()
        for _, _, out, lse, want in calls:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert ctx.device_status() == 0
