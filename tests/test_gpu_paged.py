"""New tokens into a paged cache and attention over it on the GPU, against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2401_15207_amd as H
from tests.test_gpu_rotary import DT, HALF_STEP, close, table, turned

pytestmark = pytest.mark.gpu


class Made:
    """A batch over a cache: pages in random order, slots without a token and pages of nobody full of NaN."""

    def __init__(self, tokens, heads, kv, hd, page, dtype, seed=0, spare=2, more_rows=0, more_pages=0, apart=0):
        g = torch.Generator().manual_seed(seed)
        self.tokens, self.heads, self.kv, self.hd, self.page, self.dtype = tokens, heads, kv, hd, page, DT[dtype]
        need = [-(-(c + n) // page) for c, n in tokens]
        pool, most = sum(need) + spare, max(need + [1]) + more_pages
        order = torch.randperm(pool, generator=g)
        self.pages = torch.full((len(tokens), most), -1, dtype=torch.int32)
        full = torch.full((pool, 2 * kv * page * hd + apart), math.nan).to(self.dtype)
        k, v = (full[:, i * kv * page * hd:(i + 1) * kv * page * hd].view(pool, kv, page, hd) for i in range(2))
        used, self.keys, self.values = 0, [], []
        for s, (c, n) in enumerate(tokens):
            mine = order[used:used + need[s]]
            used += need[s]
            self.pages[s, :need[s]] = mine.to(torch.int32)
            ks, vs = (torch.randn(c + n, kv, hd, generator=g).to(self.dtype) for _ in range(2))
            self.keys.append(ks)
            self.values.append(vs)
            for t in range(c + n):
                k[mine[t // page], :, t % page], v[mine[t // page], :, t % page] = ks[t], vs[t]
        full = full.cuda()
        self.k, self.v = (full[:, i * kv * page * hd:(i + 1) * kv * page * hd].view(pool, kv, page, hd) for i in range(2))
        self.pages = self.pages.cuda()
        self.lengths = torch.tensor([c for c, _ in tokens], dtype=torch.int32, device="cuda")
        self.starts = torch.tensor([0] + [n for _, n in tokens], device="cuda").cumsum(0).to(torch.int32)
        self.rows = sum(n for _, n in tokens) + more_rows
        self.max_new, self.max_length = max(n for _, n in tokens), max(c + n for c, n in tokens)
        self.cache = H.PagedCache(self.k, self.v, self.pages, self.lengths)
        self.q = (torch.randn(self.rows, heads * hd, generator=g) * 1.5).to("cuda", self.dtype)

    def attend(self, window=0, scale=None, gone=(), max_new=None, max_length=None, lse=True, **more):
        out = torch.full((self.rows, self.heads * self.hd), -7.0, device="cuda", dtype=self.dtype)
        z = torch.full((self.rows, self.heads), -7.0, device="cuda") if lse else None
        H.kernel_attention_paged(self.cache, self.starts, self.q, self.heads, out, max_new or self.max_new, max_length or self.max_length, window=window, scale=scale,
                                 lse=z, **more)
        return out, z

    def check(self, out, lse, window=0, scale=None, gone=()):
        """gone: (sequence, page index) pairs that are not there."""
        heads, kv, hd, row = self.heads, self.kv, self.hd, 0
        scale = scale or hd ** -0.5
        half = HALF_STEP[self.dtype]
        for s, (c, n) in enumerate(self.tokens):
            if n == 0:
                continue
            q = self.q[row:row + n].double().view(n, kv, heads // kv, hd)
            k, v = self.keys[s].cuda().double(), self.values[s].cuda().double()
            score = torch.einsum("nkgd,tkd->nkgt", q, k) * scale
            size = torch.einsum("nkgd,tkd->nkgt", q.abs(), k.abs()).amax(-1, keepdim=True) * scale
            at, key = torch.arange(c, c + n, device="cuda")[:, None], torch.arange(c + n, device="cuda")[None, :]
            seen = (key <= at) & ((key > at - window) if window else True)
            for s2, index in gone:
                if s2 == s:
                    seen &= key // self.page != index
            score = score.masked_fill(~seen[:, None, None, :], -math.inf)
            z = torch.logsumexp(score, -1)
            p = torch.exp(score - torch.where(torch.isinf(z), 0.0, z)[..., None])
            want, body = torch.einsum("nkgt,tkd->nkgd", p, v).reshape(n, -1), torch.einsum("nkgt,tkd->nkgd", p, v.abs()).reshape(n, -1)
            # a score is off by head_dim + 2 roundings of 2^-24 of its products, an exponential by that and 2^-22 (scaling, exp2 and the running maximum), in sums
            # above and below; sums of at most as many terms as keys; bf16: each exponential rounded for the product with v; then the result
            off = (hd + 2) * 2.0 ** -24 * size.repeat(1, 1, 1, hd).reshape(n, -1)
            tol = body * (2 * off + 2.0 ** -21 + 2 * (c + n) * 2.0 ** -24 + (half if self.dtype is torch.bfloat16 else 0)) * 1.02 + half * want.abs() + 1e-37
            far = (out[row:row + n].double() - want).abs()
            assert (far <= tol).all(), f"sequence {s}: off by up to {(far / tol).max().item():.2f} of the tolerance"
            if lse is not None:
                none = torch.isinf(z).reshape(n, -1)
                got, z = lse[row:row + n].double(), z.reshape(n, -1) / math.log(2)
                assert (got[none] == -math.inf).all() and (out[row:row + n].view(n, heads, hd)[none] == 0).all()
                tol = ((off.view(n, heads, hd)[..., 0] + (c + n) * 2.0 ** -24 + 2.0 ** -21) * 1.4427 + 2.0 ** -22 * z.abs().clamp(min=1.0))[~none]
                assert ((got - z).abs()[~none] <= tol).all()
            row += n
        assert (out[row:] == -7.0).all() and (lse is None or (lse[row:] == -7.0).all())


FEW = [  # (cached, new) of each sequence, heads, kv_heads, head_dim, page
    ([(0, 1)], 1, 1, 64, 16), ([(500, 1)], 4, 4, 128, 16), ([(31, 1), (32, 1), (33, 1), (0, 1), (1023, 1)], 8, 2, 128, 16), ([(700, 3)], 8, 2, 64, 32),
    ([(15, 1), (16, 1), (47, 1)], 4, 1, 16, 16), ([(200, 4), (5, 1), (0, 4)], 16, 2, 80, 64), ([(2000, 1)], 32, 1, 128, 128), ([(100, 1)], 6, 2, 96, 16),
    ([(130, 0), (3000, 2), (64, 1)], 4, 2, 32, 64)]
MANY = [([(0, 128)], 2, 2, 128, 16), ([(0, 33)], 1, 1, 64, 16), ([(77, 200)], 4, 2, 128, 32), ([(300, 129), (0, 1), (40, 70), (9, 0), (0, 257)], 4, 2, 64, 16),
        ([(1, 64)], 8, 1, 80, 64), ([(1000, 300)], 2, 1, 128, 128), ([(5, 40), (6, 40)], 3, 1, 16, 16)]


# enough blocks of 32 rows for the kernel of many rows (over 128 of them in bf16, over 512 in fp32), keys split over workgroups or not, short sequences among long ones
MIXED = [([(0, 200), (30, 1), (700, 130), (5, 0)], 16, 16, 64, 16), ([(2000, 150), (3, 140)], 16, 16, 128, 32), ([(1500, 300)], 64, 16, 96, 64),
         ([(900, 300), (5, 2)], 64, 32, 32, 64), ([(10, 40)] * 9 + [(2100, 1)], 64, 32, 16, 16), ([(0, 257)] * 3, 24, 8, 80, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", FEW + MANY + MIXED)
@pytest.mark.parametrize("window", [0, 1, 50])
def test_attention(dtype, case, window):
    m = Made(*case, dtype, seed=len(case[0]) + case[3], more_rows=2)
    out, lse = m.attend(window=window)
    m.check(out, lse, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_caches_in_many_parts(dtype):
    m = Made([(9000, 1), (40, 1), (4097, 2)], 4, 2, 128, 16, dtype)
    out, lse = m.attend()
    m.check(out, lse)
    again, lse2 = m.attend()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # fewer parts, as for a shorter bound; more of them; the bound is no limit
    for bound in (100, 2 ** 30):
        out, lse = m.attend(max_length=bound)
        m.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_chunk_over_a_long_cache_in_parts(dtype):
    m = Made([(5000, 40)], 2, 2, 128, 64, dtype)
    out, lse = m.attend()
    m.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_that_are_too_low_or_too_high(dtype):
    """max_length sets how the work is cut up and nothing else: eight wavefronts or four, runs, parts."""
    for tokens, heads, kv in [([(3000, 1)], 8, 8), ([(3000, 150), (0, 33)], 32, 32)]:
        m = Made(tokens, heads, kv, 64, 16, dtype)
        for bound in (0, 300, 900, 1200, 4000, 2 ** 40):
            out, lse = m.attend(max_length=bound)
            m.check(out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,heads", [([(100, 1), (60, 2)], 4), ([(100, 60), (20, 1)], 4), ([(100, 60), (1000, 60)], 256)])
def test_pages_that_are_not_there(dtype, tokens, heads):
    m = Made(tokens, heads, max(2, heads // 2), 64, 16, dtype)
    gone = [(0, 0), (0, 3), (1, 1)]
    m.pages[0, 0], m.pages[0, 3], m.pages[1, 1] = -1, m.k.shape[0], 2 ** 31 - 1
    out, lse = m.attend()
    m.check(out, lse, gone=gone)
    # nothing left at all: zeros, and -inf
    m.pages.fill_(-5)
    out, lse = m.attend()
    m.check(out, lse, gone=[(s, i) for s in range(2) for i in range(80)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_window_over_returned_pages(dtype):
    """Pages before the window may have been given back."""
    m = Made([(500, 1), (300, 50)], 4, 2, 128, 16, dtype)
    m.pages[0, :(501 - 64) // 16] = -1
    m.pages[1, :(301 - 64) // 16] = -1
    out, lse = m.attend(window=64)
    m.check(out, lse, window=64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 40])
def test_strides_in_place_and_scale(dtype, new):
    """q inside rows of a fused projection, the result in its place, pages of one layer inside pages of all, another scale."""
    m = Made([(90, new), (33, 1)], 4, 2, 64, 32, dtype, apart=64)
    want, _ = m.attend(scale=0.3)
    m.check(want, None, scale=0.3)
    wide = torch.full((m.rows, 512), -7.0, device="cuda", dtype=m.dtype)
    wide[:, :256] = m.q
    H.kernel_attention_paged(m.cache, m.starts, wide[:, :256], 4, wide[:, :256], m.max_new, m.max_length, scale=0.3)
    assert torch.equal(wide[:, :256], want) and (wide[:, 256:] == -7.0).all()


def test_large_scores_and_equal_keys():
    """Scores far above 2^8 and below: the reference moves; equal keys share the weight evenly."""
    m = Made([(200, 1)], 2, 2, 64, 16, "fp32")
    m.q.mul_(40.0)
    out, lse = m.attend()
    m.check(out, lse)
    for s in range(1):
        m.keys[s][:] = m.keys[s][:1]
    for t in range(201):
        m.k[m.pages[0, t // 16].item(), :, t % 16] = m.keys[0][t].cuda()
    out, lse = m.attend()
    m.check(out, lse)


def test_rows_limits_and_lengths_out_of_range():
    """max_new leaves the rest out; lengths beyond the pages and below zero are kept in range; starts outside the rows too."""
    m = Made([(20, 5), (10, 3)], 2, 2, 64, 16, "fp32")
    whole, _ = m.attend()
    out, _ = m.attend(max_new=2)
    keep = torch.zeros(8, dtype=torch.bool, device="cuda")
    keep[[0, 1, 5, 6]] = True
    assert (out[~keep] == -7.0).all()
    assert (out[keep].double() - whole[keep].double()).abs().max().item() <= 1e-5
    m.lengths[0], m.lengths[1] = 2 ** 31 - 1, -4
    m.k.nan_to_num_(0.0), m.v.nan_to_num_(0.0)
    out, _ = m.attend()     # sequence 0: at the end of its pages; sequence 1: as if empty
    assert not out.isnan().any()
    m.lengths[1] = 0
    assert torch.equal(m.attend()[0][5:], out[5:])
    m.starts[2] = 2 ** 31 - 1
    assert not m.attend()[0].isnan().any()
    m.starts.copy_(torch.tensor([-3, 5, 2], dtype=torch.int32))
    out, _ = m.attend()
    assert (out[5:] == -7.0).all()


def test_no_rows_and_no_sequences():
    m = Made([(20, 1)], 2, 2, 64, 16, "bf16")
    none = torch.empty(0, 128, device="cuda", dtype=torch.bfloat16)
    H.kernel_attention_paged(m.cache, m.starts, none, 2, none, 1, 21)
    H.kernel_cache_append(m.cache, m.starts, torch.empty(0, 384, device="cuda", dtype=torch.bfloat16), 2)


def test_another_stream_and_a_workspace_of_ones_own():
    m = Made([(3000, 1), (100, 1)], 8, 2, 128, 16, "bf16")
    want, _ = m.attend()
    n = H.kernel_attention_paged_bytes(m.cache, m.rows, 8, m.max_new, m.max_length)
    assert n > 0
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(m.attend(workspace=ws)[0], want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    H.kernel_attention_paged(m.cache, m.starts, m.q, 8, out, m.max_new, m.max_length, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("case", [([(0, 1)], 1, 1, 16, 16, 16), ([(15, 1), (16, 1), (100, 1)], 8, 2, 128, 16, 64), ([(30, 40), (0, 3), (7, 0), (64, 65)], 4, 4, 80, 32, 20),
                                  ([(3, 200)], 6, 3, 64, 128, 64), ([(5, 9)], 2, 1, 48, 16, 0)])
def test_append(dtype, layout, case):
    *shape, rot = case
    m = Made(*shape, dtype, more_rows=2)
    heads, kv, hd, rows = m.heads, m.kv, m.hd, m.rows
    qkv = torch.randn(rows, (heads + 2 * kv) * hd + 8, generator=torch.Generator().manual_seed(1)).to("cuda", m.dtype)
    cs = table(m.max_length, rot) if rot else None
    q = torch.full((rows, heads * hd), -7.0, device="cuda", dtype=m.dtype)
    k0, v0 = m.k.clone(), m.v.clone()
    H.kernel_cache_append(m.cache, m.starts, qkv, heads, q, cs, layout=layout, max_new=m.max_new)
    written, row = torch.zeros(m.k.shape[0], m.page, dtype=torch.bool, device="cuda"), 0
    for s, (c, n) in enumerate(m.tokens):
        x = qkv[row:row + n, :(heads + 2 * kv) * hd].reshape(n, heads + 2 * kv, hd)
        want, size = turned(x[:, :heads + kv], cs[c:c + n], layout) if rot else (x[:, :heads + kv].double(), x[:, :heads + kv].double().abs())
        close(q[row:row + n].view(n, heads, hd), want[:, :heads], size[:, :heads], m.dtype)
        at = torch.arange(c, c + n, device="cuda")
        pg = m.pages[s, at // m.page].long()
        close(m.k[pg, :, at % m.page], want[:, heads:], size[:, heads:], m.dtype)
        assert torch.equal(m.v[pg, :, at % m.page], x[:, heads + kv:])
        written[pg, at % m.page] = True
        row += n
    assert (q[row:] == -7.0).all()
    other = ~written[:, None, :, None].expand_as(m.k)
    assert torch.equal(m.k.nan_to_num(9.0)[other], k0.nan_to_num(9.0)[other]) and torch.equal(m.v.nan_to_num(9.0)[other], v0.nan_to_num(9.0)[other])
    # q in its place, and keys and values alone
    again = qkv.clone()
    m.k.copy_(k0), m.v.copy_(v0)
    H.kernel_cache_append(m.cache, m.starts, again, heads, again, cs, layout=layout)
    assert torch.equal(again[:row, :heads * hd], q[:row]) and torch.equal(again[:, heads * hd:], qkv[:, heads * hd:]) and torch.equal(again[row:], qkv[row:])
    k1 = m.k.clone()
    m.k.copy_(k0), m.v.copy_(v0)
    H.kernel_cache_append(m.cache, m.starts, qkv, heads, None, cs, layout=layout, max_new=m.max_new)
    assert torch.equal(m.k.nan_to_num(9.0), k1.nan_to_num(9.0))


def test_append_drops_what_has_no_page():
    m = Made([(14, 4), (0, 40)], 2, 1, 64, 16, "bf16")
    m.pages[0, 1], m.pages[1, 1] = -1, m.k.shape[0]
    small = H.PagedCache(m.k, m.v, m.pages[:, :2], m.lengths)     # two pages: tokens from 32 on have none
    k0 = m.k.clone()
    qkv = torch.randn(44, 256, device="cuda").bfloat16()
    q, want = torch.empty(44, 128, device="cuda", dtype=torch.bfloat16), torch.empty(44, 128, device="cuda", dtype=torch.bfloat16)
    cs = table(64, 64)
    H.kernel_cache_append(small, m.starts, qkv, 2, q, cs, max_new=40)
    at = torch.cat([torch.arange(14, 18), torch.arange(40)]).to(torch.int32).cuda()
    H.kernel_rotary(qkv[:, :128], 2, 64, want, cs, positions=at)
    assert torch.equal(q, want)
    changed = (m.k.nan_to_num(9.0) != k0.nan_to_num(9.0)).any(3).any(1)
    assert changed.sum().item() == 2 + 16
    assert changed[m.pages[0, 0].item(), 14:].all() and changed[m.pages[1, 0].item()].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_model_answers(dtype):
    """All of it as it is used: a prompt in chunks, then token by token, two sequences; each step's attention equals attention over everything so far."""
    heads, kv, hd, page = 4, 2, 64, 16
    g = torch.Generator().manual_seed(4)
    k, v = (torch.full((16, kv, page, hd), math.nan, device="cuda", dtype=DT[dtype]) for _ in range(2))
    pages = torch.randperm(16, generator=g).to(torch.int32).view(2, 8).cuda()
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache = H.PagedCache(k, v, pages, lengths)
    cs = torch.empty(128, 16, 2, device="cuda")
    H.kernel_rotary_table(dict(rot=32, scaling="linear", factor=2.0), cs)
    so_far = [torch.zeros(0, (heads + 2 * kv), hd, dtype=torch.float64, device="cuda") for _ in range(2)]
    for news in [(40, 7), (20, 30), (1, 1), (1, 1), (1, 0), (1, 1)]:
        rows = sum(news)
        qkv = torch.randn(rows, (heads + 2 * kv) * hd, generator=g).to("cuda", DT[dtype])
        starts = torch.tensor([0, news[0], rows], dtype=torch.int32, device="cuda")
        H.kernel_cache_append(cache, starts, qkv, heads, qkv, cs, layout="pairs", max_new=max(news))
        out = torch.empty(rows, heads * hd, device="cuda", dtype=DT[dtype])
        H.kernel_attention_paged(cache, starts, qkv, heads, out, max(news), 128)
        at = 0
        for s, n in enumerate(news):
            if n == 0:
                continue
            have = so_far[s].shape[0]
            x = qkv[at:at + n].view(n, heads + 2 * kv, hd).double()
            pg = pages[s, torch.arange(have, have + n, device="cuda") // page].long()
            slot = torch.arange(have, have + n, device="cuda") % page
            x[:, heads:heads + kv], x[:, heads + kv:] = k[pg, :, slot].double(), v[pg, :, slot].double()
            so_far[s] = torch.cat([so_far[s], x])
            a = so_far[s]
            score = torch.einsum("nhd,thd->nht", a[have:, :heads], a[:, heads:heads + kv].repeat_interleave(heads // kv, 1)) * hd ** -0.5
            score = score.masked_fill((torch.arange(have + n, device="cuda")[None, :] > torch.arange(have, have + n, device="cuda")[:, None])[:, None], -math.inf)
            p = torch.softmax(score, -1)
            vv = a[:, heads + kv:].repeat_interleave(heads // kv, 1)
            want, body = torch.einsum("nht,thd->nhd", p, vv).reshape(n, -1), torch.einsum("nht,thd->nhd", p, vv.abs()).reshape(n, -1)
            half = HALF_STEP[DT[dtype]]
            # scores off by 66 roundings of products whose sizes add up to at most 100
            tol = body * (2 * 66 * 2.0 ** -24 * 100 + 2.0 ** -20 + (half if dtype == "bf16" else 0)) + half * want.abs()
            assert ((out[at:at + n].double() - want).abs() <= tol).all()
            at += n
        lengths += torch.tensor(news, dtype=torch.int32, device="cuda")


def test_replayed_from_a_graph_while_answers_grow():
    """One captured step for a token each; lengths grow on the device between the replays, with the program's own work in between."""
    m = Made([(30, 1), (100, 1), (0, 1)], 4, 2, 128, 16, "bf16", more_pages=3, spare=16)
    free = sorted(set(range(m.k.shape[0])) - set(m.pages.flatten().tolist()))
    for s in range(3):
        for i in range(m.pages.shape[1]):
            if m.pages[s, i] < 0:
                m.pages[s, i] = free.pop() if free else -1
    m.k.nan_to_num_(0.0), m.v.nan_to_num_(0.0)
    qkv = torch.randn(3, 8 * 128, device="cuda").bfloat16()
    cs, one = table(256, 128), torch.ones(3, dtype=torch.int32, device="cuda")
    out = torch.zeros(3, 512, device="cuda", dtype=torch.bfloat16)
    q = torch.zeros_like(out)
    n = H.kernel_attention_paged_bytes(m.cache, 3, 4, 1, 5000)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")

    def step(out, q):
        H.kernel_cache_append(m.cache, m.starts, qkv, 4, q, cs, max_new=1)
        H.kernel_attention_paged(m.cache, m.starts, q, 4, out, 1, 5000, workspace=ws)

    step(out, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, q)
        m.lengths.add_(one)
    for k in range(5):
        qkv.copy_(torch.randn(3, 8 * 128, device="cuda").bfloat16())
        want, q2 = torch.empty_like(out), torch.empty_like(q)
        step(want, q2)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(q, q2)
    assert m.lengths.tolist() == [35, 105, 5]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_row_in_place_by_views_of_other_widths(dtype):
    """A single row has no distance to the next: its views of different widths are in place all the same, and its width need not be whole pieces."""
    m = Made([(40, 1)], 4, 2, 64, 16, dtype)
    qkv = torch.randn(1, 8 * 64 + 3, generator=torch.Generator().manual_seed(5)).to("cuda", m.dtype)
    cs, q, at = table(64, 64), torch.empty(1, 256, device="cuda", dtype=m.dtype), torch.tensor([40], device="cuda", dtype=torch.int32)
    H.kernel_cache_append(m.cache, m.starts, qkv, 4, q, cs)
    want, turned_q = torch.empty_like(q), qkv.clone()
    H.kernel_rotary(turned_q, 4, 64, turned_q[:, :256], cs, positions=at)
    assert torch.equal(turned_q[:, :256], q) and torch.equal(turned_q[:, 256:], qkv[:, 256:])
    H.kernel_cache_append(m.cache, m.starts, qkv, 4, qkv[:, :256], cs)
    assert torch.equal(qkv[:, :256], q)
    H.kernel_attention_paged(m.cache, m.starts, q, 4, want, 1, 41)
    H.kernel_attention_paged(m.cache, m.starts, qkv, 4, qkv[:, :256], 1, 41)
    assert torch.equal(qkv[:, :256], want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [1, 300])
def test_pages_beyond_32_bits(dtype, new):
    """Pages 2^30 + 64 elements apart: the last one's bytes, and with five its elements too, lie beyond 2^32."""
    heads, kv, hd, page, cached = 32, 16, 64, 512, 700
    pool = torch.empty(2, 4 * (2 ** 30 + 64) + kv * page * hd, device="cuda", dtype=DT[dtype])
    k, v = (x.as_strided((5, kv, page, hd), (2 ** 30 + 64, page * hd, hd, 1), x.storage_offset()) for x in pool)
    g = torch.Generator(device="cuda").manual_seed(6)
    for x in (k, v):
        for n in range(5):
            x[n].normal_(generator=g)
    order = torch.tensor([[4, 1, 3]], device="cuda", dtype=torch.int32)
    near = [torch.stack([x[n] for n in (4, 1, 3)]) for x in (k, v)]
    q = torch.randn(new, (heads + 2 * kv) * hd, device="cuda", generator=g).to(DT[dtype])
    starts, lengths = torch.tensor([0, new], device="cuda", dtype=torch.int32), torch.tensor([cached], device="cuda", dtype=torch.int32)
    outs = []
    for kk, vv, pages in ((k, v, order), (*near, torch.tensor([[0, 1, 2]], device="cuda", dtype=torch.int32))):
        cache, out = H.PagedCache(kk, vv, pages, lengths), torch.empty(new, heads * hd, device="cuda", dtype=DT[dtype])
        H.kernel_cache_append(cache, starts, q, heads)
        H.kernel_attention_paged(cache, starts, q[:, :heads * hd], heads, out, new, cached + new)
        outs.append(out)
    assert not outs[0].isnan().any() and torch.equal(outs[0], outs[1])
    for x, y in zip((k, v), near):
        assert all(torch.equal(x[n], y[i]) for i, n in enumerate((4, 1, 3)))


def test_two_calls_at_once():
    """Two streams with a cache each, keys of both split over workgroups: each has a workspace of its own, and the results are those of the calls alone."""
    made = [Made([(3000, 1), (100, 2)], 8, 2, 128, 16, "bf16", seed=8), Made([(2500, 150)], 16, 16, 64, 32, "bf16", seed=9)]
    want = [m.attend()[0] for m in made]
    streams, outs = [torch.cuda.Stream() for _ in made], [[torch.empty_like(w) for _ in range(8)] for w in want]
    torch.cuda.synchronize()
    for i in range(8):
        for m, st, out in zip(made, streams, outs):
            H.kernel_attention_paged(m.cache, m.starts, m.q, m.heads, out[i], m.max_new, m.max_length, stream=st)
    torch.cuda.synchronize()
    for w, out in zip(want, outs):
        assert all(torch.equal(o, w) for o in out)


# keys split over workgroups, with sequences of few rows and of none among the others; keys of one and of two blocks; rows on either side of the choice of kernel
RAGGED = [([(3000, 1), (100, 40), (2500, 0), (0, 3), (700, 17)], 4, 2, 64, 16), ([(2000, 9), (40, 1)], 4, 4, 128, 32), ([(1500, 33)], 2, 2, 80, 16), ([(900, 4), (1, 4)], 32, 8, 128, 16),
          ([(31, 1), (5, 1), (0, 1)], 4, 4, 96, 16), ([(60, 2), (33, 1)], 8, 2, 128, 32), ([(300, 65)], 1, 1, 128, 16), ([(400, 1), (150, 1)], 2, 2, 128, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", RAGGED)
@pytest.mark.parametrize("window", [0, 33, 700])
def test_sequences_of_few_rows_among_split_keys(dtype, case, window):
    m = Made(*case, dtype, seed=11, more_rows=1)
    out, lse = m.attend(window)
    m.check(out, lse, window)
    again, lse2 = m.attend(window)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens", [[(2100, 1), (700, 1), (0, 1)], [(520, 1)] * 3 + [(580, 1)], [(130 + 5 * i, 1) for i in range(17)]])
def test_caches_larger_than_the_l2(dtype, tokens):
    """Keys that go past the caches: in runs, and a workgroup a head with eight and with four wavefronts."""
    m = Made(tokens, 32, 32, 128, 16, dtype, seed=12)
    out, lse = m.attend()
    m.check(out, lse)
