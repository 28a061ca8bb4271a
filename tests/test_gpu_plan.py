"""A server step's bookkeeping on the GPU against lists, and whole steps (release, plan, 8-bit floating-point projection, norm and
rotation into the cache, attention) in one graph."""
import math
import random

import pytest
import torch

import more_ref as R
import serve_ref as S

pytestmark = pytest.mark.gpu

import paper_2609_34866_gb300 as J  # noqa: E402


@pytest.fixture(autouse=True)
def _status():
    J.jab_get_device_status()
    yield
    torch.cuda.synchronize()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class State:
    """Sequences with pages in no order, and a stack of free ones."""

    def __init__(self, lens, width, page, seed, spare=0):
        self.page = page
        rng = random.Random(seed)
        used = [-(-n // page) for n in lens]
        total = sum(used) + spare
        ids = list(range(total))
        rng.shuffle(ids)
        self.pages = [[-5] * width for _ in lens]
        for b, u in enumerate(used):
            for i in range(u):
                self.pages[b][i] = ids.pop()
        self.n_free = len(ids)
        self.free = ids + [-9] * (total - len(ids))
        self.lens, self.total = list(lens), max(total, 1)
        self.cache = J.KvCache(1, 64, 8, page, self.total)

    def device(self):
        return _i32(self.lens), _i32(self.pages), _i32(self.free), _i32([self.n_free])


@pytest.mark.parametrize("B,page,longest,most,spare,pad", [(1, 16, 1, 1, 3, 0), (1, 16, 100, 1000, 70, 1), (64, 64, 8000, 1, 40, 0), (33, 48, 300, 60, 60, 17),
                                                            (1000, 16, 500, 130, 9000, 300), (1025, 32, 64, 2, 900, 0), (8192, 16, 40, 1, 8000, 5),
                                                            (2, 4096, 9000, 30000, 20, 3), (300, 128, 0, 700, 2000, 100)])
@pytest.mark.parametrize("in_place", [False, True])
def test_release_and_plan(B, page, longest, most, spare, pad, in_place):
    rng = random.Random(B + page)
    lens = [rng.randint(0, longest) for _ in range(B)]
    ended = [int(rng.random() < 0.2) * rng.choice((1, -3, 2 ** 31 - 1)) for _ in range(B)]
    counts = [rng.choice((0, 1, most, rng.randint(0, most))) for _ in range(B)]
    width = -(-(longest + most) // page) + 1
    s = State(lens, width, page, B, spare)
    need = sum(-(-(l + c) // page) - -(-l // page) for l, c in zip(lens, counts))
    dl, dp, df, dn = s.device()
    nl, nn = (None, None) if in_place else (torch.empty_like(dl), torch.empty_like(dn))
    J.jab_kv_release(s.cache, dl, _i32(ended), dp, df, dn, new_lens=nl, new_free=nn)
    lens1, free1, n1 = R.release(s.lens, ended, s.pages, s.free, s.n_free, page, 0)
    l1, f1 = (dl, dn) if in_place else (nl, nn)
    assert l1.tolist() == lens1 and f1.tolist() == [n1] and df.tolist() == free1
    need = sum(-(-(l + c) // page) - -(-l // page) for l, c in zip(lens1, counts))
    assert need <= n1  # (what this test is made for)
    rows = sum(counts) + pad
    qs, sl, po = _i32([7] * (B + 1)), torch.full((rows,), 7, dtype=torch.int64, device="cuda"), _i32([7] * rows)
    nl, nn = (None, None) if in_place else (torch.empty_like(dl), torch.empty_like(dn))
    J.jab_kv_plan(s.cache, l1, _i32(counts), dp, df, f1, qs, sl, po, new_lens=nl, new_free=nn)
    want = R.plan(lens1, counts, s.pages, free1, n1, page, rows)
    got = (l1 if in_place else nl, dp, f1 if in_place else nn, qs, sl, po)
    for g, w in zip(got, (want[0], want[1], [want[2]], *want[3:])):
        assert g.tolist() == w
    assert df.tolist() == free1 and J.jab_get_device_status() == 0


def test_release_behind_a_shared_prefix():
    s = State([100, 64, 64, 40, 0], 8, 16, 3)
    for b in range(1, 5):  # the first four pages are everybody's
        s.pages[b][:4] = s.pages[0][:4]
    dl, dp, df, dn = s.device()
    ended = [1, 1, 0, 1, 1]
    J.jab_kv_release(s.cache, dl, _i32(ended), dp, df, dn, shared_len=64)
    lens, free, n = R.release(s.lens, ended, s.pages, s.free, s.n_free, 16, 64)
    assert lens == [64, 64, 64, 40, 0] and n == s.n_free + 3
    assert dl.tolist() == lens and df.tolist() == free and dn.tolist() == [n] and J.jab_get_device_status() == 0


@pytest.mark.parametrize("what", ["pages", "rows", "length", "count", "room", "overflow", "stack", "stack+"])
@pytest.mark.parametrize("big", [False, True])
def test_a_plan_that_cannot_be_carried_out_changes_nothing(what, big):
    B, width = (5000, 12) if big else (4, 12)
    lens, counts = [20] * B, [30] * B
    s = State(lens, width, 16, 1, spare=B * 2 - (1 if what == "pages" else 0))
    rows = 30 * B - (1 if what == "rows" else 0)
    if what == "length":
        s.lens[B - 2] = -1
    if what == "count":
        counts[B - 1] = -1
    if what == "room":
        counts[1] = 12 * 16 - 20 + 1
    if what == "overflow":
        counts[0] = 2 ** 31 - 1
    dl, dp, df, dn = s.device()
    if what == "stack":
        dn.fill_(-1)
    if what == "stack+":
        dn.fill_(len(s.free) + 1)
    n0 = dn.tolist()
    qs, sl, po = _i32([7] * (B + 1)), torch.full((rows,), 7, dtype=torch.int64, device="cuda"), _i32([7] * rows)
    J.jab_kv_plan(s.cache, dl, _i32(counts), dp, df, dn, qs, sl, po)
    assert J.jab_get_device_status() == 1
    assert dl.tolist() == s.lens and dp.tolist() == s.pages and df.tolist() == s.free and dn.tolist() == n0
    assert not qs.any() and bool((sl == -1).all()) and not po.any()


def test_a_release_that_cannot_be_carried_out_changes_nothing():
    for what in ("length", "room", "stack", "capacity"):
        s = State([20] * 40, 3, 16, 1, spare=5)
        if what == "length":
            s.lens[30] = -7
        if what == "room":
            s.lens[30] = 49
        dl, dp, df, dn = s.device()
        if what == "stack":
            dn.fill_(-1)
        if what == "capacity":
            df = df[:-1].clone()
        keep, n0 = df.tolist(), dn.tolist()
        J.jab_kv_release(s.cache, dl, _i32([1] * 40), dp, df, dn)
        assert J.jab_get_device_status() == 1
        assert dl.tolist() == s.lens and df.tolist() == keep and dn.tolist() == n0


def test_page_numbers_outside_the_cache():
    s = State([20, 20], 4, 16, 1, spare=2)
    s.pages[0][1] = s.total  # the page that sequence 0 goes on in
    s.free[s.n_free - 1] = -2  # the one that sequence 1 gets
    dl, dp, df, dn = s.device()
    qs, sl, po = _i32([0] * 3), torch.zeros(26, dtype=torch.int64, device="cuda"), _i32([0] * 26)
    J.jab_kv_plan(s.cache, dl, _i32([12, 14]), dp, df, dn, qs, sl, po)
    assert J.jab_get_device_status() == 1
    assert bool((sl[:12] == -1).all()) and bool((sl[12:24] >= 0).all()) and bool((sl[24:] == -1).all())
    assert po.tolist() == list(range(20, 32)) + list(range(20, 34)) and qs.tolist() == [0, 12, 26]


@pytest.mark.parametrize("number", ["-1", "one past the last", "least", "most"])
@pytest.mark.parametrize("B,each,page,which", [(1, 1, 16, 0), (3, 5, 16, 7), (40, 3, 64, 119), (300, 60, 16, 12345), (300, 60, 16, 17999)])
def test_a_release_of_page_numbers_outside_the_cache_changes_nothing(B, each, page, which, number):
    """One bad entry among the pages that would go back, the first and the last among them, with as many pages as stay in registers and
    with more; a bad entry that does not go back stays unseen."""
    s = State([each * page] * B, each + 2, page, 1, spare=5)
    bad = {"-1": -1, "one past the last": s.total, "least": -2 ** 31, "most": 2 ** 31 - 1}[number]
    good, s.pages[which // each][which % each] = s.pages[which // each][which % each], bad
    for in_place in (False, True):
        dl, dp, df, dn = s.device()
        keep, n0 = df.tolist(), dn.tolist()
        nl, nn = (None, None) if in_place else (torch.empty_like(dl), torch.empty_like(dn))
        J.jab_kv_release(s.cache, dl, _i32([1] * B), dp, df, dn, new_lens=nl, new_free=nn)
        assert J.jab_get_device_status() == 1
        assert (dl if in_place else nl).tolist() == s.lens and (dn if in_place else nn).tolist() == n0
        assert df.tolist() == keep and dp.tolist() == s.pages
    dl, dp, df, dn = s.device()
    ended = [int(b != which // each) for b in range(B)]
    J.jab_kv_release(s.cache, dl, _i32(ended), dp, df, dn)  # (that sequence goes on)
    lens, free, n = R.release(s.lens, ended, s.pages, s.free, s.n_free, page, 0)
    assert dl.tolist() == lens and df.tolist() == free and dn.tolist() == [n] and J.jab_get_device_status() == 0
    s.pages[which // each][which % each] = good
    s.pages[0][each] = bad  # (behind the sequence's pages)
    dl, dp, df, dn = s.device()
    J.jab_kv_release(s.cache, dl, _i32([1] * B), dp, df, dn)
    lens, free, n = R.release(s.lens, [1] * B, s.pages, s.free, s.n_free, page, 0)
    assert dl.tolist() == lens and df.tolist() == free and dn.tolist() == [n] and J.jab_get_device_status() == 0


def test_long_prompts_in_a_graph():
    """Release and plan in place with more rows than one launch writes, captured once and replayed with other counts, until the pages
    run out: that call changes nothing, and the one after a release goes on."""
    B, page, rows = 40, 16, 12000
    s = State([0] * B, 200, page, 2, spare=1500)
    dl, dp, df, dn = s.device()
    ended, counts = _i32([0] * B), _i32([0] * B)
    qs, sl, po = _i32([0] * (B + 1)), torch.empty(rows, dtype=torch.int64, device="cuda"), _i32([0] * rows)

    def step():
        J.jab_kv_release(s.cache, dl, ended, dp, df, dn)
        J.jab_kv_plan(s.cache, dl, counts, dp, df, dn, qs, sl, po)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens, pages, free, n = s.lens, s.pages, s.free, s.n_free
    rng = random.Random(3)
    refused = 0
    for t in range(6):
        e, c = [int(t == 4 and b % 2 == 0) for b in range(B)], [rng.randint(0, 300) for _ in range(B)]
        ended.copy_(_i32(e)), counts.copy_(_i32(c))
        graph.replay()
        lens, free, n = R.release(lens, e, pages, free, n, page, 0)
        if sum(-(-(l + k) // page) - -(-l // page) for l, k in zip(lens, c)) > n:
            refused += 1
            assert J.jab_get_device_status() == 1 and not qs.any() and bool((sl == -1).all())
        else:
            lens, pages, n, start, slots, positions = R.plan(lens, c, pages, free, n, page, rows)
            assert J.jab_get_device_status() == 0
            assert qs.tolist() == start and sl.tolist() == slots and po.tolist() == positions
        assert dl.tolist() == lens and dp.tolist() == pages and dn.tolist() == [n] and df.tolist()[:n] == free[:n]
    assert refused


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("bits", [8, 4])
def test_steps_of_a_server(bits):
    """Five steps of up to 8 sequences (prompts, single tokens, sequences that end and rows that begin anew, padding) in one captured
    graph, against the same calls from lists on the host bit by bit, and the attention of each against float64."""
    B, page, width, rows, d, hq, hkv, dh = 8, 16, 6, 48, 256, 4, 2, 64
    D = (hq + 2 * hkv) * dh
    g = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randn((D, d), generator=g, device="cuda") * 0.05
    codes, scales = torch.empty((D, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((D // 128, 2), device="cuda")
    J.jab_fp8_quantize(W, codes, scales)
    wq, wk = (1 + 0.2 * torch.randn(dh, generator=g, device="cuda") for _ in range(2))
    rope = tuple(torch.empty((width * page, dh // 4), device="cuda") for _ in range(2))
    J.jab_rope_table_scaled(*rope, 1e4, kind="by_parts", factor=4.0, original_length=64.0)
    n_pages = 24
    cache, twin = (J.KvCache(hkv, dh, bits, page, n_pages) for _ in range(2))
    lens, pages = _i32([0] * B + [0]), _i32([[0] * width for _ in range(B + 1)])  # (the last sequence has the padding)
    free, n_free = _i32(random.Random(1).sample(range(n_pages), n_pages)), _i32([n_pages])
    ended, counts = _i32([0] * B), _i32([0] * B)
    q_start = _i32([0] * (B + 1) + [rows])
    slots, positions = torch.empty(rows, dtype=torch.int64, device="cuda"), _i32([0] * rows)
    x = torch.zeros((rows, d), dtype=torch.float16, device="cuda")

    def buffers():
        return (torch.zeros((rows, D), dtype=torch.float16, device="cuda"), torch.zeros((rows, hq * dh), dtype=torch.float16, device="cuda"),
                torch.zeros((rows, hq, dh), dtype=torch.float16, device="cuda"),
                torch.empty(J.jab_fp8_linear_workspace_size(rows, D, d), dtype=torch.uint8, device="cuda"),
                torch.empty(J.jab_kv_attention_workspace_size(cache, B + 1, rows, hq, rows, width * page), dtype=torch.uint8, device="cuda"))

    def compute(c, b, slots, positions, q_start, pages, lens):
        qkv, q, out, w1, w2 = b
        J.jab_fp8_linear(x, codes, scales, qkv, w1)
        J.jab_kv_write_norm_rope(c, qkv, hq, slots, q_out=q, positions=positions, rope=rope, interleaved=True, norm_eps=1e-6, q_weight=wq, k_weight=wk)
        J.jab_kv_attention(c, q.view(rows, hq, dh), q_start, pages, lens, out, w2, rows, width * page)

    mine, other = buffers(), buffers()

    def step():
        J.jab_kv_release(cache, lens[:B], ended, pages[:B], free, n_free)
        J.jab_kv_plan(cache, lens[:B], counts, pages[:B], free, n_free, q_start[: B + 1], slots, positions)
        compute(cache, mine, slots, positions, q_start, pages, lens)

    step()  # (nothing to do, outside the capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    host = dict(lens=[0] * B, pages=[[0] * width for _ in range(B)], free=free.tolist(), n_free=n_pages)
    for t, (e, c) in enumerate([([0] * 8, [5, 17, 0, 1, 16, 3, 0, 2]), ([0] * 8, [1] * 8), ([0, 1, 0, 0, 1, 0, 0, 0], [1, 30, 1, 1, 0, 1, 1, 1]),
                                ([0] * 8, [1, 1, 16, 1, 0, 15, 1, 1]), ([1] * 8, [4] * 8)]):
        ended.copy_(_i32(e)), counts.copy_(_i32(c))
        x.copy_(torch.randn((rows, d), generator=g, device="cuda"))
        graph.replay()
        hl, hf, hn = R.release(host["lens"], e, host["pages"], host["free"], host["n_free"], page, 0)
        hl, hp, hn, qs, sl, po = R.plan(hl, c, host["pages"], hf, hn, page, rows)
        host = dict(lens=hl, pages=hp, free=hf, n_free=hn)
        assert lens.tolist() == hl + [0] and pages.tolist()[:B] == hp and n_free.tolist() == [hn] and slots.tolist() == sl and positions.tolist() == po
        compute(twin, other, torch.tensor(sl, device="cuda"), _i32(po), _i32(qs + [rows]), _i32(hp + [[0] * width]), _i32(hl + [0]))
        for u, v in zip(mine[:3], other[:3]):
            assert torch.equal(u[: qs[-1]], v[: qs[-1]]), t
        assert not mine[2][qs[-1] :].any()  # padding sees nothing
        k, v = (torch.empty((B, width * page, hkv, dh), device="cuda") for _ in range(2))
        J.jab_kv_read(cache, pages[:B].contiguous(), lens[:B].contiguous(), k, v)
        for b in range(B):
            n = qs[b + 1] - qs[b]
            if n == 0:
                continue
            q = mine[1][qs[b] : qs[b + 1]].double().view(n, hq, dh)
            out, _, mag = S.attention(q, k[b, : hl[b]].double(), v[b, : hl[b]].double(), 0, 1 / math.sqrt(dh))
            # weights to 2^-12 of themselves, scores of fp32 sums, half a step of fp16
            off = (mine[2][qs[b] : qs[b + 1]].double() - out).abs()
            assert bool((off <= mag * (2.0 ** -12 + 2.0 ** -16) + hl[b] * 2.0 ** -25 * mag.max() + out.abs() * 2.0 ** -11 + 2.0 ** -24).all())
        assert J.jab_get_device_status() == 0
