"""New tokens, bounds, selection, attention over lists, forks, copies and compaction together, as a serving program calls
them: eagerly, captured and replayed, on another stream, and far into a large pool."""
import pytest
import torch

from paper_2506_15745_amd import ipv
from tests import blocks as X
from tests import paged as R
from tests.test_gpu_blocks import check_attend
from tests.test_gpu_compact import kept

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "f32", "fp8", "fp4")
L, H, G, D, T, BLOCK, TOP, EPS = 2, 2, 3, 64, 64, 16, 4, 1e-6
A = H * G


class Program:
    """Conversations over one pool."""

    def __init__(self, fmt, streams, pages, columns, longest, seed):
        formats = dict(zip(FORMATS, (ipv.PAGES_BF16, ipv.PAGES_F32, ipv.PAGES_FP8, ipv.PAGES_FP4)))
        self.fmt, self.g = fmt, torch.Generator(device="cuda").manual_seed(seed)
        self.pool = ipv.PagePool.empty(pages, L, H, T, D, formats[fmt])
        self.bounds = ipv.BlockBounds(self.pool, BLOCK)
        self.tables = ipv.PageTables(self.pool, streams, columns)
        self.rotary = R.angles(columns * T, D, "cuda")
        self.norms = [torch.rand(D, generator=self.g, device="cuda") + 0.5 for _ in range(2)]
        self.page_ws = ipv.alloc_page_workspace("cuda")
        self.block_ws = ipv.alloc_blocks_workspace(self.bounds, streams, A, longest, TOP, columns * T)
        self.n = [0] * streams

    def rows(self, b, layer, h, name="K"):
        return R.rows_of(self.pool, self.fmt, self.tables.table, b, layer, h, name)[:self.n[b]]

    def everything(self):
        return {(b, layer, h, name): self.rows(b, layer, h, name) for b in range(len(self.n)) for layer in range(L) for h in range(H)
                for name in "KV"}

    def step(self, rows):
        """rows[b] new tokens of every stream, through both layers; each is checked."""
        B, M, first = len(self.n), max(rows), list(self.n)
        before, others = self.everything(), list(self.n)
        self.tables.reserve(first, rows, self.page_ws, bounds=self.bounds)
        table = self.tables.table
        self.n = [x + y for x, y in zip(first, rows)]
        for layer in range(L):
            qkv = (torch.randn(B, M, A + 2 * H, D, generator=self.g, device="cuda") * 2).to(self.pool.dtype).transpose(1, 2)
            q, k, v = qkv[:, :A], qkv[:, A:A + H], qkv[:, A + H:]  # of one projection, token by token
            turned, out = (torch.full((B, A, M, D), 777.0, dtype=q.dtype, device="cuda") for _ in range(2))
            lists = torch.full((B, H, M, TOP), 777, dtype=torch.int32, device="cuda")
            lse = torch.full((B, A, M), 777.0, device="cuda")
            ipv.ipv_qkv_write(self.pool, table, first, layer, q, k, v, turned, self.page_ws, rows=rows, q_norm=self.norms[0],
                              k_norm=self.norms[1], eps=EPS, rotary=self.rotary, bounds=self.bounds)
            ipv.ipv_attend_blocks(self.pool, table, self.n, first, layer, turned, lists, out, self.block_ws, bounds=self.bounds,
                                  q_rows=rows, first_blocks=1, lse=lse)
            torch.cuda.synchronize()
            pos = torch.tensor(first, device="cuda")[:, None] + torch.arange(M, device="cuda")
            want = X.turned(X.normed32(q, self.norms[0], EPS), self.rotary, pos.clamp_max(self.rotary.shape[0] - 1)).to(q.dtype)
            for b, m in enumerate(rows):
                assert torch.equal(turned[b, :, :m], want[b, :, :m])
                if self.fmt in ("bf16", "f32"):
                    keys = X.turned(X.normed32(k, self.norms[1], EPS), self.rotary, pos.clamp_max(self.rotary.shape[0] - 1)).to(q.dtype)
                    for h in range(H):
                        assert torch.equal(self.rows(b, layer, h)[first[b]:], keys[b, h, :m].double())
                        assert torch.equal(self.rows(b, layer, h, "V")[first[b]:], v[b, h, :m].double())
            assert torch.equal(lists.cpu(), X.select(self.bounds, table, self.n, first, layer, turned, TOP, 1, 1, rows))
            check_attend(self.fmt, self.pool, table, self.n, first, layer, turned, lists, BLOCK, out, lse, rows)
        for key, x in before.items():  # the rows that were there, shared or not
            assert torch.equal(x, self.rows(*key)[:others[key[0]]])
        self.check()

    def check(self):
        for b, n in enumerate(self.n):
            for layer in range(L):
                for h in range(H):
                    for j in range(-(-n // BLOCK)):
                        lo, hi = X.block_bounds(self.pool, self.fmt, self.tables.table, b, layer, h, j, BLOCK, n)
                        got = X.bounds_at(self.bounds, self.tables.table, b, layer, h, j).double()
                        assert torch.equal(got, torch.stack((lo, hi)))
        assert ipv.ipv_read_device_errors(self.page_ws) == 0 and ipv.ipv_read_device_errors(self.block_ws) == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_conversations(fmt):
    p = Program(fmt, 3, 14, 5, 90, 1)
    p.step([90, 0, 0])
    # two more conversations go on from the first one's tokens
    p.tables.fork(0, 1, 90)
    p.n[1] = 90
    p.tables.fork(0, 2, 70)
    p.n[2] = 70
    before = p.tables.free_pages
    # stream 2 has fewer rows of the shared page than its bounds cover: they are made anew in its own page
    p.tables.reserve(p.n, [1, 1, 1], p.page_ws, bounds=p.bounds)
    assert p.tables.free_pages == before - 2
    ipv.ipv_block_bounds(p.pool, p.tables.table, [0, 0, 64], [0, 0, 6], p.bounds, p.page_ws)
    p.check()
    p.step([1, 1, 1])
    p.step([1, 0, 5])
    p.step([33, 1, 40])  # across pages
    # two of them keep some of their rows, the rest goes back
    n, keep = [p.n[0], p.n[2]], kept(2, L, H, [p.n[0], p.n[2]], 50, 3)
    old = p.everything()
    pages = [list(x) for x in p.tables.pages]
    p.tables.compact([0, 2], n, keep, p.page_ws, rows=[50, 49], rotary=p.rotary, bounds=p.bounds)
    p.n = [50, p.n[1], 49]
    assert p.tables.pages[1] == pages[1] and len(p.tables.pages[0]) == len(p.tables.pages[2]) == 1
    for i, b in enumerate((0, 2)):
        for layer in range(L):
            for h in range(H):
                at = keep[i, layer, h, :p.n[b]].long()
                assert torch.equal(p.rows(b, layer, h, "V"), old[b, layer, h, "V"][at])
                j = torch.arange(p.n[b], device="cuda")
                x = old[b, layer, h, "K"][at].float()[None, None]
                y = X.turned(X.turned(x, p.rotary, at[None], back=True), p.rotary, j[None])[0, 0]
                assert torch.equal(p.rows(b, layer, h)[at != j], X.coded_again(y[at != j], fmt))
                assert torch.equal(p.rows(b, layer, h)[at == j], old[b, layer, h, "K"][at][at == j])
    for layer in range(L):
        for h in range(H):
            assert torch.equal(p.rows(1, layer, h), old[1, layer, h, "K"])
    p.check()
    p.step([1, 1, 1])
    p.step([20, 0, 16])
    for b in range(3):
        p.tables.free(b)
    assert p.tables.free_pages == 14


def sequence(fmt, m, seed, ws=None, page_ws=None):
    """A pool and what a step of m tokens, a copy and a compaction do to it, with fixed tensors: (run, state, results)."""
    B, n = 2, [200, 131]
    pool = R.filled_pool(fmt, 16, 1, H, T, D, seed)
    tables = R.shuffled_table(2 * B, 4, 16, seed)
    table, fresh = tables[:B].contiguous(), tables[B:].contiguous()
    bounds = ipv.BlockBounds(pool, BLOCK)
    page_ws = ipv.alloc_page_workspace("cuda") if page_ws is None else page_ws
    ipv.ipv_block_bounds(pool, table, 0, n, bounds, page_ws)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn(B, h, m, D, generator=g, device="cuda").to(pool.dtype) for h in (A, H, H))
    rotary, keep = R.angles(4 * T, D, "cuda"), kept(B, 1, H, n, 100, seed)
    turned, out = torch.zeros_like(q), torch.zeros_like(q)
    lists, lse = torch.zeros((B, H, m, TOP), dtype=torch.int32, device="cuda"), torch.zeros((B, A, m), device="cuda")
    from_pages, to_pages = table[0, :1].contiguous(), fresh[0, 3:].contiguous()
    if ws is None:
        ws = ipv.alloc_blocks_workspace(bounds, B, A, m, TOP, 4 * T)
    first = [x - m for x in n]

    def run():
        ipv.ipv_qkv_write(pool, table, first, 0, q, k, v, turned, page_ws, eps=EPS, rotary=rotary, bounds=bounds)
        ipv.ipv_attend_blocks(pool, table, n, first, 0, turned, lists, out, ws, bounds=bounds, lse=lse)
        ipv.ipv_page_copy(pool, from_pages, to_pages, page_ws, bounds=bounds)
        ipv.ipv_page_compact(pool, table, fresh, n, keep, page_ws, rotary=rotary, bounds=bounds)

    results = [turned, out, lists, lse]
    return run, X.raw(pool) + [bounds.values], results


def eager(run, state, results):
    """What the sequence gives from its state, which is put back."""
    start = [t.clone() for t in state]
    run()
    torch.cuda.synchronize()
    got = [t.clone() for t in state + results]
    for t, x in zip(state, start):
        t.copy_(x)
    return start, got


def assert_replayed(replay, start, want, state, results):
    for t, x in zip(state, start):
        t.copy_(x)
    for t in results:
        t.fill_(7)
    replay()
    torch.cuda.synchronize()
    for t, x in zip(state + results, want):
        assert torch.equal(t.view(torch.uint8), x.view(torch.uint8))


@pytest.mark.parametrize("fmt", FORMATS)
def test_two_graphs_share_workspaces(fmt):
    """Captured steps of one token and of 40, with one pair of workspaces, replayed in turn with eager work between."""
    few = sequence(fmt, 1, 5)
    many_ws, page_ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda"), ipv.alloc_page_workspace("cuda")
    calls = [sequence(fmt, m, 5 + m, ws=many_ws, page_ws=page_ws) for m in (1, 40)]
    eagers = [eager(*c) for c in calls]
    few_eager = eager(*few)
    graphs = []
    for run, _, _ in calls:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    for _ in range(4):
        for graph, c, (start, want) in zip(graphs, calls, eagers):
            assert_replayed(graph.replay, start, want, c[1], c[2])
            assert_replayed(few[0], *few_eager, few[1], few[2])  # eager work with workspaces of its own
            assert_replayed(c[0], start, want, c[1], c[2])        # and with the shared ones
    # back to back, with nothing between them
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    for graph, c, (start, want) in zip(graphs, calls, eagers):
        assert_replayed(graph.replay, start, want, c[1], c[2])
    assert ipv.ipv_read_device_errors(many_ws) == 0 and ipv.ipv_read_device_errors(page_ws) == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_on_another_stream(fmt):
    """A side stream, as the current one, and two streams at once with pools and workspaces of their own."""
    calls = [sequence(fmt, m, 9 + m) for m in (1, 17)]
    eagers = [eager(*c) for c in calls]
    sides = [torch.cuda.Stream() for _ in calls]
    for (run, state, results), (start, _) in zip(calls, eagers):
        for t, x in zip(state, start):
            t.copy_(x)
        for t in results:
            t.fill_(7)
    busy = torch.randn(2048, 2048, device="cuda")
    for _ in range(3):
        busy = (busy @ busy).clamp(-1, 1)
    inputs = torch.cuda.Event()
    inputs.record()
    for side, (run, _, _) in zip(sides, calls):
        side.wait_event(inputs)
        with torch.cuda.stream(side):
            run()
    torch.cuda.synchronize()
    for (_, state, results), (_, want) in zip(calls, eagers):
        for t, x in zip(state + results, want):
            assert torch.equal(t.view(torch.uint8), x.view(torch.uint8))


def test_another_current_device_is_refused(monkeypatch):
    """Kernels go to the current device: with another one than the pool's nothing is launched."""
    run, state, _ = sequence("bf16", 2, 1)
    before = [t.clone() for t in state]
    torch.cuda.synchronize()
    pool = R.filled_pool("bf16", 4, 1, H, T, D, 3)
    bounds, ws = ipv.BlockBounds(pool, BLOCK), ipv.alloc_page_workspace("cuda")
    block_ws = ipv.alloc_blocks_workspace(bounds, 1, A, 1, TOP, T)
    q = torch.zeros((1, A, 1, D), dtype=torch.bfloat16, device="cuda")
    lists = torch.zeros((1, H, 1, TOP), dtype=torch.int32, device="cuda")
    page = torch.zeros(1, dtype=torch.int32, device="cuda")
    keep = torch.zeros((1, 1, H, 5), dtype=torch.int32, device="cuda")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (run,
                 lambda: ipv.ipv_qkv_write(pool, None, 0, 0, q, q[:, :H], q[:, :H], q, ws),
                 lambda: ipv.ipv_block_bounds(pool, None, [0], [5], bounds, ws),
                 lambda: ipv.ipv_block_select(pool, None, bounds, 5, 0, 0, q, lists, block_ws),
                 lambda: ipv.ipv_attend_blocks(pool, None, 5, 0, 0, q, lists, q, block_ws, bounds=bounds),
                 lambda: ipv.ipv_page_compact(pool, None, page[None], 5, keep, ws),
                 lambda: ipv.ipv_page_copy(pool, page, page + 1, ws)):
        with pytest.raises(ipv.IpvError) as e:
            call()
        assert e.value.status == ipv.ERR_ARG and "current device is 1" in str(e.value)
    monkeypatch.undo()
    torch.cuda.synchronize()
    for t, x in zip(state, before):
        assert torch.equal(t, x)


def test_the_stream_argument():
    pool = R.filled_pool("bf16", 4, 1, H, T, D, 3)
    side, ws = torch.cuda.Stream(), ipv.alloc_page_workspace("cuda")
    src, dst = (torch.tensor([i], dtype=torch.int32, device="cuda") for i in (1, 3))
    torch.cuda.synchronize()
    ipv.ipv_page_copy(pool, src, dst, ws, stream=side)
    side.synchronize()
    assert torch.equal(pool.K[3], pool.K[1]) and torch.equal(pool.V[3], pool.V[1])


@pytest.mark.parametrize("fmt,pages,heads,dim", [("bf16", 36000, 8, 128), ("fp4", 270000, 8, 128)])
def test_past_32_bits(fmt, pages, heads, dim):
    """Pages whose rows (bf16: 4.7 GB of keys) or bounds (4.4 GB) lie past 32 bits give what the same ones at the start of a
    small pool give."""
    n, m, B = 150, 3, 1
    kinds = {"bf16": ipv.PAGES_BF16, "fp4": ipv.PAGES_FP4}
    small, big = R.filled_pool(fmt, 8, 1, heads, T, dim, 4), ipv.PagePool.empty(pages, 1, heads, T, dim, kinds[fmt])
    for x, y in zip(X.raw(small), X.raw(big)):
        y[-8:] = x
    table = torch.tensor([[5, 0, 7, 2]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(B, h, m, dim, generator=g, device="cuda").to(small.dtype) for h in (2 * heads, heads, heads))
    rotary, keep = R.angles(4 * T, dim, "cuda"), kept(B, 1, heads, [n], 70, 4)
    ends = []
    for pool, base in ((small, 0), (big, pages - 8)):
        at, ws = table + base, ipv.alloc_page_workspace("cuda")
        bounds = ipv.BlockBounds(pool, BLOCK)
        block_ws = ipv.alloc_blocks_workspace(bounds, B, 2 * heads, m, TOP, 4 * T)
        turned, out = torch.zeros_like(q), torch.zeros_like(q)
        lists = torch.zeros((B, heads, m, TOP), dtype=torch.int32, device="cuda")
        new = torch.tensor([[3, 6]], dtype=torch.int32, device="cuda") + base
        ipv.ipv_block_bounds(pool, at, 0, n - m, bounds, ws)
        ipv.ipv_qkv_write(pool, at, n - m, 0, q, k, v, turned, ws, rotary=rotary, bounds=bounds)
        ipv.ipv_attend_blocks(pool, at, n, n - m, 0, turned, lists, out, block_ws, bounds=bounds)
        ipv.ipv_page_compact(pool, at, new, n, keep, ws, rotary=rotary, bounds=bounds)
        ipv.ipv_page_copy(pool, new[0, :1], at[0, 3:], ws, bounds=bounds)
        torch.cuda.synchronize()
        assert ipv.ipv_read_device_errors(ws) == 0 and ipv.ipv_read_device_errors(block_ws) == 0
        ends.append([turned, out, lists] + [t[-8:].clone() for t in X.raw(pool) + [bounds.values]])
    for x, y in zip(*ends):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    for t in X.raw(big):  # and nothing went anywhere else
        assert not bool(t[:8].view(torch.uint8).any())
