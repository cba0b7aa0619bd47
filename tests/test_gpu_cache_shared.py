"""Pages that requests share, against a plain bookkeeping of who holds what; with tokens, eager and captured."""
import copy

import numpy as np
import pytest
import torch

from paper_2603_02170_amd import binding, cache
from paper_2603_02170_amd.cache import CacheParams

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Books:
    """Who holds which page, as the header has it: lists and sets, request after request."""

    def __init__(self, R, columns, page, pages, stack):
        self.page, self.pages, self.columns = page, pages, columns
        self.lengths, self.table = [0] * R, [[-1] * columns for _ in range(R)]
        self.stack = list(stack)

    def count(self, n):
        return min(-(-n // self.page), self.columns)

    def holders(self):
        who = {}
        for r, row in enumerate(self.table):
            for e in row[:self.count(self.lengths[r])]:
                if 0 <= e < self.pages:
                    who[e] = who.get(e, 0) + 1
        return who

    def shares(self):
        who = self.holders()
        return [max(0, who.get(e, 0) - 1) for e in range(self.pages)]

    def _give_back(self, before):
        after = self.holders()
        self.stack += sorted((e for e in before if e not in after), reverse=True)

    def free(self, keep):
        before = self.holders()
        for r, n in enumerate(keep):
            if 0 <= n <= self.lengths[r]:
                for c in range(self.count(n), self.count(self.lengths[r])):
                    self.table[r][c] = -1
                self.lengths[r] = n
        self._give_back(before)

    def fork(self, parents):
        before = self.holders()
        rows, sizes = copy.deepcopy(self.table), list(self.lengths)
        for r, p in enumerate(parents):
            if 0 <= p < len(rows) and p != r:
                n = self.count(sizes[p])
                self.table[r], self.lengths[r] = rows[p][:n] + [-1] * (self.columns - n), sizes[p]
        self._give_back(before)

    def own(self, added):
        """(added_out, [(from, to)])"""
        who, out, moves, wants = self.holders(), list(added), [], {}
        for r, n in enumerate(added):
            c = self.lengths[r] // self.page
            e = self.table[r][c] if n > 0 and self.lengths[r] % self.page and c < self.columns else -1
            if 0 <= e < self.pages and who[e] > 1:
                wants.setdefault(e, []).append(r)
        left, needs = len(self.stack), 0
        taken = 0
        for r in sorted(r for x in wants.values() for r in x):
            e = self.table[r][self.lengths[r] // self.page]
            e = next(k for k, x in wants.items() if r in x)
            keeps = len(wants[e]) == who[e] and wants[e][-1] == r
            needs += not keeps
            if needs > left:
                out[r] = 0
            elif not keeps:
                to = self.stack[left - needs]
                taken = needs
                moves.append((e, to))
                self.table[r][self.lengths[r] // self.page] = to
        del self.stack[left - taken:]
        return out, moves

    def grow(self, r, n):
        """Tokens with pages from the stack, as plan grants them."""
        for _ in range(self.count(self.lengths[r]), self.count(self.lengths[r] + n)):
            self.table[r][self.table[r].index(-1)] = self.stack.pop()
        self.lengths[r] += n


class Device:
    def __init__(self, b, p, pool):
        self.p, self.pool = p, pool
        self.lengths, self.table = _i32(b.lengths), _i32(b.table).reshape(len(b.lengths), b.columns)
        self.free_pages, self.free_count = _i32(b.stack + [-9] * (b.pages - len(b.stack))), _i32([len(b.stack)])
        self.shares = cache.alloc_shares(b.pages)
        self.shares[0] = _i32(b.shares())

    def state(self):
        return self.lengths, self.table, self.free_pages, self.free_count, self.shares

    def check(self, b, what=""):
        assert self.lengths.tolist() == b.lengths, what
        assert self.table.tolist() == b.table, what
        assert self.free_count.item() == len(b.stack) and self.free_pages[:len(b.stack)].tolist() == b.stack, what
        assert self.shares[0].tolist() == b.shares() and (self.shares[1:] == 0).all(), what


def _books(rng, R, columns, page, spare):
    """Requests that share pages with requests before them, and some that are empty."""
    lengths, table, fresh = [], [], 0
    for r in range(R):
        n = int(rng.choice([0, 1, page, rng.integers(0, columns * page + 1), rng.integers(0, columns * page + 1)]))
        k, row = -(-n // page), []
        if r > 0 and rng.random() < 0.6:
            other = int(rng.integers(0, r))
            row = table[other][:min(int(rng.integers(0, columns + 1)), k, -(-lengths[other] // page))]
        while len(row) < k:
            row.append(fresh if rng.random() < 0.97 else -5)
            fresh += row[-1] >= 0
        lengths.append(n)
        table.append(row + [-1] * (columns - k))
    pages = fresh + spare
    order = rng.permutation(pages).tolist()
    b = Books(R, columns, page, pages, [order[e] for e in range(fresh, pages)])
    b.lengths, b.table = lengths, [[order[e] if e >= 0 else e for e in row] for row in table]
    return b


SIZES = [(1, 1, 32, 1), (1, 3, 64, 4), (5, 4, 32, 3), (16, 40, 64, 30), (65, 7, 128, 50), (200, 30, 32, 400), (64, 600, 256, 9), (1500, 9, 64, 77), (3000, 40, 32, 1000)]


@pytest.mark.parametrize("R,columns,page,spare", SIZES)
def test_free_fork_own_and_compact_against_the_books(R, columns, page, spare):
    rng = np.random.default_rng(R + columns)
    for trial in range(3):
        b = _books(rng, R, columns, page, spare)
        p = CacheParams(H=1, d=64, page=page, block=32) if trial != 1 else CacheParams(H=1, d=64, page=page, group=32)
        pool = torch.zeros(tuple(cache.alloc_cache(p, b.pages).shape), dtype=torch.uint8, device="cuda")
        words = pool.view(torch.int32).flatten(1)
        words[:, 0], words[:, -1] = torch.arange(b.pages, device="cuda"), torch.arange(b.pages, device="cuda")      # a page's name at its both ends
        d = Device(b, p, pool)
        d.check(b)
        for what in rng.permutation(["free", "fork", "own", "fork", "own", "free", "own"]):
            names = words.clone()
            if what == "free":
                keep = [int(x) for x in rng.integers(-3, columns * page + 3, R)]
                keep = [n if rng.random() < 0.5 else int(rng.choice([0, m])) for n, m in zip(keep, b.lengths)]
                b.free(keep)
                cache.sagebwd_cache_free(_i32(keep), *d.state(), p)
            elif what == "fork":
                parents = [int(x) if rng.random() < 0.7 else r for r, x in enumerate(rng.integers(-2, R + 2, R))]
                b.fork(parents)
                cache.sagebwd_cache_fork(_i32(parents), *d.state(), p)
            else:
                added = [int(x) for x in rng.integers(-1, 3, R)]
                want, moves = b.own(added)
                got = cache.sagebwd_cache_own(_i32(added), *d.state(), pool, p)
                assert got.tolist() == want
                for e, to in moves:
                    names[to] = names[e]
            d.check(b, what)
            assert torch.equal(words, names)
        # compact, beside the state and in its place
        held = [[e if 0 <= e < b.pages and c < b.count(n) else -1 for c, e in enumerate(row)] for row, n in zip(b.table, b.lengths)]
        used = sorted({e for row in held for e in row if e >= 0})
        n = len(used)
        holes = [e for e in range(n) if e not in set(used)]
        where = {e: e for e in used if e < n}
        where.update(zip([e for e in used if e >= n], holes))
        names = words.clone()
        for e, to in where.items():
            names[to] = words[e]
        start = pool.clone()
        for in_place in (False, True):
            pool.copy_(start)
            out = None
            if in_place:
                d.shares[0].random_(0, 1000)          # (row 0 is written, not read)
                out = cache.CacheCompaction(d.table, d.free_pages, d.free_count, d.shares, _i32([-1]))
            got = cache.sagebwd_cache_compact(d.lengths, d.table, pool, p, out=out)
            assert got.used.item() == n and got.free_count.item() == b.pages - n
            assert got.block_table.tolist() == [[where[e] if e >= 0 else -1 for e in row] for row in held]
            assert got.free_pages.tolist() == list(range(b.pages - 1, n - 1, -1)) + [-1] * n
            after = Books(R, columns, page, b.pages, [])
            after.lengths, after.table = b.lengths, got.block_table.tolist()
            assert got.shares[0].tolist() == after.shares() and (got.shares[1:] == 0).all()
            assert torch.equal(words[:n], names[:n]) and torch.equal(pool[n:], start[n:])


def test_more_pages_than_a_step_settles():
    """200000 pages: their stack is settled, and moves are chosen, in several steps."""
    rng = np.random.default_rng(5)
    pages, R, columns, page = 200_000, 400, 300, 32
    p = CacheParams(H=1, d=64, page=page, group=64)
    order = rng.permutation(pages).tolist()
    b = Books(R, columns, page, pages, order[R * columns:])
    b.lengths, b.table = [columns * page] * R, [order[r * columns:(r + 1) * columns] for r in range(R)]
    pool = torch.zeros(tuple(cache.alloc_cache(p, pages).shape), dtype=torch.uint8, device="cuda")
    words = pool.view(torch.int32).flatten(1)
    words[:, 5] = torch.arange(pages, device="cuda")
    d = Device(b, p, pool)
    for call in ("fork", "free"):
        if call == "fork":
            parents = [r // 2 * 2 for r in range(R)]
            b.fork(parents)
            cache.sagebwd_cache_fork(_i32(parents), *d.state(), p)
        else:
            keep = [int(x) for x in rng.integers(0, columns * page, R)]
            b.free(keep)
            cache.sagebwd_cache_free(_i32(keep), *d.state(), p)
        d.check(b, call)
    got = cache.sagebwd_cache_compact(d.lengths, d.table, pool, p)
    n = len(b.holders())
    assert got.used.item() == n
    new, old = got.block_table, d.table
    assert torch.equal(words[new[new >= 0].long(), 5], old[old >= 0]) and torch.equal(new >= 0, old >= 0) and int(new.max()) == n - 1


def test_a_stack_that_is_full_and_bounds_that_device_memory_breaks():
    """Pages beyond the stack's capacity are lost, counts beyond it are read as it; nothing is written outside."""
    p = CacheParams(H=1, d=64, page=32, block=32)
    pool = torch.zeros(tuple(cache.alloc_cache(p, 6).shape), dtype=torch.uint8, device="cuda")
    guard = torch.full((40,), 77, dtype=torch.int32, device="cuda")
    stack = guard[8:11]
    stack.copy_(_i32([5, 4, 9]))
    shares = cache.alloc_shares(6)
    lengths, table, count = _i32([90, 1 << 30, -7]), _i32([[0, 1, 2], [3, 1 << 30, -1 << 31], [1, 1, 1]]), _i32([2])
    cache.sagebwd_cache_free(_i32([0, 1 << 30, -8]), lengths, table, stack, count, shares, p)
    assert stack.tolist() == [5, 4, 2] and count.item() == 3 and (guard[11:] == 77).all() and (guard[:8] == 77).all()
    assert table.tolist() == [[-1, -1, -1], [3, 1 << 30, -1 << 31], [1, 1, 1]] and lengths.tolist() == [0, 1 << 30, -7]
    count.fill_(1 << 30)
    shares[0, 3] = 2
    lengths.copy_(_i32([5, 33, 20]))
    table.copy_(_i32([[3, -1, -1], [0, 3, -1], [3, -1, -1]]))
    stack.copy_(_i32([5, 4, 77]))                     # (77 is no page: it is handed out, and nothing is copied there)
    before = pool.clone()
    got = cache.sagebwd_cache_own(_i32([1, 1, 0]), lengths, table, stack, count, shares, pool, p)
    assert got.tolist() == [1, 1, 0] and table.tolist() == [[77, -1, -1], [0, 4, -1], [3, -1, -1]] and count.item() == 1
    assert torch.equal(pool, before) and shares[0].tolist() == [0] * 6 and (shares[1:] == 0).all()
    for call in (lambda: cache.sagebwd_cache_free(_i32([]), _i32([]), table[:0], stack, count, shares, p),
                 lambda: cache.sagebwd_cache_fork(_i32([]), _i32([]), table[:0], stack, count, shares, p),
                 lambda: cache.sagebwd_cache_own(_i32([]), _i32([]), table[:0], stack, count, shares, pool, p)):
        call()
    assert cache.sagebwd_cache_compact(_i32([]), table[:0], pool, p).used.item() == 0


@pytest.mark.parametrize("p", [CacheParams(H=2, d=64, page=32, block=32), CacheParams(H=2, d=128, page=64, group=64)])
@pytest.mark.parametrize("captured", [False, True])
def test_a_search_over_beams_against_requests_that_share_nothing(p, captured):
    """Prompts, then steps in which beams go on from one another: attention over shared pages gives the bits of that over requests which
    hold their own copies of everything; compacted now and then; at the end every page comes back."""
    g, rng = torch.Generator().manual_seed(p.d), np.random.default_rng(p.d)
    R, Hq, columns, pages, W = 6, 4, 8, 60, 3
    H, d = p.H, p.d
    pool = torch.full(tuple(cache.alloc_cache(p, pages).shape), 0xFF, dtype=torch.uint8, device="cuda")
    lengths, table = _i32([0] * R), torch.full((R, columns), -1, dtype=torch.int32, device="cuda")
    stack, count, shares = _i32(list(range(pages))), _i32([pages]), cache.alloc_shares(pages)
    alone = torch.full(tuple(cache.alloc_cache(p, R * columns).shape), 0xFF, dtype=torch.uint8, device="cuda")      # request r: pages r * columns ..
    own_table = torch.arange(R * columns, device="cuda", dtype=torch.int32).reshape(R, columns)
    qkv, parents, added = torch.zeros((R, Hq + 2 * H, d), dtype=torch.bfloat16, device="cuda"), _i32([0] * R), _i32([1] * R)

    def step(qkv, added, rows, most):
        cache.sagebwd_cache_fork(parents, lengths, table, stack, count, shares, p)
        now = cache.sagebwd_cache_own(added, lengths, table, stack, count, shares, pool, p)
        plan = cache.sagebwd_cache_plan(lengths, now, table, stack, count, p, rows)
        cache.sagebwd_cache_append(qkv[:, Hq:Hq + H], qkv[:, Hq + H:], plan.slots, pool, p)
        O, lse = cache.sagebwd_cache_attention(qkv[:, :Hq], pool, table, plan.lengths, plan.cu_new, p, most)
        lengths.copy_(plan.lengths)
        count.copy_(plan.free_left)
        return O, lse

    def check(parent_list, added_list, qkv, before, O, lse):
        old = alone.clone()
        for r, q in enumerate(parent_list):
            if 0 <= q < R:
                alone[r * columns:(r + 1) * columns] = old[q * columns:(q + 1) * columns]
                before[r] = lens0[q]
        slots = torch.cat([torch.arange(n, device="cuda") + r * columns * p.page + before[r] for r, n in enumerate(added_list)])
        cache.sagebwd_cache_append(qkv[:, Hq:Hq + H], qkv[:, Hq + H:], slots, alone, p)
        now = [a + n for a, n in zip(before, added_list)]
        assert lengths.tolist() == now
        cu = _i32(np.concatenate([[0], np.cumsum(added_list)]).tolist())
        want, wl = cache.sagebwd_cache_attention(qkv[:, :Hq], alone, own_table, lengths, cu, p, max(added_list))
        assert torch.equal(O, want) and torch.equal(lse, wl)

    prompt = [45, 0, 0, 33, 0, 0]
    lens0 = [0] * R
    x = torch.randn((sum(prompt), Hq + 2 * H, d), generator=g).to(torch.bfloat16).cuda()
    parents.fill_(-1)
    check([-1] * R, prompt, x, [0] * R, *step(x, _i32(prompt), sum(prompt), max(prompt)))
    graph = None
    if captured:
        saved = [t.clone() for t in (pool, lengths, table, stack, count, shares)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(qkv, added, R, 1)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for t, s in zip((pool, lengths, table, stack, count, shares), saved):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            Og, lg = step(qkv, added, R, 1)
    for i in range(60):
        if i == 0:
            who = [r // W * W for r in range(R)]                       # samples of a prompt
        elif i % 3 == 0:
            who = [-1] * R
        else:
            who = [r // W * W + int(rng.integers(0, W)) for r in range(R)]
        if i % 17 == 11:
            kept = cache.sagebwd_cache_compact(lengths, table, pool, p, out=cache.CacheCompaction(table, stack, count, shares, _i32([0])))
            assert kept.used.item() == len({e for row in table.tolist() for e in row if e >= 0})
        lens0 = lengths.tolist()
        before = [lens0[q] if q >= 0 else lens0[r] for r, q in enumerate(who)]
        qkv.copy_(torch.randn((R, Hq + 2 * H, d), generator=g).to(torch.bfloat16))
        parents.copy_(_i32(who))
        if captured:
            graph.replay()
            O, lse = Og, lg
        else:
            O, lse = step(qkv, added, R, 1)
        check(who, [1] * R, qkv, before, O, lse)
        if i == 30:                                                    # drafted tokens are taken back, into pages that may be shared
            keep = [n - int(rng.integers(0, 9)) for n in lengths.tolist()]
            cache.sagebwd_cache_free(_i32(keep), lengths, table, stack, count, shares, p)
    cache.sagebwd_cache_free(_i32([0] * R), lengths, table, stack, count, shares, p)
    assert count.item() == pages and sorted(stack.tolist()) == list(range(pages)) and (shares == 0).all() and (table == -1).all()


def test_offsets_beyond_32_bits():
    p = CacheParams(H=16, d=128, page=256, block=64)
    size = cache.cache_page_bytes(p)
    pages = (5 << 30) // size
    pool = torch.empty((pages, p.H, size // p.H), dtype=torch.uint8, device="cuda")
    pool[-4:] = torch.randint(0, 256, tuple(pool[-4:].shape), dtype=torch.uint8, device="cuda")
    shares = cache.alloc_shares(pages)
    shares[0, pages - 1] = 1
    lengths, table, stack, count = _i32([100, 90]), _i32([[pages - 1], [pages - 1]]), _i32([pages - 3]), _i32([1])
    assert cache.sagebwd_cache_own(_i32([1, 1]), lengths, table, stack, count, shares, pool, p).tolist() == [1, 1]
    assert table.tolist() == [[pages - 3], [pages - 1]] and torch.equal(pool[pages - 3], pool[pages - 1])
    last = pool[-4:].clone()
    got = cache.sagebwd_cache_compact(lengths, table, pool, p)
    assert got.block_table.tolist() == [[0], [1]] and torch.equal(pool[0], last[1]) and torch.equal(pool[1], last[3])


def test_calls_on_streams_of_their_own():
    """Each call on the stream that is current, in order with that stream's other work."""
    p = CacheParams(H=1, d=64, page=32, block=32)
    pool = torch.zeros(tuple(cache.alloc_cache(p, 40).shape), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        pool.view(torch.int32).flatten(1)[:, 3] = torch.arange(40, device="cuda", dtype=torch.int32)
        lengths, table, stack, count, shares = _i32([40, 0, 0]), _i32([[7, 9], [-1, -1], [-1, -1]]), _i32([20, 21]), _i32([2]), cache.alloc_shares(40)
        cache.sagebwd_cache_fork(_i32([0, 0, 0]), lengths, table, stack, count, shares, p)
        got = cache.sagebwd_cache_own(_i32([1, 1, 0]), lengths, table, stack, count, shares, pool, p)
        cache.sagebwd_cache_free(_i32([40, 40, 0]), lengths, table, stack, count, shares, p)
        out = cache.sagebwd_cache_compact(lengths, table, pool, p)
    side.synchronize()
    assert got.tolist() == [1, 1, 0] and table.tolist() == [[7, 21], [7, 20], [-1, -1]] and shares[0, 7] == 1 and stack[:1].tolist() == [9]
    assert out.block_table.tolist() == [[0, 2], [0, 1], [-1, -1]]
    assert pool.view(torch.int32).flatten(1)[:3, 3].tolist() == [7, 9, 9]
