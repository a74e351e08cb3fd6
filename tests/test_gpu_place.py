"""Places of new tokens and pages given back, against a plain account of lists: whole numbers, compared bit for bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2403_08058_amd as C

I32 = torch.int32


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def account(counts, lens, table, free, n_free, page, N):
    """The call's outputs by the definition, row by row."""
    table, n_pages = table.copy(), len(free)
    top = min(max(int(n_free), 0), n_pages)
    out = {"new_lens": [], "granted": [], "offsets": [0], "token_rows": [], "positions": [], "slots": []}
    ended, served, top0 = 0, True, top
    for b, (n, count) in enumerate(zip(np.maximum(lens, 0).tolist(), np.maximum(counts, 0).tolist())):
        ended += count
        new = range(-(-n // page), -(-(n + count) // page))
        ok = ended <= N and n + count <= table.shape[1] * page
        if ok and len(new) > 0:
            served = served and len(new) <= top
            ok = served
            if ok:
                for block in new:
                    top -= 1
                    table[b, block] = free[top]
        out["granted"].append(int(ok))
        out["new_lens"].append(n + count if ok else n)
        out["offsets"].append(min(ended, N))
        for i in range(min(count, N - len(out["token_rows"]))):
            at = int(table[b, (n + i) // page]) if ok else -1
            out["token_rows"].append(b)
            out["positions"].append(n + i)
            out["slots"].append(at * page + (n + i) % page if 0 <= at < n_pages else -1)
    rest = N - len(out["token_rows"])
    out["token_rows"] += [-1] * rest
    out["positions"] += [0] * rest
    out["slots"] += [-1] * rest
    out.update(block_table=table, n_left=[top])
    assert top <= top0
    return {name: np.array(v, np.int32) for name, v in out.items()}


class Pool:
    """Rows with lengths and pages, a list of free ones."""

    def __init__(self, g, B, page, lens, blocks, spare):
        self.page = page
        self.lens = np.asarray(lens, np.int64)
        used = -(-np.maximum(self.lens, 0) // page)
        self.n_pages = int(used.sum()) + spare
        ids = g.permutation(self.n_pages)
        self.table = np.full((B, blocks), -1, np.int64)
        at = 0
        for b in range(B):
            self.table[b, :used[b]] = ids[at:at + used[b]]
            at += used[b]
        self.free = g.integers(-5, self.n_pages + 5, self.n_pages)
        self.free[:spare] = ids[at:]
        self.n_free = spare


def place(pool, counts, N, in_place=False, stream=None):
    B = len(pool.lens)
    whole = torch.full((3, N + 32), -77, dtype=I32, device="cuda")            # (nothing behind the block is written)
    t = {"counts": dev(counts), "seq_lens": dev(pool.lens), "block_table": dev(pool.table), "free_pages": dev(pool.free),
         "n_free": dev([pool.n_free]), "granted": dev(np.full(B, 9)), "offsets": dev(np.full(B + 1, 9))}
    t["new_lens"] = t["seq_lens"] if in_place else dev(np.full(B, 9))
    t["n_left"] = t["n_free"] if in_place else dev([9])
    t["token_rows"], t["positions"], t["slots"] = whole[0, :N], whole[1, :N], whole[2, :N]
    ws = C.alloc_paged_place_workspace(B)
    ws.fill_(0xFF)
    C.chai_paged_place_tokens(**t, page=pool.page, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert bool((whole[:, N:] == -77).all())
    assert np.array_equal(t["free_pages"].cpu().numpy(), pool.free)
    if not in_place:
        assert np.array_equal(t["seq_lens"].cpu().numpy(), pool.lens) and int(t["n_free"]) == pool.n_free
    return {n: t[n].cpu().numpy() for n in ("block_table", "new_lens", "n_left", "granted", "offsets", "token_rows", "positions", "slots")}


def check(pool, counts, N, **kw):
    got, want = place(pool, counts, N, **kw), account(np.asarray(counts), pool.lens, pool.table, pool.free, pool.n_free, pool.page, N)
    for name, v in want.items():
        assert np.array_equal(got[name].ravel(), v.ravel()), (name, got[name], v)
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,longest,most", [(1, 8, 30, 1), (3, 16, 50, 40), (16, 64, 300, 1), (63, 24, 100, 7), (64, 8, 40, 40),
                                                 (65, 16, 200, 30), (257, 16, 90, 3), (1024, 8, 33, 2), (1025, 8, 33, 2), (4096, 8, 20, 4)])
def test_rows_grow(B, page, longest, most, in_place):
    print(f"[place] {B} rows page {page} to {longest} + {most} in place {in_place}", flush=True)
    g = np.random.default_rng(B * 7 + page + most)
    lens, counts = g.integers(0, longest + 1, B), g.integers(0, most + 1, B)
    need = int((-(-(lens + counts) // page) - -(-lens // page)).sum())
    total = int(counts.sum())
    for spare, N in ((need, total), (need + 3, total + 37), (max(need // 2, 0), total + 1), (need, total // 2), (0, total)):
        pool = Pool(g, B, page, lens, -(-(longest + most) // page), spare)
        want = check(pool, counts, N, in_place=in_place)
        if spare >= need and N >= total:
            assert want["granted"].all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("N", [1, 255, 256, 257, 2047, 2048, 2049, 5000])
def test_one_row_with_many_tokens(N, in_place):
    g = np.random.default_rng(N)
    pool = Pool(g, 2, 16, [5, 3], 400, 500)
    check(pool, [N - 1, 1], N, in_place=in_place)
    check(pool, [0, N], N, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_more_tokens_than_workgroups_at_once(in_place):
    """300 000 tokens: every workgroup takes more than one stretch of them."""
    g = np.random.default_rng(8)
    pool = Pool(g, 3, 64, [100, 7, 0], 3300, 4700)
    check(pool, [200000, 1, 100000], 300010, in_place=in_place)


def test_tables_that_are_full_and_rows_without_tokens():
    g = np.random.default_rng(3)
    pool = Pool(g, 5, 8, [16, 0, 15, 9, 0], 2, 9)
    want = check(pool, [1, 0, 1, 7, 17], 30)               # no place, nothing asked for, the last place, no new page, more than a table
    assert want["granted"].tolist() == [0, 1, 1, 1, 0]
    want = check(pool, [0, 0, 0, 0, 0], 4)
    assert want["slots"].tolist() == [-1] * 4 and want["token_rows"].tolist() == [-1] * 4
    check(pool, [-3, 2, 1, -1, 4], 12)                     # (below 0: none)
    check(pool, [0, 1, 0, 0, 1], 0)                        # a block of no tokens


def test_the_first_row_without_pages_keeps_those_behind_it_from_any():
    g = np.random.default_rng(4)
    pool = Pool(g, 4, 8, [8, 8, 3, 8], 4, 2)
    want = check(pool, [1, 9, 5, 8], 40)
    assert want["granted"].tolist() == [1, 0, 1, 0] and want["n_left"].tolist() == [1]


def test_counts_and_lengths_of_any_size():
    g = np.random.default_rng(5)
    big = 2 ** 31 - 1
    pool = Pool(g, 6, 8, [3, 0, 0, 5, 2, 1], 3, 12)
    pool.lens[4], pool.table[4] = big - 4, -1              # longer than its table
    check(pool, [2, big, big, big, 1, 3], 20)
    pool.n_free = 2 ** 30                                  # the list holds n_pages at most
    check(pool, [2, 3, 4, 1, 0, 3], 20)
    pool.n_free = -4
    check(pool, [2, 3, 4, 1, 0, 3], 20)
    many = Pool(g, 4096, 8, np.zeros(4096), 2, 50)
    check(many, np.full(4096, big), 60)


def test_absent_and_foreign_pages_have_no_slots():
    g = np.random.default_rng(6)
    pool = Pool(g, 3, 8, [5, 9, 4], 3, 3)
    pool.table[0, 0], pool.table[1, 1] = -1, pool.n_pages
    pool.free[:3] = [pool.n_pages + 2, -1, 0]              # entries of the list are entered as they are
    want = check(pool, [2, 2, 9], 16)
    assert (want["slots"][:4] == -1).all()


def test_a_recorded_step_grows_rows_again_and_again():
    """Lengths and the list's top in place; a page given back and taken again; the graph against the account, replay by replay."""
    g = np.random.default_rng(7)
    B, page, N = 5, 8, 8
    pool = Pool(g, B, page, [7, 0, 3, 15, 8], 6, 8)
    t = {"seq_lens": dev(pool.lens), "block_table": dev(pool.table), "free_pages": dev(pool.free), "n_free": dev([pool.n_free])}
    counts, keep = dev([1, 1, 0, 1, 2]), dev(np.full(B, 1 << 20))
    out = {"granted": dev(np.zeros(B)), "offsets": dev(np.zeros(B + 1)), "token_rows": dev(np.zeros(N)), "positions": dev(np.zeros(N)),
           "slots": dev(np.zeros(N))}
    ws = C.alloc_paged_place_workspace(B)

    def step():
        C.chai_paged_release_pages(keep, t["seq_lens"], t["block_table"], t["free_pages"], t["n_free"], page, t["seq_lens"], t["n_free"])
        C.chai_paged_place_tokens(counts, **t, page=page, new_lens=t["seq_lens"], n_left=t["n_free"], **out, workspace=ws)

    state = {n: x.clone() for n, x in t.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n, x in state.items():
        t[n].copy_(x)
    lens, table, free, n_free = pool.lens.copy(), pool.table.copy(), pool.free.copy(), pool.n_free
    for i in range(9):
        new, kept = g.integers(0, 3, B), np.where(g.random(B) < 0.25, g.integers(0, 9, B), 1 << 20)
        counts.copy_(dev(new))
        keep.copy_(dev(kept))
        graph.replay()
        torch.cuda.synchronize()
        lens, table, free, n_free = give_back(kept, lens, table, free, n_free, page)
        want = account(new, lens, table, free, n_free, page, N)
        for name in out:
            assert np.array_equal(out[name].cpu().numpy(), want[name]), (i, name)
        lens, table, n_free = want["new_lens"].astype(np.int64), want["block_table"].astype(np.int64), int(want["n_left"][0])
        assert np.array_equal(t["seq_lens"].cpu().numpy(), lens) and np.array_equal(t["block_table"].cpu().numpy(), table)
        assert int(t["n_free"]) == n_free and np.array_equal(t["free_pages"].cpu().numpy(), free)


def give_back(keep, lens, table, free, n_free, page):
    table, free, n_pages = table.copy(), free.copy(), len(free)
    top, new = min(max(int(n_free), 0), n_pages), []
    for b, n in enumerate(np.maximum(lens, 0).tolist()):
        kept = min(max(int(keep[b]), 0), n)
        new.append(kept)
        for block in range(min(-(-kept // page), table.shape[1]), min(-(-n // page), table.shape[1])):
            if 0 <= table[b, block] < n_pages:
                if top < n_pages:
                    free[top] = table[b, block]
                top += 1
            table[b, block] = -1
    return np.array(new, np.int64), table, free, min(top, n_pages)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,longest", [(1, 8, 600), (3, 16, 50), (64, 8, 700), (257, 24, 90), (1500, 8, 20), (4096, 8, 9)])
def test_pages_given_back(B, page, longest, in_place):
    print(f"[place] release {B} rows page {page} to {longest} in place {in_place}", flush=True)
    g = np.random.default_rng(B + longest)
    lens = g.integers(0, longest + 1, B)
    pool = Pool(g, B, page, lens, -(-longest // page) + 1, 5)
    pool.table[g.random(pool.table.shape) < 0.1] = -1      # holes are nobody's
    keep = np.where(g.random(B) < 0.4, 1 << 30, g.integers(-2, longest + 1, B))
    t = {"seq_lens": dev(lens), "block_table": dev(pool.table), "free_pages": dev(pool.free), "n_free": dev([pool.n_free])}
    new_lens, n_left = (t["seq_lens"], t["n_free"]) if in_place else (dev(np.zeros(B)), dev([0]))
    C.chai_paged_release_pages(dev(keep), **t, page=page, new_lens=new_lens, n_left=n_left)
    torch.cuda.synchronize()
    want = give_back(keep, lens, pool.table, pool.free, pool.n_free, page)
    for got, x in zip((new_lens, t["block_table"], t["free_pages"]), want):
        assert np.array_equal(got.cpu().numpy(), x)
    assert int(n_left) == want[3]


def test_a_list_that_would_overflow_is_cut():
    """More entries than pages (a page in two rows): what the list has no place for is dropped, nothing is written behind it."""
    table = np.tile(np.arange(4), (3, 1))
    whole = torch.full((4 + 16,), -7, dtype=I32, device="cuda")
    left, lens = dev([0]), dev([32, 32, 32])
    t = dev(table)
    C.chai_paged_release_pages(dev([0, 0, 0]), lens, t, whole[:4], dev([2]), 8, lens, left)
    torch.cuda.synchronize()
    assert whole.tolist() == [-7, -7, 0, 1] + [-7] * 16 and int(left) == 4
    assert bool((t == -1).all()) and lens.tolist() == [0, 0, 0]


def test_another_stream():
    g = np.random.default_rng(9)
    pool = Pool(g, 20, 16, g.integers(0, 60, 20), 8, 40)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    check(pool, g.integers(0, 9, 20), 100, stream=side)
