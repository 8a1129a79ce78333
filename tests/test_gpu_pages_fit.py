"""GPU tests of page tables on the device (mtla_pages_fit) against the same rules by plain loops: tables, bounds, the ring page for page, refusals
and the slot map, over calls that build on one another."""
import numpy as np
import pytest
import torch

from paper_2505_13544_amd import binding as B
from tests import packed_reference as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Tables:
    """The library's pools and the reference's, made alike and compared after every call."""

    def __init__(self, *, max_batch, max_slots, page_slots, stride, n_pages, n_packed=0, keep=0, spill=False, seed=0):
        rng = np.random.default_rng(seed)
        self.__dict__.update(max_batch=max_batch, max_slots=max_slots, page_slots=page_slots, stride=stride, keep=keep)
        mp = -(-max_slots // page_slots)
        self.ref = P.Pool(max_batch, mp, rng.permutation(n_pages), n_pages + spill, n_pages if spill else -1)
        self.ref4 = P.Pool(max_batch, mp, rng.permutation(n_packed)) if n_packed else None
        for p in (self.ref, self.ref4):
            if p:
                p.table[:] = rng.integers(-9, 9, p.table.shape)
        self.ctx = B.Context(n_heads=4, d_head=64, r=64, d_rope=32, d_hyper=64, stride=stride, max_batch=max_batch, max_slots=max_slots, dtype="bf16",
                             page_slots=page_slots, n_pages=max(n_pages + spill, 1))
        self.ws = torch.empty(self.ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
        self.stream = torch.cuda.current_stream().cuda_stream
        self.ctx.workspace_init(self.ws, self.stream)
        up = lambda p: p and B.PagePool(dev(p.table), dev(p.first), dev(p.end), dev(p.ring), dev(np.array([p.head, p.count, 0, 0], np.int32)), dev(p.was_end), p.spill)
        self.pool, self.pool4 = up(self.ref), up(self.ref4)

    def fit(self, lens, n_new=None, n_max=0, batch=None, both=True, what=""):
        batch = batch or len(lens)
        n = np.full(len(lens), n_max) if n_new is None else np.asarray(n_new)
        rows = P.fit(self.ref, self.ref4 if both else None, lens, n, page_slots=self.page_slots, stride=self.stride, max_slots=self.max_slots, keep=self.keep,
                     batch=batch, n_max=n_max)
        got = torch.full((batch + 1, n_max), -77, dtype=torch.int64, device=DEV) if n_max else None
        self.ctx.pages_fit(self.pool, self.pool4 if both else None, dev(np.asarray(lens, np.int32)), None if n_new is None else dev(n.astype(np.int32)), n_max,
                           self.keep, batch, got, self.ws, self.stream)
        status = self.ctx.device_status(self.ws, self.stream)
        if n_max:
            assert bool((got[batch] == -77).all()), what
            assert np.array_equal(got[:batch].cpu().numpy(), rows), what
        refused = 0
        for p, r, name in ((self.pool, self.ref, "pool"), (self.pool4, self.ref4, "packed")):
            if p is None or (name == "packed" and not both):
                continue
            t = {k: v.cpu().numpy() for k, v in p.tensors.items()}
            for k in ("first", "end", "was_end", "table"):
                assert np.array_equal(t[k], getattr(r, k)), f"{what}: {name} {k}"
            assert list(t["state"][:3]) == [r.head, r.count, r.refused], f"{what}: {name} {t['state']} {r.head, r.count, r.refused}"
            at = (r.head + np.arange(r.count)) % len(r.ring)
            assert np.array_equal(t["ring"][at], r.ring[at]), f"{what}: {name} ring"
            refused += r.refused
        assert status == (B.MTLA_ERR_CAPACITY if refused else B.MTLA_OK), what
        return refused

    def no_page_is_lost(self):
        for r in (self.ref, self.ref4):
            if r is None:
                continue
            held = [int(x) for b in range(self.max_batch) for x in r.table[b, r.first[b]:r.end[b]]]
            free = [int(x) for x in r.ring[(r.head + np.arange(r.count)) % len(r.ring)]]
            assert len(set(held + free)) == len(held) + len(free)
            assert sorted(held + free) == list(range(len(held) + len(free)))


@pytest.mark.parametrize("two,keep,stride,page_slots,batch", [(False, 0, 1, 16, 5), (False, 0, 3, 64, 70), (True, 0, 2, 16, 33), (True, 1, 4, 32, 9), (True, 2, 1, 16, 64),
                                                              (True, 0, 2, 32, 1)])
def test_a_servers_life(two, keep, stride, page_slots, batch):
    # requests come with prompts, go on token by token or by drafts that are partly dropped, and leave; the rings wrap round
    rng = np.random.default_rng(batch + keep)
    max_slots = 11 * page_slots + 5
    t = Tables(max_batch=batch + 2, max_slots=max_slots, page_slots=page_slots, stride=stride, n_pages=batch * 13, n_packed=batch * 12 if two else 0, keep=keep,
               seed=batch)
    lens, room = np.zeros(batch, np.int64), max_slots * stride
    for step in range(30):
        kind = rng.random(batch)
        lens[kind < 0.1] = 0
        joins = (lens == 0) & (rng.random(batch) < 0.5)
        n_max = int(rng.choice([1, 3, stride * page_slots + 7]))
        n = np.minimum(rng.integers(0, n_max + 1, batch), room - lens)
        if step % 3 == 0:                                   # prompts
            n_max = room // 2
            n = np.where(joins, rng.integers(0, n_max, batch), 0)
        assert t.fit(lens, n, n_max, what=f"step {step}") == 0
        kept = np.where(rng.random(batch) < 0.3, rng.integers(0, 1 << 30, batch) % (n + 1), n)   # some drafts are dropped
        lens += kept
        t.no_page_is_lost()
    t.fit(np.zeros(batch, np.int64), what="end")
    t.no_page_is_lost()
    assert t.ref.count == batch * 13 and (t.ref4 is None or t.ref4.count == batch * 12)


@pytest.mark.parametrize("batch", [1023, 1024, 1025, 3001])
def test_more_sequences_than_threads(batch):
    rng = np.random.default_rng(batch)
    t = Tables(max_batch=batch, max_slots=256, page_slots=16, stride=2, n_pages=batch * 17, n_packed=batch * 16)
    for step in range(4):
        lens = rng.integers(0, 400, batch)
        lens[rng.random(batch) < 0.2] = 0
        assert t.fit(lens, rng.integers(0, 9, batch), 8, what=f"step {step}") == 0
        t.no_page_is_lost()


def test_refusals():
    # 10 pages, prompts of 4 pages each: the third sequence and the ones behind it that lack pages get none; what holds enough goes on
    t = Tables(max_batch=6, max_slots=128, page_slots=16, stride=1, n_pages=10, spill=True)
    assert t.fit([0] * 6, [64, 60, 33, 0, 1, 100], 100) == 3
    assert list(t.ref.end) == [4, 4, 0, 0, 0, 0] and (t.ref.table[2, :3] == 10).all()
    assert t.fit([64, 60, 0, 0, 0, 0], [0, 4, 17, 0, 1, 0], 17) == 1          # the second has room; two pages are left, then none for the fifth
    assert t.fit([0, 60, 17, 0, 0, 0], [0] * 6, 4) == 0                       # the first leaves ...
    assert t.fit([0, 60, 17, 0, 0, 0], [0, 0, 0, 0, 64, 0], 64) == 0          # ... and its pages go to the fifth
    t.no_page_is_lost()


def test_a_full_packed_pool_leaves_the_pages_where_they_are():
    t = Tables(max_batch=3, max_slots=256, page_slots=16, stride=2, n_pages=40, n_packed=3)
    assert t.fit([0, 0, 0], [64, 70, 33], 70) == 0
    assert t.fit([64, 70, 33], None, 1) == 2                                  # two pages fit in three; two more do not, nor does what comes behind them
    assert list(t.ref4.end) == [2, 0, 0] and list(t.ref.first) == [2, 0, 0]
    assert t.fit([65, 71, 34], None, 1) == 2
    assert t.fit([0, 72, 35], None, 1) == 2                                   # given back pages are there from the next call on
    assert t.fit([0, 73, 36], None, 1) == 0
    assert list(t.ref4.end) == [0, 2, 1]
    t.no_page_is_lost()


def test_one_pool_behind_two():
    # all pages of a sequence in one pool again (what a prefill that continues it reads), and back
    t = Tables(max_batch=4, max_slots=256, page_slots=16, stride=1, n_pages=70, n_packed=64)
    lens = [100, 16, 0, 255]
    t.fit([0] * 4, lens, 255)
    t.fit(lens, None, 1)
    assert list(t.ref.first) == [6, 1, 0, 15]
    t.fit(lens, [5, 40, 3, 0], 40, both=False)
    assert list(t.ref.first) == [0, 0, 0, 0] and list(t.ref4.end) == [6, 1, 0, 15]
    t.fit([105, 56, 3, 255], None, 1)
    t.no_page_is_lost()


def test_lengths_and_counts_outside_their_range():
    t = Tables(max_batch=5, max_slots=50, page_slots=16, stride=3, n_pages=30, n_packed=20)
    t.fit([-4, 150, 1 << 30, 149, 7], [-3, 0, 50, 1 << 30, 2], 4)
    t.fit([-(1 << 31), 150, 151, 149, 7], None, 1)
    t.no_page_is_lost()


def test_no_tokens_and_part_of_the_sequences():
    t = Tables(max_batch=8, max_slots=64, page_slots=16, stride=1, n_pages=40)
    t.fit([17, 0, 64, 1, 16, 33, 2, 48], what="no new tokens, no map")
    t.fit([0, 0, 64, 1, 16, 33, 2, 48], batch=3, what="the first three")
    assert t.ref.end[3] == 1 and t.ref.end[7] == 3
    t.no_page_is_lost()


def test_words_that_hold_anything_stay_inside_the_arrays():
    # bounds and ring words that no call left: nothing outside the arrays is touched (the neighbours of every one of them keep their values)
    n, mp, pages = 6, 4, 12
    ctx = B.Context(n_heads=4, d_head=64, r=64, d_rope=32, d_hyper=64, stride=1, max_batch=n, max_slots=64, dtype="bf16", page_slots=16, n_pages=pages)
    ws = torch.zeros(ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(0)
    for word in (-(1 << 31), -1, 3, 100, (1 << 31) - 1):
        arena = torch.full((4096,), -5, dtype=torch.int32, device=DEV)
        part = lambda at, *shape: arena[at:at + int(np.prod(shape))].view(*shape)
        t = dict(table=part(512, n, mp), first=part(1024, n), end=part(1536, n), ring=part(2048, pages), state=part(2560, 4), was_end=part(3200, n))
        for k, v in t.items():
            v.copy_(dev(rng.integers(0, pages, v.shape).astype(np.int32)))
        t["state"][0], t["state"][1] = word, word
        t["first"][1], t["end"][2], t["first"][3], t["end"][3] = word, word, word, word
        ctx.pages_fit(B.PagePool(**t), None, dev(np.array([60, 1, 0, 64, 33, 2], np.int32)), None, 4, 0, n, None, ws, torch.cuda.current_stream().cuda_stream)
        ctx.device_status(ws, torch.cuda.current_stream().cuda_stream)
        inside = torch.zeros(4096, dtype=torch.bool, device=DEV)
        for at, size in ((512, n * mp), (1024, n), (1536, n), (2048, pages), (2560, 4), (3200, n)):
            inside[at:at + size] = True
        assert bool((arena[~inside] == -5).all()), word
        assert 0 <= int(t["state"][0]) < pages and 0 <= int(t["state"][1]) <= pages


@pytest.mark.parametrize("batch", [64, 65, 80, 1024, 1025])
def test_many_sequences_and_too_few_pages(batch):
    # either pool short of pages, then both, then room for all again: who gets pages depends on who came before, across every group of sequences
    rng = np.random.default_rng(batch)
    t = Tables(max_batch=batch, max_slots=128, page_slots=16, stride=1, n_pages=batch * 5, n_packed=batch * 2, spill=True)
    lens, some = np.zeros(batch, np.int64), 0
    for step in range(6):
        n = rng.integers(0, 60, batch)
        some += t.fit(lens, n, 60, what=f"step {step}")
        lens = np.minimum(lens + n, 128)
        lens[rng.random(batch) < 0.3] = 0
        t.fit(lens, None, 1, what=f"behind step {step}")
    assert some > 0
    assert t.fit(np.zeros(batch, np.int64), what="all leave") == 0
    assert t.fit(np.zeros(batch, np.int64), np.full(batch, 30), 30, what="and come back") == 0


def test_words_that_hold_anything_among_many_sequences():
    # as above, with the sequences dealt to several workgroups and two pools
    n, mp, pages = 300, 4, 900
    ctx = B.Context(n_heads=4, d_head=64, r=64, d_rope=32, d_hyper=64, stride=1, max_batch=n, max_slots=64, dtype="bf16", page_slots=16, n_pages=pages)
    ws = torch.zeros(ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
    rng = np.random.default_rng(1)
    sizes = dict(table=(n, mp), first=(n,), end=(n,), ring=(pages,), state=(4,), was_end=(n,))
    for word in (-(1 << 31), -1, 3, 100, (1 << 31) - 1):
        arena = torch.full((16384,), -5, dtype=torch.int32, device=DEV)
        inside = torch.zeros(16384, dtype=torch.bool, device=DEV)
        at, pools = 64, []
        for _ in range(2):
            t = {}
            for k, shape in sizes.items():
                size = int(np.prod(shape))
                t[k] = arena[at:at + size].view(*shape)
                t[k].copy_(dev(rng.integers(0, mp, shape).astype(np.int32)))
                inside[at:at + size] = True
                at += size + 64
            t["state"][0], t["state"][1] = word, word
            for k in ("first", "end"):
                t[k][int(rng.integers(n))] = word
            pools.append(t)
        ctx.pages_fit(B.PagePool(**pools[0]), B.PagePool(**pools[1]), dev(rng.integers(-3, 70, n).astype(np.int32)), None, 4, 0, n, None, ws,
                      torch.cuda.current_stream().cuda_stream)
        ctx.device_status(ws, torch.cuda.current_stream().cuda_stream)
        assert bool((arena[~inside] == -5).all()), word
        for t in pools:
            assert 0 <= int(t["state"][0]) < pages and 0 <= int(t["state"][1]) <= pages
