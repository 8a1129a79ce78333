"""GPU tests of PackedSession's rows as requests change hands: a row that is released and taken over by the next call, lengths that fall, pools that have
no page left.  The contiguous session beside it holds the rows that the pages should hold."""
import numpy as np
import pytest
import torch

import workloads as W
from paper_2505_13544_amd import binding as B
from paper_2505_13544_amd.session import PackedSession
from tests import packed_reference as P
from tests.test_gpu_packed_session import check_out, check_state, rows_of, sessions, tokens

pytestmark = pytest.mark.gpu


class Served:
    """Three prompts of 40, 100 and 70 tokens and 45 steps behind them, one token a slot, pages of 16: nine complete pages of sequence 1 were packed, and of
    the bf16 pages that it gave back for them another sequence holds one (18 pages serve all three)."""

    def __init__(self, n_pages=18, steps=45):
        self.wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_rows", batch=3, d_model=96, n_heads=8, d_head=64, r=128, d_rope=32, stride=1, prefix=8, steps=4)
        self.packed, self.flat, self.wts = sessions(self.wl, page_slots=16, max_slots=160, keep=0, n_pages=n_pages)
        self.make, self.lens = tokens(self.wl, 5), np.array([40, 100, 70], np.int64)
        self.out = torch.empty(3, 8, 64, dtype=torch.bfloat16, device="cuda")
        x = self.make(100)
        n = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.hold = [self.packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=torch.empty(3, 100, 8, 64, device="cuda"), n_new=n)]
        self.flat.append(x["c"], x["kr"], n_new=n)
        for _ in range(steps):
            self.step()
        self.check("as served")

    def step(self, check=False):
        x = self.make(1)
        q, qr = x["q"][:, 0].contiguous(), x["q_rope"][:, 0].contiguous()
        self.packed.step(x["c"], x["kr"], q, qr, out=self.out)
        self.flat.append(x["c"], x["kr"])
        self.lens += 1
        if check:
            check_out(self.packed, self.flat, self.wts, self.lens, q, qr, self.out, "a step")

    def prompt(self, row, n, past=0):
        x = self.make(n)
        sub = {k: v[row:row + 1].contiguous() for k, v in x.items()}
        self.hold.append(self.packed.prefill(sub["q"], sub["q_rope"], sub["c"], sub["kr"], out=torch.empty(1, n, 8, 64, device="cuda"), at=row, max_past_slots=past))
        count = torch.zeros(3, dtype=torch.int32, device="cuda")
        count[row] = n
        self.flat.append(x["c"], x["kr"], n_new=count)
        self.lens[row] += n

    def set_len(self, row, n):
        self.packed.seq_len[row] = n
        self.flat.seq_len[row] = n
        self.lens[row] = n

    def check(self, what):
        check_state(self.packed, self.flat, self.lens, what)

    def pages(self, b):
        t = {k: v.cpu().numpy() for k, v in self.packed.pool.tensors.items()}
        return {int(x) for x in t["table"][b, t["first"][b]:t["end"][b]]}

    def stale(self, b, reach):
        """Pages that entries of row b from `reach` to the end of its packed ones name, in other sequences' hands."""
        named = {int(x) for x in self.packed.table[b, reach:int(self.packed.packed.tensors["end"][b])].cpu()}
        return named & set().union(*(self.pages(i) for i in range(3) if i != b))


@pytest.mark.parametrize("n", [20, 7, 150])
def test_a_released_row_takes_the_next_prompt_at_once(n):
    # shorter than what was there (also than a page), and longer
    s = Served()
    assert s.stale(1, 2), "the case is none: no other sequence holds a page that the row still names"
    s.packed.release(1)
    s.flat.seq_len[1] = 0
    s.lens[1] = 0
    s.prompt(1, n)
    s.check("the new prompt")
    assert int(s.packed.packed.tensors["end"][1]) == n // 16
    for _ in range(8):                       # across the end of a page of every sequence
        s.step(check=True)
    s.check("steps behind it")


def test_a_released_row_is_empty_to_unpack():
    s = Served()
    s.packed.release(1)
    s.flat.seq_len[1] = 0
    s.lens[1] = 0
    s.packed.unpack(1, 0, at=1)
    assert not s.pages(1) and int(s.packed.packed.tensors["end"][1]) == 0
    s.check("unpacked")


def test_a_length_that_falls_in_front_of_a_prefill():
    # the row's pages are unpacked, the length falls to the middle of page 3 of nine that were packed, and a prefill continues there
    s = Served()
    lat, _, n4 = rows_of(s.packed, s.flat, 1, int(s.lens[1]))
    assert n4 == 9
    s.packed.unpack(1, 0, at=1)
    s.flat.cache_c[1, :len(lat)] = torch.from_numpy(lat).cuda().bfloat16()      # (rounded as they were packed)
    s.set_len(1, 50)
    s.prompt(1, 20, past=50)
    assert int(s.packed.packed.tensors["end"][1]) == 4
    s.check("continued")
    s.step(check=True)


@pytest.mark.parametrize("as_tensor", [False, True])
def test_an_order_that_leaves_pages_out(as_tensor):
    # pages 3, 1 and 5 of eight, in this order, and no other: neither the ones left out nor the page that refused appends go to
    order = torch.tensor([3, 1, 5]) if as_tensor else [3, 1, 5]
    s = PackedSession(n_heads=8, d_head=64, r=128, d_rope=32, d_hyper=64, stride=1, max_batch=4, max_slots=48, page_slots=16, n_pages=8, n_packed_pages=4,
                      page_order=order)
    s.fit(4, 1, counts=torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda"))
    assert s.device_status() == B.MTLA_OK and s.table[1, 0] == 3 and s.table[2, 0] == 1
    s.fit(4, 1)
    assert s.refused() == (1, 0) and s.device_status() == B.MTLA_ERR_CAPACITY
    t = s.pool.tensors
    assert s.table[0, 0] == 5 and t["end"].tolist() == [1, 1, 1, 0] and s.table[3, 0] == 8       # (the page behind the pool's eight)
    s.fit(4)
    assert s.device_status() == B.MTLA_OK and int(t["state"][1]) == 3
    assert sorted(t["ring"][[(int(t["state"][0]) + i) % 9 for i in range(3)]].tolist()) == [1, 3, 5]


@pytest.mark.parametrize("order", [[0, 1, 1], [0, 8], [-1, 2], list(range(9)), [[0, 1]], [0.5, 1.0]])
def test_orders_that_are_none(order):
    with pytest.raises((ValueError, TypeError)):
        PackedSession(n_heads=8, d_head=64, r=128, d_rope=32, d_hyper=64, stride=1, max_batch=4, max_slots=48, page_slots=16, n_pages=8, n_packed_pages=4,
                      page_order=order)


def test_a_prefill_that_lacked_pages_says_how_many():
    # six bf16 pages: prompts of 40, 30 and 33 tokens need 3 + 2 + 3, so the third gets none (its tokens go to the page that is nobody's).  The fit behind
    # the prefill refuses nobody, and must not hide that; no row of the others is harmed
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_refused", batch=3, d_model=96, n_heads=8, d_head=64, r=128, d_rope=32, stride=1, prefix=8, steps=4)
    packed, flat, _ = sessions(wl, page_slots=16, max_slots=160, keep=0, n_pages=6)
    make, n = tokens(wl, 3), torch.tensor([40, 30, 33], dtype=torch.int32, device="cuda")
    x = make(40)
    hold = packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=torch.empty(3, 40, 8, 64, device="cuda"), n_new=n)
    flat.append(x["c"], x["kr"], n_new=n)
    assert packed.refused()[0] == 1 and packed.device_status() == B.MTLA_ERR_CAPACITY
    packed.release(2)
    flat.seq_len[2] = 0
    packed.fit(3)
    check_state(packed, flat, [40, 30, 0], "the others")          # (refused() == (0, 0) among it)
    del hold


def test_a_prefill_that_found_room_behind_its_packing():
    # the packed pool holds two pages: the second prompt's do not fit, and stay bf16; nothing is lost, and both pools say what they refused
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_refused", batch=2, d_model=96, n_heads=8, d_head=64, r=128, d_rope=32, stride=1, prefix=8, steps=4)
    packed, flat, _ = sessions(wl, page_slots=16, max_slots=160, keep=0, n_pages=12, n_packed=2)
    make, n = tokens(wl, 3), torch.tensor([40, 70], dtype=torch.int32, device="cuda")
    x = make(70)
    hold = packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=torch.empty(2, 70, 8, 64, device="cuda"), n_new=n)
    assert packed.refused() == (0, 1) and packed.device_status() == B.MTLA_ERR_CAPACITY
    assert packed.packed.tensors["end"].tolist() == [2, 0] and packed.pool.tensors["first"].tolist() == [2, 0]
    packed.unpack(1, 8, at=1)                                     # alone: what the last call lacked
    assert packed.refused() == (0, 1) and packed.device_status() == B.MTLA_ERR_CAPACITY
    packed.unpack(1, 8)
    assert packed.refused() == (0, 0) and packed.device_status() == B.MTLA_OK
    del hold


@pytest.mark.parametrize("n_pages,n_packed", [(3, 9), (4, 3), (3, 3), (6, 9)])
def test_pools_that_run_out_while_serving(n_pages, n_packed):
    # rows of 20, 10 and no tokens go on by 40: what the rules by plain loops refuse, step by step, in either pool.  A token of a row without a page lies in the
    # page that is nobody's; rows that never lacked one stay what they should be
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_out", batch=3, d_model=96, n_heads=8, d_head=64, r=128, d_rope=32, stride=1, prefix=8, steps=4)
    packed, flat, _ = sessions(wl, page_slots=16, max_slots=96, keep=0, n_pages=n_pages, n_packed=n_packed)
    make, n = tokens(wl, 11), torch.tensor([20, 10, 0], dtype=torch.int32, device="cuda")
    x = make(20)
    hold = packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=torch.empty(3, 20, 8, 64, device="cuda"), n_new=n)
    flat.append(x["c"], x["kr"], n_new=n)
    ref = P.Pool(3, 6, np.random.default_rng(0).permutation(n_pages), n_pages + 1, n_pages)
    ref4 = P.Pool(3, 6, np.arange(n_packed))
    fit = lambda lens, new, four=ref4, most=1: P.fit(ref, four, lens, new, page_slots=16, stride=1, max_slots=96, keep=0, batch=3, n_max=most)
    fit([0] * 3, [0] * 3), fit([0] * 3, [20, 10, 0], None, 20), fit([20, 10, 0], [0] * 3)
    lens, out = np.array([20, 10, 0]), torch.empty(3, 8, 64, dtype=torch.bfloat16, device="cuda")
    lost, spilled, refused4 = set(), 0, 0
    assert packed.device_status() == B.MTLA_OK
    for t in range(40):
        x = make(1)
        packed.step(x["c"], x["kr"], x["q"][:, 0].contiguous(), x["q_rope"][:, 0].contiguous(), out=out)
        flat.append(x["c"], x["kr"])
        rows = fit(lens, [1] * 3)
        assert packed.refused() == (ref.refused, ref4.refused), t
        assert packed.device_status() == (B.MTLA_ERR_CAPACITY if ref.refused or ref4.refused else B.MTLA_OK), t
        refused4 += ref4.refused
        where = {}
        for b in range(3):
            if rows[b, 0] < 0:                      # its token has no page
                assert int(packed.table[b, lens[b] // 16]) == n_pages
                where.setdefault(int(lens[b]) % 16, []).append(b)
                lost.add(b)
                spilled += 1
        for slot, who in where.items():             # (of two tokens of one slot either one)
            assert any(torch.equal(packed.pool_c[n_pages, slot], flat.cache_c[b, lens[b]]) for b in who), t
        lens += 1
        for b in set(range(3)) - lost:
            lat, _, n4 = rows_of(packed, flat, b, int(lens[b]))
            assert n4 == int(ref4.end[b])
            t16, t4 = packed.table[b].long(), packed.packed.tensors["table"][b].long()
            got = packed.pool_c[t16[n4:-(-int(lens[b]) // 16)]].reshape(-1, 128)[:int(lens[b]) - 16 * n4].double().cpu().numpy()
            assert np.array_equal(got, lat[16 * n4:]), (t, b)
            if n4:
                c, _ = P.page_rows(packed.codes[t4[:n4]].cpu().numpy(), packed.scales[t4[:n4]].cpu().numpy(), packed.keys[t4[:n4]].double().cpu().numpy())
                assert np.array_equal(c.reshape(-1, 128), lat[:16 * n4]), (t, b)
    assert (spilled > 0) == (n_pages < 6) and (refused4 > 0) == (n_packed < 9)
    del hold
