"""GPU tests of packed pages through the C-ABI: pages into 4 bits and back against the format's definition, decode attention over both kinds
of page against float64, and both where they can go wrong: rows that hold NaN behind the last slot, lengths and counts outside their range, tables
that hold anything, chunks and pages that end inside a tile."""
import math

import numpy as np
import pytest
import torch

from paper_2505_13544_amd import binding as B
from tests import packed_reference as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN_BITS, POOL_SPARE = 0x7fc0, 3


def stream():
    return torch.cuda.current_stream().cuda_stream


def context(*, n_heads=4, d_head=64, r=128, d_rope=32, stride=1, max_batch, max_slots, page_slots, n_pages):
    ctx = B.Context(n_heads=n_heads, d_head=d_head, r=r, d_rope=d_rope, d_hyper=64, stride=stride, max_batch=max_batch, max_slots=max_slots,
                    dtype="bf16", page_slots=page_slots, n_pages=n_pages)
    ws = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
    ctx.workspace_init(ws, stream())
    return ctx, ws


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def bits_to_bf16(bits):
    return dev(np.ascontiguousarray(bits, np.uint16).view(np.int16)).view(torch.bfloat16)


def bf16_bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


# ------------------------------------------------------------------------------------------- pack, unpack
def every_number(rng, rows, r):
    """bf16 patterns [rows, r]: all finite ones over and over, first by magnitude (a block's numbers alike), then anyhow."""
    n = rows * r
    by_size = np.sort(np.tile(np.r_[0:0x7f80], n // 0x7f80 + 1)[: n // 2])
    sign = rng.integers(0, 2, n // 2) << 15
    normal = (rng.normal(size=n - n // 2).astype(np.float32) * np.exp2(rng.integers(-3, 3, n - n // 2)).astype(np.float32)).view(np.uint32) >> 16
    return np.concatenate([by_size | sign, normal]).astype(np.uint16).reshape(rows, r)


@pytest.mark.parametrize("r,d_rope,page_slots", [(512, 64, 64), (256, 32, 16), (128, 64, 32), (64, 32, 128)])
def test_pack_and_unpack_follow_the_format(r, d_rope, page_slots):
    rng = np.random.default_rng(r + page_slots)
    Bn, mp, n_pages, n4 = 3, 4, 16, 11
    lat = every_number(rng, n_pages * page_slots, r).reshape(n_pages, page_slots, r)
    keys = rng.integers(0, 1 << 16, (n_pages, page_slots, d_rope)).astype(np.uint16)
    lat[2, 5, 40] = NAN_BITS                     # (page 2 is one of those that are packed)
    lat[2, 6, 3], lat[2, 7, 33] = 0x7f80, 0xff80
    lat[2, 8] = 0x8000                           # a row of negative zeros
    ctx, _ = context(r=r, d_rope=d_rope, max_batch=Bn, max_slots=mp * page_slots, page_slots=page_slots, n_pages=n_pages)
    table = np.array([[2, 7, 1, 99], [4, -5, 3, 6], [8, 9, 10, 11]], np.int32)          # out of range: clamped
    table4 = np.array([[0, 1, 2, 3], [4, 5, 6, 7], [8, 99, -1, 10]], np.int32)
    first, end = np.array([0, -3, 3], np.int32), np.array([3, 2, 77], np.int32)         # pages 0-2; 0-1; 3
    cache_c, cache_kr = bits_to_bf16(lat), bits_to_bf16(keys)
    codes = torch.full((n4, page_slots // 16, r // 32, 16, 16), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((n4, page_slots // 16, r // 32, 16), 0x5A, dtype=torch.uint8, device=DEV)
    keys4 = bits_to_bf16(np.full((n4, page_slots // 16, d_rope // 8, 16, 8), 0x1234, np.uint16))
    pk = B.PackedCache(codes, scales, keys4, dev(table4))
    ctx.pages_pack(cache_c, cache_kr, dev(table), pk, dev(first), dev(end), Bn, 1, stream())
    torch.cuda.synchronize()
    moved = [(2, 0), (7, 1), (1, 2), (4, 4), (0, 5), (11, 10)]
    C, S, K = codes.cpu().numpy(), scales.cpu().numpy(), bf16_bits(keys4)
    for page, to in moved:
        x = P.bf16_to_f64(lat[page])
        for t in range(page_slots // 16):
            tile = x[16 * t:16 * t + 16].reshape(16, r // 32, 32)
            good = np.isfinite(tile).all(-1)
            want, scale = P.packed_blocks(np.where(good[..., None], tile, 0.0))
            byte = C[to, t].transpose(1, 0, 2)                                          # [slot, block, 16]
            got = np.stack([byte & 15, byte >> 4], -1).reshape(16, r // 32, 32)
            assert np.array_equal(S[to, t].T, np.where(good, scale, 255)), (page, t)
            assert np.array_equal(got[good], want[good]), (page, t)
            assert np.array_equal(K[to, t].transpose(1, 0, 2).reshape(16, d_rope), keys[page, 16 * t:16 * t + 16])
    for to in set(range(n4)) - {to for _, to in moved}:                                 # nothing else is written
        assert (C[to] == 0xA5).all() and (S[to] == 0x5A).all() and (K[to] == 0x1234).all()
    assert np.array_equal(bf16_bits(cache_c), lat) and np.array_equal(bf16_bits(cache_kr), keys)

    # ... and back, into other pages
    back = np.array([[12, 13, 14, 0], [15, 3, 5, 6], [8, 9, 10, 6]], np.int32)
    ctx.pages_unpack(cache_c, cache_kr, dev(back), pk, dev(first), dev(end), Bn, 3, stream())
    torch.cuda.synchronize()
    got_c, got_k = cache_c.float().cpu().numpy().astype(np.float64), bf16_bits(cache_kr)
    where = [(0, 12), (1, 13), (2, 14), (4, 15), (5, 3), (10, 6)]
    rows, _ = P.page_rows(C[[a for a, _ in where]], S[[a for a, _ in where]], np.zeros(K[[a for a, _ in where]].shape))
    for i, (a, to) in enumerate(where):
        assert np.array_equal(got_c[to], rows[i], equal_nan=True), (a, to)
        assert np.array_equal(got_k[to], keys[dict((t, p) for p, t in moved)[a]])
    untouched = sorted(set(range(n_pages)) - {to for _, to in where})
    assert np.array_equal(bf16_bits(cache_c)[untouched], lat[untouched]) and np.array_equal(got_k[untouched], keys[untouched])


def test_packing_many_pages_with_a_small_launch():
    # pages_each 0 and 1 size the launch only: 40 pages of each sequence are moved
    ps, r, Bn, mp = 16, 64, 2, 40
    ctx, _ = context(r=r, max_batch=Bn, max_slots=mp * ps, page_slots=ps, n_pages=Bn * mp)
    lat = torch.randn(Bn * mp, ps, r, device=DEV).bfloat16()
    kr = torch.randn(Bn * mp, ps, 32, device=DEV).bfloat16()
    table = torch.randperm(Bn * mp, device=DEV).int().view(Bn, mp)
    outs = []
    for each in (0, 1, 3, 40, 1 << 30):
        pk = B.PackedCache(torch.zeros(Bn * mp, 1, 2, 16, 16, dtype=torch.uint8, device=DEV), torch.zeros(Bn * mp, 1, 2, 16, dtype=torch.uint8, device=DEV),
                           torch.zeros(Bn * mp, 1, 4, 16, 8, dtype=torch.bfloat16, device=DEV), table.flip(1).contiguous())
        ctx.pages_pack(lat, kr, table, pk, None, torch.tensor([40, 39], dtype=torch.int32, device=DEV), Bn, each, stream())
        outs.append(pk.tensors)
    torch.cuda.synchronize()
    assert (outs[0]["scales"] > 0).all(-1).all(-1).all(-1).sum() == 79
    for o in outs[1:]:
        for k in ("codes", "scales", "keys"):
            assert torch.equal(o[k], outs[0][k])


# ------------------------------------------------------------------------------------------- attention
class Case:
    """Sequences of `lens` tokens whose first packed[b] pages are packed ones; what no slot needs holds NaN, table entries beyond it anything."""

    def __init__(self, *, n_heads, d_head, r, d_rope, stride, page_slots, lens, packed, max_slots, seed=0, chunk=None, scale=0.0, spread=4.0):
        rng = np.random.default_rng(seed)
        self.__dict__.update(n_heads=n_heads, d_head=d_head, r=r, d_rope=d_rope, stride=stride, page_slots=page_slots, lens=lens, max_slots=max_slots)
        Bn, ps = len(lens), page_slots
        self.batch, mp = Bn, -(-max_slots // ps)
        self.live = [min(-(-max(n, 0) // stride), max_slots) for n in lens]
        self.packed = packed
        in4 = [min(max(p, 0), mp, -(-n // ps)) for p, n in zip(packed, self.live)]       # pages that are really read there
        in16 = [max(-(-n // ps) - p, 0) for n, p in zip(self.live, in4)]
        n4, n16 = sum(in4) + POOL_SPARE, sum(in16) + POOL_SPARE
        o4, o16 = list(rng.permutation(n4)), list(rng.permutation(n16))
        table = rng.integers(-1 << 31, 1 << 31, (Bn, mp)).astype(np.int32)
        table4 = rng.integers(-1 << 31, 1 << 31, (Bn, mp)).astype(np.int32)
        lat = np.full((n16, ps, r), NAN_BITS, np.uint16)
        kr = np.full((n16, ps, d_rope), NAN_BITS, np.uint16)
        codes = rng.integers(0, 256, (n4, ps // 16, r // 32, 16, 16)).astype(np.uint8)
        scales = np.full((n4, ps // 16, r // 32, 16), 255, np.uint8)
        keys = np.full((n4, ps // 16, d_rope // 8, 16, 8), NAN_BITS, np.uint16)
        to_bits = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)
        for b in range(Bn):
            for k in range(in4[b] + in16[b]):
                n = min(ps, self.live[b] - k * ps)
                if k < in4[b]:
                    page = table4[b, k] = o4.pop()
                    for s in range(n):
                        scales[page, s // 16, :, s % 16] = rng.integers(123, 127, r // 32)
                        keys[page, s // 16, :, s % 16] = to_bits(rng.normal(size=(d_rope // 8, 8)))
                else:
                    page = table[b, k] = o16.pop()
                    lat[page, :n], kr[page, :n] = to_bits(rng.normal(size=(n, r))), to_bits(rng.normal(size=(n, d_rope)))
        self.ctx, self.ws = context(n_heads=n_heads, d_head=d_head, r=r, d_rope=d_rope, stride=stride, max_batch=Bn + 1, max_slots=max_slots,
                                    page_slots=ps, n_pages=n16)
        if chunk:
            self.ctx.set_decode_chunk(chunk)
            self.ws = torch.empty(self.ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
            self.ctx.workspace_init(self.ws, stream())
        self.cache_c, self.cache_kr = bits_to_bf16(lat), bits_to_bf16(kr)
        self.table, self.seq_len = dev(table), dev(np.array(lens, np.int32))
        self.pk = B.PackedCache(dev(codes), dev(scales), bits_to_bf16(keys), dev(table4), dev(np.array(packed, np.int32)))
        bf = lambda *shape, s=1.0: torch.from_numpy(rng.normal(size=shape) * s).to(DEV).bfloat16()
        # logits of a standard deviation of about `spread`
        self.q, self.q_rope = bf(Bn, n_heads, d_head, s=spread / 2), bf(Bn, n_heads, d_rope)
        self.w_uk, self.w_uv = bf(n_heads, r, d_head, s=r ** -0.5), bf(n_heads, d_head, r, s=r ** -0.5)
        # what the kernels should read, in float64
        f64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        lat4, key4 = P.page_rows(codes, scales, P.bf16_to_f64(keys))
        lat16, key16 = P.bf16_to_f64(lat), P.bf16_to_f64(kr)
        self.rows = []
        for b in range(Bn):
            p = [(lat4[table4[b, k]], key4[table4[b, k]]) if k < in4[b] else (lat16[table[b, k]], key16[table[b, k]]) for k in range(in4[b] + in16[b])]
            n = self.live[b]
            self.rows.append((np.concatenate([x for x, _ in p])[:n], np.concatenate([x for _, x in p])[:n]) if p else (np.zeros((0, r)), np.zeros((0, d_rope))))
        self.f64 = {k: f64(getattr(self, k)) for k in ("q", "q_rope", "w_uk", "w_uv")}

    def run(self, out=True, latent=True, lse=True, ws=None):
        Bn, H = self.batch, self.n_heads
        full = lambda *s, dt=torch.float32: torch.full(s, 7.0, dtype=dt, device=DEV)
        o = full(Bn + 1, H, self.d_head, dt=torch.bfloat16) if out else None             # (one row more than the call has)
        ol = full(Bn + 1, H, self.r) if latent else None
        ls = full(Bn + 1, H) if lse else None
        self.ctx.decode_attn_packed(self.q, self.q_rope, self.w_uk, self.w_uv if out else None, self.cache_c, self.cache_kr, self.seq_len, self.table,
                                    self.pk, Bn, o, ol, ls, self.ws if ws is None else ws, stream())
        torch.cuda.synchronize()
        for t in (o, ol, ls):
            assert t is None or bool((t[Bn] == 7).all()), "rows behind the batch are written"
        return [None if t is None else t[:Bn].double().cpu().numpy() for t in (o, ol, ls)]

    def check(self, what=""):
        o, ol, ls = self.run()
        for b in range(self.batch):
            ro, rl, rs, bd = P.attend(self.f64["q"][b], self.f64["q_rope"][b], self.f64["w_uk"], self.f64["w_uv"], *self.rows[b], 1 / math.sqrt(self.d_head))
            where = f"{what} sequence {b} of {self.live[b]} slots"
            if self.live[b] == 0:
                assert not o[b].any() and not ol[b].any() and np.all(np.isneginf(ls[b])), where
                continue
            # logits: q~ as two bf16 numbers (off by 2^-17 of itself, 2^-16 allows for its own sum), sums of r + d_R terms in fp32
            # (over packed pages off by 2^-18.9 of the largest of 32, three to four times the mean of normal numbers: 2^-17 of itself on average)
            de = bd["logit"] * (2.0 ** -16 + (self.r + self.d_rope + self.d_head) * 2.0 ** -24) + 2.0 ** -22
            # weights: twice that (in the sum and in its normaliser), and 2^-16 for their own two bf16 numbers; partials: half (2^-11)
            dp = 2 * de + 2.0 ** -16
            dl = (dp + 2.0 ** -11)[:, None] * bd["latent"] + 2.0 ** -24
            assert np.all(np.abs(ls[b] - rs) <= de + 2.0 ** -20 * np.maximum(1, np.abs(rs))), where
            assert np.all(np.abs(ol[b] - rl) <= dl), f"{where}: latent {(np.abs(ol[b] - rl) - dl).max()}"
            # the value projection adds r terms of fp32; the output is rounded to bf16 (2^-8)
            do = np.einsum("hkr,hr->hk", np.abs(self.f64["w_uv"]), dl + self.r * 2.0 ** -24 * bd["latent"])
            assert np.all(np.abs(o[b] - ro) <= do + 2.0 ** -8 * (np.abs(ro) + do)), f"{where}: out {np.abs(o[b] - ro).max()}"
            # as a whole: the rounding of the output, and of the partials, are the largest errors
            assert np.linalg.norm(o[b] - ro) <= 2.0 ** -7 * np.linalg.norm(ro), where
            assert np.linalg.norm(ol[b] - rl) <= 2.0 ** -10 * np.linalg.norm(rl), where
        return o, ol, ls


SHAPES = [  # n_heads, d_head, r, d_rope, stride, page_slots
    (4, 64, 64, 32, 2, 16), (16, 64, 64, 64, 1, 32), (17, 128, 64, 32, 3, 16), (32, 64, 64, 64, 2, 64),
    (1, 64, 128, 32, 1, 16), (8, 128, 128, 64, 2, 32), (20, 64, 128, 32, 3, 16), (8, 64, 256, 32, 2, 64),
    (16, 128, 256, 64, 4, 16), (31, 64, 256, 32, 1, 32), (16, 128, 512, 64, 2, 64), (5, 64, 512, 32, 2, 16),
    (32, 128, 512, 64, 4, 32), (33, 64, 128, 32, 2, 32), (64, 64, 256, 64, 2, 16), (48, 128, 512, 64, 1, 16),
    (8, 32, 128, 32, 2, 16), (12, 96, 256, 32, 2, 32), (6, 256, 512, 64, 2, 64)]


@pytest.mark.parametrize("n_heads,d_head,r,d_rope,stride,page_slots", SHAPES)
def test_attention_over_both_kinds_of_page(n_heads, d_head, r, d_rope, stride, page_slots):
    ps, s = page_slots, stride
    slots = [0, 1, 15, 16, 17, ps - 1, ps, ps + 1, 3 * ps, 4 * ps + 15, 5 * ps + 1, 300]
    # all complete pages; none; half of them; also the one that is being written to (its rows beyond the last slot hold NaN)
    packed = [n // ps for n in slots]
    for i in (4, 9):
        packed[i] = 0
    for i in (8, 10):
        packed[i] = packed[i] // 2
    packed[7], packed[11] = 2, -(-300 // ps)
    lens = [max(0, n * s - (i % s if n else 0)) for i, n in enumerate(slots)]
    Case(n_heads=n_heads, d_head=d_head, r=r, d_rope=d_rope, stride=s, page_slots=ps, lens=lens, packed=packed, max_slots=max(slots) + ps + 3, seed=n_heads + r).check()


@pytest.mark.parametrize("chunk", [32, 96, 1024, 2048])
@pytest.mark.parametrize("n_heads,r", [(8, 64), (16, 256), (24, 512)])
def test_attention_in_chunks(n_heads, r, chunk):
    # one long sequence beside short ones; with pages of 16 slots a chunk of 2048 has more table entries than a wavefront has lanes
    slots = [3000, 33, 0, 1025, 2047]
    packed = [187, 1, 0, 40, 127]
    Case(n_heads=n_heads, d_head=64, r=r, d_rope=32, stride=1, page_slots=16, lens=slots, packed=packed, max_slots=3001, chunk=chunk, seed=chunk).check()


def test_counts_and_lengths_outside_their_range():
    # lengths below zero and beyond the capacity count as the nearer end, and so does the number of packed pages
    c = Case(n_heads=8, d_head=64, r=128, d_rope=32, stride=2, page_slots=16, lens=[-5, 1 << 30, 400, 77, 0, 130], packed=[3, 1 << 30, -9, 99, 5, 2],
             max_slots=100)
    assert c.live == [0, 100, 100, 39, 0, 65]
    c.check()


def test_peaked_and_flat_logits_and_a_reference_that_moves():
    # weights that differ by more than 2^40 inside a chunk move the softmax reference
    for spread in (0.0, 60.0):
        c = Case(n_heads=16, d_head=64, r=256, d_rope=32, stride=1, page_slots=16, lens=[700, 64, 5], packed=[43, 3, 0], max_slots=704, spread=spread, chunk=352)
        c.check(f"spread {spread}")


def test_a_table_that_holds_anything_stays_inside_the_pools():
    c = Case(n_heads=8, d_head=64, r=256, d_rope=32, stride=1, page_slots=16, lens=[200, 90], packed=[8, 2], max_slots=256)
    n4, n16 = c.pk.n_pages, c.cache_c.shape[0]
    wild = np.array([[-1, 1 << 30, -(1 << 31), (1 << 31) - 1] * 4] * 2, np.int32)
    c.table, table4 = dev(wild), dev(wild)
    c.pk = B.PackedCache(*[c.pk.tensors[k] for k in ("codes", "scales", "keys")], table4, c.pk.tensors["n_packed"])
    for t in (c.pk.tensors["scales"],):
        t.fill_(126)
    c.pk.tensors["keys"].zero_()
    c.cache_c.zero_(), c.cache_kr.zero_()
    f64 = lambda t: t.double().cpu().numpy()
    lat4, key4 = P.page_rows(c.pk.tensors["codes"].cpu().numpy(), c.pk.tensors["scales"].cpu().numpy(), f64(c.pk.tensors["keys"]))
    clamp = lambda k, n: min(max(int(k), 0), n - 1)
    for b in range(2):
        rows = [lat4[clamp(wild[b, k], n4)] if k < (8, 2)[b] else f64(c.cache_c)[clamp(wild[b, k], n16)] for k in range(13)]
        lat = np.concatenate(rows)[:c.live[b]]
        c.rows[b] = (lat, np.zeros((len(lat), 32)))
    c.check()


def test_outputs_one_at_a_time_and_twice():
    c = Case(n_heads=20, d_head=128, r=512, d_rope=64, stride=2, page_slots=32, lens=[900, 3, 64 * 2], packed=[14, 0, 2], max_slots=450)
    o, ol, ls = c.check()
    again = c.run()
    for x, y in zip(again, (o, ol, ls)):
        assert np.array_equal(x, y)                                    # bit for bit
    assert np.array_equal(c.run(latent=False, lse=False)[0], o)
    assert np.array_equal(c.run(out=False, lse=False)[1], ol)
    assert np.array_equal(c.run(out=False, latent=False)[2], ls)


def test_pages_past_two_to_the_31_bytes():
    # 70000 packed pages of 64 slots at r = 512: the codes alone are 1.1 GB, keys 0.57 GB; and a bf16 pool of 40000 pages (2.6 GB)
    free = torch.cuda.mem_get_info()[0]
    if free < 16 << 30:
        pytest.skip("a card with 16 GB free is needed")
    ps, r, dr, H, dh = 64, 512, 64, 8, 64
    n4, n16 = 140000, 40000
    codes = torch.zeros(n4, ps // 16, r // 32, 16, 16, dtype=torch.uint8, device=DEV)
    scales = torch.full((n4, ps // 16, r // 32, 16), 255, dtype=torch.uint8, device=DEV)
    keys = torch.zeros(n4, ps // 16, dr // 8, 16, 8, dtype=torch.bfloat16, device=DEV)
    pool_c, pool_kr = torch.full((n16, ps, r), float("nan"), dtype=torch.bfloat16, device=DEV), torch.zeros(n16, ps, dr, dtype=torch.bfloat16, device=DEV)
    assert codes.numel() > 1 << 31 and pool_c.numel() * 2 > 1 << 31
    ctx, ws = context(n_heads=H, d_head=dh, r=r, d_rope=dr, max_batch=1, max_slots=3 * ps, page_slots=ps, n_pages=n16)
    g = torch.Generator(device=DEV).manual_seed(1)
    src = torch.randn(2, ps, r, generator=g, device=DEV).bfloat16()
    pool_c[n16 - 1], pool_c[n16 - 2] = src[0], src[1]
    table = torch.tensor([[n16 - 1, n16 - 2, n16 - 2]], dtype=torch.int32, device=DEV)
    one = lambda v: torch.tensor([v], dtype=torch.int32, device=DEV)
    pk = B.PackedCache(codes, scales, keys, torch.tensor([[n4 - 1, n4 - 2, 0]], dtype=torch.int32, device=DEV), one(2))
    ctx.pages_pack(pool_c, pool_kr, table, pk, None, one(2), 1, 2, stream())
    ctx.pages_unpack(pool_c, pool_kr, torch.tensor([[n16 - 3, n16 - 4, 0]], dtype=torch.int32, device=DEV), pk, None, one(2), 1, 2, stream())
    q, qr = torch.randn(1, H, dh, generator=g, device=DEV).bfloat16(), torch.randn(1, H, dr, generator=g, device=DEV).bfloat16()
    w_uk, w_uv = ((torch.randn(*s, generator=g, device=DEV) / r ** 0.5).bfloat16() for s in ((H, r, dh), (H, dh, r)))
    out = torch.empty(1, H, dh, dtype=torch.bfloat16, device=DEV)
    ctx.decode_attn_packed(q, qr, w_uk, w_uv, pool_c, pool_kr, one(2 * ps + 5), table, pk, 1, out, None, None, ws, stream())
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()
    lat = np.concatenate([f(pool_c[n16 - 3]), f(pool_c[n16 - 4]), f(src[1])[:5]])
    ro = P.attend(f(q)[0], f(qr)[0], f(w_uk), f(w_uv), lat, np.zeros((len(lat), dr)), 1 / 8)[0]
    assert np.linalg.norm(f(out)[0] - ro) <= 2.0 ** -7 * np.linalg.norm(ro)


def test_queries_with_one_large_number_a_block():
    # the large one meets zeros in the cache, so the logits are what is left of the query beside it.  Its error there: 2^-18.9 of the block's largest times the
    # sum of the block's magnitudes (four planes of 6-bit floats: steps of 1/2, then 1/4 of a sixteenth, 1/4 of a 2^9th and 1/4 of a 2^14th, half of the last)
    H, dh, r = 16, 64, 256
    c = Case(n_heads=H, d_head=dh, r=r, d_rope=32, stride=1, page_slots=16, lens=[200, 48], packed=[12, 3], max_slots=256, spread=2.0, seed=5)
    c.w_uk[:, ::32, :] *= 512
    c.pk.tensors["codes"][..., 0] &= 0xf0                                                   # column 0 of every block
    c.cache_c[..., ::32] = 0
    c.f64["w_uk"] = c.w_uk.double().cpu().numpy()
    o, ol, ls = c.run()
    for b in range(c.batch):
        lat, key = c.rows[b][0].copy(), c.rows[b][1]
        lat[:, ::32] = 0
        ro, rl, rs, bd = P.attend(c.f64["q"][b], c.f64["q_rope"][b], c.f64["w_uk"], c.f64["w_uv"], lat, key, 1 / math.sqrt(dh))
        qt = np.abs(np.einsum("hk,hrk->hr", c.f64["q"][b], c.f64["w_uk"])).reshape(H, r // 32, 32).max(-1)
        planes = (qt @ np.abs(lat).reshape(len(lat), r // 32, 32).sum(-1).T).max(-1) * 2.0 ** -18.9 / math.sqrt(dh)
        de = planes + bd["logit"] * (2.0 ** -16 + (r + 32 + dh) * 2.0 ** -24) + 2.0 ** -22
        assert np.all(planes < 0.5)
        assert np.all(np.abs(ls[b] - rs) <= de + 2.0 ** -20 * np.maximum(1, np.abs(rs)))
        dp = np.exp(2 * de) - 1 + 2.0 ** -16                                                # (a weight and its normaliser)
        assert np.all(np.abs(ol[b] - rl) <= (dp + 2.0 ** -11)[:, None] * bd["latent"] + 2.0 ** -24)


def test_numbers_that_are_none_stay_where_they_are():
    # a NaN block of a live slot, and a query with an infinity: their sequence (their head) is NaN, the others are what they were
    c = Case(n_heads=8, d_head=64, r=128, d_rope=32, stride=1, page_slots=16, lens=[100, 90, 64], packed=[6, 5, 4], max_slots=128, seed=9)
    o, ol, ls = c.check()
    page = int(c.pk.tensors["table"][0, 2])
    before = c.pk.tensors["scales"][page, 0, 1, 7].clone()
    c.pk.tensors["scales"][page, 0, 1, 7] = 255
    no, nol, nls = c.run()
    assert np.isnan(no[0]).all() and np.isnan(nls[0]).all()
    for x, y in ((no, o), (nol, ol), (nls, ls)):
        assert np.array_equal(x[1:], y[1:])
    c.pk.tensors["scales"][page, 0, 1, 7] = before
    c.q[1, 3, 5] = float("inf")
    no, nol, nls = c.run()
    assert np.isnan(no[1, 3]).all() and np.isnan(nls[1, 3])
    keep = [i for i in range(8) if i != 3]
    assert np.array_equal(no[1, keep], o[1, keep]) and np.array_equal(no[[0, 2]], o[[0, 2]]) and np.array_equal(nls[[0, 2]], ls[[0, 2]])


@pytest.mark.parametrize("chunk", [256, 288, 1024])
@pytest.mark.parametrize("n_heads,d_rope,page_slots,slots,packed", [
    (16, 64, 16, [3000], [187]), (20, 32, 64, [1025, 40], [16, 0]), (5, 64, 32, [64, 0, 2047, 129], [2, 0, 40, 4]), (64, 32, 16, [700], [0]), (33, 64, 128, [1900], [14])])
def test_few_long_sequences_in_wide_workgroups(n_heads, d_rope, page_slots, slots, packed, chunk):
    # up to four groups of heads and sequences at r = 512, chunks of 256 slots and more: eight wavefronts, two groups of them, of which one may have no slot
    Case(n_heads=n_heads, d_head=64, r=512, d_rope=d_rope, stride=1, page_slots=page_slots, lens=slots, packed=packed, max_slots=3001, chunk=chunk, seed=n_heads).check()


def test_a_reference_that_moves_in_wide_workgroups():
    for spread in (0.0, 60.0):
        Case(n_heads=16, d_head=64, r=512, d_rope=32, stride=1, page_slots=16, lens=[900, 70], packed=[50, 4], max_slots=1024, spread=spread, chunk=512).check(f"spread {spread}")
