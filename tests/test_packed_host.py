"""Packed pages and page tables on the device: sizes, refusals and the binding's structures, no GPU needed; the scale rule compiled and run on
the host; the tests' own reference against itself and against the host's page book."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2505_13544_amd import binding as B
from tests import packed_reference as P

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_13544_amd", "csrc")
PAGED = dict(n_heads=8, d_head=64, r=256, d_rope=32, d_hyper=64, stride=2, max_batch=16, max_slots=640, dtype="bf16", page_slots=64, n_pages=40)
BAD = B.MTLA_ERR_INVALID_ARG


def pool(max_batch=16, max_pages=10, n_pages=40, **kw):
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)
    t = dict(table=ints(max_batch, max_pages), first=ints(max_batch), end=ints(max_batch), ring=ints(n_pages), state=ints(4), was_end=ints(max_batch))
    return B.PagePool(**{**t, **kw})


def packed(n_pages=7, r=256, d_rope=32, tiles=4, max_batch=16, max_pages=10, counts=True):
    return B.PackedCache(torch.zeros(n_pages, tiles, r // 32, 16, 16, dtype=torch.uint8), torch.zeros(n_pages, tiles, r // 32, 16, dtype=torch.uint8),
                         torch.zeros(n_pages, tiles, d_rope // 8, 16, 8, dtype=torch.bfloat16), torch.zeros(max_batch, max_pages, dtype=torch.int32),
                         torch.zeros(max_batch, dtype=torch.int32) if counts else None)


def edit(structure, **kw):
    for k, v in kw.items():
        setattr(structure, k, v)
    return structure


def test_packed_bytes():
    ctx = B.Context(**PAGED)
    c = packed().tensors
    assert ctx.packed_codes_bytes(7) == c["codes"].numel() == 7 * 64 * 256 // 2
    assert ctx.packed_scales_bytes(7) == c["scales"].numel() == 7 * 64 * 256 // 32
    assert ctx.packed_keys_bytes(7) == 2 * c["keys"].numel() == 7 * 64 * 32 * 2
    assert ctx.packed_codes_bytes(0) == ctx.packed_codes_bytes(-3) == 0
    flat = B.Context(**{**PAGED, "page_slots": 0, "n_pages": 0})
    assert flat.packed_codes_bytes(7) == flat.packed_scales_bytes(7) == flat.packed_keys_bytes(7) == 0
    # a slot of the large layer: 400 bytes instead of 1152
    big = B.Context(**{**PAGED, "r": 512, "d_rope": 64})
    assert (big.packed_codes_bytes(3) + big.packed_scales_bytes(3) + big.packed_keys_bytes(3)) / (3 * 64) == 400


def _fit(ctx, a, **kw):
    return ctx.pages_fit_status(*{**a, **kw}.values())


def test_fit_refuses_before_it_enqueues():
    ctx = B.Context(**PAGED)
    good = dict(pool=pool(), packed=pool(), seq_len=1024, n_new=None, n_new_max=1, keep_pages=0, batch=0, slot_map=None, workspace=1024)
    assert _fit(ctx, good) == BAD                         # batch 0: what else is wrong is refused as well, nothing runs here
    good["batch"] = 16
    for kw in (dict(batch=-1), dict(batch=17), dict(pool=None), dict(seq_len=None), dict(workspace=None), dict(n_new_max=-1), dict(keep_pages=-1),
               dict(slot_map=1024, n_new_max=0)):
        assert _fit(ctx, good, **kw) == BAD, kw
    for field in ("table", "first", "end", "ring", "state"):
        assert _fit(ctx, good, pool=edit(pool(), **{field: None})) == BAD, field
        assert _fit(ctx, good, packed=edit(pool(), **{field: None})) == BAD, field
        both = pool()                                     # two pools are two pools
        assert _fit(ctx, good, pool=both, packed=edit(pool(), **{field: getattr(both, field)})) == BAD, field
    for kw in (dict(n_pages=0), dict(n_pages=-4), dict(spill=40), dict(n_pages=1 << 26, spill=-1)):
        assert _fit(ctx, good, pool=edit(pool(), **kw)) == BAD, kw
        assert _fit(ctx, good, packed=edit(pool(), **kw)) == BAD, kw
    assert _fit(B.Context(**{**PAGED, "page_slots": 0, "n_pages": 0}), good) == BAD


@pytest.mark.parametrize("name", ["pages_pack_status", "pages_unpack_status"])
def test_pack_refuses_before_it_enqueues(name):
    good = dict(cache_c=1024, cache_kr=1024, page_table=1024, packed_cache=packed(), first=None, end=1024, batch=16, pages_each=1)
    go = lambda ctx, **kw: getattr(ctx, name)(*{**good, **kw}.values())
    ctx = B.Context(**PAGED)
    for kw in (dict(batch=0), dict(batch=17), dict(cache_c=None), dict(cache_kr=None), dict(page_table=None), dict(packed_cache=None), dict(end=None),
               dict(pages_each=-1), dict(cache_c=1032), dict(cache_kr=1032)):
        assert go(ctx, **kw) == BAD, kw
    for kw in (dict(codes=None), dict(scales=None), dict(keys=None), dict(table=None), dict(n_pages=0), dict(codes=1032), dict(scales=1025),
               dict(keys=1032), dict(n_pages=1 << 25)):
        assert go(ctx, packed_cache=edit(packed(), **kw)) == BAD, kw
    assert go(B.Context(**{**PAGED, "page_slots": 0, "n_pages": 0})) == BAD


def test_attention_refuses_before_it_enqueues():
    ctx = B.Context(**PAGED)
    a = dict(q=1024, q_rope=1024, w_uk=1024, w_uv=1024, cache_c=1024, cache_kr=1024, seq_len=1024, page_table=1024, packed_cache=packed(), batch=16,
             out=1024, out_latent=None, lse=None, workspace=1024)
    go = lambda c, **kw: c.decode_attn_packed_status(*{**a, **kw}.values())
    bad = [dict(batch=0), dict(batch=17), dict(out=None), dict(w_uv=None), dict(out=None, w_uv=None), dict(packed_cache=None),
           dict(packed_cache=packed(counts=False)), dict(packed_cache=edit(packed(), codes=None)), dict(packed_cache=edit(packed(), n_pages=0)),
           dict(packed_cache=edit(packed(), keys=1032))]
    bad += [{k: None} for k in ("q", "q_rope", "w_uk", "cache_c", "cache_kr", "seq_len", "page_table", "workspace")]
    bad += [{k: 1032} for k in ("q", "q_rope", "w_uk", "w_uv", "cache_c", "cache_kr", "workspace")]
    for kw in bad:
        assert go(ctx, **kw) == BAD, kw
    assert go(B.Context(**{**PAGED, "page_slots": 0, "n_pages": 0})) == BAD
    ctx.set_shared_prefix(1024, 1024, 16)
    assert go(ctx) == B.MTLA_ERR_UNSUPPORTED


def test_step_refuses_before_it_enqueues():
    a = dict(cache_c=1024, cache_kr=1024, tail_c=1024, seq_len=1024, page_table=1024, packed_cache=packed(), c_new=1024, kr_new=1024, hyp_A=1024,
             hyp_a=None, hyp_G=1024, q=1024, q_rope=1024, w_uk=1024, w_uv=1024, batch=16, out=1024, out_latent=None, lse=None, workspace=1024)
    go = lambda c, **kw: c.decode_step_packed_status(*{**a, **kw}.values())
    ctx = B.Context(**PAGED)
    for kw in [{k: None} for k in ("cache_c", "cache_kr", "tail_c", "seq_len", "page_table", "packed_cache", "c_new", "kr_new", "hyp_A", "hyp_G", "q",
                                   "q_rope", "w_uk", "workspace")] + [dict(batch=0), dict(batch=17), dict(out=None)]:
        assert go(ctx, **kw) == BAD, kw


def test_structures_are_structures():
    ctx = B.Context(**PAGED)
    for other in (1024, b"x" * ctypes.sizeof(B.PagePool), bytearray(8), np.zeros(4, np.int32), packed()):
        with pytest.raises((TypeError, BufferError)):
            ctx.pages_fit_status(other, None, 1024, None, 1, 0, 0, None, 1024)
    for other in (1024, bytearray(8), B.mtla_page_book()):
        with pytest.raises((TypeError, BufferError)):
            ctx.pages_pack_status(1024, 1024, 1024, other, None, 1024, 0, 1)
    with pytest.raises(AttributeError):
        ctx.pages_fit_status(pool(), None, np.zeros(16, np.int32), None, 1, 0, 0, None, 1024)


def test_structures_check_their_tensors():
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for kw in (dict(table=torch.zeros(16, 10)), dict(table=ints(16, 20)[:, ::2]), dict(table=ints(160)), dict(first=ints(16).long()), dict(ring=None),
               dict(state=np.zeros(4, np.int32)), dict(was_end=ints(16, 1))):
        with pytest.raises(TypeError):
            pool(**kw)
    for kw in (dict(first=ints(15)), dict(end=ints(17)), dict(was_end=ints(3)), dict(state=ints(3))):
        with pytest.raises(ValueError):
            pool(**kw)
    t = packed().tensors
    for kw in (dict(codes=t["codes"].int()), dict(keys=t["keys"].float()), dict(table=t["table"].t()), dict(n_packed=t["n_packed"].long())):
        with pytest.raises(TypeError):
            B.PackedCache(**{**t, **kw})
    for kw in (dict(scales=t["scales"][:3]), dict(keys=t["keys"][:3]), dict(codes=t["codes"][:, :2].contiguous())):
        with pytest.raises(ValueError):
            B.PackedCache(**{**t, **kw})


PROGRAM = r"""
#include <cstdio>
#include "packed_scale.h"
int main() {
  for (unsigned top = 0; top < 0x8000u; ++top) printf("%u\n", mtla::packed_scale_of(top));
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_scale_rule_for_every_magnitude(tmp_path):
    (tmp_path / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    got = np.array(subprocess.run([str(tmp_path / "main")], check=True, capture_output=True, text=True).stdout.split(), int)
    top = P.bf16_to_f64(np.arange(0x8000))
    for bits in list(range(0, 0x8000, 37)) + list(range(0x7f00, 0x8000)):
        x = np.zeros(32)
        x[5] = top[bits]
        assert got[bits] == P.block(x)[1], hex(bits)
    finite = np.arange(0x7f80)
    scale = 2.0 ** (got[finite].astype(float) - 127)
    assert np.all((top[finite] <= 7 * scale) | (got[finite] == 252)) and np.all((top[finite] > 3.5 * scale) | (got[finite] == 3)) and np.all(got[0x7f80:] == 255)


def test_reference_blocks_agree():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(300, 32)) * 2.0 ** rng.integers(-12, 12, (300, 1))
    x[::3] = np.round(x[::3] * 4) / 4            # ties among them
    x[5] = 0
    codes, scale = P.packed_blocks(x)
    for i in range(len(x)):
        c, s = P.block(x[i])
        assert s == scale[i] and np.array_equal(c, codes[i]), i


@pytest.mark.parametrize("seed", range(6))
def test_reference_tables_are_the_host_books(seed):
    # one pool, lengths that only grow: what mtla_pages_reserve fills, in its order
    rng = np.random.default_rng(seed)
    Bn, ps, stride, max_slots = 7, 16, int(rng.integers(1, 4)), 100
    mp, n_pages = -(-max_slots // ps), 60
    ring = rng.permutation(n_pages).astype(np.int32)
    mine = P.Pool(Bn, mp, ring)
    mine.table[:] = -1
    table, nxt = np.full((Bn, mp), -1, np.int32), np.zeros((Bn, mp), np.int32)
    length, nlen, refs, host_ring = np.zeros(Bn, np.int64), np.zeros(Bn, np.int64), np.zeros(n_pages, np.int32), ring.copy()
    at = lambda x: x.ctypes.data
    book = B.mtla_page_book(at(table), at(nxt), at(length), at(nlen), at(refs), at(host_ring), 0, n_pages, Bn, mp, n_pages, ps, stride, max_slots)
    for _ in range(12):
        n = rng.integers(0, 3 * ps, Bn).astype(np.int32)
        n = np.minimum(n, max_slots * stride - length).astype(np.int32)
        assert B.calls.mtla_pages_reserve(book, n.ctypes.data, Bn) >= 0
        P.fit(mine, None, length, n, page_slots=ps, stride=stride, max_slots=max_slots, keep=0, batch=Bn, n_max=3 * ps)
        length += n
        assert np.array_equal(mine.table, table) and mine.count == book.free_count and mine.head == book.free_head


def test_too_many_chunks_of_a_sequence():
    # 65536 pieces and more of a sequence do not fit a launch
    a = dict(q=1024, q_rope=1024, w_uk=1024, w_uv=1024, cache_c=1024, cache_kr=1024, seq_len=1024, page_table=1024, packed_cache=packed(max_pages=1), batch=0,
             out=1024, out_latent=None, lse=None, workspace=1024)
    ctx = B.Context(**{**PAGED, "max_slots": 32 * 65535 + 1, "stride": 1})
    args = {**a, "packed_cache": packed(max_pages=-(-(32 * 65535 + 1) // 64)), "batch": 16}
    ctx.set_decode_chunk(32)
    assert ctx.decode_attn_packed_status(*args.values()) == B.MTLA_ERR_UNSUPPORTED
    assert ctx.decode_attn_packed_status(*{**args, "batch": 0}.values()) == BAD


CHUNKS = r"""
#include <cstdio>
#include "decode_schedule.h"
int main() {
  int r, b, s, h;
  while (scanf("%d %d %d %d", &r, &b, &s, &h) == 4) {
    const int c = mtla::packed_chunk(r, b, s, h);
    printf("%d %d\n", c, (int)mtla::packed_wide(r, b, h, (s + c - 1) / c, c));
  }
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no host compiler")
def test_chunk_rule(tmp_path):
    (tmp_path / "main.cpp").write_text(CHUNKS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    # the shapes whose times stand beside the rule, then the ends of its range: multiples of 64, 256 of a sequence at most, wide ones on 256 units at most
    shapes = [(512, 8, 8192, 32), (512, 1, 131071, 16), (512, 256, 2048, 16), (256, 16, 640, 8), (64, 1, 75, 4), (512, 1, 65536, 16), (512, 1, 131071, 32),
              (512, 1, 32768, 16), (256, 1, 131071, 16)]
    ends = [(512, 1, 1, 1), (64, 65535, 1, 64), (64, 65535, 32767, 64)] + [(512, b, s, 16) for b in (1, 2, 3, 4, 5) for s in (65535, 65536, 99999, (1 << 31) - 1)]
    run = subprocess.run([str(tmp_path / "main")], input="\n".join("%d %d %d %d" % s for s in shapes + ends), check=True, capture_output=True, text=True)
    got = np.array(run.stdout.split(), int).reshape(-1, 2)
    assert got[:9].tolist() == [[256, 0], [576, 1], [1024, 0], [64, 0], [64, 0], [512, 1], [1088, 1], [192, 0], [512, 0]]
    for (r, b, s, h), (c, wide) in zip(shapes + ends, got):
        chunks = -(-s // c)
        assert c % 64 == 0 and c >= 64 and chunks <= 256
        assert not wide or b * -(-h // 16) * (chunks + 1) <= 256


def test_a_slot_map_of_more_tokens_than_an_index_counts():
    ctx = B.Context(**PAGED)
    good = dict(pool=pool(), packed=None, seq_len=1024, n_new=None, n_new_max=(1 << 30) + 1, keep_pages=0, batch=16, slot_map=1024, workspace=1024)
    for n in ((1 << 30) + 1, (1 << 31) - 1):
        assert _fit(ctx, good, n_new_max=n) == BAD
