"""GPU tests of what the attention over packed pages keeps of its sums: between the chunks of a sequence they are single precision, with its range.  Inputs
for which every product and sum is exact in 24 bits, and inputs that differ by a power of two alone, whose results then do too."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_packed import Case, context

pytestmark = pytest.mark.gpu

# n_heads, d_head, r, slots, packed pages, chunk (0: the call's own); pages of 16 slots
SHAPES = [(4, 64, 64, [75, 16, 0, 5], [4, 1, 0, 0], 0), (20, 64, 128, [300, 33], [18, 1], 64), (8, 128, 256, [300, 200, 17], [18, 12, 1], 0),
          (16, 128, 512, [300, 64, 129, 31, 90], [18, 4, 8, 1, 0], 96), (16, 64, 512, [700], [43], 256), (12, 96, 128, [300, 33], [18, 2], 64),
          (16, 64, 64, [300] * 20, [18] * 20, 32)]


def case(n_heads, d_head, r, slots, packed, chunk, **kw):
    return Case(n_heads=n_heads, d_head=d_head, r=r, d_rope=32, stride=1, page_slots=16, lens=slots, packed=packed, max_slots=max(slots) + 20, chunk=chunk,
                seed=r + n_heads, **kw)


@pytest.mark.parametrize("n_heads,d_head,r,slots,packed,chunk", SHAPES)
def test_the_mean_of_exact_numbers(n_heads, d_head, r, slots, packed, chunk):
    # a query of zeros gives every slot the weight 1; the latents are multiples of 2^-5 below 8, not negative, so their sums over 700 slots are exact in
    # fp32 (18 bits).  What is left is the division: a reciprocal and a product, a step each at most
    c = case(n_heads, d_head, r, slots, packed, chunk)
    c.q.zero_(), c.q_rope.zero_()
    c.pk.tensors["codes"] &= 0x77
    nan = torch.isnan(c.cache_c)
    c.cache_c.copy_(torch.where(nan, c.cache_c.float(), (c.cache_c.float().abs().clamp(max=7.0) * 32).round() / 32).bfloat16())
    o, ol, ls = c.run()
    for b, n in enumerate(slots):
        if n == 0:
            assert not ol[b].any()
            continue
        lat = np.abs(c.rows[b][0])
        n4 = min(packed[b] * 16, n)
        lat[n4:] = np.round(np.minimum(lat[n4:], 7.0) * 32) / 32
        mean = lat.sum(0) / n
        assert np.all(np.abs(ol[b] - mean) <= 2.0 ** -22 * mean), f"sequence {b}: {(np.abs(ol[b] - mean) / np.maximum(mean, 1e-9)).max()}"
        assert np.all(np.abs(ls[b] - math.log(n)) <= 2.0 ** -20 * max(1.0, math.log(n)))


@pytest.mark.parametrize("power", [20, -20, 60, -60])
@pytest.mark.parametrize("n_heads,d_head,r,slots,packed,chunk", SHAPES)
def test_latents_of_any_size(n_heads, d_head, r, slots, packed, chunk, power):
    # latents times 2^k and queries (not their RoPE part) times 2^-k: the same logits and weights, and outputs times 2^k, bit for bit
    c = case(n_heads, d_head, r, slots, packed, chunk, spread=2.0)
    o, ol, ls = c.check()
    c.q.mul_(2.0 ** -power)
    c.cache_c.mul_(2.0 ** power)
    scales = c.pk.tensors["scales"]
    scales.copy_(torch.where(scales == 255, scales, scales + power if power > 0 else scales - (-power)))
    no, nol, nls = c.run()
    assert np.array_equal(nls, ls)
    assert np.array_equal(nol, np.ldexp(ol, power)) and np.array_equal(no, np.ldexp(o, power))


@pytest.mark.parametrize("n_heads,r,max_batch,max_slots", [(16, 512, 256, 8192), (8, 256, 512, 2048), (20, 128, 64, 32768), (8, 64, 1, 60000), (16, 512, 3, 60000)])
def test_few_short_sequences_in_a_large_context(n_heads, r, max_batch, max_slots):
    # the chunk follows the context's sequences, the call's are fewer and shorter: long chunks of which one is in use, and a join of many pieces that are not there
    slots = [700, 33, 0, 1500][:max_batch]
    c = Case(n_heads=n_heads, d_head=64, r=r, d_rope=32, stride=1, page_slots=64, lens=slots, packed=[10, 0, 0, 23][:max_batch], max_slots=max_slots, seed=r)
    c.ctx, c.ws = context(n_heads=n_heads, d_head=64, r=r, d_rope=32, stride=1, max_batch=max_batch, max_slots=max_slots, page_slots=64,
                          n_pages=c.cache_c.shape[0])
    c.check()


@pytest.mark.parametrize("n_heads,r", [(8, 64), (16, 256), (20, 512), (16, 512)])
def test_a_chunk_that_holds_every_slot(n_heads, r):
    # the largest chunk that can be set is one chunk, and whole sequences in one chunk are the same whatever its size
    c = Case(n_heads=n_heads, d_head=64, r=r, d_rope=32, stride=1, page_slots=16, lens=[300, 33, 0, 64], packed=[17, 1, 0, 4], max_slots=310, chunk=320, seed=r)
    want = c.check()
    for chunk in (1024, 1 << 30, (1 << 31) - 32):
        c.ctx.set_decode_chunk(chunk)
        for x, y in zip(c.run(), want):
            assert np.array_equal(x, y), chunk
