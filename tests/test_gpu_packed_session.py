"""GPU tests of PackedSession: prompts, steps and requests that come and go over packed pages, beside a contiguous session that appends the same
tokens (its rows are what the pages should hold, packed or not) and float64; whole steps, pages changing hands among them, as a replayed graph; the
library's calls on another stream."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from paper_2505_13544_amd import binding as B
from paper_2505_13544_amd.session import PackedSession
from tests import harness as H
from tests import packed_reference as P

pytestmark = pytest.mark.gpu


def sessions(wl, *, page_slots, max_slots, keep, n_pages=None, n_packed=None, seed=0):
    pages = -(-max_slots // page_slots)
    n_pages = n_pages or wl.batch * pages
    packed = PackedSession(n_heads=wl.n_heads, d_head=wl.d_head, r=wl.r, d_rope=wl.d_rope, d_hyper=wl.d_hyper, stride=wl.stride, max_batch=wl.batch,
                           max_slots=max_slots, page_slots=page_slots, n_pages=n_pages, n_packed_pages=n_packed or wl.batch * pages, keep_pages=keep,
                           page_order=np.random.default_rng(seed).permutation(n_pages))
    flat = H.make_session(wl, max_slots=max_slots)
    wts = W.make_weights(wl, max_slots=max_slots)
    for s in (packed, flat):
        H.upload_weights(s, wts)
    return packed, flat, wts


def rows_of(packed, flat, b, length):
    """Sequence b's slots as the packed session should hold them: (latents, keys) in float64, and how many pages are packed."""
    live, ps = -(-length // packed.stride), packed.page_slots
    f = lambda t: t.double().cpu().numpy()
    lat, key = f(flat.cache_c[b, :live]), f(flat.cache_kr[b, :live])
    n4 = int(packed.packed.tensors["end"][b])
    if n4:
        x = lat[:n4 * ps]
        codes, scale = P.packed_blocks(x.reshape(-1, 32))
        signed = np.concatenate([P.VALUES, -P.VALUES])
        lat = np.concatenate([(signed[codes] * 2.0 ** (scale - 127.0)[:, None]).reshape(x.shape), lat[n4 * ps:]])
    return lat, key, n4


def check_state(packed, flat, lens, what):
    ps = packed.page_slots
    assert packed.device_status() == B.MTLA_OK and packed.refused() == (0, 0), what
    assert torch.equal(packed.seq_len.cpu(), torch.as_tensor(np.asarray(lens, np.int32))), what
    for b, n in enumerate(lens):
        live = -(-int(n) // packed.stride)
        lat, key, n4 = rows_of(packed, flat, b, int(n))
        t, t4 = packed.table[b].long(), packed.packed.tensors["table"][b].long()
        assert int(packed.pool.tensors["first"][b]) == n4, what
        got = packed.pool_c[t[n4:-(-live // ps)]].reshape(-1, packed.r)[:live - n4 * ps].double().cpu().numpy()
        assert np.array_equal(got, lat[n4 * ps:]), f"{what}: bf16 rows of sequence {b}"
        got_k = packed.pool_kr[t[n4:-(-live // ps)]].reshape(-1, packed.d_rope)[:live - n4 * ps].double().cpu().numpy()
        assert np.array_equal(got_k, key[n4 * ps:]), what
        if n4:
            c, k = P.page_rows(packed.codes[t4[:n4]].cpu().numpy(), packed.scales[t4[:n4]].cpu().numpy(), packed.keys[t4[:n4]].double().cpu().numpy())
            assert np.array_equal(c.reshape(-1, packed.r), lat[:n4 * ps]), f"{what}: packed rows of sequence {b}"
            assert np.array_equal(k.reshape(-1, packed.d_rope), key[:n4 * ps]), what


def check_out(packed, flat, wts, lens, q, q_rope, out, what):
    f = lambda t: t.double().cpu().numpy()
    w_uk, w_uv = f(packed.w_uk), f(packed.w_uv)
    for b, n in enumerate(lens):
        lat, key, _ = rows_of(packed, flat, b, int(n))
        ro = P.attend(f(q[b]), f(q_rope[b]), w_uk, w_uv, lat, key, 1 / math.sqrt(packed.d_head))[0]
        # the rounding of the output (2^-8) and of the partials (2^-11) are the largest errors
        assert np.linalg.norm(f(out[b]) - ro) <= 2.0 ** -7 * np.linalg.norm(ro) + 1e-30, f"{what} sequence {b}"


def tokens(wl, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    B_ = wl.batch
    ln = lambda x: torch.nn.functional.layer_norm(x, x.shape[-1:])
    return lambda T: dict(c=ln(n(B_, T, wl.r)).bfloat16(), kr=n(B_, T, wl.d_rope).bfloat16(), q=n(B_, T, wl.n_heads, wl.d_head).bfloat16(),
                          q_rope=n(B_, T, wl.n_heads, wl.d_rope).bfloat16())


SHAPES = [(8, 64, 256, 32, 2, 16, 0), (16, 128, 512, 64, 3, 32, 1), (4, 64, 64, 32, 1, 16, 2), (20, 64, 128, 32, 2, 32, 0)]


@pytest.mark.parametrize("n_heads,d_head,r,d_rope,stride,page_slots,keep", SHAPES)
def test_prompts_steps_and_requests_that_come_and_go(n_heads, d_head, r, d_rope, stride, page_slots, keep):
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed", batch=4, d_model=96, n_heads=n_heads, d_head=d_head, r=r, d_rope=d_rope, stride=stride, prefix=8, steps=4)
    max_slots = 9 * page_slots + 7
    packed, flat, wts = sessions(wl, page_slots=page_slots, max_slots=max_slots, keep=keep)
    make, Bn = tokens(wl, 7), wl.batch
    # prompts: one of no token, one that ends on a page, odd ones
    T = 5 * page_slots * stride
    n = np.array([0, 2 * page_slots * stride, T - 3, 7], np.int32)
    x, n_dev = make(T), torch.from_numpy(n).cuda()
    out = torch.empty(Bn, T, n_heads, d_head, device="cuda")
    hold = packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=out, n_new=n_dev)
    flat_out = torch.empty_like(out)
    hold2 = flat.prefill_chunk(x["q"], x["q_rope"], x["c"], x["kr"], out=flat_out, max_past_slots=0, n_new=n_dev)
    lens = n.astype(np.int64)
    check_state(packed, flat, lens, "prompts")
    assert torch.equal(out, flat_out)                    # the prefill itself reads bf16 rows
    assert int(packed.packed.tensors["end"][2]) == max((T - 3) // stride // page_slots - keep, 0)
    # steps, across slots and pages
    o = torch.empty(Bn, n_heads, d_head, dtype=torch.bfloat16, device="cuda")
    for t in range(page_slots * stride + 3):
        x = make(1)
        q, qr = x["q"][:, 0].contiguous(), x["q_rope"][:, 0].contiguous()
        packed.step(x["c"], x["kr"], q, qr, out=o)
        flat.append(x["c"], x["kr"])
        lens += 1
        if t % 11 == 0 or t > page_slots * stride - 2:
            check_state(packed, flat, lens, f"step {t}")
            check_out(packed, flat, wts, lens, q, qr, o, f"step {t}")
    # sequence 1 leaves; a prompt takes its place while the others stay, with its pages
    packed.release(1)
    flat.seq_len[1] = 0
    lens[1] = 0
    packed.fit(Bn)
    held = packed.pool.tensors["end"] - packed.pool.tensors["first"]
    assert int(held[1]) == 0 and int(packed.packed.tensors["end"][1]) == 0
    x = make(33)
    sub = {k: v[1:2].contiguous() for k, v in x.items()}
    out = torch.empty(1, 33, n_heads, d_head, device="cuda")
    hold = packed.prefill(sub["q"], sub["q_rope"], sub["c"], sub["kr"], out=out, at=1)
    flat.append(x["c"], x["kr"], n_new=torch.tensor([0, 33, 0, 0], dtype=torch.int32, device="cuda"))
    lens[1] = 33
    check_state(packed, flat, lens, "a new prompt")
    # sequences 2 and 3 go on by a prefill over what is packed: it reads the packed rows
    ref_lat = [rows_of(packed, flat, b, int(lens[b]))[0] for b in (2, 3)]
    before = lens.copy()
    x = make(20)
    sub = {k: v[2:].contiguous() for k, v in x.items()}
    out = torch.empty(2, 20, n_heads, d_head, device="cuda")
    past = int(before[2:].max()) // stride
    hold = packed.prefill(sub["q"], sub["q_rope"], sub["c"], sub["kr"], out=out, at=2, max_past_slots=past)
    for i, b in enumerate((2, 3)):                       # the contiguous session's cache with the rows that were packed: the same prefill
        flat.cache_c[b, :len(ref_lat[i])] = torch.from_numpy(ref_lat[i]).cuda().bfloat16()
    flat_out = torch.empty(Bn, 20, n_heads, d_head, device="cuda")
    hold2 = flat.prefill_chunk(x["q"], x["q_rope"], x["c"], x["kr"], out=flat_out, max_past_slots=max(past, int(before.max()) // stride),
                               n_new=torch.tensor([0, 0, 20, 20], dtype=torch.int32, device="cuda"))
    lens[2:] += 20
    torch.cuda.synchronize()
    assert (out - flat_out[2:]).norm() <= 2.0 ** -9 * flat_out[2:].norm()     # (fp16 operands inside: shapes of another size may add in another order)
    assert packed.device_status() == B.MTLA_OK
    for b, n_ in enumerate(lens):                        # packing what was packed before gives the same codes: nothing is rounded twice
        assert int(packed.packed.tensors["end"][b]) == max(int(n_) // stride // page_slots - keep, 0)
    check_state(packed, flat, lens, "continued")
    del hold, hold2


@pytest.mark.parametrize("side_stream", [False, True])
def test_captured_steps_turn_pages_over(side_stream):
    # 40 replays of one captured step: slots open, pages complete, are packed and handed out again, without the host; eager work in between
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_graph", batch=5, d_model=96, n_heads=8, d_head=64, r=256, d_rope=32, stride=1, prefix=8, steps=4)
    max_slots = 16 * 9
    make = tokens(wl, 3)
    start = make(40)
    n0 = torch.tensor([40, 0, 15, 16, 33], dtype=torch.int32, device="cuda")
    feed = [make(1) for _ in range(44)]
    results = []
    for captured in (False, True):
        packed, flat, wts = sessions(wl, page_slots=16, max_slots=max_slots, keep=0, n_pages=5 * 3 + 3)
        hold = packed.prefill(start["q"], start["q_rope"], start["c"], start["kr"], out=torch.empty(5, 40, 8, 64, device="cuda"), n_new=n0)
        buf = {k: v.clone() for k, v in feed[0].items()}
        q, qr = torch.empty(5, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(5, 8, 32, dtype=torch.bfloat16, device="cuda")
        out = torch.empty(5, 8, 64, dtype=torch.bfloat16, device="cuda")
        junk = torch.zeros(1000, device="cuda")
        outs = []

        def load(t):
            for k in ("c", "kr"):
                buf[k].copy_(feed[t][k])
            q.copy_(feed[t]["q"][:, 0]), qr.copy_(feed[t]["q_rope"][:, 0])

        step = lambda: packed.step(buf["c"], buf["kr"], q, qr, out=out)
        side = torch.cuda.Stream() if side_stream else torch.cuda.current_stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for t in range(4):
                load(t)
                step()
                outs.append(out.clone())
            graph = torch.cuda.CUDAGraph()
            if captured:
                state = [x.clone() for x in (packed.seq_len, packed.table)]
                torch.cuda.synchronize()
                with torch.cuda.graph(graph, stream=side if side_stream else None):
                    step()
                torch.cuda.synchronize()
                assert torch.equal(state[0], packed.seq_len) and torch.equal(state[1], packed.table)   # a capture runs nothing
            for t in range(4, 44):
                load(t)
                graph.replay() if captured else step()
                outs.append(out.clone())
                junk.add_(1.0)
                if t % 7 == 0:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert packed.device_status() == B.MTLA_OK
        results.append((torch.stack(outs), packed.seq_len.clone(), packed.packed.tensors["end"].clone(), packed.table.clone(), packed.codes.clone()))
        del hold
    for x, y in zip(*results):
        assert torch.equal(x, y)
    assert results[0][2].tolist() == [(int(n) + 44 - 1) // 16 for n in n0.tolist()]


def test_a_session_out_of_pages_says_so_and_harms_nobody():
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_full", batch=3, d_model=96, n_heads=8, d_head=64, r=128, d_rope=32, stride=1, prefix=8, steps=4)
    packed, flat, wts = sessions(wl, page_slots=16, max_slots=96, keep=0, n_pages=4, n_packed=6)
    make = tokens(wl, 11)
    x = make(32)
    n = torch.tensor([30, 31, 0], dtype=torch.int32, device="cuda")
    hold = packed.prefill(x["q"], x["q_rope"], x["c"], x["kr"], out=torch.empty(3, 32, 8, 64, device="cuda"), n_new=n)
    flat.append(x["c"], x["kr"], n_new=n)
    assert packed.device_status() == B.MTLA_OK
    # 2 + 2 pages are in use, two of them given back by the packing: one for the third sequence's first token, and the second's next page
    out = torch.empty(3, 8, 64, dtype=torch.bfloat16, device="cuda")
    lens = np.array([30, 31, 0])
    refused = 0
    for t in range(20):
        x = make(1)
        packed.step(x["c"], x["kr"], x["q"][:, 0].contiguous(), x["q_rope"][:, 0].contiguous(), out=out)
        flat.append(x["c"], x["kr"])
        lens += 1
        torch.cuda.synchronize()
        a, b4 = packed.refused()
        refused += a + b4
        status = packed.device_status()
        assert (status == B.MTLA_ERR_CAPACITY) == (a + b4 > 0), t
    # sequences 0 and 1 never lacked a page (6 packed ones hold 3 + 3; the third sequence asks behind them): their rows are right
    for b in (0, 1):
        lat, key, n4 = rows_of(packed, flat, b, int(lens[b]))
        t16, t4 = packed.table[b].long(), packed.packed.tensors["table"][b].long()
        c, _ = P.page_rows(packed.codes[t4[:n4]].cpu().numpy(), packed.scales[t4[:n4]].cpu().numpy(), packed.keys[t4[:n4]].double().cpu().numpy())
        assert np.array_equal(c.reshape(-1, 128), lat[:16 * n4])
        got = packed.pool_c[t16[n4:-(-int(lens[b]) // 16)]].reshape(-1, 128)[:int(lens[b]) - 16 * n4].double().cpu().numpy()
        assert np.array_equal(got, lat[16 * n4:])
    del hold


def test_sessions_refuse_what_they_cannot_have():
    wl = W.WORKLOADS["speech_bf16"].scaled(name="packed_bad", batch=2, d_model=96, prefix=8, steps=4)
    kw = dict(n_heads=8, d_head=64, r=256, d_rope=32, d_hyper=64, stride=2, max_batch=2, max_slots=64, page_slots=16, n_pages=8, n_packed_pages=8)
    with pytest.raises(ValueError):
        PackedSession(**kw, keep_pages=-1)
    with pytest.raises(B.MtlaError):
        PackedSession(**{**kw, "page_slots": 24})
    s = PackedSession(**kw)
    with pytest.raises(IndexError):
        s.fit(1, at=2)
    with pytest.raises(B.MtlaError):
        s.fit(3)
