"""Serving from a cache whose complete pages are held in 4 bits: what the three operators for it do, as cases that can be timed.

  attend   one new query per sequence over its slots: complete pages out of the packed pool, the rest out of the bf16 pool
  pack     complete pages into the packed pool, and back into pages of bf16
  fit      page tables and slot maps made to fit the requests' lengths, on the device

A packed page holds its latents as 4-bit floats (E2M1) with one power-of-two scale (E8M0) per 32 values of a row, and its RoPE keys in bf16,
all of them in units of 16 slots:
  codes   [pages, page_slots / 16, r / 32, 16, 16]   uint8: 32 values of a slot, the even ones in the low nibbles
  scales  [pages, page_slots / 16, r / 32, 16]       uint8: exponent + 127
  keys    [pages, page_slots / 16, d_rope / 8, 16, 8]
A block's scale is the smallest power of two whose seven-fold its largest magnitude does not exceed (6 is the largest value of the format, and
what lies above is off by no more than half of the step below it); values go to the nearest, ties to the even code.

Inputs are Gaussian tensors of the decoder's shapes, the latents layer-normalised and weighted as the merge weighs them, weights
N(0, 1) / sqrt(fan_in); lengths are spread evenly over their range, in an order that the seed gives.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
D_HYPER = 64

SPEECH = dict(heads=8, d_head=64, r=256, d_rope=32)     # the paper's decoder
LARGE = dict(heads=16, d_head=128, r=512, d_rope=64)    # a language-model layer of width 2048


# --------------------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------------------
def listed():
    return [
        # one sequence of the smallest configuration: the latency of a call
        dict(name="attend_first", kind="attend", heads=4, d_head=64, r=64, d_rope=32, stride=2, page_slots=16, batch=1, lo=150, hi=150, keep=0),
        # 16 utterances in the paper's decoder
        dict(name="attend_speech", kind="attend", **SPEECH, stride=2, page_slots=64, batch=16, lo=1024, hi=1280, keep=0),
        # an odd batch from empty sequences on, two tiles of heads of which the second is part full, small pages, the newest two of them in bf16
        dict(name="attend_odd", kind="attend", heads=20, d_head=64, r=128, d_rope=32, stride=3, page_slots=32, batch=37, lo=0, hi=3001, keep=2),
        # a full serving batch of ragged sequences
        dict(name="attend_ragged", kind="attend", **LARGE, stride=2, page_slots=64, batch=256, lo=512, hi=4096, keep=0),
        # few long documents, 32 heads, the cache compressed four times
        dict(name="attend_long", kind="attend", heads=32, d_head=128, r=512, d_rope=64, stride=4, page_slots=64, batch=8, lo=32768, hi=32768, keep=0),
        # one very long document, uncompressed in time: the work has to be split over one sequence
        dict(name="attend_document", kind="attend", **LARGE, stride=1, page_slots=128, batch=1, lo=131071, hi=131071, keep=1),
        # the pages that a batch of utterances completes at about the same time
        dict(name="pack_step", kind="pack", r=256, d_rope=32, page_slots=64, batch=16, lo=0, hi=2),
        # eight prompts of 4096 tokens, s = 2, as their prefill left them
        dict(name="pack_prompts", kind="pack", r=512, d_rope=64, page_slots=64, batch=8, lo=32, hi=32),
        # the pages of a whole serving batch
        dict(name="pack_batch", kind="pack", r=512, d_rope=64, page_slots=64, batch=256, lo=1, hi=31),
        # a decode step of 16 utterances, pages in both pools
        dict(name="fit_step", kind="fit", stride=2, page_slots=64, batch=16, lo=1024, hi=1280, n_new=1, packed=True, admit=False, keep=0),
        # 256 prompts admitted with the slots of all their tokens, and retired again
        dict(name="fit_admit", kind="fit", stride=2, page_slots=64, batch=256, lo=512, hi=4096, n_new=4096, packed=False, admit=True, keep=0),
        # a step of some thousand requests of very different lengths, eight drafted tokens each
        dict(name="fit_requests", kind="fit", stride=2, page_slots=32, batch=3001, lo=0, hi=16384, n_new=8, packed=True, admit=False, keep=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "pack", "fit"])
    page_slots, stride = rng.choice([16, 32, 64, 64, 128]), rng.choice([1, 2, 2, 3, 4])
    d_head = rng.choice([64, 128])
    r = d_head * rng.choice([2, 4, 4]) if d_head == 128 else rng.choice([64, 128, 256, 256])
    d_rope = d_head // 2
    if kind == "attend":
        heads = rng.choice([4, 8, 12, 16, 20, 32])
        batch = _log(rng, 1, 256)
        most = 300000 * 16 * stride * 256 // (max(16, heads) * max(256, r)) // batch   # tokens of a sequence
        hi = _log(rng, 16, max(17, min(131072, most)))
        return dict(kind=kind, heads=heads, d_head=d_head, r=r, d_rope=d_rope, stride=stride, page_slots=page_slots, batch=batch,
                    lo=hi // rng.choice([1, 1, 2, 8]), hi=hi, keep=rng.choice([0, 0, 1, 2]))
    if kind == "pack":
        batch = _log(rng, 1, 256)
        hi = _log(rng, 1, max(2, min(512, 4000 * 64 // page_slots // batch)))
        return dict(kind=kind, r=r, d_rope=d_rope, page_slots=page_slots, batch=batch, lo=rng.choice([0, hi // 2, hi]), hi=hi)
    batch = _log(rng, 1, 3000)
    admit = rng.random() < 0.4
    hi = _log(rng, 16, max(17, min(16384, (1000000 if admit else 20000000) // batch)))
    return dict(kind=kind, stride=stride, page_slots=page_slots, batch=batch, lo=hi // rng.choice([1, 2, 8]) if admit else rng.choice([0, hi // 2]), hi=hi,
                n_new=hi if admit else rng.choice([1, 1, 2, 5, 8]), packed=False if admit else rng.random() < 0.6, admit=admit,
                keep=0 if admit else rng.choice([0, 0, 1]))


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly spaced, both ends among them."""
    return [int(round(lo + (hi - lo) * i / (n - 1))) if n > 1 else hi for i in range(n)]


def _lengths(case, seed):
    return np.random.default_rng(seed).permutation(_spread(case["lo"], case["hi"], case["batch"])).astype(np.int32)


def _complete(length, case):
    """Complete pages of a sequence, but for the newest `keep`."""
    return np.maximum(length // case["stride"] // case["page_slots"] - case["keep"], 0)


def _pages(length, case):
    """Pages that a sequence's slots reach."""
    slots = -(-length // case["stride"])
    return -(-slots // case["page_slots"])


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _tables(pages, max_pages, rng, n_pages):
    """Rows of page numbers, sequence b's entries first[b] .. end[b] - 1 in `pages`, in an order that a long-running pool of n_pages has."""
    first, end = pages
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.zeros((len(first), max_pages), np.int32)
    at = 0
    for b, (f, e) in enumerate(zip(first, end)):
        table[b, f:e] = order[at:at + e - f]
        at += e - f
    return table


class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32).to(dtype)

    def latents(self, pages, slots, r):
        """Rows as the merge leaves them: layer-normalised latents times weights between 0 and 1, two to a slot."""
        out = torch.empty(pages, slots, r, dtype=torch.bfloat16, device=DEV)
        for lo in range(0, pages, 1024):
            n = min(1024, pages - lo)
            w = torch.rand(n, slots, 1, generator=self.g, device=DEV)
            out[lo:lo + n] = torch.randn(n, slots, r, generator=self.g, device=DEV) * (0.3 + w)
        return out


def prepare(case, seed):
    return {"attend": _prepare_attend, "pack": _prepare_pack, "fit": _prepare_fit}[case["kind"]](case, int(seed))


def _context(case, max_batch, max_slots, n_pages):
    """The library's handle and its workspace, which a program makes once."""
    from paper_2505_13544_amd import binding as B
    ctx = B.Context(n_heads=case.get("heads", 8), d_head=case.get("d_head", 64), r=case.get("r", 256), d_rope=case.get("d_rope", 32),
                    d_hyper=D_HYPER, stride=case.get("stride", 1), max_batch=max_batch, max_slots=max_slots, dtype="bf16",
                    page_slots=case["page_slots"], n_pages=n_pages)
    workspace = torch.empty(ctx.workspace_bytes(), dtype=torch.uint8, device=DEV)
    ctx.workspace_init(workspace, torch.cuda.current_stream().cuda_stream)
    return ctx, workspace


def _prepare_attend(case, seed):
    rng, rnd = np.random.default_rng(seed + 1), _Random(seed)
    B, H, dh, r, dr, ps = (case[k] for k in ("batch", "heads", "d_head", "r", "d_rope", "page_slots"))
    length = _lengths(case, seed)
    max_slots = max(1, -(-case["hi"] // case["stride"]))
    max_pages = -(-max_slots // ps)
    packed, reach = _complete(length, case), _pages(length, case)
    n_pages, n_pages4 = int((reach - packed).sum()) + 3, int(packed.sum()) + 3
    table, table4 = _tables((packed, reach), max_pages, rng, n_pages), _tables((np.zeros_like(packed), packed), max_pages, rng, n_pages4)
    s = dict(case=case, batch=B, max_slots=max_slots, n_pages=n_pages, n_pages4=n_pages4,
             seq_len=_dev(length), table=_dev(table), table4=_dev(table4), n_packed=_dev(packed.astype(np.int32)),
             cache_c=rnd.latents(n_pages, ps, r), cache_kr=rnd.normal(n_pages, ps, dr))
    codes = torch.empty(n_pages4, ps // 16, r // 32, 16, 16, dtype=torch.uint8, device=DEV)
    scales = torch.empty(n_pages4, ps // 16, r // 32, 16, dtype=torch.uint8, device=DEV)
    for lo in range(0, n_pages4, 1024):
        n = min(1024, n_pages4 - lo)
        codes[lo:lo + n], scales[lo:lo + n] = _to_codes(rnd.latents(n, ps, r))
    s.update(codes=codes, scales=scales, keys=rnd.normal(n_pages4, ps // 16, dr // 8, 16, 8),
             q=rnd.normal(B, H, dh), q_rope=rnd.normal(B, H, dr), w_uk=rnd.normal(H, r, dh, dtype=torch.float32).div(math.sqrt(r)).bfloat16(),
             w_uv=rnd.normal(H, dh, r, dtype=torch.float32).div(math.sqrt(r)).bfloat16(),
             out=torch.empty(B, H, dh, dtype=torch.bfloat16, device=DEV))
    if own:
        from paper_2505_13544_amd import binding as L
        s["ctx"], s["workspace"] = _context(case, B, max_slots, n_pages)
        s["packed_cache"] = L.PackedCache(codes, scales, s["keys"], s["table4"], s["n_packed"])
    return s


def _prepare_pack(case, seed):
    rng, rnd = np.random.default_rng(seed + 1), _Random(seed)
    B, r, dr, ps = (case[k] for k in ("batch", "r", "d_rope", "page_slots"))
    end = _lengths(case, seed)
    first = np.minimum(end, rng.integers(0, 3, B)).astype(np.int32)     # some pages were packed before
    max_pages = max(1, int(end.max()))
    n_pages = n_pages4 = int(end.sum()) + 1
    table, table4 = _tables((first, end), max_pages, rng, n_pages), _tables((np.zeros_like(end), end), max_pages, rng, n_pages4)
    s = dict(case=case, batch=B, max_pages=max_pages, n_pages=n_pages, first=_dev(first), end=_dev(end), table=_dev(table), table4=_dev(table4),
             table_back=_dev(table + np.int32(n_pages)),        # the pages that they go back to: the other half of the pool
             cache_c=torch.cat([rnd.latents(n_pages, ps, r), torch.zeros(n_pages, ps, r, dtype=torch.bfloat16, device=DEV)]),
             cache_kr=torch.cat([rnd.normal(n_pages, ps, dr), torch.zeros(n_pages, ps, dr, dtype=torch.bfloat16, device=DEV)]),
             codes=torch.zeros(n_pages4, ps // 16, r // 32, 16, 16, dtype=torch.uint8, device=DEV),
             scales=torch.zeros(n_pages4, ps // 16, r // 32, 16, dtype=torch.uint8, device=DEV),
             keys=torch.zeros(n_pages4, ps // 16, dr // 8, 16, 8, dtype=torch.bfloat16, device=DEV))
    if own:
        from paper_2505_13544_amd import binding as L
        s["ctx"], s["workspace"] = _context(case, B, max_pages * ps, 2 * n_pages)
        s["packed_cache"] = L.PackedCache(s["codes"], s["scales"], s["keys"], s["table4"], s["end"])
    return s


def _pool(max_batch, max_pages, n_pages, rng):
    """A pool nobody holds a page of."""
    return dict(table=torch.zeros(max_batch, max_pages, dtype=torch.int32, device=DEV), first=torch.zeros(max_batch, dtype=torch.int32, device=DEV),
                end=torch.zeros(max_batch, dtype=torch.int32, device=DEV), ring=_dev(rng.permutation(n_pages).astype(np.int32)),
                state=torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=DEV))


def _prepare_fit(case, seed):
    rng = np.random.default_rng(seed + 1)
    B, ps, stride = case["batch"], case["page_slots"], case["stride"]
    length = _lengths(case, seed)
    most = case["hi"] + 2 * stride * ps + case["n_new"]
    max_slots = -(-most // stride)
    max_pages = -(-max_slots // ps)
    if case["admit"]:       # prompts come into an empty pool, and leave it
        before, new = np.zeros_like(length), length
    else:                   # the requests go on by some tokens, of which the last ones are drafts: and back
        before, new = length, rng.integers(1, case["n_new"] + 1, B).astype(np.int32)
    after = before if case["admit"] else before + rng.integers(1, stride * ps // 2 + 1, B).astype(np.int32)
    n_pages = int(_pages(length + case["n_new"] + stride * ps // 2, case).sum()) + 2 * B + 8
    s = dict(case=case, batch=B, max_slots=max_slots, max_pages=max_pages, n_pages=n_pages, pool=_pool(B, max_pages, n_pages, rng),
             packed=_pool(B, max_pages, n_pages, rng) if case["packed"] else None,
             seq_len=_dev(after), n_new=_dev(new), n_new_max=int(case["n_new"]), seq_back=_dev(before),
             n_back=_dev(np.zeros_like(new) if case["admit"] else new),
             slot_map=torch.empty(B, case["n_new"], dtype=torch.int64, device=DEV))
    if not case["admit"]:
        _fit_plain(s, s["seq_back"], s["n_back"])
    if own:
        from paper_2505_13544_amd import binding as L
        s["ctx"], s["workspace"] = _context(case, B, max_slots, n_pages)
        s["pool_"] = L.PagePool(**s["pool"])
        s["packed_"] = L.PagePool(**s["packed"]) if case["packed"] else None
    return s


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["kind"] == "attend":
        if own:
            s["ctx"].decode_attn_packed(s["q"], s["q_rope"], s["w_uk"], s["w_uv"], s["cache_c"], s["cache_kr"], s["seq_len"], s["table"],
                                        s["packed_cache"], s["batch"], s["out"], None, None, s["workspace"], torch.cuda.current_stream().cuda_stream)
            return s["out"]
        return _attend_plain(s)
    if case["kind"] == "pack":
        if own:
            stream = torch.cuda.current_stream().cuda_stream
            s["ctx"].pages_pack(s["cache_c"], s["cache_kr"], s["table"], s["packed_cache"], s["first"], s["end"], s["batch"], case["hi"], stream)
            s["ctx"].pages_unpack(s["cache_c"], s["cache_kr"], s["table_back"], s["packed_cache"], s["first"], s["end"], s["batch"], case["hi"], stream)
        else:
            _pack_plain(s)
        return s["cache_c"], s["cache_kr"]
    # a pass fits the tables to the new lengths and, when the requests have left or their drafts are dropped, to the old ones again
    if own:
        stream = torch.cuda.current_stream().cuda_stream
        s["ctx"].pages_fit(s["pool_"], s["packed_"], s["seq_len"], s["n_new"], s["n_new_max"], case["keep"], s["batch"], s["slot_map"], s["workspace"], stream)
        s["ctx"].pages_fit(s["pool_"], s["packed_"], s["seq_back"], s["n_back"], s["n_new_max"], case["keep"], s["batch"], None, s["workspace"], stream)
    else:
        s["slot_map"] = _fit_plain(s, s["seq_len"], s["n_new"])
        _fit_plain(s, s["seq_back"], s["n_back"])
    return [s["slot_map"]] + [p[k] for p in (s["pool"], s["packed"]) if p for k in ("table", "first", "end", "ring", "state")]


# ---- plain forms
def _grid():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)


def _to_codes(x):
    """[pages, slots, r] -> codes and scales."""
    n, ps, r = x.shape
    v = x.float().view(n, ps // 16, 16, r // 32, 32).transpose(2, 3)                       # [n, tile, block, slot, 32]
    m, k = torch.frexp(v.abs().amax(-1))                                                   # amax = m 2^k, m in [1/2, 1)
    e = torch.where(m > 0, k - 3 + (m > 0.875).int(), -124).clamp(-124, 127)               # amax <= 7 * 2^e
    y = torch.ldexp(v, -e.unsqueeze(-1))
    a, g = y.abs(), _grid()
    mid = (g[1:] + g[:-1]) / 2
    code = torch.bucketize(a, mid, right=False)                                            # a tie goes down ...
    tie_up = (a.unsqueeze(-1) == mid[1::2]).any(-1)                                        # ... or up, where that is the even code
    code = (code + tie_up.int() + 8 * torch.signbit(y).int()).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _from_codes(codes, scales):
    """Codes and scales of pages -> [pages, slots, r] in fp32."""
    n, nt, nb = codes.shape[:3]
    c = torch.stack([codes & 15, codes >> 4], -1).view(n, nt, nb, 16, 32).int()
    v = torch.where(c < 8, 1.0, -1.0) * _grid()[c & 7]
    v = torch.ldexp(v, scales.int().unsqueeze(-1) - 127)
    return v.transpose(2, 3).reshape(n, nt * 16, nb * 32)


def _attend_plain(s):
    case, B = s["case"], s["batch"]
    r, dr, ps = case["r"], case["d_rope"], case["page_slots"]
    P = s["table"].shape[1]
    S = P * ps
    page = torch.arange(P, device=DEV)
    in_packed = page[None, :] < s["n_packed"][:, None]                                     # [B, P]
    lat4 = _from_codes(s["codes"], s["scales"])
    key4 = s["keys"].float().transpose(2, 3).reshape(s["n_pages4"], ps, dr)
    at = torch.where(in_packed, s["table4"], s["table"] + s["n_pages4"]).long().clamp(0, s["n_pages4"] + s["n_pages"] - 1)
    lat = torch.cat([lat4, s["cache_c"].float()])[at].reshape(B, S, r)
    key = torch.cat([key4, s["cache_kr"].float()])[at].reshape(B, S, dr)
    live = torch.arange(S, device=DEV)[None, :] < ((s["seq_len"] + case["stride"] - 1) // case["stride"])[:, None]
    lat, key = torch.where(live[..., None], lat, 0.0), torch.where(live[..., None], key, 0.0)
    qt = torch.bmm(s["q"].float().transpose(0, 1).contiguous(), s["w_uk"].float().transpose(1, 2).contiguous()).transpose(0, 1).contiguous()
    e = torch.bmm(qt, lat.transpose(1, 2)) + torch.bmm(s["q_rope"].float(), key.transpose(1, 2))
    e = (e / math.sqrt(case["d_head"])).masked_fill(~live[:, None, :], float("-inf"))
    m = e.amax(-1, keepdim=True)
    p = torch.exp(e - torch.where(m == float("-inf"), 0.0, m))
    o = torch.bmm(p, lat) / p.sum(-1, keepdim=True).clamp_min(1e-37)
    out = torch.bmm(o.transpose(0, 1).contiguous(), s["w_uv"].float().transpose(1, 2).contiguous())
    return out.transpose(0, 1).contiguous().bfloat16()


def _pack_plain(s):
    page = torch.arange(s["max_pages"], device=DEV)[None, :]
    b, k = torch.nonzero((page >= s["first"][:, None]) & (page < s["end"][:, None]), as_tuple=True)
    source, packed, back = (s[t][b, k].long() for t in ("table", "table4", "table_back"))
    codes, scales = _to_codes(s["cache_c"][source])
    n, ps, dr = len(source), s["cache_kr"].shape[1], s["cache_kr"].shape[2]
    s["codes"][packed], s["scales"][packed] = codes, scales
    s["keys"][packed] = s["cache_kr"][source].view(n, ps // 16, 16, dr // 8, 8).transpose(2, 3)
    s["cache_c"][back] = _from_codes(s["codes"][packed], s["scales"][packed]).bfloat16()
    s["cache_kr"][back] = s["keys"][packed].transpose(2, 3).reshape(n, ps, dr)


def _fit_pool(p, want_first, want_end):
    """Pages of one pool made to fit: entries want_first .. want_end - 1 of every row."""
    P, n = p["table"].shape[1], p["ring"].numel()
    e = torch.arange(P, dtype=torch.int32, device=DEV)[None, :]
    head, count = p["state"][0].clone(), p["state"][1].clone()
    held = (e >= p["first"][:, None]) & (e < p["end"][:, None])
    want = (e >= want_first[:, None]) & (e < want_end[:, None])
    take, give = want & ~held, held & ~want
    need = take.sum(1)
    upto = need.cumsum(0)
    granted = (need == 0) | (upto <= count)
    take &= granted[:, None]
    rank = (upto - need)[:, None] + take.cumsum(1) - 1
    page = p["ring"][(head + rank) % n]
    gone = give.view(-1)
    place = torch.where(gone, (head + count + gone.cumsum(0) - 1) % n, n)
    p["ring"].copy_(torch.cat([p["ring"], p["ring"][:1]]).index_put((place,), p["table"].view(-1))[:n])
    p["table"].copy_(torch.where(take, page, p["table"]))
    first = torch.where(granted, want_first, torch.minimum(torch.maximum(p["first"], want_first), want_end))
    p["end"].copy_(torch.where(granted, want_end, torch.maximum(first, torch.minimum(p["end"], want_end))))
    p["first"].copy_(first)
    taken = take.sum()
    p["state"].copy_(torch.stack([(head + taken) % n, count - taken + gone.sum(), (~granted).sum(), torch.zeros_like(taken)]))


def _fit_plain(s, seq_len, n_new):
    case, pool, packed = s["case"], s["pool"], s["packed"]
    stride, ps, T = case["stride"], case["page_slots"], s["n_new_max"]
    slots = torch.clamp((seq_len + n_new + stride - 1) // stride, max=s["max_slots"])
    reach = (slots + ps - 1) // ps
    start = torch.zeros_like(reach)
    if packed:
        _fit_pool(packed, start, torch.clamp(seq_len // stride // ps - case["keep"], min=0))
        start = packed["end"].clone()
    _fit_pool(pool, start, torch.maximum(start, reach))
    t = torch.arange(T, dtype=torch.int32, device=DEV)[None, :]
    slot = (seq_len[:, None] + t) // stride
    entry = slot // ps
    held = (t < n_new[:, None]) & (entry >= pool["first"][:, None]) & (entry < pool["end"][:, None])
    row = pool["table"].gather(1, entry.clamp(0, s["max_pages"] - 1).long()).long() * ps + slot % ps
    return torch.where(held, row, -1)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its exact result
# --------------------------------------------------------------------------------------------------
def work(case):
    length = np.array(_spread(case["lo"], case["hi"], case["batch"]), np.int64)
    B, ps = case["batch"], case["page_slots"]
    if case["kind"] == "attend":
        H, dh, r, dr = (case[k] for k in ("heads", "d_head", "r", "d_rope"))
        slots = -(-length // case["stride"])
        packed = _complete(length, case) * ps
        cache = packed.sum() * (r // 2 + r // 32 + 2 * dr) + (slots - packed).sum() * 2 * (r + dr)
        return dict(bytes=float(cache + 4 * H * r * dh + 2 * B * H * (2 * dh + dr)), flops=float(2 * H * (slots.sum() * (2 * r + dr) + 2 * B * r * dh)))
    if case["kind"] == "pack":  # (about one page of a sequence was packed before)
        r, dr = case["r"], case["d_rope"]
        pages = np.maximum(length - 1, 0).sum() + 1
        return dict(bytes=float(pages * ps * 2 * (2 * (r + dr) + r // 2 + r // 32 + 2 * dr)), flops=float(pages * ps * r * 4))
    # lengths and counts in, bounds in and out, two calls; what changes of the tables and the free pages; the slot map
    moved = _pages(length, case).sum() if case["admit"] else B / 2
    pools = 2 if case["packed"] else 1
    return dict(bytes=float(2 * B * (8 + 16 * pools) + 2 * pools * moved * 8 + B * case["n_new"] * 8), flops=float(B * 20))


def exact(case, seed):
    """The same in 64 bits, a sequence or a page at a time."""
    if case["kind"] == "fit":
        return None
    s = prepare(case, seed)
    value = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=DEV)
    ps, r, dr = case["page_slots"], case["r"], case["d_rope"]
    if case["kind"] == "pack":
        c, kr = s["cache_c"].double(), s["cache_kr"].double()
        first, end, table = s["first"].tolist(), s["end"].tolist(), s["table"].tolist()
        odd = torch.tensor([0, 1], dtype=torch.float64, device=DEV).repeat(8) * 1e-9                    # a tie goes to the even code
        for b in range(case["batch"]):
            for k in range(first[b], end[b]):
                page = table[b][k]
                x = c[page].view(ps, r // 32, 32)
                top = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -200)
                step = torch.pow(2.0, torch.ceil(torch.log2(top / 7)))
                step = torch.where(7 * step / 2 >= top, step / 2, step).clamp_min(2.0 ** -124)          # (the logarithm rounds)
                near = ((x[..., None] / step[..., None] - value).abs() + odd).argmin(-1)
                c[page + s["n_pages"]] = (value[near] * step).view(ps, r)
                kr[page + s["n_pages"]] = kr[page]
        return c, kr
    if case["batch"] * case["hi"] > 4_000_000:
        return None
    out = torch.zeros(case["batch"], case["heads"], case["d_head"], dtype=torch.float64, device=DEV)
    w_uk, w_uv = s["w_uk"].double(), s["w_uv"].double()
    for b in range(case["batch"]):
        n = -(-int(s["seq_len"][b]) // case["stride"])
        k4 = min(int(s["n_packed"][b]), -(-n // ps))
        if n == 0:
            continue
        p4, p16 = s["table4"][b, :k4].long(), s["table"][b, k4:-(-n // ps)].long()
        byte = s["codes"][p4].long()
        x = torch.empty(k4, ps // 16, r // 32, 16, 32, dtype=torch.float64, device=DEV)
        x[..., 0::2], x[..., 1::2] = value[byte % 16], value[byte // 16]
        x *= torch.pow(2.0, s["scales"][p4].double() - 127)[..., None]
        lat = torch.cat([x.permute(0, 1, 3, 2, 4).reshape(-1, r), s["cache_c"][p16].double().view(-1, r)])[:n]
        key = torch.cat([s["keys"][p4].double().permute(0, 1, 3, 2, 4).reshape(-1, dr), s["cache_kr"][p16].double().view(-1, dr)])[:n]
        qt = torch.matmul(w_uk, s["q"][b].double()[:, :, None])[:, :, 0]                                # [H, r]
        w = torch.softmax((qt @ lat.T + s["q_rope"][b].double() @ key.T) / math.sqrt(case["d_head"]), -1)
        out[b] = torch.matmul(w_uv, (w @ lat)[:, :, None])[:, :, 0]
    return out
