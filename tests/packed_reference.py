"""Packed pages and page tables as the tests expect them: float64 and plain loops, from the format's and the rules' definitions."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16_to_f64(bits):
    return (np.asarray(bits, np.uint32) << 16).view(np.float32).astype(np.float64)


def block(x):
    """32 numbers -> (codes 0..15, scale byte)."""
    x = np.asarray(x, np.float64)
    if not np.all(np.isfinite(x)):
        return None, 255
    top = np.abs(x).max()
    e = -124
    while top > 7 * 2.0 ** e and e < 125:
        e += 1
    y = np.abs(x) / 2.0 ** e
    d = np.abs(y[:, None] - VALUES)
    best = d.min(1)
    code = np.empty(32, int)
    for i in range(32):
        near = [c for c in range(8) if d[i, c] == best[i]]
        code[i] = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
    return code + 8 * np.signbit(x), e + 127


def packed_blocks(x):
    """The same for many blocks [n, 32] at once (finite numbers): (codes, scale bytes), in steps that a search over a table makes."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    e = np.full(top.shape, -124)
    for _ in range(260):
        e = np.where((top > 7 * 2.0 ** e) & (e < 125), e + 1, e)
    y = np.abs(x) / 2.0 ** e[..., None]
    code = np.zeros(x.shape, int)
    for c, mid in enumerate((VALUES[1:] + VALUES[:-1]) / 2):
        code += (y > mid) | ((y == mid) & (c % 2 == 1))
    return code + 8 * np.signbit(x), e + 127


def page_rows(codes, scales, keys):
    """Packed arrays (numpy; keys as float64) -> latents [pages, slots, r] and keys [pages, slots, d_rope], slot by slot."""
    n, nt, nb = scales.shape[:3]
    lat, kr = np.empty((n, nt * 16, nb * 32)), np.empty((n, nt * 16, keys.shape[2] * 8))
    signed = np.concatenate([VALUES, -VALUES])
    for t in range(nt):
        for s in range(16):
            for u in range(nb):
                byte = codes[:, t, u, s]
                v = np.empty((n, 32))
                v[:, 0::2], v[:, 1::2] = signed[byte & 15], signed[byte >> 4]
                sc = scales[:, t, u, s].astype(np.float64)
                lat[:, 16 * t + s, 32 * u:32 * u + 32] = v * np.where(sc == 255, np.nan, 2.0 ** (sc - 127))[:, None]
            kr[:, 16 * t + s] = keys[:, t, :, s].reshape(n, -1)
    return lat, kr


def attend(q, q_rope, w_uk, w_uv, lat, key, scale):
    """One sequence: q [H, dh], lat [n, r], key [n, d_R] -> (out [H, dh], out_latent [H, r], lse [H], and what their errors scale with)."""
    H = q.shape[0]
    if len(lat) == 0:
        z = np.zeros((H, w_uk.shape[1]))
        return np.zeros((H, w_uv.shape[1])), z, np.full(H, -np.inf), dict(logit=np.zeros(H), latent=z, top=z, out=np.zeros((H, w_uv.shape[1])))
    qt = np.einsum("hrk,hk->hr", w_uk, q)
    e = (qt @ lat.T + q_rope @ key.T) * scale
    m = e.max(1, keepdims=True)
    p = np.exp(e - m)
    l = p.sum(1, keepdims=True)
    p /= l
    o = p @ lat
    bounds = dict(logit=((np.abs(qt) @ np.abs(lat).T + np.abs(q_rope) @ np.abs(key).T) * scale).max(1),   # sum of a logit's terms
                  qt=np.einsum("hrk,hk->hr", np.abs(w_uk), np.abs(q)),
                  latent=p @ np.abs(lat), top=np.broadcast_to(np.abs(lat).max(0), o.shape))
    return np.einsum("hkr,hr->hk", w_uv, o), o, (m + np.log(l))[:, 0], bounds


class Pool:
    """One pool of pages by plain loops (the rules of mtla_pages_fit)."""

    def __init__(self, max_batch, max_pages, ring, n_pages=None, spill=-1):
        n = n_pages or len(ring)
        self.table = np.zeros((max_batch, max_pages), np.int32)
        self.first, self.end, self.was_end = (np.zeros(max_batch, np.int32) for _ in range(3))
        self.ring = np.concatenate([np.asarray(ring, np.int32), np.full(n - len(ring), -7, np.int32)])
        self.head, self.count, self.refused, self.spill = 0, len(ring), 0, spill

    def fit(self, want, batch):
        """want[b] = (first, end) -> ends as they are afterwards."""
        n, avail, asked, back = len(self.ring), self.count, 0, []
        self.refused = 0
        head = self.head
        for b in range(batch):
            f, e = int(self.first[b]), int(self.end[b])
            self.was_end[b] = e
            wf, we = want[b]
            held, wanted = set(range(f, e)), set(range(wf, we))
            take, give = sorted(wanted - held), sorted(held - wanted)
            back += [int(self.table[b, k]) for k in give]
            asked += len(take)
            if not take or asked <= avail:
                for k in take:
                    self.table[b, k] = self.ring[head % n]
                    head += 1
                self.first[b], self.end[b] = wf, we
            else:
                self.refused += 1
                if self.spill >= 0:
                    for k in take:
                        self.table[b, k] = self.spill
                self.first[b] = min(max(f, wf), we)
                self.end[b] = max(int(self.first[b]), min(e, we))
        for i, page in enumerate(back):
            self.ring[(self.head + self.count + i) % n] = page
        self.count += len(back) - (head - self.head)
        self.head = head % n


def fit(pool, packed, seq_len, n_new, *, page_slots, stride, max_slots, keep, batch, n_max=0):
    """mtla_pages_fit on two Pools (packed may be None) -> slot map [batch, n_max]."""
    room = max_slots * stride
    have = [min(max(int(x), 0), room) for x in seq_len[:batch]]
    n = [min(max(int(x), 0), n_max) for x in n_new[:batch]]
    start = [0] * batch
    if packed is not None:
        packed.fit([(0, max(h // stride // page_slots - keep, 0)) for h in have], batch)
        start = [int(x) for x in packed.end[:batch]]
    reach = [-(-(-(-min(h + k, room) // stride)) // page_slots) for h, k in zip(have, n)]
    pool.fit([(s, max(s, r)) for s, r in zip(start, reach)], batch)
    rows = np.full((batch, n_max), -1, np.int64)
    for b in range(batch):
        for t in range(n[b]):
            at = int(seq_len[b]) + t
            if at < 0 or at >= room:
                continue
            slot = at // stride
            k = slot // page_slots
            if pool.first[b] <= k < pool.end[b]:
                rows[b, t] = int(pool.table[b, k]) * page_slots + slot % page_slots
    return rows
