"""References of the paged-cache operators: numpy in 64 bits over a cache that the
CPU oracle quantizes.  Slots that no sequence owns hold random codes and
not-a-number parameters."""
import numpy as np

import oracle

HALF_STEP = 2.0 ** -11  # of fp16, relative


def f64(u16):
    return np.asarray(u16, np.uint16).view(np.float16).astype(np.float64)


def to16(x):
    return np.asarray(x, np.float32).astype(np.float16).view(np.uint16)


def kv_rows(rng, n, kvh, D):
    """fp16 rows [n][kvh][D] with per-channel ranges."""
    span = np.exp2(3.0 * rng.random((kvh, D)))
    return to16(rng.standard_normal((n, kvh, D)) * span + rng.standard_normal((kvh, D)))


class Paged:
    """Sequences of (rows, tokens) in a cache of pages in random order.  `holes`:
    (sequence, page index) entries replaced by invalid ones after the tokens were
    stored."""

    def __init__(self, seed, seqs, kvh=2, D=128, G=128, page=16, max_pages=None, spare=3,
                 holes=()):
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.seqs, self.kvh, self.D, self.G, self.page = list(seqs), kvh, D, G, page
        B = len(self.seqs)
        need = [max(0, -(-L // page)) for _, L in self.seqs]
        self.max_pages = max_pages or max(max(need), 1)
        self.num_pages = sum(min(n, self.max_pages) for n in need) + spare
        order = rng.permutation(self.num_pages)
        # entries behind a sequence's tokens are garbage that must not be followed
        self.table = rng.integers(-9, 2 ** 31 - 1, (B, self.max_pages)).astype(np.int64)
        self.table[:, :] = np.where(self.table < self.num_pages, -1, self.table)
        at = 0
        for b, n in enumerate(need):
            n = min(n, self.max_pages)
            self.table[b, :n] = order[at:at + n]
            at += n
        self.table = self.table.astype(np.int32)
        shape = (self.num_pages, kvh, page)
        self.codes = [rng.integers(0, 256, shape + (D // 2,)).astype(np.uint8) for _ in "kv"]
        self.params = [np.full(shape + (D // G, 2), 0x7E00, np.uint16) for _ in "kv"]
        for i in (0, 1):
            for b, (_, L) in enumerate(self.seqs):
                L = min(L, self.max_pages * page)
                if L > 0:
                    c, p = oracle.kv4_quantize(kv_rows(rng, L, kvh, D).reshape(L * kvh, D), G)
                    self.store(i, b, np.arange(L), c.reshape(L, kvh, -1),
                               p.reshape(L, kvh, D // G, 2))
        for k, (b, j) in enumerate(holes):
            self.table[b, j] = (-1, self.num_pages, 2 ** 31 - 1, -2 ** 31)[k % 4]
        n = [max(0, r) for r, _ in self.seqs]
        self.row_start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.lens = np.array([L for _, L in self.seqs], np.int32)
        self.M = int(self.row_start[-1])

    def page_of(self, b, j):
        if j < 0 or j >= self.max_pages * self.page:
            return -1
        p = int(self.table[b, j // self.page])
        return p if 0 <= p < self.num_pages else -1

    def store(self, i, b, tokens, codes, params):
        for j, c, p in zip(tokens, codes, params):
            page = self.page_of(b, int(j))
            if page >= 0:
                self.codes[i][page, :, j % self.page] = c
                self.params[i][page, :, j % self.page] = p

    def rows(self):
        """(row, sequence, position) of every row."""
        for b, (n, L) in enumerate(self.seqs):
            for r in range(max(0, n)):
                yield int(self.row_start[b]) + r, b, L - n + r

    def tokens(self, i, b, js):
        """(codes, s, mn) fp64 [tokens][kvh][D] of tokens js of sequence b (no holes)."""
        at = [(self.page_of(b, int(j)), int(j) % self.page) for j in js]
        c = np.array([self.codes[i][p, :, t] for p, t in at])
        prm = f64(np.array([self.params[i][p, :, t] for p, t in at]))
        q = np.stack([c & 15, c >> 4], axis=-1).reshape(len(js), self.kvh, self.D)
        prm = np.repeat(prm, self.G, axis=2)
        return q.astype(np.float64), prm[..., 0], prm[..., 1]

    def dequantized(self, i, M=None):
        """What reading the rows back gives, fp16 bits [M][kvh][D]; rows in no sequence: 0x1234."""
        out = np.full((M or self.M, self.kvh, self.D), 0x1234, np.uint16)
        for m, b, p in self.rows():
            page = self.page_of(b, p)
            out[m] = 0
            if page >= 0:
                out[m] = oracle.kv4_dequantize(self.codes[i][page, :, p % self.page],
                                               self.params[i][page, :, p % self.page], self.G)
        return out

    def attention(self, q16, H, scale, window=0, rows=None):
        """(out, bound) fp64 [M][H][D]; bound: what fp16 weights and output and fp32 sums may
        be off by, element by element.  rows: only these (others zero)."""
        q = f64(q16)
        out, bound = (np.zeros((self.M, H, self.D)) for _ in range(2))
        R = H // self.kvh
        cached = {}
        for m, b, p in self.rows():
            if rows is not None and m not in rows:
                continue
            lo = max(0, p - window + 1) if window else 0
            js = [j for j in range(lo, p + 1) if self.page_of(b, j) >= 0]
            if not js:
                continue
            if b not in cached:
                every = [j for j in range(max(0, self.lens[b])) if self.page_of(b, j) >= 0]
                cached[b] = ({j: n for n, j in enumerate(every)}, self.tokens(0, b, every),
                             self.tokens(1, b, every))
            index, K, V = cached[b]
            at = np.array([index[j] for j in js])
            kc, ks, km = (a[at] for a in K)
            vc, vs, vm = (a[at] for a in V)
            n = len(js)
            for h in range(H):
                g = h // R
                terms = np.abs(q[m, h]) * (ks[:, g] * kc[:, g] + np.abs(km[:, g]))
                x = scale * (ks[:, g] * kc[:, g] + km[:, g]) @ q[m, h]
                w = np.exp(x - x.max())
                w /= w.sum()
                out[m, h] = w @ (vs[:, g] * vc[:, g] + vm[:, g])
                # a score is off by its fp32 sum's rounding (D + 16 steps at most on terms
                # of this size), which scales a weight and the sum of the weights
                dx = (abs(scale) * terms.sum(axis=1).max() * (self.D + 16) + 2 * np.abs(x).max()
                      + 4) * 2.0 ** -24
                size = w @ (vs[:, g] * vc[:, g] + np.abs(vm[:, g]))
                bound[m, h] = (HALF_STEP * np.abs(out[m, h]) + 2.0 ** -25
                               + (HALF_STEP + 2 * dx + n * 2.0 ** -24) * size)
        return out, bound


def check_attention(got16, ref, bound, what=""):
    got = f64(got16)
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    over = np.abs(got - ref) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, (f"{what}: {got[at]} at {at}, expected {ref[at]} within {bound[at]}; "
                           f"{np.mean(over > 0):.2g} of the values are off")
