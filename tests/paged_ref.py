"""The caches in pages in plain form: the state changed view by view and page by
page on the host, attention of the new tokens in 64 bits, and the bounds on what a
kernel's arithmetic may add to it."""
import numpy as np
import torch

D = 128


def pages_of(rows, page):
    return -(-rows // page)


class Pages:
    """Mirror of a cache on the host (rows as fp32 values, which hold bf16 exactly)."""

    def __init__(self, n_pages, page, n_slots, hkv, max_pages):
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.k, self.v = (np.zeros((n_pages, page, D), np.float32) for _ in "kv")
        self.table = np.full((n_slots, hkv, max_pages), -1, np.int32)
        self.lens = np.zeros((n_slots, hkv), np.int64)
        self.refs = np.zeros(n_pages, np.int32)

    @classmethod
    def of(cls, c):
        """What a PagedCache on the GPU holds now."""
        s = cls(c.n_pages, c.page, c.n_slots, c.hkv, c.max_pages)
        s.k, s.v = c.k.float().cpu().numpy().copy(), c.v.float().cpu().numpy().copy()
        s.table, s.lens, s.refs = (t.cpu().numpy().copy() for t in (c.table, c.lens, c.refs))
        return s

    def bits(self):
        b = np.zeros(pages_of(self.n_pages, 64) * 64, np.uint64)
        b[:self.n_pages] = self.refs == 0
        return (b.reshape(-1, 64) << np.arange(64, dtype=np.uint64)).sum(axis=1, dtype=np.uint64).view(np.int64)

    def free(self):
        return [int(p) for p in np.flatnonzero(self.refs == 0)]

    def rows(self, slot, h):
        """The rows of a view, K and V."""
        L = int(self.lens[slot, h])
        ids = self.table[slot, h, :pages_of(L, self.page)]
        return self.k[ids].reshape(-1, D)[:L], self.v[ids].reshape(-1, D)[:L]

    def append(self, slots, new, k_new, v_new):
        """k_new, v_new [tokens][hkv][D]; returns whether a sequence was left."""
        P, hkv = self.page, self.lens.shape[1]
        free, used, left, first, gone, stop = self.free(), 0, False, 0, [], False
        refs = self.refs.copy()
        for x, m in zip(slots, new):
            L = [int(self.lens[x, h]) for h in range(hkv)]
            if m and any(n < 0 or n + m > self.max_pages * P for n in L):
                left, first = True, first + m
                continue
            copied = [m > 0 and n % P > 0 and refs[self.table[x, h, n // P]] > 1 for h, n in enumerate(L)]
            need = sum(pages_of(n + m, P) - pages_of(n, P) + c for n, c in zip(L, copied))
            if need and (stop or used + need > len(free)):
                left, stop, first = True, True, first + m
                continue
            for h, n in enumerate(L if m else []):
                if copied[h]:
                    old, to = int(self.table[x, h, n // P]), free[used]
                    used += 1
                    self.k[to, :n % P], self.v[to, :n % P] = self.k[old, :n % P], self.v[old, :n % P]
                    self.table[x, h, n // P] = to
                    self.refs[to] = 1
                    gone.append(old)
                for p in range(pages_of(n, P), pages_of(n + m, P)):
                    self.table[x, h, p] = free[used]
                    self.refs[free[used]] = 1
                    used += 1
                for j in range(m):
                    p, r = int(self.table[x, h, (n + j) // P]), (n + j) % P
                    self.k[p, r], self.v[p, r] = k_new[first + j, h], v_new[first + j, h]
                self.lens[x, h] = n + m
            first += m
        for p in gone:
            self.refs[p] -= 1
        return left

    def fork(self, src, dst):
        refused = False
        for a, b in zip(src, dst):
            for h in range(self.lens.shape[1]):
                if self.lens[b, h]:
                    refused = True
                    continue
                n = pages_of(int(self.lens[a, h]), self.page)
                self.table[b, h, :n] = self.table[a, h, :n]
                np.add.at(self.refs, self.table[a, h, :n], 1)
                self.lens[b, h] = self.lens[a, h]
        return refused

    def drop(self, rows):
        for x, r in enumerate(rows):
            for h in range(self.lens.shape[1]):
                L = int(self.lens[x, h])
                left = max(L - max(int(r), 0), 0)
                for p in range(pages_of(left, self.page), pages_of(L, self.page)):
                    self.refs[self.table[x, h, p]] -= 1
                    self.table[x, h, p] = -1
                self.lens[x, h] = left

    def compact(self, slot, heads, idx, cs, tail):
        free, used, left, gone, stop = self.free(), 0, False, [], False
        for h, chunks in zip(heads, idx):
            L, P = int(self.lens[slot, h]), self.page
            if L < tail:
                left = True
                continue
            rows = [t for c in chunks if c >= 0 for t in range(c * cs, min((c + 1) * cs, L - tail))]
            rows += range(L - tail, L)
            need = pages_of(len(rows), P)
            if need > self.max_pages:
                left = True
                continue
            if need and (stop or used + need > len(free)):
                left = stop = True
                continue
            k, v = (x[rows] for x in self.rows(slot, h))
            old, new = self.table[slot, h, :pages_of(L, P)].copy(), free[used:used + need]
            used += need
            for i in range(len(rows)):
                self.k[new[i // P], i % P], self.v[new[i // P], i % P] = k[i], v[i]
            self.table[slot, h] = -1
            self.table[slot, h, :need] = new
            self.refs[new] = 1
            self.lens[slot, h] = len(rows)
            gone.append(old)
        for old in gone:
            np.subtract.at(self.refs, old, 1)
        return left

    def same(self, c):
        """Everything of the PagedCache c, bit for bit."""
        got = Pages.of(c)
        for name in ("table", "lens", "refs"):
            a, b = getattr(got, name), getattr(self, name)
            assert np.array_equal(a, b), f"{name}: {np.argwhere(a != b)[:5].tolist()} {a[a != b][:5]} for {b[a != b][:5]}"
        assert np.array_equal(c.free_bits.cpu().numpy(), self.bits()), "free_bits"
        for name in "kv":
            a, b = getattr(got, name), getattr(self, name)
            assert np.array_equal(a, b, equal_nan=True), f"{name}: pages {np.unique(np.argwhere(a != b)[:, 0])[:8]}"


def attention(q, k, v, m, scale):
    """q [m][G][D], one view's rows k, v -> out, log-sum-exp and what bounds the
    error of a computation in fewer bits: A = sum softmax |v| [m][G][D], and the
    largest sum of |q k| [m][G]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    G, L = q.shape[1], len(k)
    out, A = np.zeros((m, G, D)), np.zeros((m, G, D))
    lse, B = np.full((m, G), -np.inf), np.zeros((m, G))
    for j in range(m):
        n = L - m + j + 1
        if n <= 0:
            continue
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            s = q[j] @ k[:n].T * scale
            B[j] = (np.abs(q[j]) @ np.abs(k[:n]).T).max(axis=1) * scale
            top = s.max(axis=1)
            none = top == -np.inf
            p = np.exp(s - np.where(none, 0.0, top)[:, None])
            l = p.sum(axis=1)
            lse[j] = top + np.log(l)
            w = np.where(none[:, None], 0.0, p / l[:, None])
            out[j] = np.where(none[:, None], 0.0, w @ v[:n])
            A[j] = np.where(none[:, None], 0.0, w @ np.abs(v[:n]))
    return out, lse, A, B


def bounds(out, lse, A, B, n, dtype, rows):
    """Largest errors of out and lse that the arithmetic of csrc allows.  A score is
    off by at most d: 130 roundings of 2^-24 of the sum of |q k|, and of a few of its
    own size on the way through exp2 (units of log2: 1.45); exp2 itself 2^-22.  Sums
    over n rows in fp32 add n 2^-24 each, in the product and in the weights' sum.  The
    weights are rounded to bf16 (2^-8; kept to 16 bits, 2^-16, for up to 16 rows of
    new tokens), the result to its type."""
    d = 130 * 2.0 ** -24 * B + 6 * 2.0 ** -24 * 1.45 * np.nan_to_num(B) + 2.0 ** -21
    sums = (n + 200) * 2.0 ** -24
    w = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8 if rows > 16 else 2.0 ** -16}[dtype]
    half = torch.finfo(dtype).eps / 2
    return (w + 2 * d[..., None] + 2 * sums) * A * 1.01 + half * np.abs(out) * 1.01 + 1e-30, \
        d + sums + 2.0 ** -22 * np.abs(lse) + 2.0 ** -22
