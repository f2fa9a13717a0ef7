"""Plain 64-bit forms, in numpy, of what a 4-bit cache holds and of how a cache's pages are looked after."""
import numpy as np

PAGE, D, GROUP = 64, 576, 16
CODE_ROW, SCALE_ROW = D // 2, D // GROUP
CODE_BYTES = PAGE * CODE_ROW
PAGE_BYTES = CODE_BYTES + PAGE * SCALE_ROW

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3(byte):
    """Value of E4M3 bytes (NaN for S.1111.111)."""
    b = np.asarray(byte).astype(np.int64)
    e, m, s = (b >> 3) & 15, b & 7, 1.0 - 2.0 * (b >> 7)
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0)) * s
    return np.where((b & 127) == 127, np.nan, v)


E4M3 = e4m3(np.arange(127))           # 0 .. 448


def nearest(v, grid):
    """Index of the grid's nearest number, ties to the even index; beyond the last: the last."""
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = v - grid[lo], grid[hi] - v
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantise(x, kv_scale):
    """float64 [..., 576] -> (codes uint8 [..., 288], scales uint8 [..., 36]); x is finite."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], SCALE_ROW, GROUP) / kv_scale
    sc = nearest(np.minimum(np.abs(g).max(-1) / 6.0, 448.0), E4M3)
    step = E4M3[sc][..., None]
    idx = np.where(step > 0, nearest(np.minimum(np.abs(g) / np.where(step > 0, step, 1.0), 6.0), E2M1), 0)
    code = (idx + 8 * (np.signbit(g))).astype(np.uint8).reshape(*x.shape[:-1], D)
    return code[..., 0::2] | (code[..., 1::2] << 4), sc.astype(np.uint8)


def values(codes, scales):
    """What codes [..., 288] and scales [..., 36] stand for, without kv_scale: float64 [..., 576]."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D)
    v = E2M1[n & 7] * np.where(n & 8, -1.0, 1.0)
    return v * np.repeat(e4m3(scales), GROUP, -1)


def pack(codes, scales):
    """[pages, 64, 288], [pages, 64, 36] -> uint8 [pages, 20736]."""
    n = codes.shape[0]
    return np.ascontiguousarray(np.concatenate([codes.reshape(n, -1), scales.reshape(n, -1)], 1))


def unpack(cache):
    n = cache.shape[0]
    return cache[:, :CODE_BYTES].reshape(n, PAGE, CODE_ROW), cache[:, CODE_BYTES:].reshape(n, PAGE, SCALE_ROW)


def bf16_bits(x):
    """float64 -> bf16 bit patterns, for numbers that bf16 holds exactly."""
    f = np.asarray(x, np.float32)
    bits = f.view(np.uint32)
    assert np.isnan(f).any() or not (bits & 0xFFFF).any()
    return (bits >> 16).astype(np.uint16)


def bf16_values(bits):
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ------------------------------------------------------------------------------------------ pages

def pages_of(n):
    return max(0, (n + PAGE - 1) // PAGE)


class Books:
    """Block table, lengths and reference counts (and the cache as one number per page), looked after one request at a time."""

    def __init__(self, table, lens, refs, cache):
        self.table, self.lens, self.refs, self.cache = table.copy(), lens.copy(), refs.copy(), cache.copy()

    def free_list(self):
        return [int(p) for p in np.flatnonzero(self.refs <= 0)]

    def free(self, rows):
        for r in rows:
            if 0 <= r < len(self.lens):
                for i in range(pages_of(self.lens[r])):
                    self.refs[self.table[r, i]] -= 1
                    self.table[r, i] = -1
                self.lens[r] = 0

    def fork(self, parents, children):
        served, pool, lens = [], self.free_list(), self.lens.copy()
        for p, c in zip(parents, children):
            B = len(lens)
            if not (0 <= p < B and 0 <= c < B) or p == c:
                served.append(0)
                continue
            n, full = int(lens[p]), int(lens[p]) // PAGE
            self.table[c] = -1
            self.lens[c] = 0
            if n % PAGE and not pool:
                served.append(0)
                continue
            self.table[c, :full] = self.table[p, :full]
            np.add.at(self.refs, self.table[p, :full], 1)
            if n % PAGE:
                page = pool.pop(0)
                self.table[c, full] = page
                self.refs[page] = 1
                self.cache[page] = self.cache[self.table[p, full]]
            self.lens[c] = n
            served.append(1)
        return np.array(served, np.int32)

    def reserve(self, new):
        granted, pool, at = [], self.free_list(), 0
        for b, then in enumerate(new):
            now = int(self.lens[b])
            if then > self.table.shape[1] * PAGE:
                granted.append(0)
                continue
            more = max(0, pages_of(then) - pages_of(now))
            first, at = at, at + more
            if more and at > len(pool):
                granted.append(0)
                continue
            for i in range(more):
                self.table[b, pages_of(now) + i] = pool[first + i]
                self.refs[pool[first + i]] = 1
            self.lens[b] = max(now, then)
            granted.append(1)
        return np.array(granted, np.int32)

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] <= 0]
        high = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        to = dict(zip(high, holes))
        for s, d in to.items():
            self.cache[d] = self.cache[s]
            self.refs[d], self.refs[s] = self.refs[s], 0
        for b in range(len(self.lens)):
            for i in range(pages_of(self.lens[b])):
                self.table[b, i] = to.get(int(self.table[b, i]), self.table[b, i])
        return live
