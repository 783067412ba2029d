"""What lies between the dense layers of a decoder block, in 64 bits and written out plainly: root-mean-square
normalisation, rotary positions, a paged cache in 8 bits with power-of-two scales, attention over it, and the
bookkeeping of pages.  Independent of the library: numpy and the E4M3 decoder of `reference` only."""
import numpy as np

from . import reference

PAGE, BLOCK = 64, 32
TOP = 448.0
E_MIN, E_MAX = -96, 120


# ---- E4M3 --------------------------------------------------------------------------------------------------------

_CODES = np.arange(256, dtype=np.uint8)
_VALUES = reference.e4m3_decode(_CODES[:127], 1.0)          # 0 .. 448, ascending; 0x7f is the NaN


def e4m3_encode(x):
    """Round to the nearest code (ties to the even one), saturating at +-448; NaN -> 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), TOP)
    hi = np.clip(np.searchsorted(_VALUES, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _VALUES[hi] - a, a - _VALUES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (a == _VALUES[hi]), hi, lo).astype(np.uint8)
    code = np.where(np.signbit(x), code | 0x80, code)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def e4m3_decode(codes):
    codes = np.asarray(codes, dtype=np.uint8)
    mag = codes & 0x7F
    v = np.where(mag == 0x7F, np.nan, _VALUES[np.minimum(mag, 126)])
    return np.where(codes & 0x80, -v, v)


# ---- normalisation -----------------------------------------------------------------------------------------------

def add_rms_norm(x, r, gamma, eps):
    """-> (s, y)."""
    s = x if r is None else x + r
    return s, s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps) * gamma


# ---- rotary positions --------------------------------------------------------------------------------------------

def rotary_table(n_positions, head_dim, base=10000.0):
    """[n_positions, head_dim / 2, 2]: cos and sin."""
    angle = np.arange(n_positions)[:, None] * base ** (-np.arange(head_dim // 2) * 2.0 / head_dim)[None]
    return np.stack([np.cos(angle), np.sin(angle)], axis=-1)


def rotate(x, table, positions, axis_pairs):
    """x [rows, heads, D]; positions [rows, 3]: pair (i, i + D / 2) turns by the angle of its axis's position."""
    half = x.shape[2] // 2
    axis = np.repeat(np.arange(3), axis_pairs)
    at = np.clip(positions[:, axis], 0, len(table) - 1)                      # [rows, half]
    cs = table[at, np.arange(half)[None]]                                    # [rows, half, 2]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


# ---- the cache ---------------------------------------------------------------------------------------------------

def block_exponent(amax):
    """The smallest e in [-96, 120] with amax <= 448 * 2^e."""
    e = E_MIN
    while e < E_MAX and amax > TOP * 2.0 ** e:
        e += 1
    return e


class Cache:
    """codes [n_pages, kv_heads, 2, 64, D] in the order of tokens, exponents [n_pages, kv_heads, 2, 2]."""

    def __init__(self, n_pages, kv_heads, head_dim, rng=None):
        shape = (n_pages, kv_heads, 2, PAGE, head_dim)
        self.codes = np.zeros(shape, dtype=np.uint8) if rng is None else rng.integers(0, 256, shape).astype(np.uint8)     # NaN codes too: nobody may look
        self.scales = np.full((n_pages, kv_heads, 2, 2), 0 if rng is None else 255, dtype=np.uint8)

    def append(self, pages, start, K, V):
        """Tokens K, V [n, kv_heads, D] (rotated) join a sequence with these pages at positions start ..; negative positions are padding."""
        n = len(K)
        for block in range(max(start, 0) // BLOCK, (start + n - 1) // BLOCK + 1 if start + n > 0 else 0):
            lo, hi = max(start, 0, block * BLOCK), min(start + n, (block + 1) * BLOCK)
            page, half, had = pages[block * BLOCK // PAGE], block % 2, max(max(start, 0) - block * BLOCK, 0)
            at = half * BLOCK
            for h in range(K.shape[1]):
                broken = np.isnan(K[lo - start: hi - start, h]).any(axis=1) | np.isnan(V[lo - start: hi - start, h]).any(axis=1)
                for which, X in ((0, K), (1, V)):
                    x = X[lo - start: hi - start, h].copy()
                    finite = np.abs(x[np.isfinite(x)])
                    e = block_exponent(finite.max() if finite.size else 0.0)
                    if had:
                        before = int(self.scales[page, h, which, half]) - 127
                        if e > before:
                            old = self.codes[page, h, which, at: at + had]
                            self.codes[page, h, which, at: at + had] = e4m3_encode(e4m3_decode(old) * 2.0 ** (before - e))
                        e = max(e, before)
                    code = e4m3_encode(np.where(np.isnan(x), 0.0, x) * 2.0 ** -e)
                    if which == 0:
                        code[broken, 0] = 0x7F
                    self.codes[page, h, which, at + had: at + had + hi - lo] = code
                    self.scales[page, h, which, half] = e + 127

    def values(self, pages, tokens):
        """-> K, V [tokens, kv_heads, D]."""
        out = []
        for which in (0, 1):
            rows = []
            for t in range(tokens):
                page = pages[t // PAGE]
                e = self.scales[page, :, which, t % PAGE // BLOCK].astype(np.float64) - 127
                rows.append(e4m3_decode(self.codes[page, :, which, t % PAGE]) * 2.0 ** e[:, None])
            out.append(np.array(rows).reshape(tokens, self.codes.shape[1], self.codes.shape[4]))
        return out

    def packed(self):
        """codes in the library's order inside a page: [n_pages, kv_heads, 2, 64 D]."""
        P, H, _, _, D = self.codes.shape
        out = np.zeros((P, H, 2, PAGE * D), dtype=np.uint8)
        t, d = np.arange(PAGE)[:, None], np.arange(D)[None]
        key = ((((t // 4) % 4) * (D // 16) + d // 16) * 16 + 4 * (t // 16) + t % 4) * 16 + d % 16
        value = ((d // 16 * 4 + t // 16) * 16 + d % 16) * 16 + t % 16
        out[:, :, 0, key.reshape(-1)] = self.codes[:, :, 0].reshape(P, H, -1)
        out[:, :, 1, value.reshape(-1)] = self.codes[:, :, 1].reshape(P, H, -1)
        return out


# ---- attention ---------------------------------------------------------------------------------------------------

def attention(Q, K, V, start, scale, window=0, softcap=0.0):
    """Q [rows, heads, D] of one sequence at positions start .., K, V [tokens, kv_heads, D] -> (o, a) [rows, heads, D]: the outputs, and the same
    weighted means of |v| (what the rounding of the weights is relative to).  A row sees keys 0 .. its own position (window: the last `window` of
    them); a row that sees none is zeros."""
    rows, H, D = Q.shape
    group = H // K.shape[1]
    out, mass = np.zeros((rows, H, D)), np.zeros((rows, H, D))
    for i in range(rows):
        hi = start + i + 1
        lo = max(0, hi - window) if window else 0
        if hi <= lo:
            continue
        for h in range(H):
            z = K[lo:hi, h // group] @ Q[i, h] * scale
            if softcap:
                z = softcap * np.tanh(z / softcap)
            w = np.exp(z - z.max()) if not np.isnan(z).any() else np.full_like(z, np.nan)
            w = w / w.sum()
            out[i, h], mass[i, h] = w @ V[lo:hi, h // group], w @ np.abs(V[lo:hi, h // group])
    return out, mass


# ---- pages -------------------------------------------------------------------------------------------------------

class Pages:
    """How many sequences hold each page, and the free ones in the order in which they are taken (last first)."""

    def __init__(self, n):
        self.refs, self.free_pages = [0] * n, list(range(n))[::-1]

    def take(self, n):
        out = [self.free_pages.pop() for _ in range(n)]
        for p in out:
            self.refs[p] = 1
        return out

    def fork(self, pages, tokens):
        whole, n = tokens // PAGE, -(-tokens // PAGE)
        for p in pages[:whole]:
            if p != -1:
                self.refs[p] += 1
        child, moves = list(pages[:whole]), []
        if n > whole:
            child += self.take(1)
            moves = [(pages[whole], child[-1])]
        return child, moves

    def free(self, pages):
        for p in pages:
            if p == -1:
                continue
            self.refs[p] -= 1
            if self.refs[p] == 0:
                self.free_pages.append(p)

    def compact(self, tables):
        used = sum(r > 0 for r in self.refs)
        holes = [p for p in range(used) if self.refs[p] == 0]
        far = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        moves = list(zip(far, holes))
        name = dict(moves)
        for src, dst in moves:
            self.refs[dst], self.refs[src] = self.refs[src], 0
        self.free_pages = list(range(used, len(self.refs)))[::-1]
        return moves, [[name.get(p, p) for p in t] for t in tables]
