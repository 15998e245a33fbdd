"""Plain model of the paged 8-bit cache for the tests: a dictionary per (page, head), numpy in the precision that the definition
states (binary32 for what is stored, binary64 for the attention), token by token."""
import numpy as np
import torch

QMAX = {"int8": np.float32(127), "e4m3": np.float32(448)}
FLOOR = np.float32(2.0 ** -60)
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _e4m3_values():
    out = np.zeros(256, np.float32)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = np.nan if (c & 0x7f) == 0x7f else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -x if c & 128 else x
    return out


E4M3 = _e4m3_values()
_POS = E4M3[:127].astype(np.float64)  # ascending, code = index
_MID = (_POS[:-1] + _POS[1:]) / 2


def decode(codes, fmt):
    return codes.view(np.int8).astype(np.float32) if fmt == "int8" else E4M3[codes]


def encode(x, fmt):
    """x fp32, divided by its scale already -> codes uint8; nearest, ties to even."""
    if fmt == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(x.astype(np.float64)), 448.0)
    lo = np.searchsorted(_MID, a, side="left")   # a on a midpoint: the lower code
    hi = np.searchsorted(_MID, a, side="right")  # ... the upper one
    code = np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def v_place(token, dim, D):
    """Byte of V's code inside its (page, head)."""
    group, r = divmod(token, 32)
    tile, r = divmod(r, 16)
    g, i = divmod(r, 4)
    return ((((group * (D // 2) + dim // 2) * 4 + g) * 2 + dim % 2) * 2 + tile) * 4 + i


def v_index(P, D):
    return np.array([[v_place(t, d, D) for d in range(D)] for t in range(P)])


def rotate(x, table, pos, interleaved):
    """x fp32 [..., D], table [positions][rot / 2][2] -> fp32, one rounding per operation."""
    y = x.copy()
    half = table.shape[1]
    c, s = table[pos, :, 0], table[pos, :, 1]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Model:
    """Codes as [page][head][token][dim] for K and V alike, scales [page][head]."""

    def __init__(self, pages, heads, D, P, fmt):
        self.heads, self.D, self.P, self.fmt = heads, D, P, fmt
        self.codes = [np.zeros((pages, heads, P, D), np.uint8) for _ in range(2)]
        self.scale = [np.zeros((pages, heads), np.float32) for _ in range(2)]
        self.known = np.zeros((pages, P), bool)

    def append(self, which, rows, length, table):
        """rows fp32 [n][heads][D] (K after the rotation) behind `length` tokens of the sequence with this table."""
        codes, scale, P = self.codes[which], self.scale[which], self.P
        n = rows.shape[0]
        for b in range(length // P, -(-(length + n) // P)):
            lo, hi = max(length, b * P), min(length + n, (b + 1) * P)
            if lo >= hi or b >= len(table) or not 0 <= table[b] < codes.shape[0]:
                continue
            page, new = table[b], rows[lo - length:hi - length]
            self.known[page, lo - b * P:hi - b * P] = True
            if lo == b * P:
                self.known[page, hi - b * P:] = False
            for h in range(self.heads):
                x = new[:, h]
                opens = lo == b * P
                with np.errstate(invalid="ignore", over="ignore"):
                    finite = np.isfinite(x).all() and (opens or np.isfinite(scale[page, h]))
                    need = max(np.float32(np.abs(x).max() / QMAX[self.fmt]), FLOOR) if finite else np.float32(np.nan)
                if not finite:
                    scale[page, h] = np.nan
                    codes[page, h, lo - b * P:hi - b * P] = 0
                    continue
                if opens:
                    scale[page, h] = need
                else:
                    k = 0
                    while np.float64(scale[page, h]) * 2.0 ** k < np.float64(need):
                        k += 1
                    if k:
                        scale[page, h] = np.float32(np.float64(scale[page, h]) * 2.0 ** k)
                        old = decode(codes[page, h, :lo - b * P], self.fmt)
                        codes[page, h, :lo - b * P] = encode((old.astype(np.float64) * 2.0 ** -k).astype(np.float32), self.fmt)
                codes[page, h, lo - b * P:hi - b * P] = encode((x / scale[page, h]).astype(np.float32), self.fmt)

    def value(self, which, length, table):
        """fp64 [tokens][heads][D] of the first `length` tokens, and whether each is there."""
        out = np.zeros((length, self.heads, self.D))
        there = np.zeros(length, bool)
        for t in range(length):
            b = t // self.P
            if b < len(table) and 0 <= table[b] < self.codes[which].shape[0]:
                there[t] = True
                out[t] = decode(self.codes[which][table[b], :, t % self.P], self.fmt).astype(np.float64) * \
                    self.scale[which][table[b]].astype(np.float64)[:, None]
        return out, there

    def device(self, dtype, dev, fill=None):
        """The framework's cache with these contents; codes of tokens that nobody wrote are `fill` (a byte), or left zero."""
        import paper_2505_05950_amd as F
        k, v = self.codes[0].copy(), self.codes[1].copy()
        if fill is not None:
            for c in (k, v):
                c[np.broadcast_to(~self.known[:, None, :, None], c.shape)] = fill
        vt = np.zeros_like(v).reshape(*v.shape[:2], -1)
        vt[..., v_index(self.P, self.D).ravel()] = v.reshape(*v.shape[:2], -1)
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        return F.KVCache(k.shape[0], self.heads, self.D, self.P, F.KV_INT8 if self.fmt == "int8" else F.KV_E4M3, DTYPES[dtype],
                         tensors=(up(k), up(vt), up(self.scale[0]), up(self.scale[1])))


def codes_of_device(cache):
    """(K codes, V codes) [page][head][token][dim] and the scales, as numpy."""
    k = cache.k.cpu().numpy().reshape(cache.n_pages, cache.kv_heads, cache.block, cache.head_dim)
    v = cache.v.cpu().numpy().reshape(cache.n_pages, cache.kv_heads, -1)[..., v_index(cache.block, cache.head_dim).ravel()]
    return (k, v.reshape(k.shape)), (cache.k_scale.cpu().numpy().reshape(-1, cache.kv_heads), cache.v_scale.cpu().numpy().reshape(-1, cache.kv_heads))


def attention(q, k, v, there, length, causal, window, scale):
    """One sequence in fp64: q [n][H][D], k / v [length][heads][D] -> out [n][H][D], lse [n][H], and sum p |v| / sum p, the size that the
    rounding of the weights is measured against."""
    n, H, D = q.shape
    G = H // (k.shape[1] or 1)
    out, size, lse = np.zeros((n, H, D)), np.zeros((n, H, D)), np.full((n, H), -np.inf)
    for i in range(n):
        pos = length - n + i
        j = np.arange(length)
        see = there & (j <= pos if causal else j >= 0)
        if window:
            see &= j > pos - window
        j = j[see]
        if not j.size:
            continue
        for h in range(H):
            with np.errstate(invalid="ignore"):
                s = (k[j, h // G] @ q[i, h]) * scale
                top = s.max()
                p = np.exp(s - top)
                out[i, h] = p @ v[j, h // G] / p.sum()
                size[i, h] = p @ np.abs(v[j, h // G]) / p.sum()
                lse[i, h] = top + np.log(p.sum()) + 0 * out[i, h].sum()  # a block whose scale is NaN, of K or of V, makes both NaN
    return out, lse, size
