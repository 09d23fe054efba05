"""Plain forms, in 64 bits and on the host, of what st_attn_* computes, and the cache layout of include/st_lm.h.

The oracle of the 4-bit cache works on the definition: it looks for the nearest of the sixteen elements under the group's scale."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x):
    """[..., dim] float64 values -> (codes [..., dim], scale codes [..., dim / 32])."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    most = np.abs(b).max(-1)
    e = np.full(most.shape, -126, dtype=np.int64)
    some = most > 0
    mantissa, exponent = np.frexp(most)                  # 0.5 <= mantissa < 1
    m, k = 2 * mantissa, exponent - 1
    e[some] = np.clip(np.where(m <= 1.5, k - 2, k - 1), -126, 125)[some]
    size = np.minimum(np.abs(b) / np.exp2(e.astype(np.float64))[..., None], 6.0)
    off = np.abs(size[..., None] - GRID)
    low = off.argmin(-1)                                  # the lower of two that are equally near
    high = 7 - off[..., ::-1].argmin(-1)
    code = np.where(low % 2 == 0, low, high)              # ties to the even code
    code = code + 8 * np.signbit(b)
    return code.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def encode_token_head(k, v):
    """Keys and values [..., dim] as the library writes them, with the rule for values that are not finite."""
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
    clean = lambda x: np.where(bad[..., None], 0.0, x)  # noqa: E731
    (kc, ks), (vc, vs) = encode(clean(k)), encode(clean(v))
    kc[bad] = vc[bad] = 0
    ks[bad], vs[bad] = 255, 1
    return kc, ks, vc, vs


def decode(code, scale):
    size = GRID[code % 8] * np.where(code >= 8, -1.0, 1.0)
    f = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return (size.reshape(*code.shape[:-1], code.shape[-1] // 32, 32) * f[..., None]).reshape(code.shape)


def block_bytes(dim):
    return 16 * (dim + dim // 16)


class Pool:
    """A page pool on the host as the layout describes it, byte by byte."""

    def __init__(self, n_pages, kv_heads, page_tokens, dim, fill=0):
        self.kv, self.page, self.dim = kv_heads, page_tokens, dim
        self.bytes = np.full((n_pages, kv_heads, page_tokens // 16, block_bytes(dim)), fill, dtype=np.uint8)

    def _places(self, t):
        """Byte offsets in a block of token t's parts: keys' codes, values' codes (one per pair of elements), scales of both."""
        d = self.dim
        pair = np.arange(d // 2)
        in_group = d // 32                                # bytes of a token's part of a group
        kc = t * (d // 2) + pair
        vc = 8 * d + (pair // in_group * 16 + t) * in_group + pair % in_group
        ks = 16 * d + t * (d // 32) + np.arange(d // 32)
        vs = 16 * d + d // 2 + np.arange(d // 32) * 16 + t
        return kc, vc, ks, vs

    def write(self, page, t, kc, ks, vc, vs):
        """A token's codes and scales, [head][...], to place t of a page."""
        block = self.bytes[page, :, t // 16]
        a, b, c, e = self._places(t % 16)
        block[:, a] = kc[:, 0::2] | kc[:, 1::2] << 4
        block[:, b] = vc[:, 0::2] | vc[:, 1::2] << 4
        block[:, c], block[:, e] = ks, vs

    def read(self, page, t):
        block = self.bytes[page, :, t // 16]
        a, b, c, e = self._places(t % 16)
        both = [np.stack([block[:, x] & 15, block[:, x] >> 4], -1).reshape(self.kv, self.dim) for x in (a, b)]
        return decode(both[0], block[:, c]), decode(both[1], block[:, e])


def attend(q, k, v, p0, scale, causal, window, bits):
    """q [new, heads, dim]; k, v [kv, tokens, dim] (NaN keys allowed): outputs, and the tolerance of each.  bits: bits of the type's significand.

    With e = 2^-24: a score is a sum of dim exact products, off by at most 2 e (dim + 4) sum|q k| |scale|, and its weight's
    exponent is rounded twice more, |s| e each (s relative to the row's largest, and the largest itself); the weight is rounded to
    the type, half a step, and the exponential adds a few e.  Numerator and denominator have each the weights' relative error, the
    sum over tokens adds 2 e per token, and the result is rounded to the type.  fp16 weights may lose what is below 2^-34 of the largest."""
    new, heads, dim = q.shape
    kv, tokens, _ = k.shape
    e, half = 2.0 ** -24, 2.0 ** -bits
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    place = np.arange(tokens)
    for j in range(new):
        p = p0 + j
        seen = np.ones(tokens, bool) if not causal else (place <= p) & ((place > p - window) if window else True)
        if p < 0 and causal or not seen.any():
            continue
        for h in range(heads):
            kk, vv = k[h // (heads // kv)][seen], v[h // (heads // kv)][seen]
            s = kk @ q[j, h] * scale
            if np.isnan(s).any():
                out[j, h], tol[j, h] = np.nan, 0.0
                continue
            w = np.exp(s - s.max())
            total = w.sum()
            out[j, h] = w @ vv / total
            mixed = w @ np.abs(vv) / total
            score = 2 * e * (dim + 4) * (np.abs(kk) @ np.abs(q[j, h])).max() * abs(scale) + 4 * e * np.abs(s).max() + 2 * e * (s.max() - s.min())
            rel = 2 * (half + score + 8 * e) + 2 * e * len(s)
            tol[j, h] = rel * mixed + half * np.abs(out[j, h]) + len(s) * 2.0 ** -34 * np.abs(vv).max() * (bits == 11) + 2.0 ** -24
    return out, tol


class Tenant:
    """One tenant's cache and sequences: (new, length) pairs; the cache is filled on the host and checked on the way back."""

    def __init__(self, heads, kv_heads, dim, dtype, seqs, page=16, causal=True, window=0, scale=None, seed=0, spare=3, garbage=True, pad=0, gain=1.0, max_new=None,
                 filled=True, spread=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.heads, self.kv, self.dim, self.dtype, self.seqs, self.page = heads, kv_heads, dim, dtype, list(seqs), page
        self.causal, self.window, self.scale = causal, window, dim ** -0.5 if scale is None else scale
        self.tt = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
        self.bits = {"bf16": 8, "f16": 11}[dtype]
        need = [-(-length // page) for _, length in self.seqs]
        self.columns = max([1] + need) + 1
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((max(1, len(self.seqs)), self.columns), 1 << 30, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.first = np.concatenate([[0], np.cumsum([n for n, _ in self.seqs])]).astype(np.int32)
        self.length = np.array([n for _, n in self.seqs] or [0], dtype=np.int32)
        self.tokens = int(self.first[-1]) + 2              # two rows that belong to nobody
        self.max_new = max_new or max([1] + [n for n, _ in self.seqs])
        rounded = lambda x: torch.from_numpy(x).to(self.tt).double().numpy()  # noqa: E731
        # all tokens' keys and values of every sequence; the last ones are the new ones
        self.k = [rounded(rng.standard_normal((length, kv_heads, dim)) * spread) for _, length in self.seqs]
        self.v = [rounded(rng.standard_normal((length, kv_heads, dim))) for _, length in self.seqs]
        self.q = rounded(rng.standard_normal((self.tokens, heads, dim)) * gain)
        # memory that was never written holds anything: every byte 255 is a scale that is no number
        self.pool = Pool(self.n_pages, kv_heads, page, dim, 255 if garbage else 0)
        self.pad = pad
        if filled:
            self.fill([length for _, length in self.seqs])

    def fill(self, upto):
        for s in range(len(self.seqs)):
            kc, ks, vc, vs = encode_token_head(self.k[s], self.v[s])
            for t in range(upto[s]):
                self.pool.write(self.table[s, t // self.page], t % self.page, kc[t], ks[t], vc[t], vs[t])

    def held(self, s):
        """What the host's pool holds of sequence s: keys and values [kv, tokens, dim]."""
        n = self.seqs[s][1]
        k, v = np.zeros((self.kv, n, self.dim)), np.zeros((self.kv, n, self.dim))
        for t in range(n):
            k[:, t], v[:, t] = self.pool.read(self.table[s, t // self.page], t % self.page)
        return k, v

    def upload(self):
        import torch

        def rows(x):
            whole = torch.full((x.shape[0], x[0].size + self.pad), float("nan"), dtype=self.tt)
            whole[:, :x[0].size] = torch.from_numpy(x.reshape(x.shape[0], -1)).to(self.tt)
            return whole.cuda()
        new = lambda all_: np.concatenate([np.zeros((0, self.kv, self.dim))] + [x[len(x) - n:] if len(x) >= n else np.concatenate([np.zeros((n - len(x), *x.shape[1:])), x])  # noqa: E731
                                                                               for x, (n, _) in zip(all_, self.seqs)] + [np.zeros((2, self.kv, self.dim))])
        self.d = {"q": rows(self.q), "k": rows(new(self.k)), "v": rows(new(self.v))}
        for name, like in (("out", "q"), ("k_out", "k"), ("v_out", "v")):
            self.d[name] = torch.full_like(self.d[like], float("nan"))
        self.d["pages"] = torch.from_numpy(self.pool.bytes).cuda()
        for name in ("table", "first", "length"):
            self.d[name] = torch.from_numpy(getattr(self, name)).cuda()
        return self

    def desc(self, **changes):
        from paper_1901_00041_amd import st_lm
        wide, narrow = self.heads * self.dim + self.pad, self.kv * self.dim + self.pad
        args = dict(n_seqs=len(self.seqs), max_tokens=self.tokens, max_new=self.max_new, n_pages=self.n_pages, page_tokens=self.page, table_pages=self.columns,
                    scale=self.scale, window=self.window, flags=st_lm.ST_ATTN_CAUSAL if self.causal else 0, ldq=wide, ldk=narrow, ldv=narrow, ldo=wide, **self.d)
        args.update(changes)
        return st_lm.make_attn_desc(self.heads, self.kv, self.dim, self.dtype, **args)

    def outputs(self, name="out"):
        heads = self.heads if name == "out" else self.kv
        return self.d[name][:, :heads * self.dim].double().cpu().numpy().reshape(self.tokens, heads, self.dim)

    def check_out(self, what="", skip=()):
        got = self.outputs()
        for s, (n, length) in enumerate(self.seqs):
            if s in skip:
                continue
            k, v = self.held(s)
            rows = slice(self.first[s], self.first[s] + n)
            want, tol = attend(self.q[rows], k, v, length - n, self.scale, self.causal, self.window, self.bits)
            mine = got[rows]
            assert np.array_equal(np.isnan(want), np.isnan(mine)), f"{what}: sequence {s}: not a number where it should be one, or not written"
            over = np.where(np.isnan(want), 0.0, np.abs(mine - want) / np.maximum(tol, 1e-300))
            assert over.size == 0 or over.max() <= 1.0, f"{what}: sequence {s} ({n}, {length}): {over.max():.3g} tolerances off at {np.unravel_index(over.argmax(), over.shape)}"
        self.check_untouched(what, "out")

    def check_untouched(self, what="", *names):
        import torch
        for name in names:
            whole = self.d[name].clone()
            width = (self.heads if name == "out" else self.kv) * self.dim
            whole[:int(self.first[-1]), :width] = float("nan")
            assert torch.isnan(whole).all(), f"{what}: wrote rows of {name} that belong to nobody"
