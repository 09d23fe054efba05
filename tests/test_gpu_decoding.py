"""The operators of language models together, as a server runs them: two tenants' decoder layers step by step, prompts of unlike lengths
first and then a token at a time, every step one product for queries, keys and values, the cache, attention and three products more, each a
call for both tenants.  Every stage is compared with the formula in 64 bits on the very inputs that the GPU gave it."""
import math

import numpy as np
import pytest

from paper_1901_00041_amd import st_lm
from tests.attn_helpers import Pool, attend, encode_token_head

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


class Layer:
    def __init__(self, heads, kv, dim, wide, dtype, lengths, page, seed, rows):
        import torch
        gen = torch.Generator().manual_seed(seed)
        self.heads, self.kv, self.dim, self.dtype, self.page = heads, kv, dim, dtype, page
        self.tt, self.bits = {"bf16": (torch.bfloat16, 8), "f16": (torch.float16, 11)}[dtype]
        self.size, self.cols, self.wide, self.rows = heads * dim, (heads + 2 * kv) * dim, wide, rows
        rand = lambda *s: (torch.randn(*s, generator=gen) * s[-1] ** -0.5).to(self.tt).cuda()  # noqa: E731
        self.w = {"qkv": rand(self.cols, self.size), "out": rand(self.size, self.size), "up": rand(wide, self.size), "down": rand(self.size, wide)}
        self.b = {"qkv": rand(self.cols), "up": rand(wide)}
        new = lambda n: torch.full((rows, n), float("nan"), dtype=self.tt, device="cuda")  # noqa: E731
        self.x, self.qkv, self.mixed, self.mid, self.h, self.y = new(self.size), new(self.cols), new(self.size), new(self.size), new(wide), new(self.size)
        self.gen, self.n_seqs = gen, len(lengths)
        columns = -(-(max(lengths) + 8) // page)
        self.pages = torch.full((self.n_seqs * columns + 1, kv, page // 16, 16 * (dim + dim // 16)), 255, dtype=torch.uint8, device="cuda")
        order = torch.randperm(self.n_seqs * columns, generator=gen).to(torch.int32)
        self.table = order.view(self.n_seqs, columns).cuda()
        self.first = torch.zeros(self.n_seqs + 1, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(self.n_seqs, dtype=torch.int32, device="cuda")
        # what the cache should hold, in float64: [seq] -> ([kv, tokens, dim] keys, values)
        self.held = [(np.zeros((kv, 0, dim)), np.zeros((kv, 0, dim))) for _ in lengths]

    def products(self):
        make = st_lm.make_matmul_desc
        bias, gelu, last = st_lm.ST_EPI_BIAS, st_lm.ST_EPI_GELU, st_lm.ST_EPI_RESIDUAL_LAST
        return [make(self.rows, self.cols, self.size, self.dtype, self.dtype, self.x, self.w["qkv"], self.qkv, bias=self.b["qkv"], epilogue=bias),
                make(self.rows, self.size, self.size, self.dtype, self.dtype, self.mixed, self.w["out"], self.mid, residual=self.x, epilogue=last),
                make(self.rows, self.wide, self.size, self.dtype, self.dtype, self.mid, self.w["up"], self.h, bias=self.b["up"], epilogue=bias | gelu),
                make(self.rows, self.size, self.wide, self.dtype, self.dtype, self.h, self.w["down"], self.y, residual=self.mid, epilogue=last)]

    def attn(self, max_new):
        q, k, v = self.qkv, self.qkv[:, self.size:], self.qkv[:, self.size + self.kv * self.dim:]
        return st_lm.make_attn_desc(self.heads, self.kv, self.dim, self.dtype, self.n_seqs, self.rows, max_new, self.pages.shape[0], self.page,
                                    self.table.shape[1], self.pages, self.table, self.first, self.length, q=q, k=k, v=v, out=self.mixed, scale=self.dim ** -0.5,
                                    flags=st_lm.ST_ATTN_CAUSAL, ldq=self.cols, ldk=self.cols, ldv=self.cols)

    def set_step(self, new):
        import torch
        self.new = new
        self.x[:sum(new)] = torch.randn(sum(new), self.size, generator=self.gen).to(self.tt).cuda()
        self.first.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        self.length.copy_(torch.tensor([h[0].shape[1] + n for h, n in zip(self.held, new)], dtype=torch.int32))
        for t in (self.qkv, self.mixed, self.mid, self.h, self.y):
            t.fill_(float("nan"))
        self.mixed[sum(new):] = 0.0
        self.x[sum(new):] = 0.0

    def check(self, what):
        n = sum(self.new)
        f = {k: getattr(self, k)[:n].double().cpu().numpy() for k in ("x", "qkv", "mixed", "mid", "h", "y")}
        w, b = ({k: t.double().cpu().numpy() for k, t in d.items()} for d in (self.w, self.b))

        def product(name, x, got, bias=None, gelu=False, residual=None):
            import torch
            v = x @ w[name].T
            # as in test_gpu_matmul: the sum, the bias, the activation (slope at most 1.13), the residual, the last rounding
            off = 2 * E * (x.shape[1] + 4) * (np.abs(x) @ np.abs(w[name]).T)
            if bias is not None:
                v, off = v + bias, off + E * np.abs(v + bias)
            if gelu:
                g = (0.5 * torch.from_numpy(v) * torch.erfc(torch.from_numpy(v) / -math.sqrt(2.0))).numpy()
                v, off = g, 1.13 * off + E * (8 * v * v + 32) * np.abs(g)
            if residual is not None:
                v, off = v + residual, off + E * np.abs(v + residual)
            tol = off + (np.abs(v) + off) * 2.0 ** -self.bits + 2.0 ** -24
            assert np.isfinite(got).all() and (np.abs(got - v) <= tol).all(), f"{what}: {name}"

        product("qkv", f["x"], f["qkv"], bias=b["qkv"])
        at = 0
        for s, m in enumerate(self.new):
            rows = slice(at, at + m)
            at += m
            old_k, old_v = self.held[s]
            k, v = (f["qkv"][rows, i:i + self.kv * self.dim].reshape(m, self.kv, self.dim) for i in (self.size, self.size + self.kv * self.dim))
            pool = Pool(1, self.kv, 1024, self.dim)
            kc, ks, vc, vs = encode_token_head(k, v)
            for t in range(m):
                pool.write(0, t, kc[t], ks[t], vc[t], vs[t])
            held = [pool.read(0, t) for t in range(m)]
            both = [np.concatenate([old] + [h[i][:, None] for h in held], 1) for i, old in ((0, old_k), (1, old_v))]
            self.held[s] = tuple(both)
            want, tol = attend(f["qkv"][rows, :self.size].reshape(m, self.heads, self.dim), *both, both[0].shape[1] - m, self.dim ** -0.5, True, 0, self.bits)
            got = f["mixed"][rows].reshape(m, self.heads, self.dim)
            assert (np.abs(got - want) <= tol).all(), f"{what}: attention of sequence {s}"
        product("out", f["mixed"], f["mid"], residual=f["x"])
        product("up", f["mid"], f["h"], bias=b["up"], gelu=True)
        product("down", f["h"], f["y"], residual=f["mid"])


@pytest.mark.parametrize("graphs", [False, True])
def test_prompts_and_then_tokens(graphs):
    import torch
    prompts = [[37, 5, 0, 130], [1, 70]]
    layers = [Layer(8, 2, 64, 700, "bf16", prompts[0], 16, 1, sum(prompts[0])), Layer(4, 4, 128, 1024, "f16", prompts[1], 64, 2, sum(prompts[1]))]
    products = [st_lm.st_matmul_plan([layer.products()[i] for layer in layers], keep=layers) for i in range(4)]
    plans = {most: st_lm.st_attn_plan([layer.attn(most) for layer in layers], keep=layers) for most in (1, 130)}
    stream = torch.cuda.Stream()

    def step(most):
        st_lm.st_matmul_run(products[0], stream)
        st_lm.st_attn_append(plans[most], stream)
        st_lm.st_attn_run(plans[most], stream)
        for p in products[1:]:
            st_lm.st_matmul_run(p, stream)

    graph = torch.cuda.CUDAGraph()
    if graphs:
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step(1)
    for turn in range(6):
        for layer, prompt in zip(layers, prompts):
            layer.set_step(prompt if turn == 0 else [0 if (turn + s) % 4 == 3 else 1 for s in range(len(prompt))])
        torch.cuda.synchronize()
        if turn == 0 or not graphs:
            step(130 if turn == 0 else 1)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for i, layer in enumerate(layers):
            layer.check(f"step {turn}, tenant {i}")
    assert all(st_lm.st_attn_status(p) == 0 for p in plans.values())
