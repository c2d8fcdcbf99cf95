"""Models on 8-bit projections whose arithmetic loses next to nothing before the 8-bit codes, in 64 bits, for the tests.

A value that arithmetic moves by 1e-6 of itself takes another code in one of 1e5 cases, and from there on a row is 1e-3 and more
off: with dense weights, sums rounded to bf16 (as passes of more than 64 rows hand them on) leave no row alone.  Here a row
of weights has one value in every 64, each of four significant bits and all of one power: they are 8-bit rows as they
are, a sum has few terms, none next to another in an eight, and is exact in fp32; rounded to bf16 it is the same on both sides.
What is left is the fp32 of attention and of silu, 1e-6 and less, so that most rows are equal to some 1e-6, and a mistake of a
per cent anywhere moves all of them."""
import math

import numpy as np
import torch

import scaled_ref as ref
import workloads as wl

PROJECTIONS = ("wq", "wk", "wv", "wo", "wg", "wu", "wd")
FP32_ROWS = 64      # passes of more rows hand sums on in bf16


def sparse(layers, n, k, g):
    w = torch.zeros(layers, n, k)
    for c in range(0, k, 64):
        width = min(64, k - c)
        at = c + torch.randint(0, width, (layers, n, 1), generator=g)
        if c:      # never beside the value of the 64 before it, in the same eight
            at = torch.maximum(at, torch.full_like(at, min(c + 8, k - 1)))
        v = (8 + torch.randint(0, 8, (layers, n, 1), generator=g)).float() / 8
        w.scatter_(2, at, torch.where(torch.rand(layers, n, 1, generator=g) < 0.5, -v, v))
    return w * 2.0 ** -math.ceil(math.log2(1.5 * (k / 64) ** 0.5))


def bits_of(t):
    return t.bfloat16().view(torch.int16).numpy().view(np.uint16)


def weights(shape, seed):
    """as workloads.make_weights, the projections sparse and the embedding of size 1"""
    out = wl.make_weights(shape, seed=seed, gain_std=0.1)
    g = torch.Generator().manual_seed(seed)
    for name in PROJECTIONS:
        L, n, k = out[name].shape
        out[name] = bits_of(sparse(L, n, k, g))
    out["embed"] = bits_of(torch.randn(out["embed"].shape, generator=g))
    return out


def tensor(a):
    a = np.asarray(a)
    return torch.from_numpy(a.view(np.int16).copy()).view(torch.bfloat16).double() if a.dtype == np.uint16 else torch.from_numpy(a).double()


def hold(v):
    return ref.values(*ref.quantise(v))[:, :v.shape[1]]


class Model:
    """`wrong`: a mistake to plant; `noise`: what attention and silu are off by, relative, to see how far that leads"""

    def __init__(self, shape, w, wrong=None, noise=0.0):
        self.s, self.w, self.wrong, self.noise = shape, {k: tensor(v) for k, v in w.items()}, wrong, noise
        self.gen = torch.Generator().manual_seed(1)

    def norm(self, x, gain):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + self.s.rms_eps) * gain

    def off(self, v):
        return v * (1 + self.noise * torch.randn(v.shape, generator=self.gen, dtype=v.dtype)) if self.noise else v

    def forward(self, ids, many_lower, many_upper, exit_layer, depth=None):
        """one causal forward; many_lower, many_upper [T]: whether the pass that took a row through the layers below and above the exit
        had more than 64 rows.  (logits of the last row, K and V per layer [T][kv heads][head size])"""
        s, w = self.s, self.w
        T, hd, nq, nkv = len(ids), s.head_dim, s.n_q_heads, s.n_kv_heads
        depth = depth or s.n_layers
        inv = torch.tensor([s.rope_base ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float64).float()
        angle = (torch.arange(T).float()[:, None] * inv[None]).double()
        cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        many_lower, many_upper = (torch.as_tensor(m, dtype=torch.bool)[:, None] for m in (many_lower, many_upper))

        def rope(x):
            a, b = x[..., :hd // 2], x[..., hd // 2:]
            return x if self.wrong == "no rotation" else torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        x = w["embed"][torch.as_tensor(ids).long()]
        mask = torch.triu(torch.ones(T, T, dtype=torch.bool), 1)
        cache = []
        for l in range(depth):
            many = many_lower if l < exit_layer else many_upper

            def handed(y):
                if self.wrong == "never in bf16":
                    return y
                return torch.where(many, ref.to_type(y, torch.bfloat16), y.float().double())

            n = hold(self.norm(x, w["attn_norm"][l]))
            q, k = rope(handed(n @ w["wq"][l].T).view(T, nq, hd)), rope(handed(n @ w["wk"][l].T).view(T, nkv, hd))
            k, v = ref.to_type(k, torch.bfloat16), ref.to_type(handed(n @ w["wv"][l].T).view(T, nkv, hd), torch.bfloat16)
            cache.append((k, v))
            out = torch.empty(T, nq, hd, dtype=torch.float64)
            for h in range(nq):
                sc = q[:, h] @ k[:, h // (nq // nkv)].T / math.sqrt(hd)
                if self.wrong == "queries of zeros":
                    sc = sc * 0
                out[:, h] = torch.softmax(sc.masked_fill(mask, -math.inf), -1) @ v[:, h // (nq // nkv)]
            a = out.view(T, nq * hd)
            a[1:] = self.off(a[1:])     # (the first row's is its own values, exactly)
            a = a if self.wrong == "attention not in 8 bits" else hold(a)
            x = (x + handed(a @ w["wo"][l].T)).float().double()
            n = hold(self.norm(x, w["mlp_norm"][l]))
            g, u = n @ w["wg"][l].T, n @ w["wu"][l].T
            if self.wrong == "gate and up exchanged":
                g, u = u, g
            y = handed(hold(self.off(g * torch.sigmoid(g) * u)) @ w["wd"][l].T)
            if self.wrong == "1 % of down":
                y = y * 1.01
            if not (self.wrong == "the last residual left out" and l == depth - 1):
                x = (x + y).float().double()
        h = x[-1:]
        if depth == s.n_layers:
            return (self.norm(h, w["final_norm"]) @ w["lm_head"].T)[0], cache
        u = h + h @ w["lens_a"].T + w["lens_b"]
        return (self.norm(u, w["lens_norm"]) @ w["lens_head"].T)[0], cache


def off(got, want):
    """relative 2-norm over the last side"""
    got, want = torch.as_tensor(got).double(), torch.as_tensor(want).double()
    return (got - want).norm(dim=-1) / want.norm(dim=-1)


def rows_agree(errors):
    """Arithmetic of 1e-5 of itself leaves at least half of the rows where they are (test_scaled_model_checks.py); the others may have
    taken other codes, 2^-4 of a value along three layers of four quantisations each."""
    e = torch.as_tensor(errors).flatten().sort()[0]
    return bool(torch.isfinite(e).all()) and float(e[len(e) // 2]) <= 1e-4 and float(e[-1]) <= 0.1
