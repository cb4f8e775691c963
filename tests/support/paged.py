"""A layer's keys and values in scattered pages, on the device and beside it on the CPU, for tests of the operators that read them."""
import math

import numpy as np
import torch

from paper_2604_06664_amd import decode as fdd

DEV = "cuda:0"
DTYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f8=torch.float8_e4m3fn)
ROUND = dict(bf16=2.0 ** -8, f16=2.0 ** -11)  # half a step, of the value


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """Rows of the given lengths; everything in the pools that no row holds is NaN."""

    def __init__(self, lens, H, D, pt=16, order="token", cache="bf16", seed=1, row_pages=None, pad=0, spare=3):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.D, self.pt, self.cache = list(lens), H, D, pt, cache
        pages = [-(-n // pt) for n in lens]
        P = row_pages or max(pages + [1]) + 2
        self.n_pages = sum(pages) + spare
        order_of = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), P), -1, np.int32)
        at = 0
        for r, n in enumerate(pages):
            self.table[r, :n] = order_of[at:at + n]
            at += n
        wide = D + pad
        self.strides = (pt * H * wide + pad, H * wide if order == "token" else wide, wide if order == "token" else pt * wide)
        bits = torch.uint8 if cache == "f8" else torch.int16
        nan = torch.tensor([0x7F], dtype=torch.uint8) if cache == "f8" else torch.tensor([math.nan]).to(DTYPES[cache]).view(bits)
        self.pools, self.views = [], []
        for _ in "kv":
            pool = nan.repeat(self.n_pages * self.strides[0])
            view = torch.as_strided(pool, (self.n_pages, pt, H, D), (*self.strides, 1))
            for r, n in enumerate(lens):
                x = torch.from_numpy(rng.standard_normal((pages[r] * pt, H, D)).astype(np.float32)).to(DTYPES[cache]).view(bits)
                for j in range(pages[r]):
                    m = min(pt, n - j * pt)
                    view[self.table[r, j], :m] = x[j * pt:j * pt + m]
            self.pools.append(pool)
            self.views.append(view.view(DTYPES[cache]))
        self.scales = [torch.from_numpy(rng.uniform(0.5, 1.5, H).astype(np.float32)) if cache == "f8" else None for _ in "kv"]
        self.upload()

    def upload(self):
        """The pools as they are on the CPU now."""
        self.d_pools = [p.to(DEV) for p in self.pools]
        self.d_scales = [None if s is None else s.to(DEV) for s in self.scales]
        self.d_table, self.d_lens = torch.from_numpy(self.table).to(DEV), int32(self.lens)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def kv(self, **kw):
        f = dict(type=fdd.TYPES[self.cache], n_pages=self.n_pages, page_tokens=self.pt, n_heads=self.H, head_dim=self.D,
                 page_stride=self.strides[0], token_stride=self.strides[1], head_stride=self.strides[2],
                 k_scale=self.d_scales[0], v_scale=self.d_scales[1])
        f.update(kw)
        return fdd.make_kv(*self.d_pools, **f)


def near(got, want, kind):
    """Scores are sums of up to 256 products in 32 bits whose sizes, times the softmax factor, add up to at most 16: each is off by up to
    258 roundings of 2^-24 of that, 2^-12.  All weights moved by so much move the output by at most twice that of the largest |v| seen;
    a weight loses 2^-15 in its product with v; the result is rounded once.  The logarithm of the sum: 2^-12 and its own rounding."""
    (out, lse), (o, l, spread) = got[:2], want
    bound = spread[..., None] * (2.0 ** -11 + 2.0 ** -15) + ROUND[kind] * o.abs() + 2.0 ** -24
    err = (out.double() - o).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), int((~(err <= bound)).sum()))
    none = l == -math.inf
    assert torch.equal(lse == -math.inf, none)
    assert bool(((lse.double() - l).abs()[~none] <= 3e-4).all())
    assert bool((out[none] == 0).all())
