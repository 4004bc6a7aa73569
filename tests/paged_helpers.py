"""Shared plumbing of the tests of the paged 8-bit cache: small caches drawn on the host, tolerances."""
import numpy as np
import torch

from oracle import paged_oracle as PO
from paper_2502_14882_amd import paged

# a rounding is off by at most half a step
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}       # half the smallest subnormal


class Case:
    """Host and device side of one step over a paged cache.  lens: tokens in the cache (new ones included), new: new tokens.  Slots
    without a token hold NaN codes, the scales of pages without one NaN."""

    def __init__(self, seed, lens, new, hq, hk, d, page, dtype=torch.float16, spread=3, extra_rows=0, extra_pages=2, normal=False):
        r = np.random.RandomState(seed)
        self.lens, self.new, self.hq, self.hk, self.d, self.page, self.dtype = list(lens), list(new), hq, hk, d, page, dtype
        self.q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.t = int(self.q_start[-1]) + extra_rows
        used = [-(-l // page) for l in self.lens]
        self.max_pages = max(max(used), 1) + 1
        self.n_pages = sum(used) + extra_pages
        ids = r.permutation(self.n_pages)
        self.table = np.full((len(lens), self.max_pages), 1 << 29, np.int32)          # entries behind the end: nothing there
        self.kc = np.full((self.n_pages, hk, page, d), 0x7f, np.uint8)
        self.vc = np.full((self.n_pages, hk, page, d), 0xff, np.uint8)
        self.ks = np.full((self.n_pages, hk), np.nan, np.float32)
        self.vs = np.full((self.n_pages, hk), np.nan, np.float32)
        at = 0
        for b, l in enumerate(self.lens):
            for i in range(used[b]):
                pid = ids[at]
                at += 1
                self.table[b, i] = pid
                live = min(page, l - i * page)
                for c in (self.kc, self.vc):
                    if normal:
                        c[pid, :, :live] = PO.encode_e4m3(np.clip(r.standard_normal((hk, live, d)) * 100, -448, 448))
                    else:
                        x = r.randint(0, 254, (hk, live, d))
                        c[pid, :, :live] = np.where(x < 127, x, x + 1)                    # every finite code
                low = -7 if normal else -12
                self.ks[pid] = np.exp2(r.randint(low - spread, low + 1, hk))
                self.vs[pid] = np.exp2(r.randint(-spread, spread + 1, hk))
        self.q = torch.from_numpy(r.standard_normal((self.t, hq, d)).astype(np.float32)).to(dtype)

    def device(self):
        dev = "cuda"
        cache = paged.PagedCache(torch.from_numpy(self.kc).to(dev),
                                 torch.from_numpy(np.ascontiguousarray(self.vc.transpose(0, 1, 3, 2))).to(dev),
                                 torch.from_numpy(self.ks.copy()).to(dev), torch.from_numpy(self.vs.copy()).to(dev))
        batch = paged.PagedBatch(torch.from_numpy(self.table).to(dev),
                                 torch.tensor(self.lens, dtype=torch.int32, device=dev),
                                 torch.from_numpy(self.q_start).to(dev), max(max(self.new), 1), max(max(self.lens), 1))
        return cache, batch

    def expected(self, causal=True, scale=None, q=None):
        return PO.attend((self.q if q is None else q).double().numpy(), self.kc, self.vc, self.ks.astype(np.float64),
                         self.vs.astype(np.float64), self.table, self.lens, self.q_start, causal, scale)


def assert_attention_close(out, lse, want, case, pair):
    """Against PO.attend.  pair: the weights are pairs of fp16.

    A logit: fp32 sums of d exact products and the factors behind them: (d + 4) 2^-24 of sum |q k| at most.  exp2 of it: the same
    in the exponent, 2^-22 for the function.  The sums of weights: 2^-24 for each addition of a lane (a sixteenth of the
    tokens) and of the joins (below 64 + tokens / 64), of the products as many.  A weight in fp16: 2^-11 of it, or 2^-25 where it is subnormal (the
    largest weight of a part of a row is 1 at least, so that is 2^-25 of the row's sum at most); as a pair 2^-22 and 2^-25 * 2^-11.  Where the
    sum is taken of the rounded weights w (1 + e), it is off by 2^-11 of itself at most as well, which moves the result by 2^-11 |o| <=
    2^-11 of the weighted mean of |v|: 2^-10 together.
    The result: half a step of its type."""
    ref, ref_lse, mean_v, most_v, reach = want
    live = ~np.isnan(ref_lse) if not np.isnan(ref).any() else np.isfinite(ref_lse) | np.isneginf(ref_lse)
    n = max(case.lens)
    logit = (case.d + 4) * 2.0 ** -24 * reach
    sums = (n / 16 + n / 64 + 80) * 2.0 ** -24
    weight, least = (2.0 ** -22, 2.0 ** -36) if pair else (2.0 ** -10, 2.0 ** -25)
    rel = 2 * logit + 2 * sums + 2.0 ** -21 + weight
    tol = HALF_STEP[case.dtype] * np.abs(ref) + LEAST[case.dtype] + (rel[..., None] * mean_v + n * least * most_v) * 1.01
    got = out.double().cpu().numpy()
    err = np.abs(got - ref)
    bad = ~(err <= tol) & live[..., None]
    assert not bad.any(), "%d of %d elements off, worst %.3g of its tolerance; first at %s: got %.6g, want %.6g" % (
        bad.sum(), bad.size, np.nanmax(np.where(live[..., None], err / tol, 0)), np.argwhere(bad)[0], got[bad][0], ref[bad][0])
    if lse is not None:
        got = lse.double().cpu().numpy()
        empty = np.isneginf(ref_lse)
        assert np.array_equal(np.isneginf(got) & live, empty & live)
        with np.errstate(invalid="ignore"):
            off = np.abs(got - ref_lse)
        tol = logit + sums + 2.0 ** -21 + (0 if pair else 2.0 ** -11) + 2.0 ** -22 * np.abs(np.where(empty, 0, ref_lse))
        assert (off[live & ~empty] <= tol[live & ~empty]).all(), (off[live & ~empty] / tol[live & ~empty]).max()
