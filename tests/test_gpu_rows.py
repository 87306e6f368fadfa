"""GPU parity of the operators on rows of logits (adjusting, recording, distilling) with the oracle, through the C ABI.

Bounds.  u = 2^-24 is half a step of fp32, h = 2^-8 of bf16, relative to the value.
  adjust   at most four roundings of values no larger than `size`: 4 u size, and h of the result where it is stored as bf16
  sums     an exponential 2^x of the hardware is off by 2 u and its argument x = (z - m) c2 by 3 u |x|; no entry passes through more than
           V / 256 + 96 additions and joins; so a log-sum-exp is off by at most e = u (V / 256 + 100 + 3 X) with X the mean of |x| (base e)
           under the row's distribution, and by three roundings of its own value
  distill  ln p and ln q are off by at most e + u (4 + 4 |ln|) each, so a probability by that relative amount, a divergence sum p ln(p / q) by
           that times (2 + sum p |ln p / q|), a gradient q P - p by that times q + p (+ the rest's mass likewise)
"""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2510_12966_amd as psd
from paper_2510_12966_amd import synth

pytestmark = pytest.mark.gpu

U, H = 2.0 ** -24, 2.0 ** -8
INF = np.inf
DTYPES = (psd.F32, psd.BF16)


def to_bf16(a):
    b = np.ascontiguousarray(a, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def rounded(a, dtype):
    """The values a row of the type holds, as float32."""
    a = np.asarray(a, np.float32)
    return a if dtype == psd.F32 else synth.bf16_to_f32(to_bf16(a))


def raw(a, dtype):
    return np.ascontiguousarray(a, np.float32) if dtype == psd.F32 else to_bf16(a)


GAP = -77.0   # what stands between rows


class Rows:
    """n rows of V logits, `stride` apart, `lead` elements into a device buffer; the gaps hold a value that must stay."""

    def __init__(self, rows, dtype, stride=None, lead=0):
        self.n, self.V = rows.shape
        self.dtype, self.stride, self.lead = dtype, stride or self.V, lead
        whole = np.full(lead + self.n * self.stride, GAP, np.float32)
        whole[lead:].reshape(self.n, self.stride)[:, :self.V] = rows
        self.buf = psd.DeviceBuffer.from_numpy(raw(whole, dtype))
        self.el = 4 if dtype == psd.F32 else 2

    def data_ptr(self):
        return self.buf.data_ptr() + self.lead * self.el

    def get(self):
        size = self.lead + self.n * self.stride
        a = self.buf.to_numpy(np.float32 if self.dtype == psd.F32 else np.uint16, size)
        a = a if self.dtype == psd.F32 else synth.bf16_to_f32(a)
        body = a[self.lead:].reshape(self.n, self.stride)
        assert (a[:self.lead] == GAP).all() and (body[:, self.V:] == GAP).all(), "written outside the rows"
        return body[:, :self.V].copy()


def dev(a, dtype=None):
    return None if a is None else psd.DeviceBuffer.from_numpy(np.ascontiguousarray(a, dtype))


def sync_get(buf, dtype, shape):
    psd.dev_sync()
    return buf.to_numpy(dtype, shape)


# ---- adjusting -----------------------------------------------------------------------------------------

class Batch:
    """Random edits of S sequences of R rows: histories of the given lengths, biases, masks."""

    def __init__(self, rng, S, R, V, lengths, n_bias=0, n_masks=0, wild=True):
        self.S, self.R, self.V = S, R, V
        self.off = np.concatenate(([0], np.cumsum(lengths))).astype(np.int64)
        lo, hi = (-3, V + 3) if wild else (0, V)      # some tokens outside the vocabulary
        self.history = np.where(rng.random(self.off[-1]) < 0.5, rng.integers(0, min(V, 7), self.off[-1]), rng.integers(lo, hi, self.off[-1])).astype(np.int32)
        self.n_prompt = np.array([rng.integers(0, n + 2) for n in lengths], np.int32)
        self.window = rng.integers(lo, hi, (S, max(R - 1, 1) + 2)).astype(np.int32)
        self.window[:, 1::2] = self.window[:, :1]      # the same proposal again and again
        self.penalties = np.stack((rng.uniform(0.5, 2, S), rng.uniform(-1, 1, S), rng.uniform(-0.5, 0.5, S)), 1).astype(np.float32)
        self.boff = (np.arange(S + 1) * n_bias).astype(np.int64)
        self.btok = np.where(rng.random(S * n_bias) < 0.5, rng.integers(0, min(V, 5), S * n_bias), rng.integers(lo, hi, S * n_bias)).astype(np.int32)
        self.bias = rng.normal(0, 3, S * n_bias).astype(np.float32)
        self.bias[::7] = -INF
        self.n_masks = n_masks
        self.masks = rng.integers(0, 2 ** 32, (n_masks, (V + 31) // 32), dtype=np.uint64).astype(np.uint32)
        if n_masks > 1:
            self.masks[1] = 0                          # allows nothing
        self.mask_index = rng.integers(-1, n_masks + (2 if wild else 0), S * R).astype(np.int32)

    def device(self):
        nb = self.bias.size
        a = psd.Adjust(history=dev(self.history) if self.history.size else None, history_offsets=dev(self.off), n_history=self.history.size,
                       n_prompt=dev(self.n_prompt), window=dev(self.window) if self.R > 1 else None, window_stride=self.window.shape[1],
                       penalties=dev(self.penalties), bias_tokens=dev(self.btok) if nb else None, bias=dev(self.bias) if nb else None,
                       bias_offsets=dev(self.boff) if nb else None, n_bias=nb, masks=dev(self.masks) if self.n_masks else None,
                       mask_index=dev(self.mask_index) if self.n_masks else None, n_masks=self.n_masks)
        return a

    def oracle(self, z):
        """(result, size) of every row: `size` is the largest value that its roundings are relative to."""
        out, size = np.empty(z.shape), np.empty(z.shape)
        for s in range(self.S):
            h = self.history[self.off[s]:self.off[s + 1]]
            bt, b = (x[self.boff[s]:self.boff[s + 1]] for x in (self.btok, self.bias))
            r, p, f = (float(x) for x in self.penalties[s])
            for j in range(self.R):
                i = s * self.R + j
                m = int(self.mask_index[i]) if self.n_masks else -1
                mask = self.masks[m] if 0 <= m < self.n_masks else None
                w = self.window[s, :j]
                out[i] = oracle.adjust_row(z[i], h, int(self.n_prompt[s]), w, (r, p, f), bt, b, mask, closed=m < -1 or m >= max(self.n_masks, 0) and self.n_masks > 0)
                plain = np.abs(np.where(np.isfinite(z[i]), z[i], 0).astype(np.float64)) * max(r, 1 / r)
                size[i] = plain + abs(p) + abs(f) * (len(h) + j) + np.abs(np.where(np.isfinite(b), b, 0)).max(initial=0)
        return out, size


def check_adjusted(got, want, size, dtype):
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fine = np.isfinite(want)
    assert np.isfinite(got[fine]).all() and np.array_equal(np.isnan(got), np.isnan(want))
    err = np.abs(got[fine] - want[fine])
    tol = 4 * U * size[fine] + (H * np.abs(want[fine]) * (1 + 2 * U) if dtype == psd.BF16 else 0)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("S,R,V,lengths,n_bias,n_masks,stride,lead", [
    (1, 1, 1, [0], 0, 0, None, 0),                       # one logit
    (1, 1, 97, [1], 3, 1, None, 0),
    (1, 9, 512, [40], 0, 0, None, 0),                    # a verify pass of the tiny stack
    (3, 4, 4095, [0, 17, 900], 5, 3, None, 0),           # an empty history in the middle of the batch's lists, odd rows
    (2, 3, 4096, [5, 0], 64, 0, 4101, 3),                # padded rows that start off a 16-byte boundary
    (2, 5, 4097, [100, 33], 1, 4, 4099, 1),              # one entry in the last chunk
    (1, 32, 8200, [3000], 20, 9, None, 0),               # the widest window
    (2, 11, 32003, [511, 4100], 300, 5, None, 0),
    (1, 2, 128256, [70000], 0, 2, None, 0),              # a long history: counts of thousands
    (2, 3, 20001, [9000, 14000], 1500, 3, None, 0),      # long histories and long lists of biases
    (2, 3, 9001, [700, 0], 6000, 2, 9004, 2),            # more biases than a chunk has entries
    (1, 2, 40003, [20000], 40000, 2, None, 0),           # the same in the largest chunks
    (24, 12, 20001, [17000] * 23 + [3], 40, 5, None, 0), # several rows of such chunks by one workgroup
    (300, 1, 32003, [9] * 299 + [5000], 3, 4, None, 0),  # many sequences of one row
])
def test_adjust_matches_oracle(dtype, S, R, V, lengths, n_bias, n_masks, stride, lead):
    rng = np.random.default_rng(V + S)
    z = rounded(rng.normal(0, 4, (S * R, V)), dtype)
    z[:, ::11] = -INF
    b = Batch(rng, S, R, V, lengths, n_bias, n_masks)
    x, y = Rows(z, dtype, stride, lead), Rows(np.zeros_like(z), dtype, stride, lead)
    a = b.device()
    psd.adjust_logits(x, y, S, R, V, a, dtype=dtype, logits_stride=stride, out_stride=stride)
    psd.dev_sync()
    got = y.get()
    want, size = b.oracle(z)
    check_adjusted(got, want, size, dtype)
    assert np.array_equal(x.get(), z)
    psd.adjust_logits(x, x, S, R, V, a, dtype=dtype, logits_stride=stride, out_stride=stride)    # in place: the same bits
    psd.dev_sync()
    assert np.array_equal(x.get(), got)


def test_adjust_one_kind_at_a_time_and_none():
    rng = np.random.default_rng(2)
    S, R, V = 2, 3, 5000
    z = rng.normal(0, 4, (S * R, V)).astype(np.float32)
    z[0, 5], z[1, 6], z[2, 7] = np.nan, INF, -3.402823466e38
    full = Batch(rng, S, R, V, [30, 400], 10, 3, wild=False)
    x, y = Rows(z, psd.F32), Rows(np.zeros_like(z), psd.F32, V + 1)
    keep = full.device()
    none = psd.Adjust()
    psd.adjust_logits(x, y, S, R, V, none, out_stride=V + 1)
    psd.dev_sync()
    assert np.array_equal(y.get(), z, equal_nan=True)      # nothing asked for: a copy
    for kind in ("history", "window", "bias", "masks"):
        b = Batch(rng, S, R, V, [0, 0], 0, 0, wild=False)
        b.window[:] = -1
        a = psd.Adjust(penalties=dev(full.penalties))
        if kind == "history":                              # without n_prompt: everything counts
            b.off, b.history, b.n_prompt = full.off, full.history, np.zeros(S, np.int32)
            a = psd.Adjust(history=dev(full.history), history_offsets=dev(full.off), n_history=full.history.size, penalties=dev(full.penalties))
        if kind == "window":
            b.window = full.window
            a = psd.Adjust(window=dev(full.window), window_stride=full.window.shape[1], penalties=dev(full.penalties))
        if kind == "bias":
            b.boff, b.btok, b.bias = full.boff, full.btok, full.bias
            a = psd.Adjust(bias_tokens=dev(full.btok), bias=dev(full.bias), bias_offsets=dev(full.boff), n_bias=full.bias.size)
        if kind == "masks":
            b.masks, b.mask_index, b.n_masks = full.masks, full.mask_index, 3
            a = psd.Adjust(masks=dev(full.masks), mask_index=dev(full.mask_index), n_masks=3)
        b.penalties = full.penalties
        psd.adjust_logits(x, y, S, R, V, a, out_stride=V + 1)
        psd.dev_sync()
        want, size = b.oracle(z)
        got = y.get()
        bad = ~np.isfinite(z)
        check_adjusted(np.where(bad, 0, got), np.where(bad, 0, want), size, psd.F32)
        assert np.array_equal(np.isnan(got[bad]), np.isnan(want[bad])) and np.array_equal(np.isneginf(got), np.isneginf(want))
    # penalties without anything to penalise, history without penalties: copies again
    for a in (psd.Adjust(penalties=dev(full.penalties)), psd.Adjust(history=dev(full.history), history_offsets=dev(full.off), n_history=full.history.size)):
        psd.adjust_logits(x, y, S, R, V, a, out_stride=V + 1)
        psd.dev_sync()
        assert np.array_equal(y.get(), z, equal_nan=True)
    del keep


@pytest.mark.parametrize("dtype", DTYPES)
def test_adjust_penalties_far_from_one(dtype):
    """Results beyond the largest float are infinite, as in the formula, never NaN; small ones keep their precision."""
    reps = np.array([0.5, 1e-30, 1e30, 1.0, 1e-3, 65504], np.float32)
    z = np.tile(np.array([3e38, -3e38, 1e30, 5, 0, -0.0, -5, 1e-30, -INF, 7.3], np.float32), (reps.size, 1))
    z = rounded(z, dtype)
    S, V = z.shape
    x, y = Rows(z, dtype), Rows(np.zeros((S, V)), dtype)
    history = np.tile(np.arange(V, dtype=np.int32), S)
    pen = np.stack((reps, 0 * reps, 0 * reps), 1)
    psd.adjust_logits(x, y, S, 1, V, psd.Adjust(history=dev(history), history_offsets=dev(np.arange(S + 1, dtype=np.int64) * V), n_history=history.size, penalties=dev(pen)), dtype=dtype)
    psd.dev_sync()
    r = reps[:, None].astype(np.float64)
    want = np.where(z > 0, z / r, z * r)
    big = float(np.finfo(np.float32).max) if dtype == psd.F32 else 3.3895313892515355e38
    got = y.get()
    inside = np.abs(want) <= big
    assert np.array_equal(got[~inside], np.sign(want[~inside]) * INF)
    err = np.abs(got[inside] - want[inside])
    assert (err <= np.abs(want[inside]) * ((H if dtype == psd.BF16 else 0) + 2 * U) + 2e-38).all()   # two roundings, and what lies below the smallest normal


@pytest.mark.parametrize("dtype", DTYPES)
def test_adjust_the_smallest_repetitions(dtype):
    """Quotients by numbers whose inverse no float holds, with the bounds of the test above."""
    reps = np.array([1.17549435e-38, 5e-39, 2.9e-39, 1e-40, 1.4e-45, 2.0 ** -100, 1e-31], np.float32)
    z = np.tile(np.array([1e-3, 0.25, 1e-7, 5, 0, -0.0, -5, 1e-20, -INF, 3e38, -3e38, 1e-37, 0.9], np.float32), (reps.size, 1))
    z = rounded(z, dtype)
    S, V = z.shape
    x, y = Rows(z, dtype), Rows(np.zeros((S, V)), dtype)
    history = np.tile(np.arange(V, dtype=np.int32), S)
    pen = np.stack((reps, 0 * reps, 0 * reps), 1)
    psd.adjust_logits(x, y, S, 1, V, psd.Adjust(history=dev(history), history_offsets=dev(np.arange(S + 1, dtype=np.int64) * V), n_history=history.size, penalties=dev(pen)), dtype=dtype)
    psd.dev_sync()
    r = reps[:, None].astype(np.float64)
    want = np.where(z > 0, z / r, z * r)
    big = float(np.finfo(np.float32).max) if dtype == psd.F32 else 3.3895313892515355e38
    got = y.get()
    inside = np.abs(want) <= big
    assert np.array_equal(got[~inside], np.sign(want[~inside]) * INF)
    err = np.abs(got[inside] - want[inside])
    assert (err <= np.abs(want[inside]) * ((H if dtype == psd.BF16 else 0) + 2 * U) + 2e-38).all()


def test_rows_far_apart():
    """Rows more than 2^31 elements apart: every offset is taken in 64 bits."""
    rng = np.random.default_rng(9)
    n, V, k, stride = 2, 3000, 5, 2 ** 31 + 5
    t, z = pair(rng, n, V, psd.BF16)
    z = rounded(z, psd.BF16)
    buf = psd.DeviceBuffer((stride + V) * 2)
    L = psd.lib()
    for r in range(n):
        bits = to_bf16(z[r])
        psd.binding._check(L.psd_dev_copy(buf.data_ptr() + r * stride * 2, bits.ctypes.data, bits.nbytes, 0))

    def rows():
        out = np.empty((n, V), np.uint16)
        for r in range(n):
            psd.binding._check(L.psd_dev_copy(out[r].ctypes.data, buf.data_ptr() + r * stride * 2, V * 2, 1))
        return synth.bf16_to_f32(out)

    got = run_top(buf, n, V, k, 1.0, psd.BF16, stride)
    check_top(z, k, 1.0, got)
    values, ids, lse = records(t, k, 1.0)
    loss, nb = dev(np.zeros(n, np.float32)), psd.distill_workspace_bytes(n, V, k)
    ws = psd.DeviceBuffer(nb)
    small = Rows(z * 0, psd.BF16)
    psd.distill(buf, n, V, dev(values), dev(ids), dev(lse), k, 1.0, psd.DIV_KL, None, loss, small, ws, nb, dtype=psd.BF16, stride=stride)
    grad = small.get()
    check_distill(z, values, ids, lse, 1.0, psd.DIV_KL, None, sync_get(loss, np.float32, n), grad, psd.BF16)
    psd.adjust_logits(buf, buf, 1, n, V, psd.Adjust(bias=dev(np.array([2.0], np.float32)), bias_tokens=dev(np.array([7], np.int32)), bias_offsets=dev(np.array([0, 1], np.int64)), n_bias=1),
                      dtype=psd.BF16, logits_stride=stride, out_stride=stride)
    psd.dev_sync()
    want = z.copy()
    want[:, 7] = rounded(want[:, 7] + 2, psd.BF16)
    assert np.array_equal(rows(), want)
    psd.distill(buf, n, V, dev(values), dev(ids), dev(lse), k, 1.0, psd.DIV_KL, None, loss, buf, ws, nb, dtype=psd.BF16, stride=stride, grad_stride=stride)
    psd.dev_sync()
    check_distill(want, values, ids, lse, 1.0, psd.DIV_KL, None, loss.to_numpy(np.float32, n), rows(), psd.BF16)


def test_adjust_brings_bad_offsets_into_range():
    z = np.arange(12, dtype=np.float32).reshape(2, 6)
    x, y = Rows(z, psd.F32), Rows(z * 0, psd.F32)
    hist = dev(np.array([1, 2, 3, 4], np.int32))
    pen = dev(np.array([[1, 1, 0], [1, 1, 0]], np.float32))
    for off, sets in (([-5, 2, 99], ({1, 2}, {3, 4})), ([3, 1, 2], (set(), {2})), ([99, -1, 2 ** 40], (set(), {1, 2, 3, 4}))):
        psd.adjust_logits(x, y, 2, 1, 6, psd.Adjust(history=hist, history_offsets=dev(np.array(off, np.int64)), n_history=4, penalties=pen))
        psd.dev_sync()
        want = z - np.array([[v in s for v in range(6)] for s in sets])
        assert np.array_equal(y.get(), want), off


# ---- recording -----------------------------------------------------------------------------------------

def run_top(x, n, V, k, T, dtype, stride=None, want_lse=True, stream=None):
    values, ids = dev(np.full((n, k), 7.0, np.float32)), dev(np.full((n, k), -9, np.int32))
    lse = dev(np.full(n, 7.0, np.float32)) if want_lse else None
    nb = psd.top_logits_workspace_bytes(n, V, k)
    ws = dev(np.full(max(nb // 4, 4), 0x7fc00000, np.uint32))
    psd.top_logits(x, n, V, k, T, values, ids, lse, ws, nb, dtype=dtype, stride=stride, stream=stream)
    psd.dev_sync()
    return values.to_numpy(np.float32, (n, k)), ids.to_numpy(np.int32, (n, k)), lse.to_numpy(np.float32, n) if want_lse else None


def want_top(z, k):
    """The record's values and tokens by a stable sort; entries of -inf are none."""
    ids = np.argsort(-z, axis=-1, kind="stable")[:, :k].astype(np.int32)
    values = np.take_along_axis(z, ids, -1)
    return values, np.where(values == -INF, -1, ids)


def lse_bound(z, T):
    a = z.astype(np.float64) / T
    m = a.max()
    p = np.exp(a - m)
    X = (p * np.where(np.isfinite(a), m - a, 0)).sum() / p.sum()
    lse = m + np.log(p.sum())
    return lse, U * (z.size / 256 + 100 + 3 * X) + 3 * U * (abs(lse) + abs(m))


def check_top(z, k, T, got):
    values, ids, lse = got
    wv, wi = want_top(z, k)
    assert np.array_equal(ids, wi)
    assert np.array_equal(values, wv)
    if lse is not None:
        for r in range(z.shape[0]):
            if (z[r] == -INF).all():
                assert lse[r] == -INF
                continue
            want, tol = lse_bound(z[r], T)
            assert abs(lse[r] - want) <= tol, (r, lse[r], want, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,V,k,T,stride,lead", [
    (1, 1, 1, 1.0, None, 0), (3, 2, 2, 1.0, None, 0), (2, 255, 255, 1.0, None, 0), (4, 256, 256, 0.5, None, 0), (2, 257, 256, 1.0, None, 1),
    (5, 4095, 20, 1.0, 4103, 3), (1, 4097, 256, 1.0, None, 0), (17, 32003, 8, 0.7, None, 0), (1, 128256, 20, 1.0, None, 0), (3, 128255, 256, 2.0, None, 0),
    (1100, 9000, 5, 1.0, None, 0), (1030, 4500, 256, 1.0, 4507, 0),       # enough rows for one workgroup each
])
def test_top_matches_a_stable_sort(dtype, n, V, k, T, stride, lead):
    rng = np.random.default_rng(V + k)
    z = rounded(rng.normal(0, 3, (n, V)), dtype)
    x = Rows(z, dtype, stride, lead)
    got = run_top(x, n, V, k, T, dtype, stride)
    check_top(z, k, T, got)
    again = run_top(x, n, V, k, T, dtype, stride, want_lse=False)
    assert np.array_equal(again[0], got[0]) and np.array_equal(again[1], got[1])


def orders(V, n):
    rng = np.random.default_rng(V)
    z = np.empty((9, V), np.float32)
    z[0] = 0.0                                                       # all equal
    z[1] = np.arange(V)                                              # ascending: every block beats what came before
    z[2] = -np.arange(V)                                             # descending
    z[3] = np.where(np.arange(V) % 3 == 0, 0.0, -0.0)                # zeros of both signs are equal
    z[4] = rng.integers(0, 3, V)                                     # three values
    z[5] = -INF
    z[6] = np.where(rng.random(V) < 0.001, rng.normal(0, 1, V), -INF)   # a handful of entries
    z[7] = -3.402823466e38                                           # the lowest finite value throughout
    z[8] = np.where(np.arange(V) >= V - 40, 1e-42 * np.arange(V), -1.0)  # denormals at the end
    return np.tile(z, (n, 1))


@pytest.mark.parametrize("reps", [1, 120])   # several segments a row, one segment a row
@pytest.mark.parametrize("V,k", [(5000, 256), (20000, 64), (20000, 1)])
def test_top_ties_orders_and_short_rows(V, k, reps):
    z = orders(V, reps)
    x = Rows(z, psd.F32)
    check = z[:9]
    values, ids, lse = run_top(x, z.shape[0], V, k, 1.0, psd.F32)
    assert np.array_equal(ids.reshape(reps, 9, k), np.broadcast_to(ids[:9], (reps, 9, k)))
    assert np.array_equal(lse.reshape(reps, 9), np.broadcast_to(lse[:9], (reps, 9)))
    check_top(check, k, 1.0, (values[:9], ids[:9], lse[:9]))


@pytest.mark.parametrize("T", [0.7, 3.0, 0.013, 1.0])
def test_top_lse_of_one_entry_is_its_quotient_rounded_once(T):
    z = np.random.default_rng(1).normal(0, 300, (500, 1)).astype(np.float32)
    _, _, lse = run_top(Rows(z, psd.F32), 500, 1, 1, T, psd.F32)
    want = z[:, 0].astype(np.float64) / float(np.float32(T))
    assert (np.abs(lse - want) <= U * np.abs(want) * (1 + 2.0 ** -20)).all()


# ---- distilling ----------------------------------------------------------------------------------------

def run_distill(x, n, V, values, ids, lse, k, T, div, weights, dtype, stride=None, want_grad=True, in_place=False, gstride=None, stream=None):
    loss = dev(np.full(n, 7.0, np.float32))
    grad = None if not want_grad else x if in_place else Rows(np.full((n, V), 5.0), dtype, gstride or stride)
    nb = psd.distill_workspace_bytes(n, V, k)
    ws = dev(np.full(nb // 4, 0x7fc00000, np.uint32))
    psd.distill(x, n, V, dev(values, np.float32), dev(ids, np.int32), dev(lse, np.float32), k, T, div, dev(weights, np.float32), loss, grad, ws, nb,
                dtype=dtype, stride=stride, grad_stride=gstride or stride, stream=stream)
    psd.dev_sync()
    return loss.to_numpy(np.float32, n), grad.get() if want_grad else None


def distill_bounds(z, values, ids, lse, T, div, weight):
    """Loss, gradient and their bounds for one row with a distribution on both sides."""
    loss, grad = oracle.distill_row(z, values, ids, lse, T, div, weight)
    V = z.size
    a = z.astype(np.float64) / T
    with np.errstate(divide="ignore", invalid="ignore"):   # -inf logits
        lq = a - a.max() - np.log(np.exp(a - a.max()).sum())   # the largest entry first: it may be the type's lowest value
    q = np.exp(lq)
    seen, first = set(), []
    for i, v in enumerate(ids):
        if 0 <= v < V and v not in seen:
            seen.add(int(v))
            first.append(i)
    tok, val = np.asarray(ids)[first], np.asarray(values, np.float64)[first] / T
    lp = val - (float(np.float32(lse)) if lse is not None else np.logaddexp.reduce(val))
    p = np.exp(lp)
    outside = np.ones(V, bool)
    outside[tok] = False
    q_rest = q[outside].sum()
    p_rest = max(0.0, 1 - p.sum()) if lse is not None and (np.asarray(ids) >= 0).all() and outside.any() else 0.0
    mean_x = (q * np.where(np.isfinite(lq), np.abs(lq), 0)).sum()
    e = U * (V / 256 + 100 + 3 * mean_x)
    big = lambda l: np.abs(np.where(np.isfinite(l), l, 0))  # noqa: E731
    d_l = big(lp - np.where(np.isfinite(lq[tok]), lq[tok], 0))
    e_p, e_q = U * (4 + 4 * big(lp)), e + U * (4 + 4 * big(lq[tok]))
    # the rest of the teacher is a difference from 1: absolute error of the sum of p; its logarithm then is off by that over p_rest
    d_rest = (e_p * p).sum() + 2 * U
    lqr = np.log(q_rest) if q_rest > 0 else 0.0
    lpr = np.log(p_rest) if p_rest > 0 else 0.0
    e_qr = 2 * e + U * (4 + 4 * abs(lqr))
    tol = (p * (e_p + e_q) * (2 + d_l)).sum() + d_rest * (2 + abs(lpr - lqr)) + p_rest * (e_qr + 4 * U * (1 + abs(lpr))) + (q[tok] * e_q * 3).sum() + 3 * q_rest * e_qr
    tol = abs(weight) * tol + 2 * U * abs(loss)
    share = np.where(outside, q / max(q_rest, 1e-300), 0.0)
    gt = np.empty(V)
    x_err = e + U * (4 + 4 * big(lq))
    gt[:] = share * (q_rest * (x_err + e_qr) * 4 + p_rest * x_err * 4 + 3 * d_rest) + 2 * U * np.abs(grad) * T / abs(weight)
    gt[tok] = 4 * (q[tok] * (e_q + d_rest) + p * (e_p + e_q))
    return loss, grad, tol, abs(weight) / T * gt * (1 if div == 0 else 2)


def check_distill(z, values, ids, lse, T, div, weights, loss, grad, dtype):
    for r in range(z.shape[0]):
        w = 1.0 if weights is None else float(np.float32(weights[r]))
        ls = None if lse is None else lse[r]
        if w == 0.0 or not ((ids[r] >= 0) & (ids[r] < z.shape[1])).any():
            assert loss[r] == 0.0 and (grad is None or (grad[r] == 0).all())
            continue
        want, wg, tol, gtol = distill_bounds(z[r], values[r], ids[r], ls, T, div, w)
        assert abs(loss[r] - want) <= tol, (r, loss[r], want, tol)
        if grad is not None:
            err = np.abs(grad[r] - wg)
            gtol = gtol + 1e-38 + (H * (np.abs(wg) + gtol) if dtype == psd.BF16 else 0)
            assert (err <= gtol).all(), (r, int((err - gtol).argmax()), (err / gtol).max())


def pair(rng, n, V, dtype, spread=3.0):
    t = rng.normal(0, spread, (n, V)).astype(np.float32)
    return t, rounded(0.8 * t + rng.normal(0, 1, (n, V)), dtype)


def records(t, k, T):
    values, ids = want_top(t, k)
    a = t.astype(np.float64) / T
    m = a.max(-1, keepdims=True)
    return values.astype(np.float32), ids, (m[:, 0] + np.log(np.exp(a - m).sum(-1))).astype(np.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("div", [psd.DIV_KL, psd.DIV_JSD])
@pytest.mark.parametrize("n,V,k,T,whole,stride,lead", [
    (1, 1, 1, 1.0, False, None, 0), (2, 5, 5, 1.0, False, None, 0), (3, 512, 256, 1.0, False, None, 0), (2, 1001, 1, 2.0, False, 1003, 3),
    (4, 8191, 64, 1.0, True, None, 0), (3, 8192, 100, 1.0, False, 8197, 1), (3, 8193, 7, 0.5, False, None, 0), (9, 32003, 32, 1.0, False, None, 0),
    (2, 128256, 256, 1.0, False, None, 0), (1, 128255, 128, 2.0, True, 128257, 0), (300, 700, 20, 1.0, False, None, 0), (600, 9001, 16, 1.0, False, None, 0),
])
def test_distill_matches_oracle(dtype, div, n, V, k, T, whole, stride, lead):
    rng = np.random.default_rng(V + k)
    t, z = pair(rng, n, V, dtype)
    values, ids, lse = records(t, k, T)
    lse = None if whole else lse
    weights = rng.uniform(-1, 2, n).astype(np.float32)
    weights[n // 2] = 0.0 if n > 2 else weights[n // 2]
    x = Rows(z, dtype, stride, lead)
    loss, grad = run_distill(x, n, V, values, ids, lse, k, T, div, weights, dtype, stride)
    check_distill(z, values, ids, lse, T, div, weights, loss, grad, dtype)
    only, _ = run_distill(x, n, V, values, ids, lse, k, T, div, weights, dtype, stride, want_grad=False)
    again, other = run_distill(x, n, V, values, ids, lse, k, T, div, weights, dtype, stride, gstride=(stride or V) + 5)
    assert np.array_equal(only, loss) and np.array_equal(again, loss) and np.array_equal(other, grad)
    inside, gi = run_distill(x, n, V, values, ids, lse, k, T, div, weights, dtype, stride, in_place=True)
    assert np.array_equal(inside, loss) and np.array_equal(gi, grad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("div", [psd.DIV_KL, psd.DIV_JSD])
@pytest.mark.parametrize("reps", [1, 70])
def test_distill_odd_records_and_rows(dtype, div, reps):
    rng = np.random.default_rng(4)
    V, k, T = 9000, 12, 1.0
    t, z = pair(rng, 8, V, dtype)
    values, ids, lse = records(t, k, T)
    ids[0, 5], ids[0, 9], values[0, 9] = ids[0, 2], ids[0, 2], 99.0     # the same token three times
    ids[1, 3], ids[1, 4] = V, 2 ** 31 - 1                               # tokens the student does not have
    ids[2, 4:], values[2, 4:] = -1, -INF                                # a short record
    lse[2] = np.logaddexp.reduce(values[2, :4].astype(np.float64))
    ids[3, :] = -1                                                      # none at all
    z[4, :] = -INF                                                      # the student's tail is closed except for a few entries
    z[4, ids[4]], z[4, :7] = 1.0, 0.25
    z[5, ids[5]] = -30.0                                                # the student all but excludes the teacher's tokens
    z[6, ids[6]] = 60.0                                                 # or everything else
    weights = np.array([1, 0.5, 2, 1, 1, 1, 1, 0], np.float32)
    z[7] = np.nan                                                       # padding is not looked at
    z = rounded(z, dtype)
    big = lambda a: np.tile(a, (reps,) + (1,) * (a.ndim - 1))  # noqa: E731
    x = Rows(big(z), dtype)
    loss, grad = run_distill(x, 8 * reps, V, big(values), big(ids), big(lse), k, T, div, big(weights), dtype)
    assert np.array_equal(loss.reshape(reps, 8), np.broadcast_to(loss[:8], (reps, 8))) and np.array_equal(grad.reshape(reps, 8, V), np.broadcast_to(grad[:8], (reps, 8, V)))
    check_distill(z, values, ids, lse, T, div, weights, loss[:8], grad[:8], dtype)


# enough bytes for every way a call can go: rows that pass by workgroups of three sizes, rows that are held by three sizes, chunks; a few
# rows over and over, so that all but the first few need only be the same
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,row_bytes,odd,k", [
    (257, 30 << 10, 1, 20), (300, 100 << 10, 3, 255), (300, 60 << 10, 0, 256), (2600, 100 << 10, 2, 64), (1300, 200 << 10, 1, 255), (1300, 200 << 10, 0, 256),
    (560, 500 << 10, 3, 100), (40, 300 << 10, 1, 256), (300, 900 << 10, 2, 30), (5, 1100 << 10, 1, 256),
])
def test_distill_every_way(dtype, n, row_bytes, odd, k):
    rng = np.random.default_rng(k)
    V = row_bytes // (4 if dtype == psd.F32 else 2) - odd
    few = 5
    t, z = pair(rng, few, V, dtype)
    values, ids, lse = records(t, k, 1.0)
    ids[1, :12] = (np.arange(12) // 3 * 2 + V - 12) % V      # neighbours and repetitions, up to the row's end
    z[2, ids[2]] = -40.0
    z = rounded(z, dtype)
    weights = np.array([1.0, 0.7, 2.0, 0.0, 1.5], np.float32)
    at = np.arange(n) % few
    x = Rows(z[at], dtype)
    for div in (psd.DIV_KL, psd.DIV_JSD):
        loss, grad = run_distill(x, n, V, values[at], ids[at], lse[at], k, 1.0, div, weights[at], dtype)
        check_distill(z, values, ids, lse, 1.0, div, weights, loss[:few], grad[:few], dtype)
        assert np.array_equal(loss, loss[at]) and all(np.array_equal(grad[i], grad[i % few]) for i in range(n))
        only, _ = run_distill(x, n, V, values[at], ids[at], lse[at], k, 1.0, div, weights[at], dtype, want_grad=False)
        assert np.array_equal(only, loss)
    inside, gi = run_distill(x, n, V, values[at], ids[at], lse[at], k, 1.0, psd.DIV_JSD, weights[at], dtype, in_place=True)
    assert np.array_equal(inside, loss) and np.array_equal(gi, grad)


def test_distill_without_student_mass():
    V = 5000
    z = np.zeros((4, V), np.float32)
    z[0, 3] = -INF                    # a token of the teacher is closed
    z[1] = -INF                       # nothing but the record's tokens; the record has something left for the others
    z[1, [3, 9]] = 1.0
    z[2] = z[1]                       # the same, and the record is complete
    z[3] = -INF                       # no distribution
    values = np.tile(np.array([2.0, 1.0, -INF], np.float32), (4, 1))
    ids = np.tile(np.array([3, 9, 11], np.int32), (4, 1))
    ids[2, 2] = -1
    lse = np.full(4, 3.0, np.float32)
    lse[2] = np.logaddexp(2.0, 1.0)
    x = Rows(z, psd.F32)
    loss, grad = run_distill(x, 4, V, values, ids, lse, 3, 1.0, psd.DIV_KL, None, psd.F32)
    assert loss[0] == INF and loss[1] == INF and np.isfinite(loss[2]) and np.isnan(loss[3])
    assert np.isfinite(grad[:3]).all() and abs(grad[0, 3] + np.exp(-1.0)) < 1e-6 and (grad[2, np.setdiff1d(np.arange(V), [3, 9])] == 0).all()
    check_distill(z[2:3], values[2:3], ids[2:3], lse[2:3], 1.0, psd.DIV_KL, None, loss[2:3], grad[2:3], psd.F32)
    loss, grad = run_distill(x, 4, V, values, ids, lse, 3, 1.0, psd.DIV_JSD, None, psd.F32)
    assert np.isfinite(loss[:3]).all() and np.isfinite(grad[:3]).all() and np.isnan(loss[3])
    check_distill(z[:3], values[:3], ids[:3], lse[:3], 1.0, psd.DIV_JSD, None, loss[:3], grad[:3], psd.F32)


def test_distill_lowest_values_and_tiny_vocabularies():
    low = -3.402823466e38
    V, k = 5000, 4
    z = np.zeros((4, V), np.float32)
    z[0] = low                                      # the lowest value throughout is a uniform row
    z[1, 100:] = low                                # a mask of the lowest value
    z[2] = -1e30
    z[2, 3] = -2e30
    z[3] = np.linspace(-3, 3, V)
    values = np.array([[1, 0.5, 0, low], [2, 1, 0, -1], [1, 1, 1, 1], [0.5, 0.25, -np.inf, 1]], np.float32)
    ids = np.array([[3, 9, 200, 4999], [0, 99, 100, 5], [3, 4, 5, 6], [4999, 0, 17, 18]], np.int32)
    for lse in (None, np.array([3.0, 2.5, 3.0, 2.0], np.float32)):
        for div in (psd.DIV_KL, psd.DIV_JSD):
            loss, grad = run_distill(Rows(z, psd.F32), 4, V, values, ids, lse, k, 1.0, div, None, psd.F32)
            kl_inf = div == psd.DIV_KL               # rows 1 and 2 have tokens of the teacher that underflow to no mass at all
            for r in (0, 3) if kl_inf else range(4):
                ls = None if lse is None else lse[r:r + 1]
                check_distill(z[r:r + 1], values[r:r + 1], ids[r:r + 1], ls, 1.0, div, None, loss[r:r + 1], grad[r:r + 1], psd.F32)
            assert np.isfinite(grad).all() and not np.isnan(loss).any()
    # a record longer than the vocabulary: repetitions, tokens that are none
    rng = np.random.default_rng(3)
    for V in (1, 3, 9):
        z = rng.normal(0, 1, (2, V)).astype(np.float32)
        ids = rng.integers(0, V + 2, (2, 200)).astype(np.int32)
        values = rng.normal(0, 1, (2, 200)).astype(np.float32)
        for div in (psd.DIV_KL, psd.DIV_JSD):
            loss, grad = run_distill(Rows(z, psd.F32), 2, V, values, ids, None, 200, 1.0, div, None, psd.F32)
            check_distill(z, values, ids, None, 1.0, div, None, loss, grad, psd.F32)


def test_distill_a_record_that_just_holds_a_grammars_tokens():
    """Masks that leave k tokens, recorded with that k: no place says that the record is complete, and the sum of its probabilities is off 1 by roundings."""
    rng = np.random.default_rng(31)
    for n, V, k in ((64, 1000, 2), (64, 5000, 7), (300, 5000, 64), (20, 128256, 3)):
        t, z = pair(rng, n, V, psd.F32, spread=8)
        allowed = np.argpartition(rng.random((n, V)), k, axis=1)[:, :k]
        closed = np.ones((n, V), bool)
        np.put_along_axis(closed, allowed, False, axis=1)
        t[closed] = z[closed] = -INF
        values, ids, lse = run_top(Rows(t, psd.F32), n, V, k, 1.0, psd.F32)
        a, b = (np.take_along_axis(y, ids, 1).astype(np.float64) for y in (t, z))
        lp, lq = a - np.logaddexp.reduce(a, 1, keepdims=True), b - np.logaddexp.reduce(b, 1, keepdims=True)
        want = (np.exp(lp) * (lp - lq)).sum(1)
        loss, grad = run_distill(Rows(z, psd.F32), n, V, values, ids, lse, k, 1.0, psd.DIV_KL, None, psd.F32)
        # every ln p off by the record's lse and a few roundings more, the remainder left out
        tol = 2.0 ** -20 * (2 + np.abs(lse)) * (1 + np.abs(lp - lq).max(1))
        assert (np.abs(loss - want) <= tol).all() and (grad[closed] == 0).all()
        assert (np.abs(np.take_along_axis(grad, ids, 1) - (np.exp(lq) - np.exp(lp))) <= tol[:, None]).all()
        # a record with a true remainder: the student has no mass for it
        loss, _ = run_distill(Rows(z, psd.F32), n, V, values, ids, lse + np.float32(0.01), k, 1.0, psd.DIV_KL, None, psd.F32)
        assert np.isposinf(loss).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("closed", [-1e9, -3.3895313892515355e38, -INF])
def test_distill_grammar_records_under_masks_of_any_low_value(dtype, closed):
    """A mask may be a large negative number as well as -inf: what roundings leave of a record that holds all of its row is not held against a
    student that has no mass beside it either.  The bounds are those of the test above, h of a gradient stored as bf16 more."""
    rng = np.random.default_rng(37)
    for n, V, allow, k in ((64, 1000, 2, 2), (64, 5000, 7, 7), (64, 5000, 7, 10), (300, 5000, 64, 64), (20, 128256, 3, 3)):
        t, z = pair(rng, n, V, dtype, spread=8)
        allowed = np.argpartition(rng.random((n, V)), allow, axis=1)[:, :allow]
        shut = np.ones((n, V), bool)
        np.put_along_axis(shut, allowed, False, axis=1)
        t[shut], z[shut] = closed, rounded(closed, dtype)
        values, ids, lse = run_top(Rows(t, psd.F32), n, V, k, 1.0, psd.F32)
        a, b = (np.take_along_axis(y, allowed, 1).astype(np.float64) for y in (t, z))
        lp, lq = a - np.logaddexp.reduce(a, 1, keepdims=True), b - np.logaddexp.reduce(b, 1, keepdims=True)
        p, q = np.exp(lp), np.exp(lq)
        mid = np.log((p + q) / 2)
        kl_p, kl_q = p * (lp - mid), q * (lq - mid)
        tol = 2.0 ** -20 * (2 + np.abs(lse)) * (1 + np.abs(lp - lq).max(1))
        for div, want, wg in ((psd.DIV_KL, (p * (lp - lq)).sum(1), q - p), (psd.DIV_JSD, (kl_p + kl_q).sum(1) / 2, (kl_q - q * kl_q.sum(1, keepdims=True)) / 2)):
            loss, grad = run_distill(Rows(z, dtype), n, V, values, ids, lse, k, 1.0, div, None, dtype)
            assert (np.abs(loss - want) <= tol).all(), (V, div, np.abs(loss - want).max())
            assert (grad[shut] == 0).all()
            assert (np.abs(np.take_along_axis(grad, allowed, 1) - wg) <= tol[:, None] + (H * (np.abs(wg) + tol[:, None]) if dtype == psd.BF16 else 0)).all()


@pytest.mark.parametrize("n,V", [(5, 3), (5, 5000), (20, 128256)])
def test_distill_a_record_without_probability(n, V):
    """Places whose p fp32 does not hold are outcomes of probability 0, whatever the student has there."""
    rng = np.random.default_rng(V)
    k, low = 2, -3.402823466e38
    z = rng.normal(0, 2, (5, V)).astype(np.float32)
    ids = np.array([[1, V], [1, V], [0, 1], [1, -1], [1, 0]], np.int32)
    values = np.array([[-INF, 5], [-200, 5], [-88, -300], [-200, -INF], [-200, -120]], np.float32)
    for r in range(5):
        z[r, [v for v in ids[r] if 0 <= v < V]] = -INF if r < 4 else low
    lse = np.zeros(5, np.float32)
    at = np.arange(n) % 5
    for T in (1.0, 0.5):
        loss, grad = run_distill(Rows(z[at], psd.F32), n, V, values[at], ids[at], lse[at], k, T, psd.DIV_KL, None, psd.F32)
        # 1 ln(1 / q_rest) with q_rest = 1: a logarithm of at most ln V in fp32 (off by 2 u of itself) less the same in 64 bits; the complete record has nothing
        assert (np.abs(loss) <= 4 * U * (1 + np.log(V))).all(), loss
        assert (np.abs(grad) <= 2 * U / T).all()
        loss, grad = run_distill(Rows(z[at], psd.F32), n, V, values[at], ids[at], lse[at], k, T, psd.DIV_JSD, None, psd.F32)
        assert (np.abs(loss - np.where(at == 3, np.log(2) / 2, 0)) <= 8 * U).all() and (np.abs(grad) <= 8 * U / T).all()


@pytest.mark.parametrize("n,V", [(3, 5000), (20, 128256)])
@pytest.mark.parametrize("div", [psd.DIV_KL, psd.DIV_JSD])
def test_distill_a_whole_record_without_an_entry_is_no_distribution(n, V, div):
    rng = np.random.default_rng(V)
    z = rng.normal(0, 2, (n, V)).astype(np.float32)
    values = np.tile(np.array([-INF, -INF, -INF], np.float32), (n, 1))
    ids = np.tile(np.array([4, 9, 7], np.int32), (n, 1))
    values[1, 1] = 0.5                              # one entry is a distribution
    ids[2] = -1                                     # no place at all is padding
    loss, grad = run_distill(Rows(z, psd.F32), n, V, values, ids, None, 3, 1.0, div, None, psd.F32)
    assert np.isnan(loss[0]) and np.isnan(grad[0]).all()
    assert loss[2] == 0 and (grad[2] == 0).all()
    check_distill(z[1:2], values[1:2], ids[1:2], None, 1.0, div, None, loss[1:2], grad[1:2], psd.F32)
    only, _ = run_distill(Rows(z, psd.F32), n, V, values, ids, None, 3, 1.0, div, None, psd.F32, want_grad=False)
    assert only.tobytes() == loss.tobytes()


@pytest.mark.parametrize("div", [psd.DIV_KL, psd.DIV_JSD])
def test_distill_student_logits_far_below_the_rest(div):
    """A student's logit whose probability fp32 does not hold has a finite logarithm, and so a finite divergence."""
    rng = np.random.default_rng(12)
    V = 3000
    z = rng.normal(0, 1, (4, V)).astype(np.float32)
    values, ids = np.tile(np.array([2.0, 1.0, 0.5], np.float32), (4, 1)), np.tile(np.array([5, 9, 2999], np.int32), (4, 1))
    lse = np.full(4, 3.0, np.float32)
    z[0, 5] = -1000.0                               # one of them
    z[1, [5, 9, 2999]] = -1000.0                    # all of them
    z[2] = -1000.0                                  # all but them
    z[2, [5, 9, 2999]] = 1.0
    z[3, 9] = -3.402823466e38                       # the difference, scaled, is no float
    loss, grad = run_distill(Rows(z, psd.F32), 4, V, values, ids, lse, 3, 1.0, div, None, psd.F32)
    for r in range(3):
        want, wg, tol, gtol = distill_bounds(z[r], values[r], ids[r], lse[r], 1.0, div, 1.0)
        # sum p ln q, where ln q is 1000 and its argument three roundings (sum p |ln p| is below 5)
        tol += 3 * U * (abs(want) + 5)
        assert abs(loss[r] - want) <= tol, (r, loss[r], want, tol)
        assert (np.abs(grad[r] - wg) <= gtol + 1e-38).all()
    assert np.isposinf(loss[3]) if div == psd.DIV_KL else 0 < loss[3] < np.log(2)
    assert np.isfinite(grad).all()


def test_distill_gradient_is_that_of_differences_of_its_own_loss():
    rng = np.random.default_rng(8)
    V, k, T = 300, 9, 1.0
    t, z = pair(rng, 1, V, psd.F32, 2.0)
    z = (np.round(z * 64) / 64).astype(np.float32)
    values, ids, lse = records(t, k, T)
    h = 2.0 ** -4
    for div in (psd.DIV_KL, psd.DIV_JSD):
        _, grad = run_distill(Rows(z, psd.F32), 1, V, values, ids, lse, k, T, div, None, psd.F32)
        steps = np.concatenate([z + h * np.eye(V, dtype=np.float32), z - h * np.eye(V, dtype=np.float32)])
        loss, _ = run_distill(Rows(steps, psd.F32), 2 * V, V, np.tile(values, (2 * V, 1)), np.tile(ids, (2 * V, 1)), np.tile(lse, 2 * V), k, T, div, None, psd.F32, want_grad=False)
        fd = (loss[:V].astype(np.float64) - loss[V:]) / (2 * h)
        # h^2 / 6 times a third derivative below 1 (the variable enters through probabilities only) + the losses' own error over 2 h
        tol = h * h / 6 + 2 * distill_bounds(z[0], values[0], ids[0], lse[0], T, div, 1.0)[2] / (2 * h)
        off = float(np.abs(fd - grad[0]).max())
        assert off <= tol and off < 0.1 * float(np.abs(grad[0]).max()), (off, tol)


# ---- together, on streams, in graphs -----------------------------------------------------------------------

def test_decoding_step_and_distillation_on_the_models_rows(tiny_stack):
    """As they are used: a verify pass's rows of target and draft are adjusted alike and judged, the target's are recorded, and the draft's
    are measured against the record."""
    cfg, d, q, t, prompt = tiny_stack
    shapes = (cfg.draft, cfg.qualifier, cfg.target)
    descs = [psd.ModelDesc(s.n_layers, s.d_model, s.n_heads, s.n_kv_heads, s.d_ffn, s.vocab, cfg.rope_theta, cfg.dtype, b) for s, b in zip(shapes, (d, q, t))]
    ctx = psd.Context(*descs, 0.3, 0.2, 4, 8, len(prompt) + 40)
    k, V = 6, cfg.target.vocab
    rng = np.random.default_rng(0)
    props = rng.integers(0, V, k).astype(np.int32)
    props[3] = props[1]
    ctx.forward(2, prompt[:-1], 0, want_logits=False)
    ctx.forward(0, prompt[:-1], 0, want_logits=False)
    seq = np.concatenate((prompt[-1:], props))
    zt, zd = 40 * ctx.forward(2, seq, len(prompt) - 1), 40 * ctx.forward(0, seq[:-1], len(prompt) - 1)   # scaled: the stack's rows are flat
    ctx.close()
    masks = np.full((2, V // 32), 0xffffffff, np.uint32)
    masks[1, ::2] = 0x0f0f0f0f
    index = np.array([-1, 0, 1, 0, 1, -1, 0], np.int32)
    edit = dict(history=dev(np.asarray(prompt, np.int32)), history_offsets=dev(np.array([0, len(prompt)], np.int64)), n_history=len(prompt),
                penalties=dev(np.array([[1.2, 0.5, 0.25]], np.float32)), masks=dev(masks), n_masks=2)
    bt, bd = Rows(zt, psd.F32), Rows(zd, psd.F32)
    window = dev(props)
    psd.adjust_logits(bt, bt, 1, k + 1, V, psd.Adjust(window=window, window_stride=k, mask_index=dev(index), **edit))
    psd.adjust_logits(bd, bd, 1, k, V, psd.Adjust(window=window, window_stride=k, mask_index=dev(index[:k].copy()), **edit))
    nacc, ntok, div = dev(np.full(1, -7, np.int32)), dev(np.full(1, -7, np.int32)), dev(np.full(k, -7, np.float32))
    wsb = psd.accept_workspace_bytes(1, k, V)
    ws = psd.DeviceBuffer(wsb)
    psd.accept_batch(bt, bd, window, 1, k, V, 0.1, 1.0, 5, 50, 2, True, nacc, ntok, div, ws, wsb)
    psd.dev_sync()
    at, ad = bt.get(), bd.get()
    for j in range(k + 1):
        m = None if index[j] < 0 else masks[index[j]]
        for z, a in ((zt, at), (zd, ad))[:2 if j < k else 1]:
            want = oracle.adjust_row(z[j], prompt, 0, props[:j], (1.2, 0.5, 0.25), mask=m)
            assert np.array_equal(np.isneginf(a[j]), np.isneginf(want))
            ok = np.isfinite(want)
            assert (np.abs(a[j][ok] - want[ok]) <= 4 * U * (1.3 * np.abs(z[j][ok]) + 0.5 + 0.25 * 30)).all()
    res, odiv = oracle.accept(at, ad, props, 0.1, 1.0, 5, 50, 2, True)
    assert np.abs(div.to_numpy(np.float32, k) - odiv).max() <= 1e-5
    if min(res.margin_div, res.margin_coin) > 1e-6 and res.margin_race > 1e-5:
        assert nacc.to_numpy(np.int32, 1)[0] == res.n_accepted and ntok.to_numpy(np.int32, 1)[0] == res.next_token
    # the target's first k rows are the teacher of the draft's
    K = 40
    rec = run_top(bt, k, V, K, 1.0, psd.F32)
    check_top(at[:k], K, 1.0, rec)
    for div_kind in (psd.DIV_KL, psd.DIV_JSD):
        loss, grad = run_distill(bd, k, V, *rec, K, 1.0, div_kind, None, psd.F32)
        check_distill(ad, *rec, 1.0, div_kind, None, loss, grad, psd.F32)
        if div_kind == psd.DIV_JSD:      # K + 1 outcomes never see more than the whole rows
            assert (loss <= odiv + 1e-5).all() and (loss > 0).all()


class Hip:
    """The few runtime calls a capturing program makes, on the runtime that the library has loaded."""

    def __init__(self):
        name = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
        self.L = ctypes.CDLL(name)

    def __call__(self, fn, *args):
        rc = getattr(self.L, fn)(*args)
        assert rc == 0, (fn, rc)

    def stream(self):
        s = ctypes.c_void_p()
        self("hipStreamCreateWithFlags", ctypes.byref(s), ctypes.c_uint(1))
        return s


def test_on_streams_and_in_replayed_graphs():
    psd.lib()
    hip = Hip()
    rng = np.random.default_rng(6)
    n, V, k = 5, 20001, 33
    t, z = pair(rng, n, V, psd.F32)
    b = Batch(rng, n, 1, V, [50] * n, 4, 2, wild=False)
    want = []
    sides = []              # (rows under the mask that allows nothing have loss NaN: the comparison is by bits)
    for i in range(2):      # two captured chains on two streams, each with buffers of its own
        zi = np.roll(z, i, 1)
        src, x, y, g = Rows(zi, psd.F32), Rows(zi, psd.F32), Rows(np.roll(t, i, 1), psd.F32), Rows(zi * 0, psd.F32)
        values, ids, lse, loss = dev(np.zeros((n, k), np.float32)), dev(np.zeros((n, k), np.int32)), dev(np.zeros(n, np.float32)), dev(np.zeros(n, np.float32))
        wt, wd = psd.top_logits_workspace_bytes(n, V, k), psd.distill_workspace_bytes(n, V, k)
        sides.append(dict(src=src, x=x, y=y, g=g, values=values, ids=ids, lse=lse, loss=loss, ws=psd.DeviceBuffer(wt), wd=psd.DeviceBuffer(wd), wt=wt, wdb=wd,
                          adjust=b.device(), stream=hip.stream()))

    def chain(s):
        st = s["stream"]
        psd.adjust_logits(s["src"], s["x"], n, 1, V, s["adjust"], stream=st)
        psd.top_logits(s["y"], n, V, k, 1.0, s["values"], s["ids"], s["lse"], s["ws"], s["wt"], stream=st)
        psd.distill(s["x"], n, V, s["values"], s["ids"], s["lse"], k, 1.0, psd.DIV_JSD, None, s["loss"], s["g"], s["wd"], s["wdb"], stream=st)

    def results(s):
        return [s["x"].get(), s["values"].to_numpy(np.float32, (n, k)), s["ids"].to_numpy(np.int32, (n, k)), s["lse"].to_numpy(np.float32, n),
                s["loss"].to_numpy(np.float32, n), s["g"].get()]

    for s in sides:
        chain(s)
        psd.dev_sync()
        want.append(results(s))
    graphs = []
    for s in sides:
        g, e = ctypes.c_void_p(), ctypes.c_void_p()
        hip("hipStreamBeginCapture", s["stream"], ctypes.c_int(2))      # relaxed: other threads' calls are none of its business
        chain(s)
        hip("hipStreamEndCapture", s["stream"], ctypes.byref(g))
        hip("hipGraphInstantiate", ctypes.byref(e), g, None, None, ctypes.c_size_t(0))
        graphs.append((g, e))
    for turn in range(4):      # both at once, again and again, with eager work between
        for s, (g, e) in zip(sides, graphs):
            hip("hipGraphLaunch", e, s["stream"])
        for s in sides:
            hip("hipStreamSynchronize", s["stream"])
        for s, w in zip(sides, want):
            same = {name: a.tobytes() == c.tobytes() for name, a, c in zip(("x", "values", "ids", "lse", "loss", "g"), results(s), w)}
            assert all(same.values()), (turn, sides.index(s), same)
        psd.row_stats(t)
        for s in sides:     # spoil what the next replay has to write
            zero = np.zeros((n, V), np.float32)
            for name in ("x", "g"):
                psd.binding._check(psd.lib().psd_dev_copy(s[name].data_ptr(), zero.ctypes.data, zero.nbytes, 0))
    for g, e in graphs:
        hip("hipGraphExecDestroy", e)
        hip("hipGraphDestroy", g)
    for s in sides:
        hip("hipStreamDestroy", s["stream"])
