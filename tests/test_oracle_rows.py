"""Pins of the oracle's operators on rows of logits (adjusting, recording, distilling) and, without a GPU, their refusals."""
import numpy as np
import pytest
import scipy.spatial.distance
import scipy.special

import oracle
import paper_2510_12966_amd as psd

INF = np.inf


# ---- adjusting -----------------------------------------------------------------------------------------

def test_adjust_row_worked_by_hand():
    z = [2.0, -2.0, 1.0, 0.0, 4.0, 3.0, 0.5]
    #     token 0: twice counted, 1: once in the prompt only, 2: in the window, 3: never, 4: prompt and counted, 5: biased twice, 6: masked
    out = oracle.adjust_row(z, history=[1, 4, 0, 0, 4, -1, 7], n_prompt=2, window=[2], penalties=(2.0, 0.5, 0.25), bias_tokens=[5, 5, 9],
                            bias=[7.0, -1.0, 3.0], mask=[0b0111111])
    assert out.tolist() == [2.0 / 2 - (0.5 + 2 * 0.25), -4.0, 0.5 - 0.75, 0.0, 4.0 / 2 - 0.75, 2.0, -INF]


def test_adjust_row_edges():
    z = np.array([1.0, -1.0, -INF, np.nan], np.float32)
    assert np.array_equal(oracle.adjust_row(z), z.astype(np.float64), equal_nan=True)
    assert np.array_equal(oracle.adjust_row(z, mask=[0b0111]), [1.0, -1.0, -INF, -INF])       # a masked NaN is closed like any other
    assert (oracle.adjust_row(z, closed=True) == -INF).all() and (oracle.adjust_row(z, mask=[0]) == -INF).all()
    assert np.array_equal(oracle.adjust_row(z[:3], history=[0, 1, 2], penalties=(0.0, 0.0, 0.0)), z[:3])   # a repetition of 0 counts as 1
    assert oracle.adjust_row([0.0], bias_tokens=[0], bias=[-INF])[0] == -INF


# ---- recording -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("V,k,T", [(1, 1, 1.0), (5, 5, 0.7), (97, 10, 1.0), (1000, 256, 2.0)])
def test_top_row_against_a_stable_sort_and_logsumexp(V, k, T):
    rng = np.random.default_rng(V)
    z = (np.round(rng.normal(0, 3, V) * 4) / 4).astype(np.float32)     # many equal entries
    values, ids, lse = oracle.top_row(z, k, T)
    order = np.argsort(-z, kind="stable")[:k]
    assert np.array_equal(ids, order) and np.array_equal(values, z[order].astype(np.float64))
    assert abs(lse - scipy.special.logsumexp(z.astype(np.float64) / T)) < 1e-12


def test_top_row_short_and_empty_rows():
    values, ids, lse = oracle.top_row([-INF, 2.0, -INF, 3.0], 3)
    assert ids.tolist() == [3, 1, -1] and values.tolist() == [3.0, 2.0, -INF] and abs(lse - np.logaddexp(2.0, 3.0)) < 1e-14
    values, ids, lse = oracle.top_row([-INF] * 3, 2)
    assert ids.tolist() == [-1, -1] and (values == -INF).all() and lse == -INF


# ---- distilling ----------------------------------------------------------------------------------------

def _pair(rng, V, k, T):
    t = rng.normal(0, 2, V).astype(np.float32)
    z = (0.7 * t + rng.normal(0, 1, V)).astype(np.float32)
    return t, z, oracle.top_row(t, k, T)


@pytest.mark.parametrize("T", [1.0, 2.0])
def test_a_record_of_the_whole_row_gives_the_divergence_of_the_rows(T):
    rng = np.random.default_rng(3)
    t, z, (values, ids, lse) = _pair(rng, 60, 60, T)
    p, q = scipy.special.softmax(t.astype(np.float64) / T), scipy.special.softmax(z.astype(np.float64) / T)
    for rec in (np.float32(lse), None):
        assert abs(oracle.distill_row(z, values, ids, rec, T, 0)[0] - scipy.special.rel_entr(p, q).sum()) < 1e-6
        assert abs(oracle.distill_row(z, values, ids, rec, T, 1)[0] - scipy.spatial.distance.jensenshannon(p, q) ** 2) < 1e-6


@pytest.mark.parametrize("div", [0, 1])
def test_a_coarser_record_never_sees_more(div):
    # joining outcomes cannot raise a divergence (data processing); k = V is the divergence of the rows
    rng = np.random.default_rng(5)
    t, z, _ = _pair(rng, 80, 80, 1.0)
    losses = [oracle.distill_row(z, *oracle.top_row(t, k), 1.0, div)[0] for k in (1, 2, 5, 20, 60, 80)]
    assert all(a <= b + 1e-6 for a, b in zip(losses, losses[1:])) and losses[0] >= -1e-9
    if div == 1:
        p, q = (scipy.special.softmax(x.astype(np.float64)) for x in (t, z))
        assert losses[-1] <= oracle.jsd(p, q) + 1e-6


@pytest.mark.parametrize("div", [0, 1])
@pytest.mark.parametrize("T", [1.0, 0.5])
@pytest.mark.parametrize("k,whole", [(1, False), (7, False), (7, True), (30, False)])
def test_the_gradient_is_that_of_central_differences(div, T, k, whole):
    rng = np.random.default_rng(k)
    V, w = 30, 1.7
    t, z, (values, ids, lse) = _pair(rng, V, k, T)
    rec = None if whole else lse
    loss, grad = oracle.distill_row(z, values, ids, rec, T, div, w)
    # steps of a power of two are exact in fp32; z is made of multiples of 2^-8 so that z +- h is exact as well
    z = (np.round(z * 256) / 256).astype(np.float32)
    loss, grad = oracle.distill_row(z, values, ids, rec, T, div, w)
    h = 2.0 ** -9
    for v in range(V):
        up, down = z.copy(), z.copy()
        up[v] += h
        down[v] -= h
        fd = (oracle.distill_row(up, values, ids, rec, T, div, w, False)[0] - oracle.distill_row(down, values, ids, rec, T, div, w, False)[0]) / (2 * h)
        # the error of a central difference is h^2 / 6 times the third derivative, which is below 8 w / T^3 here
        assert abs(fd - grad[v]) < h * h / 6 * 8 * w / T ** 3 + 1e-10, (v, fd, grad[v])
    assert abs(grad.sum()) < 1e-5 * w / T      # softmax does not change when all logits move together (mass of the record: fp32 lse)


def test_distill_row_edges():
    z = np.array([1.0, 0.0, -1.0, 0.5], np.float32)
    # duplicates, tokens outside the vocabulary and empty places are passed over
    a = oracle.distill_row(z, [2.0, 1.0], [0, 3], 3.0)
    b = oracle.distill_row(z, [2.0, 9.0, 1.0, 9.0], [0, 0, 3, 4], 3.0)
    assert a[0] == b[0] and np.array_equal(a[1], b[1])
    # a negative token: the record is complete, nothing is left for the others
    c = oracle.distill_row(z, [2.0, 1.0, -INF], [0, 3, -1], np.logaddexp(2.0, 1.0))
    d = oracle.distill_row(z, [2.0, 1.0], [0, 3], None)
    assert abs(c[0] - d[0]) < 1e-6 and np.abs(c[1] - d[1]).max() < 1e-6 and c[0] != a[0]
    # nothing valid, weight 0
    for args in (dict(ids=[-1, 7]), dict(ids=[0, 3], weight=0.0)):
        loss, grad = oracle.distill_row(z, [2.0, 1.0], args["ids"], 3.0, weight=args.get("weight", 1.0))
        assert loss == 0.0 and (grad == 0).all()
    # no student mass for an outcome of the teacher: KL infinite with a finite gradient, JSD finite
    gone = np.array([1.0, 0.0, -INF, 0.5], np.float32)
    loss, grad = oracle.distill_row(gone, [2.0, 2.0], [0, 2], None)
    assert loss == INF and np.isfinite(grad).all() and abs(grad[2] + 0.5) < 1e-12
    loss, grad = oracle.distill_row(gone, [2.0, 2.0], [0, 2], None, divergence=1)
    assert 0 < loss < np.log(2) and grad[2] == 0.0
    assert np.isnan(oracle.distill_row(np.full(4, -INF, np.float32), [2.0], [0], 3.0)[0])
    # identical rows: no divergence, no gradient
    loss, grad = oracle.distill_row(z, *oracle.top_row(z, 2), divergence=1)
    assert abs(loss) < 1e-12 and np.abs(grad).max() < 1e-7


@pytest.mark.parametrize("closed", [-INF, -1e9, -3.402823466e38])
def test_a_record_that_just_holds_a_grammars_tokens(closed):
    """Its fp32 lse leaves a remainder of up to some 2^-24: the student, closed in the same places, is not held to it."""
    rng = np.random.default_rng(7)
    left = 0
    for _ in range(100):
        V, k = 200, 8
        allowed = rng.choice(V, k, replace=False)
        t, z = np.full((2, V), closed, np.float32)
        t[allowed], z[allowed] = rng.normal(0, 4, (2, k))
        values, ids, lse = oracle.top_row(t, k)
        p, q = scipy.special.softmax(t[allowed].astype(np.float64)), scipy.special.softmax(z[allowed].astype(np.float64))
        left += np.exp(values - float(np.float32(lse))).sum() < 1
        # every ln p is off by 2^-24 |lse|, and that much of the mass is left out
        tol = 2.0 ** -23 * (1 + abs(lse)) * (1 + np.abs(np.log(p / q)).max())
        loss, grad = oracle.distill_row(z, values, ids, lse)
        assert abs(loss - scipy.special.rel_entr(p, q).sum()) <= tol and np.abs(grad[allowed] - (q - p)).max() <= tol
        assert (np.delete(grad, allowed) == 0).all()
        assert abs(oracle.distill_row(z, values, ids, lse, divergence=1)[0] - scipy.spatial.distance.jensenshannon(p, q) ** 2) <= tol
    assert 20 < left < 80
    # a true remainder counts: the student has e^closed for it
    loss, _ = oracle.distill_row(z, values, ids, lse + 0.01)
    assert loss > 1e6 if np.isfinite(closed) else loss == INF


@pytest.mark.parametrize("low", [-INF, -1e9, -3.402823466e38])
def test_outcomes_of_no_probability_cost_nothing(low):
    """A teacher's place whose exponential fp32 does not hold, at a token that the student has closed."""
    z = np.array([1.0, low, 0.5, low], np.float32)
    lq = np.log(np.exp([1.0, 0.5]).sum())
    for v in (-INF, -200.0, -88.0):
        loss, grad = oracle.distill_row(z, [v, v], [1, 3], 0.0)              # all of the teacher lies beside its record
        assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
        loss, grad = oracle.distill_row(z, [1.0, v], [0, 1], np.float32(1.0))   # one sure token: p = 1
        assert abs(loss - (lq - 1.0)) < 1e-12 and grad[1] == 0
        loss, grad = oracle.distill_row(z, [2.0, v], [0, 1], None)
        assert abs(loss - (lq - 1.0)) < 1e-12 and grad[1] == 0
    if low == -INF:
        assert oracle.distill_row(z, [1.0, -80.0], [0, 1], np.float32(1.0))[0] == INF      # e^-81 is held


@pytest.mark.parametrize("div", [0, 1])
def test_a_side_without_an_entry_is_no_distribution(div):
    z = np.array([1.0, 0.0, -1.0, 0.5], np.float32)
    for args in ((z, [-INF, -INF], [0, 3], None), (np.full(4, -INF, np.float32), [2.0, 1.0], [0, 3], 3.0)):
        loss, grad = oracle.distill_row(*args, divergence=div)
        assert np.isnan(loss) and np.isnan(grad).all()
    loss, grad = oracle.distill_row(z, [-INF, -3.402823466e38], [0, 3], None, divergence=div)     # the lowest value is an entry
    assert np.isfinite(loss) and abs(grad.sum()) < 1e-12
    loss, grad = oracle.distill_row(z, [-INF, -INF], [0, 3], 3.0, divergence=div)                 # with the row's lse all of it lies outside
    assert np.isfinite(loss) and abs(grad.sum()) < 1e-12


# ---- refusals (argument checks come before anything touches a GPU) ----------------------------------------

class _At:
    """Stands in for a device buffer at an address; nothing looks at what is there."""

    def __init__(self, at=0x10000):
        self.at = at

    def data_ptr(self):
        return self.at


A, B = _At(), _At(0x40000000)


def _refused(code, fn, *args, **kw):
    with pytest.raises(psd.PsdError) as e:
        fn(*args, **kw)
    assert e.value.code == code, str(e.value)
    return str(e.value)


def test_adjust_refusals():
    none = psd.Adjust()
    ok = dict(logits=A, out=B, n_seqs=2, rows=3, vocab=100, adjust=none)

    def bad(**kw):
        return _refused(-1, psd.adjust_logits, **{**ok, **kw})

    bad(logits=None), bad(out=None), bad(n_seqs=0), bad(rows=0), bad(vocab=0), bad(n_seqs=256, rows=256), bad(dtype=2)
    bad(logits_stride=99), bad(out_stride=99), bad(logits=_At(0x10002)), bad(out=_At(0x40000001), dtype=psd.BF16)
    assert "overlap" in bad(out=_At(0x10000 + 4)) and "overlap" in bad(out=A, out_stride=128)
    assert "overlap" in bad(out=_At(0x10000 + 4 * 599))
    bad(adjust=psd.Adjust(history=A, n_history=5)), bad(adjust=psd.Adjust(history_offsets=A, n_history=5)), bad(adjust=psd.Adjust(n_history=-1))
    bad(adjust=psd.Adjust(bias=A, bias_tokens=A, n_bias=5)), bad(adjust=psd.Adjust(bias=A, bias_offsets=A, n_bias=5)), bad(adjust=psd.Adjust(n_bias=-2))
    bad(adjust=psd.Adjust(bias=A, bias_tokens=A, bias_offsets=A, n_bias=2 ** 30 + 1)), bad(adjust=psd.Adjust(masks=A, mask_index=A, n_masks=2 ** 31))
    bad(adjust=psd.Adjust(masks=A, n_masks=2)), bad(adjust=psd.Adjust(mask_index=A)), bad(adjust=psd.Adjust(n_masks=1, mask_index=A))
    bad(adjust=psd.Adjust(window=A, window_stride=1)), bad(adjust=psd.Adjust(penalties=_At(0x10002)))
    bad(adjust=psd.Adjust(history=A, history_offsets=_At(0x10004), n_history=5))


def test_top_refusals():
    n, V, k = 4, 1000, 8
    ws = psd.top_logits_workspace_bytes(n, V, k)
    ok = dict(logits=A, n_rows=n, vocab=V, k=k, temperature=1.0, values=B, ids=B, lse=None, workspace=B, workspace_bytes=ws)

    def bad(code=-1, **kw):
        return _refused(code, psd.top_logits, **{**ok, **kw})

    bad(logits=None), bad(values=None), bad(ids=None), bad(workspace=None), bad(n_rows=0), bad(n_rows=65536), bad(k=0), bad(k=257), bad(dtype=-1)
    bad(vocab=7, stride=1000), bad(temperature=0.0), bad(temperature=float("nan")), bad(stride=999), bad(workspace=_At(0x40000008)), bad(values=_At(0x40000002))
    if ws > 16:
        bad(-3, workspace_bytes=ws - 1)
    assert bad(-3, workspace_bytes=0)
    for args in ((0, V, k), (n, 0, k), (n, V, 0), (n, V, 257), (n, 7, 8), (65536, V, k)):
        assert psd.top_logits_workspace_bytes(*args) == 0


def test_distill_refusals():
    n, V, k = 4, 1000, 8
    ws = psd.distill_workspace_bytes(n, V, k)
    ok = dict(logits=A, n_rows=n, vocab=V, top_values=B, top_ids=B, top_lse=None, k=k, temperature=1.0, divergence=psd.DIV_KL, row_weights=None,
              loss=B, grad=None, workspace=B, workspace_bytes=ws)

    def bad(code=-1, **kw):
        return _refused(code, psd.distill, **{**ok, **kw})

    bad(logits=None), bad(top_values=None), bad(top_ids=None), bad(loss=None), bad(workspace=None), bad(n_rows=0), bad(n_rows=65536), bad(k=0), bad(k=257)
    bad(temperature=-1.0), bad(divergence=2), bad(stride=999), bad(grad=B, grad_stride=999), bad(dtype=3), bad(row_weights=_At(0x10001))
    assert "overlap" in bad(grad=_At(0x10000 + 4)) and "overlap" in bad(grad=A, grad_stride=1024)
    assert bad(-3, workspace_bytes=ws - 1)
    for args in ((0, V, k), (n, 0, k), (n, V, 0), (n, V, 257), (65536, V, k)):
        assert psd.distill_workspace_bytes(*args) == 0


def test_temperatures_without_a_finite_scale_are_refused():
    """0 * inf would be the exponent of a row's largest entry, or of an entry of -inf."""
    n, V, k = 4, 1000, 8
    for T in (float("inf"), 1e-39, -0.0, -float("inf")):
        _refused(-1, psd.top_logits, A, n, V, k, T, B, B, None, B, 1 << 20)
        _refused(-1, psd.distill, A, n, V, B, B, None, k, T, psd.DIV_JSD, None, B, None, B, 1 << 20)


def test_host_arrays_are_refused():
    host = np.zeros(100, np.float32)
    with pytest.raises(TypeError):
        psd.adjust_logits(host, A, 1, 1, 100, psd.Adjust())
    with pytest.raises(TypeError):
        psd.Adjust(penalties=host)
    with pytest.raises(TypeError):
        psd.top_logits(host, 1, 100, 4, 1.0, A, A, A, A, 1 << 20)
    with pytest.raises(TypeError):
        psd.distill(A, 1, 100, A, A, A, 4, 1.0, psd.DIV_KL, None, A, host, A, 1 << 20)


class _OnHost(_At):
    """What a tensor in host memory looks like: it has an address, but not one for a kernel."""
    is_cuda = False


def test_tensors_in_host_memory_are_refused():
    torch = pytest.importorskip("torch")
    ws = 1 << 20
    for host in (_OnHost(), torch.zeros(100), torch.zeros(100, device="meta")):
        for name in ("history", "history_offsets", "n_prompt", "window", "penalties", "bias_tokens", "bias", "bias_offsets", "masks", "mask_index"):
            with pytest.raises(TypeError):
                psd.Adjust(**{name: host})
        calls = [(psd.adjust_logits, dict(logits=A, out=B, n_seqs=1, rows=1, vocab=100, adjust=psd.Adjust()), ("logits", "out")),
                 (psd.top_logits, dict(logits=A, n_rows=1, vocab=100, k=4, temperature=1.0, values=B, ids=B, lse=B, workspace=B, workspace_bytes=ws),
                  ("logits", "values", "ids", "lse", "workspace")),
                 (psd.distill, dict(logits=A, n_rows=1, vocab=100, top_values=B, top_ids=B, top_lse=B, k=4, temperature=1.0, divergence=psd.DIV_KL, row_weights=B,
                                    loss=B, grad=None, workspace=B, workspace_bytes=ws),
                  ("logits", "top_values", "top_ids", "top_lse", "row_weights", "loss", "grad", "workspace"))]
        for fn, ok, names in calls:
            for name in names:
                # (a dtype that does not exist: were the buffer taken, the call would still be refused, by another error)
                with pytest.raises(TypeError):
                    fn(**{**ok, name: host, "dtype": 9})


def test_adjust_struct_has_the_layout_of_the_header():
    import ctypes
    A = psd.Adjust
    assert ctypes.sizeof(A) == 14 * 8 and [getattr(A, n).offset for n, _ in A._fields_] == list(range(0, 112, 8))
    assert [n for n, _ in A._fields_] == ["history", "history_offsets", "n_history", "n_prompt", "window", "window_stride", "penalties", "bias_tokens", "bias",
                                          "bias_offsets", "n_bias", "masks", "mask_index", "n_masks"]
