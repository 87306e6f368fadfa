"""The operators on rows of logits around the acceptance stage, as cases that can be timed and compared.

  adjust   penalties for repeated tokens, biases and grammar masks on the rows of a pass, before they are judged or sampled
  top      the k largest entries of every row with the row's log-sum-exp: top log-probabilities, and the record that distillation reads
  distill  divergence between such a record of a teacher (the verifier) and a student's (the proposer's) rows, and its gradient

A case is a dict of plain values.  Vocabularies are those of the package's stack configurations (512, 32000, 128256), of the other measured
cases (32003, 50257, 128255) and the generic 65536; windows, prompt lengths and numbers of trials are theirs too; rows of a
training batch are generic.  Logits are normal with a few outstanding entries per row, as a model's are; a bf16 row has many equal ones.
"""
import math

import torch

own = False

VOCABS = (32000, 32003, 50257, 65536, 128255, 128256)
KL, JSD = "kl", "jsd"


def listed():
    return [
        # a verify pass of the tiny stack (k2 = 8): the smallest call, latency is everything
        dict(name="adjust_tiny", kind="adjust", seqs=1, rows=9, vocab=512, dtype="f32", history=40, bias=0, masks=0, pad=0),
        # one token of plain sampling at the headline vocabulary, a prompt of 512 behind it: penalties alone
        dict(name="adjust_token", kind="adjust", seqs=1, rows=1, vocab=128256, dtype="f32", history=513, bias=0, masks=0, pad=0),
        # the target's rows of a verify pass (k2 = 10) on a long prompt, with biases and a grammar state for every row
        dict(name="adjust_window", kind="adjust", seqs=1, rows=11, vocab=128256, dtype="f32", history=4101, bias=300, masks=11, pad=0),
        # windows of many requests at once, ragged histories, rows padded to a wider stride
        dict(name="adjust_many", kind="adjust", seqs=48, rows=9, vocab=128255, dtype="f32", history=2000, bias=64, masks=96, pad=1),
        # one token of many requests with long histories, bf16 rows
        dict(name="adjust_long", kind="adjust", seqs=64, rows=1, vocab=128256, dtype="bf16", history=30000, bias=16, masks=8, pad=0),
        # the top log-probabilities of one served token
        dict(name="top_token", kind="top", n=1, vocab=128256, dtype="f32", k=20, T=1.0, masked=0.0),
        # those of a verify pass's rows, most of them closed by a mask, bf16
        dict(name="top_window", kind="top", n=17, vocab=32003, dtype="bf16", k=8, T=0.7, masked=0.97),
        # the teacher's record of a prompt: what a distillation run keeps of the target's rows
        dict(name="top_record", kind="top", n=2048, vocab=128256, dtype="f32", k=64, T=1.0, masked=0.0),
        # a small step on the small stack's vocabulary
        dict(name="distill_small", kind="distill", n=48, vocab=32000, dtype="f32", k=32, T=1.0, div=KL, tail=True, grad=True, pad=0.0, skip=0.0),
        # a training step of the draft on a batch of one prompt of 1024 tokens, fp32 rows
        dict(name="distill_step", kind="distill", n=1024, vocab=128256, dtype="f32", k=64, T=1.0, div=KL, tail=True, grad=True, pad=0.0, skip=0.0),
        # a larger step, by the divergence that acceptance goes by, bf16 rows, a quarter of them padding
        dict(name="distill_jsd", kind="distill", n=4096, vocab=128256, dtype="bf16", k=128, T=1.0, div=JSD, tail=True, grad=True, pad=0.25, skip=0.0),
        # evaluation: the loss alone, an odd vocabulary, records cut to their k entries and partly short, temperature 2
        dict(name="distill_eval", kind="distill", n=777, vocab=50257, dtype="bf16", k=100, T=2.0, div=KL, tail=False, grad=False, pad=0.1, skip=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("adjust", "top", "distill", "distill"))
    vocab = rng.choice(VOCABS + (512, 1001))
    dtype = rng.choice(("f32", "bf16"))
    if kind == "adjust":
        seqs, rows = _log_int(rng, 1, 64), _log_int(rng, 1, 32)
        rows = max(1, min(rows, 48 * 9 * 128256 // (seqs * vocab)))
        return dict(kind="adjust", seqs=seqs, rows=rows, vocab=vocab, dtype=dtype, history=rng.choice((0, _log_int(rng, 1, 30000), _log_int(rng, 1, 30000))),
                    bias=rng.choice((0, _log_int(rng, 1, 300))), masks=rng.choice((0, rng.randint(1, 96))), pad=rng.choice((0, 0, 1, 5)))
    if kind == "top":
        n = _log_int(rng, 1, min(4096, 2048 * 128256 // vocab))
        return dict(kind="top", n=n, vocab=vocab, dtype=dtype, k=_log_int(rng, 1, 256), T=rng.choice((1.0, 0.7, 2.0)), masked=rng.choice((0.0, 0.0, 0.97)))
    n = _log_int(rng, 1, min(4096, 2048 * 128256 // vocab))
    return dict(kind="distill", n=n, vocab=vocab, dtype=dtype, k=_log_int(rng, 1, 256), T=rng.choice((1.0, 1.0, 2.0)), div=rng.choice((KL, JSD)),
                tail=rng.choice((True, True, False)), grad=rng.choice((True, True, False)), pad=rng.choice((0.0, 0.25)), skip=rng.choice((0.0, 0.1)))


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(n, vocab, g, dtype, stride=None):
    """Rows of logits: normal, and up to 48 places of each raised by an exponential variate: some tokens stand out from the rest."""
    z = torch.empty(n, stride or vocab, device="cuda").normal_(0.0, 2.0, generator=g)
    m = min(48, vocab)
    at = torch.randint(0, vocab, (n, m), generator=g, device="cuda")
    z.scatter_reduce_(1, at, 4.0 + torch.empty(n, m, device="cuda").exponential_(0.35, generator=g), "amax")
    return z if dtype == torch.float32 else z.to(dtype)


def _offsets(n, mean, g):
    """Offsets of n ragged lists of `mean` entries on average; a single list has just as many."""
    length = torch.randint(mean // 2, mean + mean // 2 + 1, (n,), generator=g, device="cuda") if n > 1 else torch.full((1,), mean, device="cuda")
    return torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), length.cumsum(0)))


def _adjust_inputs(case, g):
    S, R, V = case["seqs"], case["rows"], case["vocab"]
    stride = V + case["pad"]
    rand = lambda hi, *shape: torch.randint(0, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    s = dict(logits=_rows(S * R, V, g, _type(case), stride), stride=stride)
    s["offsets"] = _offsets(S, case["history"], g)
    n = int(s["offsets"][-1])
    # text repeats itself: half of its tokens come from a hundredth of the vocabulary
    s["history"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, rand(max(1, V // 100), n), rand(V, n))
    s["n_prompt"] = ((s["offsets"][1:] - s["offsets"][:-1]) // 2).int()
    s["window"] = rand(V, S, max(R - 1, 1))
    u = torch.rand(S, 3, generator=g, device="cuda")
    s["penalties"] = torch.stack((1.0 + 0.3 * u[:, 0], u[:, 1], 0.5 * u[:, 2]), 1).contiguous()   # repetition, presence, frequency
    if case["bias"]:
        s["bias_offsets"] = _offsets(S, case["bias"], g)
        m = int(s["bias_offsets"][-1])
        s["bias_tokens"], s["bias"] = rand(V, m), torch.empty(m, device="cuda").normal_(0.0, 3.0, generator=g)
    if case["masks"]:
        M, words = case["masks"], (V + 31) // 32
        bits = torch.randint(-2 ** 31, 2 ** 31, (M, words), generator=g, device="cuda", dtype=torch.int64).int()
        few = bits & torch.randint(-2 ** 31, 2 ** 31, (M, words), generator=g, device="cuda", dtype=torch.int64).int()
        few &= torch.randint(-2 ** 31, 2 ** 31, (M, words), generator=g, device="cuda", dtype=torch.int64).int()
        s["masks"] = torch.where(torch.arange(M, device="cuda")[:, None] % 2 == 0, few, bits | few).contiguous()   # a state opens an eighth or half
        s["mask_index"] = (torch.randint(0, M + 1, (S * R,), generator=g, device="cuda") - 1).int()               # -1: no mask
    s["out"] = torch.empty_like(s["logits"])
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    V = case["vocab"]
    if case["kind"] == "adjust":
        return dict(case=case, **_adjust_inputs(case, g))
    n, k = case["n"], case["k"]
    if case["kind"] == "top":
        z = _rows(n, V, g, _type(case))
        if case["masked"]:
            z.masked_fill_(torch.rand(n, V, generator=g, device="cuda") < case["masked"], -math.inf)
        return dict(case=case, logits=z, values=torch.empty(n, k, device="cuda"), ids=torch.empty(n, k, dtype=torch.int32, device="cuda"), lse=torch.empty(n, device="cuda"))
    teacher = _rows(n, V, g, torch.float32)
    values, ids = teacher.topk(k, -1)
    ids = ids.int()
    if case["skip"]:   # rows whose teacher has fewer than k entries, under a mask
        short = torch.rand(n, generator=g, device="cuda") < case["skip"]
        gone = short[:, None] & (torch.arange(k, device="cuda") >= (k + 1) // 2)
        values, ids = values.masked_fill(gone, -math.inf), ids.masked_fill(gone, -1)
    lse = torch.where((ids < 0).any(-1), (values / case["T"]).logsumexp(-1), (teacher / case["T"]).logsumexp(-1))
    student = torch.empty_like(teacher).normal_(0.0, 1.2, generator=g).add_(teacher, alpha=0.8).to(_type(case))
    weights = torch.rand(n, generator=g, device="cuda") + 0.5
    weights[n - _padding(case):] = 0.0
    return dict(case=case, logits=student, values=values.contiguous(), ids=ids.contiguous(), lse=lse, weights=weights, loss=torch.empty(n, device="cuda"),
                grad=torch.empty_like(student) if case["grad"] else None)


def _padding(case):
    return int(case["n"] * case["pad"])


# ---- the framework's calls ----------------------------------------------------------------------------------------------
def _run_own(s):
    import paper_2510_12966_amd as psd
    case = s["case"]
    V, dtype = case["vocab"], psd.F32 if case["dtype"] == "f32" else psd.BF16
    stream = torch.cuda.current_stream().cuda_stream
    if case["kind"] == "adjust":
        if "adjust" not in s:   # the description of a request batch: kept while the batch lives
            s["adjust"] = psd.Adjust(history=s["history"], history_offsets=s["offsets"], n_history=s["history"].numel(), n_prompt=s["n_prompt"],
                                     window=s["window"] if case["rows"] > 1 else None, window_stride=s["window"].shape[1], penalties=s["penalties"],
                                     bias_tokens=s.get("bias_tokens"), bias=s.get("bias"), bias_offsets=s.get("bias_offsets"),
                                     n_bias=s["bias"].numel() if case["bias"] else 0, masks=s.get("masks"), mask_index=s.get("mask_index"), n_masks=case["masks"])
        psd.adjust_logits(s["logits"], s["out"], case["seqs"], case["rows"], V, s["adjust"], dtype=dtype, logits_stride=s["stride"], out_stride=s["stride"], stream=stream)
        return dict(out=s["out"][:, :V])
    n, k = case["n"], case["k"]
    if case["kind"] == "top":
        if "ws" not in s:
            s["ws"] = torch.empty(psd.top_logits_workspace_bytes(n, V, k), dtype=torch.uint8, device="cuda")
        psd.top_logits(s["logits"], n, V, k, case["T"], s["values"], s["ids"], s["lse"], s["ws"], s["ws"].numel(), dtype=dtype, stream=stream)
        return dict(values=s["values"], ids=s["ids"], lse=s["lse"])
    if "ws" not in s:
        s["ws"] = torch.empty(psd.distill_workspace_bytes(n, V, k), dtype=torch.uint8, device="cuda")
    psd.distill(s["logits"], n, V, s["values"], s["ids"], s["lse"] if case["tail"] else None, k, case["T"], psd.DIV_KL if case["div"] == KL else psd.DIV_JSD, s["weights"],
                s["loss"], s["grad"], s["ws"], s["ws"].numel(), dtype=dtype, stream=stream)
    return dict(loss=s["loss"], grad=s["grad"]) if case["grad"] else dict(loss=s["loss"])


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def _of_lists(offsets, n):
    """Which list each of n entries belongs to."""
    return torch.searchsorted(offsets[1:].contiguous(), torch.arange(n, device="cuda"), right=True)


def _plain_adjust(s):
    case = s["case"]
    S, R, V = case["seqs"], case["rows"], case["vocab"]
    z = s["logits"][:, :V].float().view(S, R, V)
    n = s["history"].numel()
    seq = _of_lists(s["offsets"], n)
    flat = seq * V + s["history"]
    seen = torch.zeros(S * V, dtype=torch.int32, device="cuda").scatter_add_(0, flat, torch.ones_like(s["history"])).view(S, 1, V)
    late = (torch.arange(n, device="cuda") >= (s["offsets"][:-1] + s["n_prompt"])[seq]).int()
    count = torch.zeros(S * V, dtype=torch.int32, device="cuda").scatter_add_(0, flat, late).view(S, 1, V)
    if R > 1:   # row j has the j proposals before it too
        w = torch.zeros(S, R, V, dtype=torch.int32, device="cuda")
        w[:, 1:].scatter_(2, s["window"].view(S, R - 1, 1).long(), 1)
        w = w.cumsum(1, dtype=torch.int32)
        seen, count = seen + w, count + w
    r, p, f = (x.view(S, 1, 1) for x in s["penalties"].unbind(1))
    z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
    z = torch.where(count > 0, z - (count * f + p), z)
    if case["bias"]:
        m = s["bias"].numel()
        at = _of_lists(s["bias_offsets"], m) * V + s["bias_tokens"]
        order = torch.arange(1, m + 1, device="cuda")
        last = torch.zeros(S * V, dtype=torch.int64, device="cuda").scatter_reduce_(0, at, order, "amax")   # the last entry of a token counts
        z = z + torch.cat((torch.zeros(1, device="cuda"), s["bias"]))[last].view(S, 1, V)
    z = z.view(S * R, V)
    if case["masks"]:
        mi = s["mask_index"].long()
        bits = (s["masks"][mi.clamp(min=0)][:, :, None] >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
        z = z.masked_fill((bits.view(S * R, -1)[:, :V] == 0) & (mi >= 0)[:, None], -math.inf)
    return dict(out=z.to(s["logits"].dtype))


def _plain_top(s):
    case = s["case"]
    z = s["logits"].float()
    values, ids = z.sort(dim=-1, descending=True, stable=True)   # stable: equal entries stay in the order of their ids
    values, ids = values[:, :case["k"]].contiguous(), ids[:, :case["k"]].int()
    a = z / case["T"]
    m = a.amax(-1, keepdim=True)
    lse = m[:, 0] + (a - m).exp().sum(-1).log()
    return dict(values=values, ids=ids.masked_fill(values == -math.inf, -1), lse=lse)


def _plain_distill(s):
    case = s["case"]
    T, w = case["T"], s["weights"]
    valid = s["ids"] >= 0
    ids = s["ids"].clamp(min=0).long()
    t = (s["values"].double() / T).masked_fill(~valid, -math.inf)
    if case["tail"]:
        lp = t - s["lse"].double()[:, None]
        lpr = (1.0 - lp.exp().sum(-1)).clamp(min=0.0).log().masked_fill(~valid.all(-1), -math.inf)   # a short record is all there is
    else:
        m = t.amax(-1, keepdim=True)
        lp = t - m - (t - m).exp().sum(-1, keepdim=True).log()
        lpr = torch.full_like(w, -math.inf, dtype=torch.float64)
    a = s["logits"].float() / T
    m = a.amax(-1, keepdim=True)
    e = (a - m).exp()
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    in_s = torch.zeros_like(a, dtype=torch.int8).scatter_add_(1, ids, valid.to(torch.int8)) > 0
    rest = e.masked_fill(in_s, 0.0).sum(-1, dtype=torch.float64)
    lq = (a - m).gather(1, ids) - total.log()     # ln q of the record's entries
    lqr = rest.log() - total[:, 0].log()          # and of all others together
    # K + 1 outcomes: the record's entries and the rest; places without an entry have p = q = 0
    lp = torch.cat((lp, lpr[:, None]), 1)
    lq = torch.cat((lq.masked_fill(~valid, -math.inf), lqr[:, None]), 1)
    p, q = lp.exp(), lq.exp()
    if case["div"] == KL:
        loss = torch.where(p > 0, p * (lp - lq), 0.0).sum(-1)
        g = q * p.sum(-1, keepdim=True) - p       # q_b (w_b - sum q w)
    else:
        d = torch.where((p > 0) | (q > 0), lq - lp, 0.0)          # in (-inf, inf]
        up = math.log(2.0) - torch.where(d > 0, d + (-d).exp().log1p(), d.exp().log1p())      # ln(2 p / (p + q))
        uq = math.log(2.0) - torch.where(d > 0, (-d).exp().log1p(), -d + d.exp().log1p())     # ln(2 q / (p + q))
        kl_p, kl_q = torch.where(p > 0, p * up, 0.0), torch.where(q > 0, q * uq, 0.0)
        loss = 0.5 * (kl_p + kl_q).sum(-1)
        g = 0.5 * (kl_q - q * kl_q.sum(-1, keepdim=True))
    loss = (loss * w).float().masked_fill(w == 0, 0.0)
    if not case["grad"]:
        return dict(loss=loss)
    scale = (w / T).double()[:, None]
    out = e * ((g[:, -1:] / rest[:, None].clamp(min=1e-300)) * scale).float()
    here = torch.where(valid, (g[:, :-1] * scale).float(), 0.0)
    out = out.masked_fill_(in_s, 0.0).scatter_add_(1, ids, here)
    return dict(loss=loss, grad=out.masked_fill_((w == 0)[:, None], 0.0).to(s["logits"].dtype))


def run(state):
    if own:
        return _run_own(state)
    return {"adjust": _plain_adjust, "top": _plain_top, "distill": _plain_distill}[state["case"]["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case):
    el, V = 4 if case["dtype"] == "f32" else 2, case["vocab"]
    if case["kind"] == "adjust":
        n, lists = case["seqs"] * case["rows"], case["seqs"] * (case["history"] * 4 + case["bias"] * 8)
        masks = min(case["masks"], n) * ((V + 31) // 32) * 4
        return {"bytes": 2.0 * n * V * el + lists + masks, "flops": 2.0 * n * V}
    n, k = case["n"], case["k"]
    if case["kind"] == "top":
        return {"bytes": float(n * V * el + n * (8 * k + 4)), "flops": 4.0 * n * V}
    live = n - _padding(case)
    return {"bytes": float(live * V * el + (n * V * el if case["grad"] else 0) + live * (8 * k + 8) + 4 * n), "flops": (8.0 if case["grad"] else 5.0) * live * V}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def _exact_adjust(case, s):
    R, V = case["rows"], case["vocab"]
    off, history, window = s["offsets"].tolist(), s["history"].long(), s["window"].long()
    out = torch.empty(case["seqs"] * R, V, dtype=torch.float64, device="cuda")
    for i in range(case["seqs"]):
        r, p, f = s["penalties"][i].double().tolist()
        mine = history[off[i]:off[i + 1]]
        counted = mine[int(s["n_prompt"][i]):]
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        if case["bias"]:
            lo, hi = s["bias_offsets"][i:i + 2].tolist()
            given = dict(zip(s["bias_tokens"][lo:hi].tolist(), s["bias"][lo:hi].tolist()))
            bias[torch.tensor(list(given), dtype=torch.int64, device="cuda")] = torch.tensor(list(given.values()), dtype=torch.float64, device="cuda")
        for j in range(R):
            z = s["logits"][i * R + j, :V].double()
            known = torch.cat((mine, window[i, :j])).unique()
            z[known] = torch.where(z[known] > 0, z[known] / r, z[known] * r)
            tok, c = torch.cat((counted, window[i, :j])).unique(return_counts=True)
            z[tok] -= p + f * c.double()
            z += bias
            m = int(s["mask_index"][i * R + j]) if case["masks"] else -1
            if m >= 0:
                v = torch.arange(V, device="cuda")
                z[(s["masks"][m][v // 32] >> (v % 32)) & 1 == 0] = -math.inf
            out[i * R + j] = z
    return dict(out=out)


def _exact_top(case, s):
    z = s["logits"].double()
    return dict(values=z.topk(case["k"], -1)[0], ids=None, lse=(z / case["T"]).logsumexp(-1))


def _exact_distill(case, s):
    """The divergence over K + 1 outcomes as it is defined, row by row group; the gradient by differentiating it."""
    n, V, T = case["n"], case["vocab"], case["T"]
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    grad = torch.zeros(n, V, dtype=torch.float64, device="cuda") if case["grad"] else None
    live = n - _padding(case)
    for lo in range(0, live, 256):
        part = slice(lo, min(lo + 256, live))
        ids, valid, w = s["ids"][part].long(), s["ids"][part] >= 0, s["weights"][part].double()
        t = s["values"][part].double() / T
        z = s["logits"][part].double().requires_grad_(case["grad"])
        logq = (z / T).log_softmax(-1)
        chosen = torch.zeros_like(z, dtype=torch.bool)
        chosen[valid.nonzero()[:, 0], ids[valid]] = True
        p = torch.zeros_like(z.detach())
        if case["tail"]:
            p[valid.nonzero()[:, 0], ids[valid]] = (t - s["lse"][part].double()[:, None]).exp()[valid]
            left = (1.0 - p.sum(-1)).clamp(min=0.0) * valid.all(-1)
        else:
            p[valid.nonzero()[:, 0], ids[valid]] = t.masked_fill(~valid, -math.inf).softmax(-1)[valid]
            left = torch.zeros_like(w)
        log_left = logq.masked_fill(chosen, -math.inf).logsumexp(-1)
        if case["div"] == KL:
            each = torch.where(chosen, torch.special.xlogy(p, p) - p * logq, 0.0).sum(-1) + torch.special.xlogy(left, left) - left * log_left
        else:
            q, q_left = logq.exp(), log_left.exp()
            mid, mid_left = (p + q) / 2, (left + q_left) / 2
            log_mid = mid.clamp(min=1e-300).log()
            kl = (torch.special.xlogy(p, p) - p * log_mid) + q * (logq - log_mid)
            each = torch.where(chosen, kl, 0.0).sum(-1) + torch.special.xlogy(left, left) - left * mid_left.log() + q_left * (log_left - mid_left.log())
            each = each / 2
        if case["grad"]:
            (each * w).sum().backward()
            grad[part] = z.grad
        loss[part] = (each * w).detach()
    return dict(loss=loss, grad=grad) if case["grad"] else dict(loss=loss)


def exact(case, seed):
    s = prepare(case, seed)
    return {"adjust": _exact_adjust, "top": _exact_top, "distill": _exact_distill}[case["kind"]](case, s)
