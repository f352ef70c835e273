"""The operators that say how probable items are under a trained model, as timed cases: predictions at the factors'
own precision with the model's offsets, the log probabilities of given items with the entropy and the best
alternatives, and their gradient.

A case is a dict; ``kind`` says which operator it is:

``predict``   out[i, j] = act(sum_k x_uk t_jk + a_u + b_j) + residual[i, j], u = users[i] or i, from factors in
              32 or 16 bits.
``log_prob``  a row of scores as a distribution over its columns, p = softmax(z / T) with some columns left out: log p
              of the given columns (one a row, the same number for all, or a CSR row of them), the entropy, and the
              `top` most probable columns with their log p, ties to the lower column.
``grad``      the gradient of sum_e g_e log p(given_e) + sum_r h_r entropy_r with respect to the scores, or its
              sums over the rows (the gradient of the items' offsets), or both.
``fit``       a step of fitting the items' offsets: predictions of a batch of users, the log probabilities of the
              items that they chose, and the gradient of their mean with respect to the offsets.

A column with -inf or NaN is left out, too.  A row without any column has log p = -inf, entropy 0 and gradient 0;
so have given columns that are left out, which then weigh nothing in the gradient.
"""
import math

import torch

own = False
DEVICE = 0

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    movie = dict(of=480_000, n=17_770, f=100)
    return [
        # one user against the movie shape's items: the smallest call
        dict(movie, name="predict_one_movie_f100", kind="predict", m=1, dtype="f32", out="f32", offsets=True,
             activation="none", residual=False),
        # a batch of users, ratings clipped to their scale
        dict(movie, name="predict_batch_movie_f100", kind="predict", m=1_024, dtype="f32", out="f32", offsets=True,
             activation="clip", residual=False),
        # a large batch at the largest rank against the wiki shape's columns, in bf16 throughout
        dict(name="predict_batch_wiki_f128_bf16", kind="predict", m=4_096, of=0, n=40_000, f=128, dtype="bf16",
             out="bf16", offsets=True, activation="sigmoid", residual=False),
        # a few tokens through a wide layer: the weights' bytes bound it
        dict(name="predict_few_wide_bf16", kind="predict", m=5, of=0, n=8_192, f=8_192, dtype="bf16", out="bf16",
             offsets=True, activation="silu", residual=False),
        # many tokens through it, with the residual stream: the products bound it
        dict(name="predict_many_wide_bf16", kind="predict", m=4_096, of=0, n=8_192, f=8_192, dtype="bf16", out="bf16",
             offsets=True, activation="gelu", residual=True),
        # one row of the tiny shape's columns
        dict(name="log_prob_one_tiny", kind="log_prob", rows=1, n=500, dtype="f32", temperature=0.3, given=1,
             ragged=False, top=5, rated=25),
        # held-out items of a batch of users of the movie shape, training items left out, best 20 for the hit rate
        dict(name="log_prob_batch_movie", kind="log_prob", rows=1_024, n=17_770, dtype="f32", temperature=0.3,
             given=20, ragged=True, top=20, rated=208),
        # a small batch over the music shape's items in bf16: long rows
        dict(name="log_prob_long_music_bf16", kind="log_prob", rows=64, n=625_000, dtype="bf16", temperature=0.2,
             given=1, ragged=False, top=20, rated=250),
        # the gradient with respect to the scores of a batch of the movie shape
        dict(name="grad_batch_movie", kind="grad", rows=1_024, n=17_770, dtype="f32", temperature=0.3, given=20,
             ragged=True, rated=208, entropy=False, scores=True, columns=False),
        # long rows in bf16, with the entropy's gradient (a bonus for spread)
        dict(name="grad_long_music_bf16", kind="grad", rows=64, n=625_000, dtype="bf16", temperature=0.2, given=1,
             ragged=False, rated=250, entropy=True, scores=True, columns=False),
        # the gradient of the items' offsets alone
        dict(name="grad_offsets_movie", kind="grad", rows=1_024, n=17_770, dtype="f32", temperature=0.3, given=20,
             ragged=True, rated=208, entropy=False, scores=False, columns=True),
        # a whole step of fitting them
        dict(name="fit_batch_movie_f100", kind="fit", rows=1_024, of=480_000, n=17_770, f=100, temperature=0.3, given=1,
             ragged=False, rated=0),
    ]


_RANKS = (5, 8, 10, 16, 20, 24, 32, 37, 40, 50, 64, 72, 80, 96, 100, 113, 120, 128)
_ACTIVATIONS = ("none", "none", "clip", "relu", "gelu", "silu", "sigmoid", "tanh")


def draw(rng):
    """One more case: 1 to 4,096 rows against 300 to 625,000 columns, ranks or rows of 5 to 8,192 values; 1 to 2,048 rows
    of 300 to 625,000 scores; no more scores or products than the largest listed case of its kind."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def asked():
        return dict(temperature=rng.choice((0.05, 0.1, 0.3, 1.0)), given=rng.choice((1, 1, 2, 20)),
                    ragged=rng.choice((False, True)), rated=rng.choice((0, 20, 200)))

    kind = rng.choice(("predict",) * 6 + ("log_prob",) * 5 + ("grad",) * 4 + ("fit",) * 2)
    dtype = rng.choice(("f32", "f16", "bf16"))
    while True:
        if kind == "predict":
            m, n = spread(1, 4_096), spread(300, 625_000)
            f = rng.choice((rng.choice(_RANKS), spread(5, 8_192)))
            if m * n <= 100_000_000 and m * n * f <= 1.5e11 and n * f <= 150_000_000:
                return dict(kind=kind, m=m, of=rng.choice((0, 3)) * m, n=n, f=f, dtype=dtype,
                            out=rng.choice((dtype, dtype, "f32", "bf16")), offsets=rng.choice((True, True, False)),
                            activation=rng.choice(_ACTIVATIONS), residual=rng.choice((False, False, True)))
        elif kind == "fit":
            rows, n = spread(1, 2_048), spread(300, 625_000)
            if rows * n <= 18_000_000:
                return dict(asked(), kind=kind, rows=rows, of=4 * rows + 100, n=n, f=rng.choice(_RANKS))
        else:
            rows, n = spread(1, 2_048), spread(300, 625_000)
            if rows * n <= 40_000_000:
                case = dict(asked(), kind=kind, rows=rows, n=n, dtype=dtype)
                if kind == "log_prob":
                    return dict(case, top=rng.choice((0, 1, 5, 20, 50)))
                scores, columns = rng.choice(((True, False), (True, False), (False, True), (True, True)))
                return dict(case, entropy=rng.choice((False, True)), scores=scores, columns=columns)


# ------------------------------------------------------------------------------- inputs --


def _generator(seed):
    gen = torch.Generator(device=torch.device("cuda", DEVICE))
    gen.manual_seed(seed)
    return gen


def _normal(gen, *size):
    return torch.randn(*size, generator=gen, device=gen.device)


def _values(gen, rows, f):
    """Factors at ranks: a common scale and mean, as training leaves them for uncentred ratings.  Wider rows as
    activations and weights are, with products of about 1."""
    x = _normal(gen, rows, f)
    return x.add_(1.0).mul_(1.0 / math.sqrt(f)) if f <= 128 else x.mul_(f ** -0.25)


def _lengths(gen, rows, mean, most):
    lens = torch.exp(0.8 * _normal(gen, rows)) * mean * 0.726
    return lens.round().clamp_(max=most).to(torch.int64)


def _shares(gen, rows, total):
    """Row lengths of that sum, lognormal but for the longest."""
    upto = torch.cumsum(torch.exp(0.8 * _normal(gen, rows)).clamp_(max=4.0).double(), 0)
    return torch.diff((upto / upto[-1] * total).round().to(torch.int64), prepend=upto.new_zeros(1, dtype=torch.int64))


def _lists(gen, lens, n, step):
    """A CSR of these row lengths, each column once a row, and not in order of the columns."""
    rows = lens.numel()
    ptr = torch.zeros(rows + 1, dtype=torch.int64, device=gen.device)
    ptr[1:] = torch.cumsum(lens, 0)
    at = torch.arange(int(ptr[-1]), device=gen.device)
    row = torch.repeat_interleave(torch.arange(rows, device=gen.device), lens)
    start = torch.randint(0, n, (rows,), generator=gen, device=gen.device)
    # a row's columns: an arithmetic progression modulo n, its step having no factor in common with n
    while math.gcd(step, n) != 1:
        step += 2
    return ptr, ((start[row] + (at - ptr[row]) * step) % n).to(torch.int32)


def _scores(gen, rows, n):
    """Scores as a factor model gives them: the mean, an effect of the item, one of the pair."""
    z = _normal(gen, rows, n).mul_(0.6)
    z += 3.5 + 0.5 * _normal(gen, n)
    if rows >= 8:
        z[rows - 1] = float("-inf")     # a row with nothing left
        z[rows // 2, ::3] = float("-inf")
        z[rows // 3, 1::5] = float("nan")
    return z


def _asked(case, gen, rows, n):
    """The rows' temperatures, left-out columns and given ones, and what the loss weighs them with."""
    dev = gen.device
    s = dict(temperature=case["temperature"] * (0.5 + torch.rand(rows, generator=gen, device=dev)), rated=None)
    if case["rated"]:
        s["rated"] = _lists(gen, _lengths(gen, rows, case["rated"], n // 2), n, 7_919)
    if case["ragged"]:
        s["given"] = _lists(gen, _shares(gen, rows, rows * case["given"]), n, 5_003)
        entries = rows * case["given"]
    else:
        shape = (rows,) if case["given"] == 1 else (rows, case["given"])
        s["given"] = torch.randint(0, n, shape, generator=gen, device=dev, dtype=torch.int32)
        entries = shape
    # a mean over the entries, with a weight each (a rating's, or an advantage)
    s["grad_log"] = torch.randn(entries, generator=gen, device=dev).add_(1.0).div_(max(1, rows * case["given"]))
    s["grad_entropy"] = 0.01 / rows * (0.5 + torch.rand(rows, generator=gen, device=dev))
    return s


def _inputs(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    if kind == "predict":
        m, n, f = case["m"], case["n"], case["f"]
        s = dict(activation=case["activation"], out=_DTYPES[case["out"]], users=None, user_offset=None,
                 item_offset=None, residual=None)
        s["x"] = _values(gen, case["of"] or m, f).to(_DTYPES[case["dtype"]])
        s["theta"] = _values(gen, n, f).to(_DTYPES[case["dtype"]])
        if case["of"]:
            s["users"] = torch.randint(0, case["of"], (m,), generator=gen, device=gen.device, dtype=torch.int32)
        if case["offsets"]:
            s["item_offset"] = 0.5 * _normal(gen, n)
            if f <= 128:      # a layer has a bias for its outputs only
                s["user_offset"] = 2.0 + 0.4 * _normal(gen, case["of"] or m)
        if case["residual"]:
            s["residual"] = _normal(gen, m, n).to(s["out"])
        return s
    s = _asked(case, gen, case["rows"], case["n"])
    if kind == "fit":
        s["x"], s["theta"] = _values(gen, case["of"], case["f"]), _values(gen, case["n"], case["f"])
        s["users"] = torch.randint(0, case["of"], (case["rows"],), generator=gen, device=gen.device, dtype=torch.int32)
        s["item_offset"] = 0.5 * _normal(gen, case["n"])
    else:
        s["z"] = _scores(gen, case["rows"], case["n"]).to(_DTYPES[case["dtype"]])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_1603_03820_amd import predict
        s["ctx"] = predict.Context(DEVICE)
    if case["kind"] == "grad":      # the forward pass was before it
        if own:
            s["forward"] = predict.als_log_prob(s["ctx"], s["z"], s["given"], temperature=s["temperature"],
                                                rated=s["rated"])
        else:
            row, col = _entries(s["given"], case["rows"])
            s["forward"] = _distribution(s["z"], s["temperature"], s["rated"], row, col)
    return s


# --------------------------------------------------------------------------- plain forms --


def _activate(y, name):
    if name == "none":
        return y
    if name == "clip":
        return torch.clamp(y, 1.0, 5.0)
    if name == "relu":
        return torch.clamp(y, min=0.0)
    if name == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if name == "silu":
        return y / (1.0 + torch.exp(-y))
    if name == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-y))
    return torch.tanh(y)


def _predict(s):
    x = s["x"] if s["users"] is None else s["x"][s["users"].long()]
    y = x.float() @ s["theta"].float().t()
    if s["user_offset"] is not None:
        a = s["user_offset"] if s["users"] is None else s["user_offset"][s["users"].long()]
        y += a[:, None]
    if s["item_offset"] is not None:
        y += s["item_offset"]
    y = _activate(y, s["activation"])
    if s["residual"] is not None:
        y += s["residual"].float()
    return y.to(s["out"])


def _rows_of(ptr):
    return torch.repeat_interleave(torch.arange(ptr.numel() - 1, device=ptr.device), ptr[1:] - ptr[:-1])


def _entries(given, rows):
    """(row, column) of the given entries, in their order."""
    if isinstance(given, tuple):
        return _rows_of(given[0]), given[1].long()
    per = given.numel() // rows
    return torch.arange(rows, device=given.device).repeat_interleave(per), given.reshape(-1).long()


def _masked(z, rated):
    z = z.float()
    z = torch.where(torch.isnan(z), float("-inf"), z)
    if rated is not None:
        z = z.index_put((_rows_of(rated[0]), rated[1].long()), torch.full((), float("-inf"), device=z.device))
    return z


def _distribution(z, temperature, rated, row, col):
    """(log p of the entries, entropy, log p of all columns)."""
    z = _masked(z, rated)
    top = z.amax(1, keepdim=True)
    there = z > float("-inf")
    x = torch.where(there, torch.where(z == top, 0.0, (z - top) / temperature[:, None]), float("-inf"))
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    some = total > 0
    size = torch.log(torch.where(some, total, 1.0))
    log = x - size
    spread = (e * torch.where(e > 0, x, 0.0)).sum(1, keepdim=True)
    entropy = torch.where(some, size - spread / torch.where(some, total, 1.0), 0.0)
    return log[row, col], entropy[:, 0], log


def _best(z, log, rated, k):
    """The k columns that come first by their scores, and their log p; -1 and -inf where there are no more."""
    rows, n = z.shape
    z, order = torch.sort(_masked(z, rated), dim=1, descending=True, stable=True)
    order = order[:, :k]
    none = ~(z[:, :k] > float("-inf"))
    index = torch.full((rows, k), -1, dtype=torch.int32, device=z.device)
    best = torch.full((rows, k), float("-inf"), device=z.device)
    index[:, :order.shape[1]] = torch.where(none, -1, order).to(torch.int32)
    best[:, :order.shape[1]] = torch.where(none, float("-inf"), torch.gather(log, 1, order))
    return index, best


def _gradient(forward, s, row, col, with_entropy):
    entry, entropy, log = forward
    p = torch.exp(log)
    g = torch.where(entry > float("-inf"), s["grad_log"].reshape(-1), 0.0)
    total = torch.zeros(p.shape[0], device=p.device).index_put((row,), g, accumulate=True)
    d = (p * -total[:, None]).index_put((row, col), g, accumulate=True)
    if with_entropy:
        d -= s["grad_entropy"][:, None] * p * (torch.where(p > 0, log, 0.0) + entropy[:, None])
    return d / s["temperature"][:, None]


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "predict":
        return _predict(s)
    row, col = _entries(s["given"], case["rows"])
    if case["kind"] == "log_prob":
        entry, entropy, log = _distribution(s["z"], s["temperature"], s["rated"], row, col)
        out = dict(log=entry.reshape(s["grad_log"].shape), entropy=entropy)
        if case["top"]:
            out["top_index"], out["top_log"] = _best(s["z"], log, s["rated"], case["top"])
        return out
    if case["kind"] == "grad":
        d = _gradient(s["forward"], s, row, col, case["entropy"])
        out = {}
        if case["scores"]:
            out["grad"] = d.to(s["z"].dtype)
        if case["columns"]:
            out["columns"] = d.double().sum(0).float()
        return out
    z = s["x"][s["users"].long()] @ s["theta"].t() + s["item_offset"]
    forward = _distribution(z, s["temperature"], s["rated"], row, col)
    d = _gradient(forward, s, row, col, False)
    return dict(log=forward[0].reshape(s["grad_log"].shape), entropy=forward[1], columns=d.double().sum(0).float())


def _run_own(s, case):
    from paper_1603_03820_amd import predict
    ctx = s["ctx"]
    if case["kind"] == "predict":
        limits = dict(low=1.0, high=5.0) if s["activation"] == "clip" else {}
        return predict.als_predict(ctx, s["x"], s["theta"], users=s["users"], user_offset=s["user_offset"],
                                   item_offset=s["item_offset"], activation=s["activation"], residual=s["residual"],
                                   dtype=s["out"], **limits)
    if case["kind"] == "log_prob":
        r = predict.als_log_prob(ctx, s["z"], s["given"], temperature=s["temperature"], rated=s["rated"],
                                 top=case["top"])
        out = dict(log=r.log, entropy=r.entropy)
        if case["top"]:
            out["top_index"], out["top_log"] = r.top_index, r.top_log
        return out
    if case["kind"] == "grad":
        grad, columns = predict.als_log_prob_grad(
            ctx, s["z"], s["given"], s["forward"], s["grad_log"],
            grad_entropy=s["grad_entropy"] if case["entropy"] else None, temperature=s["temperature"],
            rated=s["rated"], grad=case["scores"], columns=case["columns"])
        out = {}
        if case["scores"]:
            out["grad"] = grad
        if case["columns"]:
            out["columns"] = columns
        return out
    z = predict.als_predict(ctx, s["x"], s["theta"], users=s["users"], item_offset=s["item_offset"])
    r = predict.als_log_prob(ctx, z, s["given"], temperature=s["temperature"], rated=s["rated"])
    _, columns = predict.als_log_prob_grad(ctx, z, s["given"], r, s["grad_log"], temperature=s["temperature"],
                                           rated=s["rated"], grad=False, columns=True)
    return dict(log=r.log, entropy=r.entropy, columns=columns)


# -------------------------------------------------------------------- work and precision --


def work(case):
    """Each input once, each output once; of a matrix that rows are taken from, those rows."""
    kind = case["kind"]
    if kind == "predict":
        m, n, f = case["m"], case["n"], case["f"]
        offsets = 4 * n + (4 * m if f <= 128 else 0) if case["offsets"] else 0
        users = 4 * m if case["of"] else 0
        return {"bytes": (m + n) * f * _BYTES[case["dtype"]] + offsets + users
                + m * n * _BYTES[case["out"]] * (2 if case["residual"] else 1), "flops": 2 * m * n * f}
    rows, n = case["rows"], case["n"]
    entries = rows * case["given"]
    lists = rows * 4 + entries * 4 + (rows * (4 * case["rated"] + 8) if case["rated"] else 0) \
        + (8 * rows if case["ragged"] else 0)
    if kind == "log_prob":
        # difference, scale, exponential and two sums of a score
        return {"bytes": rows * n * _BYTES[case["dtype"]] + lists + 4 * entries + 4 * rows + 8 * rows * case["top"],
                "flops": 6 * rows * n}
    if kind == "grad":
        per = _BYTES[case["dtype"]]
        return {"bytes": rows * n * per * (2 if case["scores"] else 1) + lists + 8 * entries + 12 * rows
                + (4 * n if case["columns"] else 0), "flops": 5 * rows * n}
    f = case["f"]
    return {"bytes": (rows + n) * 4 * f + 4 * rows + 4 * n + lists + 8 * entries + 4 * rows + 4 * n,
            "flops": 2 * rows * n * f + 11 * rows * n}


def _softmax64(z, s):
    """(p, log p) of every column in 64 bits, zero and -inf where it is left out."""
    z = z.double()
    left = torch.isnan(z) | (z == float("-inf"))
    if s["rated"] is not None:
        ptr, cols = s["rated"]
        lens = ptr.diff()
        left[torch.arange(z.shape[0], device=z.device).repeat_interleave(lens), cols.long()] = True
    y = (z / s["temperature"].double()[:, None]).masked_fill_(left, float("-inf"))
    size = torch.logsumexp(y, 1, keepdim=True)
    log = (y - torch.where(size > float("-inf"), size, 0.0)).masked_fill_(left, float("-inf"))
    return log.exp(), log


def _entropy64(p, log):
    return -(p * torch.where(p > 0, log, 0.0)).sum(1)


def _of_entries(log, s, rows):
    if isinstance(s["given"], tuple):
        row = torch.arange(rows, device=log.device).repeat_interleave(s["given"][0].diff())
        return row, log[row, s["given"][1].long()]
    given = s["given"].long().view(rows, -1)
    row = torch.arange(rows, device=log.device)[:, None].expand_as(given)
    return row.reshape(-1), torch.gather(log, 1, given).view(s["given"].shape)


def _columns_of(s):
    given = s["given"]
    return (given[1] if isinstance(given, tuple) else given).long().reshape(-1)


def _gradient64(p, log, row, entry, s, with_entropy):
    g = s["grad_log"].double().reshape(-1).clone()
    g[entry.reshape(-1) == float("-inf")] = 0.0
    total = torch.zeros(p.shape[0], dtype=torch.float64, device=p.device).index_add_(0, row, g)
    d = p * -total[:, None]
    if with_entropy:
        d -= (s["grad_entropy"].double()[:, None] * p) * (torch.where(p > 0, log, 0.0) + _entropy64(p, log)[:, None])
    at = row * p.shape[1] + _columns_of(s)
    d.view(-1).index_add_(0, at, g)
    return d.div_(s["temperature"].double()[:, None])


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("predict", "fit"):
        x, theta = s["x"].double(), s["theta"].double()
        users = s["users"]
        if users is not None:
            x = x.index_select(0, users.long())
        y = torch.mm(x, theta.t())
        if s["item_offset"] is not None:
            y.add_(s["item_offset"].double())
        if kind == "predict":
            if s["user_offset"] is not None:
                a = s["user_offset"].double()
                y.add_((a if users is None else a.index_select(0, users.long())).view(-1, 1))
            name = s["activation"]
            if name == "clip":
                y.clamp_(1.0, 5.0)
            elif name == "relu":
                y.clamp_(min=0.0)
            elif name == "gelu":
                y.mul_(0.5 * torch.special.erfc(y * -math.sqrt(0.5)))
            elif name == "silu":
                y.mul_(torch.special.expit(y))
            elif name == "sigmoid":
                y = torch.special.expit(y)
            elif name == "tanh":
                y = y.tanh_()
            if s["residual"] is not None:
                y.add_(s["residual"].double())
            return y
    else:
        y = s["z"]
    rows = case["rows"]
    p, log = _softmax64(y, s)
    row, entry = _of_entries(log, s, rows)
    out = {}
    if kind != "grad":
        out["log"], out["entropy"] = entry, _entropy64(p, log)
    if kind == "log_prob":
        k = case["top"]
        if k:
            best, order = torch.sort(-log, dim=1, stable=True)
            best, order = -best[:, :k], order[:, :k].to(torch.int32)
            # the order is by the scores themselves: equal probabilities in 64 bits are equal scores
            out["top_index"] = torch.where(best > float("-inf"), order, -1)
            out["top_log"] = best
        return out
    d = _gradient64(p, log, row, entry, s, kind == "grad" and case["entropy"])
    if kind == "fit":
        out["columns"] = d.sum(0)
        return out
    if case["scores"]:
        out["grad"] = d
    if case["columns"]:
        out["columns"] = d.sum(0)
    return out
