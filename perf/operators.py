"""The operators that answer with a trained model, as timed cases: factor rows held in 8 bits, the scores of
users against items from them, and the draw of an item from a row of scores.

A case is a dict; ``kind`` says which operator it is:

``quantize``   rows of X (or the rows ``users`` of it) to 8-bit integers with one scale a row:
               a = max |x|, q = rint(127 x / a), s = a / 127.  127 x and its quotient by a are each rounded to 32
               bits: a step of q would otherwise hang on the last bit of a tie.
``score``      out[i, j] = s_i t_j sum_k x_ik t_jk from 8-bit rows of both sides with a scale for each row.
``sample``     one column a row from its scores, with temperature, top-k, top-p and min-p and the columns of a
               CSR row left out, from one given uniform number a row.
``recommend``  the three in a row, as a serving loop calls them: the users' rows to 8 bits, their scores against
               all items (held in 8 bits from before), and a draw among the items a user has not rated.

The draw's weights are whole numbers, 2^40 exp((z - max) / T) rounded down, so that sums of them do not depend
on their order: the set that top-p keeps and the column that a uniform number meets are the same however a
row is cut up.  Columns with -inf or NaN are never drawn; a row without any other column gives index -1.
"""
import math

import torch

own = False
DEVICE = 0

_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # one user's factor row, as a request brings it: the smallest call
        dict(name="quantize_one_f100", kind="quantize", rows=1, of=0, f=100, dtype="f32"),
        # the item factors of the music shape, laid out once after training
        dict(name="quantize_music_items_f100", kind="quantize", rows=625_000, of=0, f=100, dtype="f32"),
        # wide activation rows in bf16
        dict(name="quantize_wide_bf16", kind="quantize", rows=8_192, of=0, f=8_192, dtype="bf16"),
        # one user against the movie shape's items
        dict(name="score_one_movie_f100", kind="score", m=1, n=17_770, f=100, dtype="f32"),
        # a batch of users against them
        dict(name="score_batch_movie_f100", kind="score", m=1_024, n=17_770, f=100, dtype="f32"),
        # a large batch at the largest rank against the wiki shape's columns, scores in bf16
        dict(name="score_batch_wiki_f128_bf16", kind="score", m=4_096, n=40_000, f=128, dtype="bf16"),
        # a few tokens through a wide layer: the weights' bytes bound it
        dict(name="score_few_wide_bf16", kind="score", m=5, n=8_192, f=8_192, dtype="bf16"),
        # many tokens through it: the products bound it
        dict(name="score_many_wide_bf16", kind="score", m=8_192, n=8_192, f=8_192, dtype="bf16"),
        # one row of the tiny shape's columns
        dict(name="sample_one_tiny", kind="sample", rows=1, n=500, dtype="f32", temperature=0.3, top_k=50,
             top_p=0.95, min_p=0.0, rated=25),
        # a batch over the movie shape's items, top-k then top-p, rated items left out
        dict(name="sample_batch_movie", kind="sample", rows=1_024, n=17_770, dtype="f32", temperature=0.3,
             top_k=200, top_p=0.9, min_p=0.0, rated=208),
        # a small batch over the music shape's items in bf16: long rows, top-p and min-p over all of them
        dict(name="sample_long_music_bf16", kind="sample", rows=64, n=625_000, dtype="bf16", temperature=0.2,
             top_k=0, top_p=0.9, min_p=0.02, rated=250),
        # the whole path for a batch of users of the movie shape
        dict(name="recommend_batch_movie_f100", kind="recommend", rows=1_024, of=480_000, n=17_770, f=100,
             temperature=0.3, top_k=200, top_p=0.9, min_p=0.0, rated=208),
    ]


_RANKS = (5, 8, 10, 16, 20, 24, 32, 37, 40, 50, 64, 72, 80, 96, 100, 113, 120, 128)


def draw(rng):
    """One more case: 1 to 1M rows of 5 to 8,192 values; 1 to 8,192 rows against 300 to 625,000; 1 to 2,048
    rows of 300 to 625,000 scores; no more values or products than the largest listed case of its kind."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def limits():
        return dict(temperature=rng.choice((0.05, 0.1, 0.3, 1.0)), top_k=rng.choice((0, 0, 1, 20, 50, 200, 1_000)),
                    top_p=rng.choice((1.0, 0.95, 0.9, 0.5)), min_p=rng.choice((0.0, 0.0, 0.02, 0.1)),
                    rated=rng.choice((0, 20, 200)))

    kind = rng.choice(("quantize",) * 3 + ("score",) * 5 + ("sample",) * 5 + ("recommend",) * 2)
    dtype = rng.choice(("f32", "f16", "bf16"))
    while True:
        if kind == "quantize":
            rows, f = spread(1, 1_000_000), spread(5, 8_192)
            if rows * f <= 60_000_000:
                return dict(kind=kind, rows=rows, of=rng.choice((0, 0, 2)) * rows, f=f, dtype=dtype)
        elif kind == "score":
            m, n = spread(1, 8_192), spread(300, 625_000)
            f = rng.choice((rng.choice(_RANKS), spread(5, 8_192)))
            if m * n <= 100_000_000 and m * n * f <= 4e11 and n * f <= 300_000_000:
                return dict(kind=kind, m=m, n=n, f=f, dtype=dtype)
        elif kind == "sample":
            rows, n = spread(1, 2_048), spread(300, 625_000)
            if rows * n <= 40_000_000:
                return dict(limits(), kind=kind, rows=rows, n=n, dtype=dtype)
        else:
            rows, n = spread(1, 2_048), spread(300, 625_000)
            if rows * n <= 20_000_000:
                return dict(limits(), kind=kind, rows=rows, of=4 * rows + 100, n=n, f=rng.choice(_RANKS))


# ------------------------------------------------------------------------------- inputs --


def _generator(seed):
    gen = torch.Generator(device=torch.device("cuda", DEVICE))
    gen.manual_seed(seed)
    return gen


def _normal(gen, *size):
    return torch.randn(*size, generator=gen, device=gen.device)


def _factor(gen, rows, f):
    """Factors as training leaves them for uncentred ratings: a common scale and mean."""
    return _normal(gen, rows, f).add_(1.0).mul_(1.0 / math.sqrt(f))


def _values(gen, rows, f):
    """Rows of factors at ranks; wider rows as activations are, with a few large columns."""
    if f <= 128:
        return _factor(gen, rows, f)
    x = _normal(gen, rows, f)
    return x.mul_(torch.exp(0.5 * _normal(gen, f)))


def _choice(gen, rows, n, rated):
    """A CSR of `rated` columns a row on average, lognormal lengths, each column once a row, and not in order
    of the columns."""
    lens = torch.exp(0.8 * _normal(gen, rows)) * rated * 0.726
    lens = lens.round().clamp_(max=n // 2).to(torch.int64)
    ptr = torch.zeros(rows + 1, dtype=torch.int64, device=gen.device)
    ptr[1:] = torch.cumsum(lens, 0)
    at = torch.arange(int(ptr[-1]), device=gen.device)
    row = torch.repeat_interleave(torch.arange(rows, device=gen.device), lens)
    start = torch.randint(0, n, (rows,), generator=gen, device=gen.device)
    # a row's columns: an arithmetic progression modulo n, its step having no factor in common with n
    step = 7_919 if n % 7_919 else 7_927
    return ptr, ((start[row] + (at - ptr[row]) * step) % n).to(torch.int32)


def _limits(case, gen, rows):
    """What the requests of a batch ask for: one temperature, k, p and least probability a row."""
    dev = gen.device
    temperature = case["temperature"] * (0.5 + torch.rand(rows, generator=gen, device=dev))
    temperature[torch.arange(rows, device=dev) % 16 == 5] = 0.0      # these ask for the best column
    top_k = torch.full((rows,), case["top_k"], dtype=torch.int32, device=dev)
    if case["top_k"] > 1:
        top_k = torch.randint(1, 2 * case["top_k"], (rows,), generator=gen, device=dev, dtype=torch.int32)
    top_p = torch.full((rows,), case["top_p"], device=dev)
    if case["top_p"] < 1.0:
        top_p -= 0.1 * torch.rand(rows, generator=gen, device=dev)
    min_p = case["min_p"] * torch.rand(rows, generator=gen, device=dev)
    u = torch.rand(rows, generator=gen, device=dev)
    return dict(u=u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def _scores(gen, rows, n):
    """Scores as a factor model gives them: the mean, an effect of the item, one of the pair."""
    z = _normal(gen, rows, n).mul_(0.6)
    z += 3.5 + 0.5 * _normal(gen, n)
    if rows >= 8:
        z[rows - 1] = float("-inf")     # a row with nothing left to draw
        z[rows // 2, ::3] = float("-inf")
        z[rows // 3, 1::5] = float("nan")
    return z


def _inputs(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    if kind == "quantize":
        of = case["of"] or case["rows"]
        x = _values(gen, of, case["f"]).to(_DTYPES[case["dtype"]])
        users = None
        if case["of"]:
            users = torch.randint(0, of, (case["rows"],), generator=gen, device=gen.device, dtype=torch.int32)
        elif case["rows"] >= 8:
            x[case["rows"] // 2] = 0
        return dict(x=x, users=users)
    if kind == "score":
        x, theta = _values(gen, case["m"], case["f"]), _values(gen, case["n"], case["f"])
        return dict(x=x, theta=theta, dtype=_DTYPES[case["dtype"]])
    s = _limits(case, gen, case["rows"])
    if kind == "sample":
        s["z"] = _scores(gen, case["rows"], case["n"]).to(_DTYPES[case["dtype"]])
        s["rated"], s["users"] = None, None
        if case["rated"]:
            s["rated"] = _choice(gen, case["rows"], case["n"], case["rated"])
        return s
    s["x"] = _factor(gen, case["of"], case["f"])
    s["theta"] = _factor(gen, case["n"], case["f"])
    s["users"] = torch.randint(0, case["of"], (case["rows"],), generator=gen, device=gen.device, dtype=torch.int32)
    s["rated"] = _choice(gen, case["of"], case["n"], case["rated"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["kind"] = case["kind"]
    quantize = _quantize
    if own:
        from paper_1603_03820_amd import serve
        s["ctx"] = serve.Context(DEVICE)

        def quantize(x):
            return serve.als_quantize(s["ctx"], x)
    # a serving program holds the items' rows in 8 bits; a product's users are in 8 bits before it, too
    if case["kind"] in ("score", "recommend"):
        s["tq"], s["ts"] = quantize(s.pop("theta"))
    if case["kind"] == "score":
        s["xq"], s["xs"] = quantize(s.pop("x"))
    return s


# --------------------------------------------------------------------------- plain forms --


def _quantize(x):
    x = x.float()
    big = x.abs().amax(1, keepdim=True)
    q = torch.round((x * 127.0) / torch.where(big > 0, big, torch.ones_like(big)))
    return q.to(torch.int8), (big / 127.0)[:, 0]


def _score(xq, xs, tq, ts, dtype):
    out = xq.float() @ tq.float().t()
    return out.mul_(xs[:, None]).mul_(ts).to(dtype)


def _share(total, part):
    """floor(total part / 2^24) of whole numbers, part < 2^25, without a product past 64 bits."""
    return (total >> 24) * part + (((total & 0xFFFFFF) * part) >> 24)


def _sample(z, u, temperature, top_k, top_p, min_p, rated, users):
    rows, n = z.shape
    z = z.float()
    z = torch.where(torch.isnan(z), float("-inf"), z)
    if rated is not None:
        ptr, col = rated
        of = torch.arange(rows, device=z.device) if users is None else users.long()
        lens = ptr[of + 1] - ptr[of]
        row = torch.repeat_interleave(torch.arange(rows, device=z.device), lens)
        first = torch.cumsum(lens, 0) - lens
        at = torch.arange(row.numel(), device=z.device) - first[row] + ptr[of][row]
        z = z.index_put((row, col[at].long()), torch.full((), float("-inf"), device=z.device))
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    top = z[:, :1]
    greedy = ~(temperature > 0)
    scale = 1.0 / torch.where(greedy, torch.ones_like(temperature), temperature)
    x = torch.where(z == top, 0.0, (z - top) * scale[:, None])
    e = torch.where(z > float("-inf"), torch.exp(x), 0.0)
    place = torch.arange(n, device=z.device)
    k = torch.where(greedy, 1, torch.where(top_k > 0, top_k, n))
    weight = torch.where(place < k[:, None], (e * 2.0 ** 40).to(torch.int64), 0)
    # top-p: a column stays while the weight before it has not reached the share
    upto = torch.cumsum(weight, 1)
    total = upto[:, -1:]
    part = (top_p.clamp(0.0, 1.0) * 2.0 ** 24).to(torch.int64)[:, None]
    stays = (upto - weight < _share(total, part).clamp(min=1)) & (e >= min_p.clamp(max=1.0)[:, None])
    weight = torch.where(stays, weight, 0)
    # the uniform number's place among the weights, in the columns' own order
    weight = torch.zeros_like(weight).scatter_(1, order, weight)
    upto = torch.cumsum(weight, 1)
    total = upto[:, -1:]
    target = _share(total, (u * 2.0 ** 24).to(torch.int64)[:, None])
    at = torch.searchsorted(upto, target, right=True).clamp_(max=n - 1)
    x = torch.zeros_like(x).scatter_(1, order, x)
    log = torch.gather(x, 1, at) - torch.log(total.float() * 2.0 ** -40)
    none = total <= 0
    return torch.where(none, -1, at)[:, 0].to(torch.int32), torch.where(none, float("-inf"), log)[:, 0]


def run(s):
    kind = s["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "quantize":
        x = s["x"] if s["users"] is None else s["x"][s["users"].long()]
        q, scale = _quantize(x)
        return q * scale[:, None], scale
    if kind == "score":
        return _score(s["xq"], s["xs"], s["tq"], s["ts"], s["dtype"])
    if kind == "sample":
        z = s["z"]
    else:
        xq, xs = _quantize(s["x"][s["users"].long()])
        z = _score(xq, xs, s["tq"], s["ts"], torch.float32)
    return _sample(z, s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["rated"], s["users"])


def _run_own(s, kind):
    from paper_1603_03820_amd import serve
    ctx = s["ctx"]
    if kind == "quantize":
        q, scale = serve.als_quantize(ctx, s["x"], users=s["users"])
        return q * scale[:, None], scale
    if kind == "score":
        return serve.als_score(ctx, s["xq"], s["xs"], s["tq"], s["ts"], dtype=s["dtype"])
    if kind == "sample":
        z = s["z"]
    else:
        xq, xs = serve.als_quantize(ctx, s["x"], users=s["users"])
        z = serve.als_score(ctx, xq, xs, s["tq"], s["ts"])
    return serve.als_sample(ctx, z, s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                            min_p=s["min_p"], rated=s["rated"], users=s["users"])


# -------------------------------------------------------------------- work and precision --


def work(case):
    """Each input once, each output once; of a matrix that rows are taken from, those rows."""
    kind = case["kind"]
    if kind == "quantize":
        rows, f = case["rows"], case["f"]
        users = 4 * rows if case["of"] else 0
        return {"bytes": rows * f * (_BYTES[case["dtype"]] + 1) + 4 * rows + users, "flops": 4 * rows * f}
    if kind == "score":
        m, n, f = case["m"], case["n"], case["f"]
        return {"bytes": (m + n) * (f + 4) + m * n * _BYTES[case["dtype"]], "flops": 2 * m * n * (f + 1)}
    rows, n = case["rows"], case["n"]
    limits = rows * 5 * 4
    left_out = rows * (4 * case["rated"] + 8) if case["rated"] else 0
    draw_bytes = limits + left_out + rows * 8
    # difference, scale, exponential and sum of a score
    if kind == "sample":
        return {"bytes": rows * n * _BYTES[case["dtype"]] + draw_bytes, "flops": 4 * rows * n}
    f = case["f"]
    return {"bytes": rows * (4 * f + 4) + n * (f + 4) + draw_bytes, "flops": 2 * rows * n * (f + 1) + 4 * rows * n}


def _quantize64(x):
    x = x.double()
    big = x.abs().max(dim=1).values
    # the definition's two roundings to 32 bits; of a quotient of such numbers, 64 bits hold enough
    q = (x * 127.0).float().double().div_(torch.where(big > 0, big, 1.0)[:, None]).float().double()
    low = torch.floor(q)
    up = (q - low > 0.5) | ((q - low == 0.5) & (low % 2 == 1))
    return low + up, big / 127.0


def _sample64(z, s):
    """Row by row: the allowed columns, best first; the cuts; the uniform number among what is left."""
    rows, n = z.shape
    index = torch.full((rows,), -1, dtype=torch.int32, device=z.device)
    log = torch.full((rows,), float("-inf"), dtype=torch.float64, device=z.device)
    host = {name: s[name].tolist() for name in ("u", "temperature", "top_k", "top_p", "min_p")}
    users = range(rows) if s["users"] is None else s["users"].tolist()
    if s["rated"] is not None:
        ptr, col = s["rated"][0].tolist(), s["rated"][1].long()
    for r in range(rows):
        v = z[r].double()
        allowed = v > float("-inf")
        if s["rated"] is not None:
            allowed[col[ptr[users[r]]:ptr[users[r] + 1]]] = False
        cols = torch.nonzero(allowed)[:, 0]
        if cols.numel() == 0:
            continue
        v, order = torch.sort(-v[cols], stable=True)
        cols, v = cols[order], -v
        temperature, k = host["temperature"][r], host["top_k"][r]
        if temperature <= 0:
            index[r], log[r] = cols[0], 0.0
            continue
        if k > 0:
            cols, v = cols[:k], v[:k]
        share = torch.exp((v - v[0]) / temperature)
        before = torch.cat((torch.zeros(1, device=z.device, dtype=torch.float64), torch.cumsum(share, 0)[:-1]))
        stays = (before < host["top_p"][r] * share.sum()) & (share >= host["min_p"][r])
        cols, order = torch.sort(cols[stays])
        share = share[stays][order]
        upto = torch.cumsum(share, 0)
        at = torch.searchsorted(upto, host["u"][r] * upto[-1:], right=True).clamp_(max=cols.numel() - 1)
        index[r] = cols[at][0]
        log[r] = torch.log(share[at] / upto[-1])[0]
    return index, log


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        x = s["x"] if s["users"] is None else s["x"].index_select(0, s["users"].long())
        q, scale = _quantize64(x)
        return q.mul_(scale[:, None]), scale
    if kind == "score":
        # the 8-bit rows and their scales, which are held in 32 bits, are the call's inputs
        xq, xs = _quantize64(s["x"])
        tq, ts = _quantize64(s["theta"])
        return torch.mm(xq, tq.t()).mul_(xs.float().double()[:, None]).mul_(ts.float().double())
    if case["rows"] * 2e-3 + case["rows"] * case["n"] * 2e-8 > 15:
        return None    # over about 20 seconds row by row
    if kind == "sample":
        return _sample64(s["z"], s)
    q, scale = _quantize64(s["x"].index_select(0, s["users"].long()))
    tq, ts = _quantize64(s["theta"])
    z = torch.mm(q, tq.t()).mul_(scale[:, None]).mul_(ts.float().double())   # the items' are inputs
    return _sample64(z, s)
