"""The paged compressed cache of an attention layer, as cases to time and to compare.

A cache holds the keys and values of many sequences as compressed arrays: one block a token and head, its largest
coefficient in N and the 8-bit bin indices of all its coefficients in F, in pages of `page` tokens that any sequence may
own.  With r = 127 and an orthonormal transform H (DCT-II, or Haar), of a head's D values x:

  append   C = x H,  N = max |C|,  F = rint(r C / N) (an all-zero line: N = 0, F = 0), stored at the token's slot,
           slot = page number * page + place in the page, for keys and for values
  attend   out_i = sum_j softmax_j(scale <q_i, k_j>) v_j,  k_j = H (N F / r) and v_j likewise, over the cached positions
           j <= p_i (and j > p_i - window where there is a window); p_i is the position of new token i, the last of
           which is the last position of its sequence; a group of query heads shares each head of the cache
  copy     page `to` becomes what page `from` is, keys and values: the copy that a write to a shared page needs, and the
           moves that bring pages together

A case is a dict of plain values:

  op          "append", "attend" or "copy"
  dim, heads  D, heads of the cache;  groups: query heads to each
  page        tokens to a page
  array       type of q, k, v and of the output;  work: type of N;  transform: "dct" or "haar"
  seqs, new   sequences, new tokens of each;  context: tokens that each has before those
  ragged      sequences differ in both (`new` and `context` are then the largest)
  window      0, or how many positions back a token sees, itself among them
  pairs       pages copied;  pool: pages there are
"""
import math

import numpy as np
import torch

own = False

FLOATS = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f64": 8, "f32": 4, "bf16": 2, "f16": 2}
RADIUS = 127.0


def _attend(name, seqs, new, context, heads=8, groups=4, dim=128, page=64, array="bf16", work="f32", transform="dct",
            ragged=False, window=0):
    case = {"op": "attend", "seqs": seqs, "new": new, "context": context, "heads": heads, "groups": groups, "dim": dim,
            "page": page, "array": array, "work": work, "transform": transform, "ragged": ragged, "window": window}
    return case if name is None else dict(case, name=name)


def _append(name, seqs, new, heads=8, dim=128, page=64, array="bf16", work="f32", ragged=False, context=0):
    # the transform is the codec's default.  (Under Haar, sums of 16-bit values meet exact rounding ties, which the last bit of
    # an irrational factor then decides: nothing to compare.)
    case = {"op": "append", "seqs": seqs, "new": new, "context": context, "heads": heads, "dim": dim, "page": page,
            "array": array, "work": work, "transform": "dct", "ragged": ragged}
    return case if name is None else dict(case, name=name)


def _copy(name, pairs, pool, heads=8, dim=128, page=64, work="f32"):
    case = {"op": "copy", "pairs": pairs, "pool": pool, "heads": heads, "dim": dim, "page": page, "work": work}
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # one sequence's next token, early on: what one call costs
        _attend("attend_token_short", 1, 1, 300, heads=2, dim=64, page=16),
        # a server's step: one token of each of 64 sequences of all ages
        _attend("attend_tokens_batch", 64, 1, 8192, ragged=True),
        # one token of one long document: nothing to split but its length
        _attend("attend_token_long", 1, 1, 131072, array="f16"),
        # one token of sequences that share one wide head of the cache
        _attend("attend_tokens_wide_head", 16, 1, 5000, heads=1, groups=16, dim=256, page=32, ragged=True),
        # four prompts continued by a chunk, as they are while others are served
        _attend("attend_chunks", 4, 512, 4096, page=32, work="f16", ragged=True),
        # chunks of odd lengths with a window, small heads, N in 16 bits, the other transform
        _attend("attend_odd_window", 7, 77, 1003, heads=5, groups=3, dim=64, page=16, array="f16", work="bf16",
                transform="haar", ragged=True, window=257),
        # a whole prompt at once
        _attend("attend_prompt", 1, 8192, 0),
        # the step's new keys and values, each to a page of its own
        _append("append_step", 64, 1, context=4000, ragged=True),
        # a prompt's keys and values
        _append("append_prompt", 1, 8192),
        # few tokens of 32-bit values, small heads, odd counts
        _append("append_odd", 3, 111, heads=5, dim=64, page=16, array="f32", work="f16", ragged=True, context=50),
        # sequences forked in the middle of a page
        _copy("copy_fork", 3, 64, page=16),
        # a fragmented pool brought together
        _copy("copy_compact", 2048, 6000),
    ]


def _log(rng, low, high):
    return int(round(2.0 ** rng.uniform(math.log2(low), math.log2(high))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "copy"])
    heads, dim = rng.choice([1, 2, 3, 5, 8, 8, 16]), rng.choice([32, 64, 128, 128, 256])
    page, work = rng.choice([16, 32, 64, 128]), rng.choice(["f32", "f32", "f16", "bf16"])
    if op == "copy":
        pairs = _log(rng, 1, 3000)
        case = _copy(None, pairs, 2 * pairs + rng.randrange(1, 200), heads, dim, page, work)
        limit = _copy(None, 2048, 6000)
    elif op == "append":
        seqs = _log(rng, 1, 64)
        case = _append(None, seqs, _log(rng, 1, 8192), heads, dim, page, rng.choice(["bf16", "f16", "f32"]), work,
                       rng.random() < 0.5, _log(rng, 1, 1000))
        limit = _append(None, 1, 8192)
    else:
        seqs = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.5 else _log(rng, 2, 4000)
        case = _attend(None, seqs, new, _log(rng, 1, 100000), heads, rng.choice([1, 2, 3, 4, 6, 8]), dim, page,
                       rng.choice(["bf16", "f16"]), work, rng.choice(["dct", "haar"]), rng.random() < 0.6,
                       rng.choice([0, 0, 0, 1, 100, 1024]))
        limit = None
    # no more than the largest listed case of its kind does
    while True:
        if limit is None:
            positions = case["seqs"] * (case["context"] + case["new"])
            products = case["seqs"] * case["new"] * case["heads"] * case["groups"] * (case["context"] + case["new"])
            fits = (positions * heads * dim <= 64 * 8192 * 8 * 128 and products * dim <= 32 * 8192 * 4096 * 128)
        else:
            fits = work_bytes(case) <= work_bytes(limit)
        if fits:
            return case
        if op == "copy":
            case["pairs"] = case["pairs"] * 2 // 3
        elif op == "append" or case["new"] > 64:
            key = "new" if case["new"] > 1 else "seqs"
            case[key] = case[key] * 2 // 3
        else:
            key = "context" if case["context"] > 2000 else "seqs"
            case[key] = case[key] * 2 // 3


def _lengths(case):
    """(new tokens, tokens before them) of every sequence; uneven sequences differ by low-discrepancy fractions."""
    new, before = [], []
    for b in range(case["seqs"]):
        if case["ragged"]:
            before.append(int(case["context"] * (0.05 + 0.95 * ((b + 1) * 0.6180339887498949 % 1.0))))
            new.append(max(1, int(math.ceil(case["new"] * ((b + 1) * 0.7548776662466927 % 1.0)))))
        else:
            before.append(case["context"])
            new.append(case["new"])
    return new, before


def _visible(new, before, window):
    """Pairs of a new token and a cached position that it sees, and positions that any of them sees."""
    pairs = 0
    for i in range(new):
        pairs += min(before + i + 1, window) if window else before + i + 1
    return pairs, min(before + new, window + new - 1) if window else before + new


def work_bytes(case):
    if case["op"] == "copy":
        return case["pairs"] * case["page"] * case["heads"] * (case["dim"] + BYTES[case["work"]]) * 2 * 2
    line = case["dim"] + BYTES[case["work"]]
    new, before = _lengths(case)
    if case["op"] == "append":
        return sum(new) * (8 + 2 * case["heads"] * (line + case["dim"] * BYTES[case["array"]]))
    read = sum(_visible(n, c, case["window"])[1] for n, c in zip(new, before)) * case["heads"] * line * 2
    return read + 2 * sum(new) * case["heads"] * case["groups"] * case["dim"] * BYTES[case["array"]]


def work(case):
    if case["op"] == "copy":
        flops = 0
    elif case["op"] == "append":
        # a line's transform by a fast algorithm, its maximum and its quotients
        flops = sum(_lengths(case)[0]) * 2 * case["heads"] * case["dim"] * (2 * math.log2(case["dim"]) + 3)
    else:
        pairs = sum(_visible(n, c, case["window"])[0] for n, c in zip(*_lengths(case)))
        flops = 4 * pairs * case["heads"] * case["groups"] * case["dim"]
    return {"bytes": work_bytes(case), "flops": flops}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _matrix(transform, n):
    """H[m][q]: coefficient q of x is sum_m x[m] H[m][q]."""
    m, q = np.meshgrid(np.arange(n, dtype=np.float64), np.arange(n, dtype=np.float64), indexing="ij")
    if transform == "dct":
        H = np.where(q == 0, math.sqrt(1.0 / n), math.sqrt(2.0 / n) * np.cos(math.pi * (2 * m + 1) * q / (2 * n)))
    else:
        H = np.zeros((n, n))
        H[:, 0] = math.sqrt(1.0 / n)
        column, runs = 1, 1
        while runs < n:
            width = n // runs
            for j in range(runs):
                H[j * width:j * width + width // 2, column] = math.sqrt(runs / n)
                H[j * width + width // 2:(j + 1) * width, column] = -math.sqrt(runs / n)
                column += 1
            runs *= 2
    return torch.from_numpy(H)


def _lines(rng, count, dim, channels):
    """Keys or values: normal, with a few channels that are several times the others, as projections have them."""
    return torch.randn(count, dim, generator=rng, device="cuda") * channels


def _channels(rng, dim):
    gain = torch.ones(dim, device="cuda")
    gain[torch.randperm(dim, generator=rng, device="cuda")[:max(1, dim // 32)]] = 6.0
    return gain


def _fill(rng, n_lines, dim, work, H):
    """A pool of compressed lines."""
    N = torch.empty(n_lines, dtype=FLOATS[work], device="cuda")
    F = torch.empty(n_lines, dim, dtype=torch.int8, device="cuda")
    gain = _channels(rng, dim)
    for at in range(0, n_lines, 1 << 20):
        C = _lines(rng, min(1 << 20, n_lines - at), dim, gain) @ H
        top = C.abs().amax(1)
        N[at:at + C.shape[0]] = top.to(N.dtype)
        F[at:at + C.shape[0]] = torch.round(C * (RADIUS / top[:, None])).to(torch.int8)
    return N, F


def prepare(case, seed):
    rng = torch.Generator(device="cuda").manual_seed(seed)
    host = np.random.default_rng(seed)
    heads, dim, page = case["heads"], case["dim"], case["page"]
    transform = case.get("transform", "dct")
    H = _matrix(transform, dim)
    state = {"case": case, "H": H.cuda()}
    if case["op"] == "copy":
        n_pages = case["pool"]
        picked = host.permutation(n_pages)[:2 * case["pairs"]].reshape(case["pairs"], 2)
        state["pairs"] = np.ascontiguousarray(picked, dtype=np.int32)
        state["from"], state["to"] = (torch.from_numpy(picked[:, i].astype(np.int64)).cuda() for i in (0, 1))
    else:
        new, before = _lengths(case)
        owned = [-(-(n + c) // page) for n, c in zip(new, before)]
        n_pages = sum(owned) + 3
        places = host.permutation(n_pages)[:sum(owned)].astype(np.int64)
        state["new"], state["before"] = new, before
        state["pages"] = np.split(places, np.cumsum(owned)[:-1])
    pools = []
    for _ in range(2):
        N, F = _fill(rng, n_pages * heads * page, dim, case["work"], state["H"].float())
        pools += [N.view(n_pages, heads, page), F.view(n_pages, heads, page, dim)]
    state["pools"] = tuple(pools)
    if case["op"] == "append":
        slots = [p[np.arange(c, c + n) // page] * page + np.arange(c, c + n) % page
                 for n, c, p in zip(new, before, state["pages"])]
        state["slots"] = torch.from_numpy(np.concatenate(slots)).cuda()
        kv = _lines(rng, sum(new) * 2 * heads, dim, _channels(rng, dim)).to(FLOATS[case["array"]])
        kv = kv.view(sum(new), 2, heads, dim)            # as one projection leaves them: keys and values side by side
        state["k"], state["v"] = kv[:, 0], kv[:, 1]
    elif case["op"] == "attend":
        state["q"] = torch.randn(sum(new), heads * case["groups"], dim, generator=rng, device="cuda").to(FLOATS[case["array"]])
        table = np.full((len(new), max(owned)), -1, dtype=np.int32)
        for b, p in enumerate(state["pages"]):
            table[b, :len(p)] = p
        state["table"] = torch.from_numpy(table).cuda()
        state["lengths"] = torch.tensor([n + c for n, c in zip(new, before)], dtype=torch.int32, device="cuda")
        state["starts"] = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        state["most"] = max(new)
        state["pages"] = [torch.from_numpy(p).cuda() for p in state["pages"]]
        state["scale"] = 1.0 / math.sqrt(dim)
    if own:
        from paper_2406_11209_amd.cache import PagedCache
        state["cache"] = PagedCache(dim, heads, n_pages, page, work_type=case["work"], transform=transform,
                                    pools=state["pools"])
        if case["op"] == "attend":
            state["out"] = torch.empty_like(state["q"])
    return state


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        cache = state["cache"]
        if case["op"] == "append":
            cache.append(state["k"], state["v"], state["slots"])
        elif case["op"] == "copy":
            cache.copy_pages(state["pairs"])
        else:
            return cache.attend(state["q"], state["table"], state["lengths"], starts=state["starts"],
                                max_new=state["most"], window=case["window"], scale=state["scale"], out=state["out"])
        return state["pools"]
    return {"append": _run_append, "copy": _run_copy, "attend": _run_attend}[case["op"]](state)


def _run_append(state):
    k_N, k_F, v_N, v_F = state["pools"]
    page = k_N.shape[2]
    at, place = state["slots"] // page, state["slots"] % page
    for x, N, F in ((state["k"], k_N, k_F), (state["v"], v_N, v_F)):
        C = torch.matmul(x.double(), state["H"])         # in 64 bits: values next to a rounding border
        top = C.abs().amax(-1)
        scaled = RADIUS * C / torch.where(top > 0, top, torch.ones_like(top))[..., None]
        N[at, :, place] = top.to(N.dtype)
        F[at, :, place] = torch.round(scaled).to(torch.int8)
    return state["pools"]


def _run_copy(state):
    for pool in state["pools"]:
        pool[state["to"]] = pool[state["from"]]
    return state["pools"]


def _gather(N, F, pages, length, H):
    """The first `length` lines of a sequence, decompressed: [heads, length, D]."""
    heads, dim = F.shape[1], F.shape[3]
    C = N[pages].to(H.dtype)[..., None] * F[pages].to(H.dtype) / RADIUS
    return (C.transpose(0, 1).reshape(heads, -1, dim)[:, :length] @ H.t())


def _run_attend(state):
    case, q = state["case"], state["q"]
    heads, groups, dim = case["heads"], case["groups"], case["dim"]
    k_N, k_F, v_N, v_F = state["pools"]
    H = state["H"].float()
    out = torch.empty_like(q)
    first = 0
    for new, before, pages in zip(state["new"], state["before"], state["pages"]):
        length = new + before
        k = _gather(k_N, k_F, pages, length, H)
        v = _gather(v_N, v_F, pages, length, H)
        at = torch.arange(before, length, device=q.device)[:, None]
        j = torch.arange(length, device=q.device)[None, :]
        hidden = j > at
        if case["window"]:
            hidden = hidden | (j <= at - case["window"])
        for h in range(heads):
            rows = q[first:first + new, h * groups:(h + 1) * groups].float()          # [new, groups, D]
            s = (rows.reshape(new * groups, dim) @ k[h].t()).view(new, groups, length) * state["scale"]
            s = s.masked_fill(hidden[:, None], -math.inf)
            s = (s - s.amax(-1, keepdim=True)).exp_()
            p = s / s.sum(-1, keepdim=True)
            o = p.view(new * groups, length) @ v[h]
            out[first:first + new, h * groups:(h + 1) * groups] = o.view(new, groups, dim).to(out.dtype)
        first += new
    return out


# ---- what the operators are defined to give, in 64 bits ----------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    H = _matrix(case.get("transform", "dct"), case["dim"]).cuda()
    pools = state["pools"]
    heads, page, dim = case["heads"], case["page"], case["dim"]
    if case["op"] == "copy":
        want = [pool.clone() for pool in pools]
        for pool, old in zip(want, pools):
            pool.index_copy_(0, state["to"], old.index_select(0, state["from"]))
        return tuple(want)
    if case["op"] == "append":
        want = []
        for x, N, F in ((state["k"], pools[0], pools[1]), (state["v"], pools[2], pools[3])):
            lines = x.to(torch.float64).reshape(-1, dim)
            C = torch.zeros_like(lines)
            for m in range(dim):                         # the sum of the definition, term by term
                C += lines[:, m:m + 1] * H[m]
            top = C.abs().max(1).values
            F_new = torch.where(top[:, None] > 0, torch.round(C * RADIUS / top[:, None]), torch.zeros_like(C))
            row = (state["slots"] // page)[:, None] * (heads * page) + torch.arange(heads, device="cuda") * page + \
                (state["slots"] % page)[:, None]
            N_all, F_all = N.reshape(-1).double(), F.reshape(-1, dim).clone()
            N_all[row.reshape(-1)] = top
            F_all[row.reshape(-1)] = F_new.to(torch.int8)
            want += [N_all.view(N.shape), F_all.view(F.shape)]
        return tuple(want)
    # in coefficients: <q, k> = <q H, N F / r> and the sum of values is transformed back once
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    q_all = (state["q"].double().reshape(-1, dim) @ H).view(state["q"].shape)
    starts = np.concatenate([[0], np.cumsum(state["new"])])
    for b, (new, before, pages) in enumerate(zip(state["new"], state["before"], state["pages"])):
        j = torch.arange(before + new, device="cuda")
        at, place = pages[j // page], j % page
        for h in range(heads):
            k = pools[0][at, h, place].double()[:, None] * pools[1][at, h, place].double() / RADIUS
            v = pools[2][at, h, place].double()[:, None] * pools[3][at, h, place].double() / RADIUS
            for g in range(h * case["groups"], (h + 1) * case["groups"]):
                for low in range(0, new, 2048):
                    i = torch.arange(low, min(low + 2048, new), device="cuda")
                    seen = j[None, :] <= before + i[:, None]
                    if case["window"]:
                        seen &= j[None, :] > before + i[:, None] - case["window"]
                    logits = torch.where(seen, state["scale"] * (q_all[starts[b] + i, g] @ k.t()), -math.inf)
                    out[starts[b] + i, g] = torch.softmax(logits, dim=-1) @ v @ H.t()
    return out
