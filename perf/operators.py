"""What a server that keeps its requests' caches in pages asks of this library, one layer at a time: writing new tokens'
keys and values into pages (as they are, or as 8-bit codes), attention of one new token of every request over its pages,
both in one call, and reading pages back.

A case is a plain dict.  "path" names the call; sizes are B rows (requests), H heads, k clusters (k = H: a layer without
clusters), T the longest row's cached tokens (in attention calls the new one included), page the tokens of a page.  "lengths"
says how the rows' lengths are spread, "cache" how keys and values are held ("f32", "bf16" or "e4m3", the latter with queries
and new rows in bf16).  "holes": some pages inside the rows are absent, as after an eviction.  All tensors come from the seed.

run() computes the plain form in torch where `own` is false, and calls the library where it is true.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.bfloat16}     # of queries and new rows
E4M3 = torch.float8_e4m3fn
LARGEST = 448.0                    # largest finite E4M3 value


def listed():
    return [
        # one request soon after its start, fp32: nothing but latency
        {"name": "attend_one_f32", "path": "attention", "B": 1, "H": 32, "k": 8, "T": 256, "page": 16, "cache": "f32",
         "lengths": "equal", "holes": False},
        # an unclustered layer, a small batch of ordinary lengths
        {"name": "attend_dense_8x52", "path": "attention", "B": 8, "H": 52, "k": 52, "T": 1777, "page": 32, "cache": "bf16",
         "lengths": "uniform", "holes": False},
        # a large batch, most requests short and a few long, over 8-bit caches that have lost some pages
        {"name": "attend_tail_64x32_e4m3", "path": "attention", "B": 64, "H": 32, "k": 8, "T": 4096, "page": 16,
         "cache": "e4m3", "lengths": "tail", "holes": True},
        # long documents: the largest call
        {"name": "attend_long_4x32", "path": "attention", "B": 4, "H": 32, "k": 4, "T": 32768, "page": 128, "cache": "bf16",
         "lengths": "equal", "holes": False},
        # the ordinary decode step of a full batch: the new token is written and attended to
        {"name": "step_16x32", "path": "step", "B": 16, "H": 32, "k": 8, "T": 2048, "page": 64, "cache": "bf16",
         "lengths": "uniform", "holes": False},
        # the same over 8-bit caches
        {"name": "step_16x32_e4m3", "path": "step", "B": 16, "H": 32, "k": 8, "T": 2048, "page": 64, "cache": "e4m3",
         "lengths": "uniform", "holes": False},
        # a small batch of many heads soon after its prompts
        {"name": "step_4x72_short", "path": "step", "B": 4, "H": 72, "k": 16, "T": 577, "page": 16, "cache": "bf16",
         "lengths": "uniform", "holes": False},
        # the prompts of a small batch, written into pages as they are
        {"name": "append_prompt_4x72", "path": "append", "B": 4, "H": 72, "k": 16, "T": 512, "start": 0, "page": 16,
         "cache": "bf16", "lengths": "equal", "holes": False},
        # the prompts of a full batch, quantised on their way into pages
        {"name": "append_prompt_16x32_e4m3", "path": "append", "B": 16, "H": 32, "k": 8, "T": 2043, "start": 5, "page": 64,
         "cache": "e4m3", "lengths": "uniform", "holes": False},
        # the new token of every request
        {"name": "append_token_16x32_e4m3", "path": "append", "B": 16, "H": 32, "k": 8, "T": 1, "start": 1023, "page": 64,
         "cache": "e4m3", "lengths": "equal", "holes": False},
        # a full batch of 8-bit caches read back, for prompt attention over them
        {"name": "gather_16x32_e4m3", "path": "gather", "B": 16, "H": 32, "k": 8, "T": 2048, "start": 0, "page": 64,
         "cache": "e4m3", "lengths": "uniform", "holes": False},
        # one request's fp32 pages read back, from a position inside a page on
        {"name": "gather_one_f32", "path": "gather", "B": 1, "H": 32, "k": 8, "T": 250, "start": 5, "page": 16,
         "cache": "f32", "lengths": "equal", "holes": False},
    ]


MOST_BYTES = 1.2e9                 # of the largest listed case
MOST_PADDED = 2 ** 31              # elements of all rows at the longest one's length


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    while True:
        H = rng.choice([32, 52, 72])
        case = {"path": rng.choice(["attention", "attention", "attention", "step", "step", "step", "append", "append", "gather"]),
                "B": _log_int(rng, 1, 64), "H": H, "k": rng.choice([4, 8, 16, H]), "T": _log_int(rng, 1, 32768),
                "page": rng.choice([16, 16, 24, 32, 64, 128, 256]), "cache": rng.choice(["bf16", "bf16", "e4m3", "e4m3", "f32"]),
                "lengths": rng.choice(["equal", "uniform", "tail"]), "holes": rng.random() < 0.25}
        if case["path"] in ("append", "gather"):
            case["start"] = rng.choice([0, 5, rng.randrange(1, 2048)])
            if rng.random() < 0.3:
                case["T"] = 1
        padded = case["B"] * (case["T"] + case.get("start", 0)) * (H + case["k"]) * D
        if work(case)["bytes"] <= MOST_BYTES and padded <= MOST_PADDED:
            return case


# ------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Every row's tokens: a fixed spread from 0 or 1 to T, so that the work of a case does not hang on the seed."""
    B, T = case["B"], case["T"]
    if case["lengths"] == "equal":
        return np.full(B, T, np.int64)
    at = (np.arange(B) + 1.0) / B                          # the last row has T
    if case["lengths"] == "uniform":
        return np.maximum(1, np.ceil(T * at)).astype(np.int64)
    n = np.ceil(T * at ** 4).astype(np.int64)              # "tail": most rows short, and a place without a request
    if B > 2:
        n[0] = 0
    return n


def _maps(case, g):
    """Head -> cluster maps, a partition of its own for every row, no cluster empty; a cluster's representative is its lowest
    member and the clusters are numbered by it."""
    B, H, k = case["B"], case["H"], case["k"]
    h2c, rep = np.empty((B, H), np.int32), np.empty((B, k), np.int32)
    for b in range(B):
        raw = np.concatenate([np.arange(k), g.integers(0, k, H - k)])[g.permutation(H)]
        first = np.array([np.flatnonzero(raw == j)[0] for j in range(k)])
        label = np.empty(k, np.int64)
        label[np.argsort(first)] = np.arange(k)
        h2c[b], rep[b] = label[raw], np.sort(first)
    return torch.from_numpy(h2c).cuda(), torch.from_numpy(rep).cuda()


def _pool(g, shape, cache):
    """Pages that have been in use: values as a model's, or codes of every size and a scale for each row of them."""
    if cache != "e4m3":
        return torch.randn(shape, generator=g, device="cuda").to(TYPES[cache]), None
    x = torch.randn(shape, generator=g, device="cuda")
    x.mul_(150.0).clamp_(-LARGEST, LARGEST)
    return x.to(E4M3).view(torch.uint8), torch.rand(shape[:3], generator=g, device="cuda").add_(0.5).mul_(0.0065)


def prepare(case, seed):
    path, B, H, k, T, page = (case[n] for n in ("path", "B", "H", "k", "T", "page"))
    host = np.random.default_rng(int(seed))
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    start = case.get("start", 0)
    lengths = host.permutation(_lengths(case))
    blocks = -(-(start + T) // page)
    used = -(-(start + lengths) // page) * (lengths > 0)
    n_pages = int(used.sum()) + 1 + B // 2                 # some pages are free
    free = host.permutation(n_pages)
    table = host.integers(0, n_pages, (B, blocks))         # places that no row has reached hold what they held before
    at = 0
    for b in range(B):
        table[b, :used[b]] = free[at:at + used[b]]
        at += used[b]
    if case["holes"]:
        table[host.random((B, blocks)) < 0.2] = -1
    s = {"case": case, "page": page, "k": k, "T": T, "table": ints(table), "maps": _maps(case, host) if k < H else (None, None)}
    s["k_pages"], s["k_scales"] = _pool(g, (n_pages, k, page, D), case["cache"])
    s["v_pages"], s["v_scales"] = _pool(g, (n_pages, H, page, D), case["cache"])
    dt = TYPES[case["cache"]]
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)  # noqa: E731
    if path in ("attention", "step"):
        s["q"], s["lengths"] = new(B, H, D), ints(lengths)
        s["out"] = torch.empty((B, H, D), dtype=torch.float32, device="cuda")
    if path == "step":
        s["k_new"], s["v_new"] = new(B, H, D), new(B, H, D)
    if path in ("append", "gather"):
        s["start"], s["count"] = ints(np.full(B, start)), ints(lengths)
    if path == "append":
        s["k_new"], s["v_new"] = new(B, H, T, D), new(B, H, T, D)
    if path == "gather":
        s["k_out"] = torch.zeros((B, k, T, D), dtype=dt, device="cuda")
        s["v_out"] = torch.zeros((B, H, T, D), dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------- plain form
def _places(table, pos, valid, page, n_pages):
    """Page and place of positions [B,N] of every row, and which of them there are."""
    block = (pos // page).clamp(0, table.shape[1] - 1)
    at = torch.gather(table.long(), 1, block)
    there = valid & (pos < table.shape[1] * page) & (at >= 0) & (at < n_pages)
    return at.clamp(0, n_pages - 1), pos % page, there


def _rows(pages, scales, at, slot):
    """Rows [B,N,heads,128] in 32 bits."""
    x = pages[at, :, slot]
    if scales is None:
        return x.float()
    return x.view(E4M3).float() * scales[at, :, slot].unsqueeze(-1)


def _stored(rows):
    """E4M3 codes and scales of rows [...,128]."""
    x = rows.float()
    amax = x.abs().amax(-1, keepdim=True)
    largest = torch.full_like(amax, LARGEST)               # (a quotient with a number would be a product with its inverse)
    inv = torch.where(amax == 0, torch.zeros_like(amax), largest / amax)
    return (x * inv).clamp(-LARGEST, LARGEST).to(E4M3).view(torch.uint8), (amax / largest).squeeze(-1)


def _write(pages, scales, rows, at, slot, there):
    """rows [B,N,heads,128] into their places."""
    b, i = there.nonzero(as_tuple=True)
    rows = rows[b, i]
    if scales is None:
        pages[at[b, i], :, slot[b, i]] = rows
    else:
        pages[at[b, i], :, slot[b, i]], scales[at[b, i], :, slot[b, i]] = _stored(rows)


def _plain_append(s, k_new, v_new, pos, valid):
    """k_new, v_new [B,H,N,128] at positions pos [B,N]."""
    at, slot, there = _places(s["table"], pos, valid, s["page"], s["k_pages"].shape[0])
    rep = s["maps"][1]
    if rep is not None:
        k_new = torch.gather(k_new, 1, rep.long()[:, :, None, None].expand(-1, -1, *k_new.shape[2:]))
    _write(s["k_pages"], s["k_scales"], k_new.transpose(1, 2), at, slot, there)
    _write(s["v_pages"], s["v_scales"], v_new.transpose(1, 2), at, slot, there)


def _plain_attention(s):
    h2c, rep = s["maps"]
    q, n = s["q"].float(), s["lengths"].long()
    pos = torch.arange(s["T"], device=q.device).expand(q.shape[0], -1)
    at, slot, there = _places(s["table"], pos, pos < n[:, None], s["page"], s["k_pages"].shape[0])
    if rep is not None:
        q = torch.gather(q, 1, rep.long()[:, :, None].expand(-1, -1, D))
    keys = _rows(s["k_pages"], s["k_scales"], at, slot).transpose(1, 2).contiguous()
    scores = SCALE * torch.matmul(keys, q.unsqueeze(-1)).squeeze(-1)
    scores = scores.masked_fill(~there[:, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = weights.sum(-1, keepdim=True)
    p = torch.where(total == 0, torch.zeros_like(weights), weights / total)
    if h2c is not None:
        p = torch.gather(p, 1, h2c.long()[:, :, None].expand(-1, -1, p.shape[2]))
    values = _rows(s["v_pages"], s["v_scales"], at, slot).transpose(1, 2)
    values = values.masked_fill(~there[:, None, :, None], 0.0)
    return torch.matmul(p.unsqueeze(2), values.contiguous()).squeeze(2)


def _plain_gather(s):
    pos = s["start"].long()[:, None] + torch.arange(s["T"], device="cuda")
    valid = pos < (s["start"] + s["count"]).long()[:, None]
    at, slot, there = _places(s["table"], pos, valid, s["page"], s["k_pages"].shape[0])
    got = []
    for pages, scales, out in ((s["k_pages"], s["k_scales"], s["k_out"]), (s["v_pages"], s["v_scales"], s["v_out"])):
        x = _rows(pages, scales, at, slot).masked_fill(~there[:, :, None, None], 0.0).transpose(1, 2).to(out.dtype)
        got.append(torch.where(valid[:, None, :, None], x, out))
    return {"k": got[0], "v": got[1]}


def _held(s):
    """The pages as the values that they hold (codes as 8-bit floating point values, beside their scales)."""
    if s["k_scales"] is None:
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {"k_pages": s["k_pages"].view(E4M3), "v_pages": s["v_pages"].view(E4M3), "k_scales": s["k_scales"],
            "v_scales": s["v_scales"]}


def run(s):
    path = s["case"]["path"]
    if own:
        return _own(s, path)
    if path == "attention":
        return {"out": _plain_attention(s)}
    if path == "gather":
        return _plain_gather(s)
    if path == "step":
        last = s["lengths"].long()[:, None] - 1
        _plain_append(s, s["k_new"].unsqueeze(2), s["v_new"].unsqueeze(2), last.clamp(min=0), last >= 0)
        return {"out": _plain_attention(s), **_held(s)}
    pos = s["start"].long()[:, None] + torch.arange(s["T"], device="cuda")
    _plain_append(s, s["k_new"], s["v_new"], pos, pos < (s["start"] + s["count"]).long()[:, None])
    return _held(s)


# ------------------------------------------------------------------------------------------------- the library
def _own(s, path):
    import paper_2403_08058_amd as C
    h2c, rep = s["maps"]
    pages = (s["k_pages"], s["v_pages"])
    scales = {"k_scales": s["k_scales"], "v_scales": s["v_scales"]}
    if path == "append":
        C.chai_paged_append_kv(s["k_new"], s["v_new"], rep, s["table"], s["start"], s["count"], *pages, **scales)
        return _held(s)
    if path == "gather":
        C.chai_paged_gather_kv(*pages, s["table"], s["start"], s["count"], s["k_out"], s["v_out"], **scales)
        return {"k": s["k_out"], "v": s["v_out"]}
    if "workspace" not in s:                               # kept from step to step, as a server does
        s["workspace"] = C.alloc_paged_workspace(*s["q"].shape[:2], s["k"], s["T"])
    if path == "attention":
        C.chai_paged_decode_attention(s["q"], *pages, h2c, rep, s["table"], s["lengths"], s["T"], SCALE, s["out"],
                                      s["workspace"], **scales)
        return {"out": s["out"]}
    C.chai_paged_decode_step(s["q"], s["k_new"], s["v_new"], *pages, h2c, rep, s["table"], s["lengths"], s["T"], SCALE,
                             s["out"], s["workspace"], **scales)
    return {"out": s["out"], **_held(s)}


def work(case):
    """One pass's bytes, each once: cached rows, new rows, queries, maps, places and results; its multiplications and additions."""
    B, H, k, page = (case[n] for n in ("B", "H", "k", "page"))
    n = _lengths(case)
    tokens, rows = int(n.sum()), int((n > 0).sum())
    new, held = {"f32": (4, 512), "bf16": (2, 256), "e4m3": (2, 132)}[case["cache"]]
    maps = 4 * B * (H + k) if k < H else 0
    places = 4 * int((-(-(case.get("start", 0) + n) // page)).sum())
    cached = tokens * (k + H) * held
    if case["path"] == "gather":
        return {"bytes": cached + tokens * (k + H) * D * new + places, "flops": tokens * (k + H) * D}
    if case["path"] == "append":
        return {"bytes": cached + tokens * (k + H) * D * new + places + maps, "flops": tokens * (k + H) * D}
    grown = rows * (k + H) * D * new if case["path"] == "step" else 0      # (the row written is among the cached ones)
    return {"bytes": cached + grown + places + maps + B * k * D * new + B * H * D * 4 + 4 * B,
            "flops": 2 * tokens * (k + H) * D}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_codes(x):
    """The E4M3 values nearest to x * 448 / (largest of the row), ties to even, and the scale.  What is rounded to 8 bits is
    the product of 32-bit factors, as the codes are defined: those beside a tie would else go by the last bit of it."""
    top = x.abs().amax(-1, keepdim=True)
    y = torch.where(top > 0, x.float() * torch.full_like(top, LARGEST).float().div(top.float()), 0.0).double()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, (top / LARGEST)[..., 0]


def exact(case, seed):
    s = prepare(case, seed)
    path, B, H, k, page = (case[n] for n in ("path", "B", "H", "k", "page"))
    table, n_pages, coded = s["table"].tolist(), s["k_pages"].shape[0], s["k_scales"] is not None
    if s["maps"][0] is None:
        h2c, rep = [list(range(H))] * B, [list(range(H))] * B
    else:
        h2c, rep = s["maps"][0].tolist(), s["maps"][1].tolist()
    held = {n: (s[n].view(E4M3) if coded else s[n]).double() for n in ("k_pages", "v_pages")}
    if coded:
        held.update({n: s[n].double() for n in ("k_scales", "v_scales")})

    def positions(b, first, count):
        """(offset in the block of rows, page, place) of the positions first .. first+count-1 that are there."""
        found = [(t - first, table[b][t // page], t % page) for t in range(first, first + count)]
        found = [f for f in found if 0 <= f[1] < n_pages]
        return [torch.tensor(v, dtype=torch.long, device="cuda") for v in (zip(*found) if found else ([], [], []))]

    def put(b, first, count, k_rows, v_rows):
        i, at, slot = positions(b, first, count)
        for name, rows in (("k", k_rows[rep[b]]), ("v", v_rows)):
            x = rows.double()[:, i].permute(1, 0, 2)
            if coded:
                x, held[name + "_scales"][at, :, slot] = _exact_codes(x)
            held[name + "_pages"][at, :, slot] = x

    def take(b, first, count, name):
        i, at, slot = positions(b, first, count)
        x = held[name + "_pages"][at, :, slot]
        return i, x * held[name + "_scales"][at, :, slot][..., None] if coded else x

    if path == "append":
        for b, n in enumerate(s["count"].tolist()):
            put(b, case["start"], n, s["k_new"][b], s["v_new"][b])
        return held
    if path == "gather":
        got = {"k": s["k_out"].double(), "v": s["v_out"].double()}
        for b, n in enumerate(s["count"].tolist()):
            for name in ("k", "v"):
                i, x = take(b, case["start"], n, name)
                got[name][b][:, i] = x.permute(1, 0, 2)
        return got
    lengths = s["lengths"].tolist()
    if path == "step":
        for b, n in enumerate(lengths):
            if n > 0:
                put(b, n - 1, 1, s["k_new"][b].unsqueeze(1), s["v_new"][b].unsqueeze(1))
    out = torch.zeros((B, H, D), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lengths):
        i, keys = take(b, 0, n, "k")
        if not len(i):
            continue
        scores = SCALE * (keys * s["q"][b].double()[rep[b]]).sum(-1)
        p = torch.softmax(scores, 0)[:, h2c[b]]
        out[b] = (p[..., None] * take(b, 0, n, "v")[1]).sum(0)
    return {"out": out} if path == "attention" else {"out": out, **held}
