"""What stands between a layer's activations and its attention in a server whose requests have lengths of their own: places in
pages for a batch's new tokens, their queries and keys turned by their positions, both on the way into pages, and the
projections that make queries and keys with a low-rank adapter of every request's own.

A case is a plain dict.  "path" names the call; sizes are B rows (requests), H heads, k clusters (k = H: a layer without
clusters), Tn new tokens of a row, page the tokens of a page.  All tensors come from the seed.

  place    B rows of up to T cached tokens; "prompts" of them get up to Tn new tokens, the others one (or, now and then, none).
           "short": the free pages do not suffice for all of them.
  rotate   blocks of Tn tokens, queries [B,H,Tn,128] and compact keys [B,k,Tn,128] into a contiguous cache from pos0 on.
           "layout": pairs of neighbours or halves of the rotated part, "rot" elements of 128; "scaling" of the angles; "far": positions
           of their own for every row, up to a million.
  packed   the tokens of all rows one behind the other ("prompts" rows with up to Tn, the others one each), turned and written into
           pages.  "cache": how keys and values are held ("f32", "bf16", "e4m3").  "by_slot": keys come as projections of the
           representatives give them, [N,k,128], else of all heads.
  adapted  projections of the representatives from [B,Tn,D] activations, adapters of rank R ("parts": of queries, keys or both),
           "adapters" of them for the B rows; "bare": some rows have none.

run() computes the plain form in torch where `own` is false, and calls the library where it is true.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128                            # head dimension
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.bfloat16}     # of queries and new rows
E4M3 = torch.float8_e4m3fn
LARGEST = 448.0                    # largest finite E4M3 value
THETA = 10000.0


def listed():
    return [
        # the decode step of a full batch: a token for every request, few of which need a page
        {"name": "place_token_16", "path": "place", "B": 16, "T": 2048, "Tn": 1, "prompts": 0, "page": 64, "short": False},
        # a busy server: requests that decode, and prompts among them, more than there are pages for
        {"name": "place_mixed_256", "path": "place", "B": 256, "T": 4096, "Tn": 2043, "prompts": 24, "page": 16, "short": True},
        # one request's new token, fp32: nothing but latency
        {"name": "rotate_one_f32", "path": "rotate", "B": 1, "H": 32, "k": 8, "Tn": 1, "pos0": 255, "dtype": "f32", "rot": 128,
         "layout": "halves", "scaling": "none", "far": False},
        # a layer without clusters, a block of a long document: far positions, scaled angles, part of the head in pairs
        {"name": "rotate_dense_4x52_far", "path": "rotate", "B": 4, "H": 52, "k": 52, "Tn": 777, "pos0": 0, "dtype": "bf16",
         "rot": 64, "layout": "pairs", "scaling": "turns", "far": True},
        # the prompts of a full batch behind the positions that membership was decided on
        {"name": "rotate_prompt_16x32", "path": "rotate", "B": 16, "H": 32, "k": 8, "Tn": 2043, "pos0": 5, "dtype": "bf16",
         "rot": 128, "layout": "halves", "scaling": "none", "far": False},
        # the decode step of a full batch, keys as the projections leave them
        {"name": "packed_token_16x32", "path": "packed", "B": 16, "H": 32, "k": 8, "Tn": 1, "prompts": 0, "page": 64,
         "cache": "bf16", "by_slot": True, "rot": 128, "layout": "halves", "scaling": "none"},
        # prompts and decoding rows in one block, quantised on their way into pages
        {"name": "packed_mixed_64x32_e4m3", "path": "packed", "B": 64, "H": 32, "k": 8, "Tn": 2043, "prompts": 8, "page": 64,
         "cache": "e4m3", "by_slot": False, "rot": 128, "layout": "halves", "scaling": "linear"},
        # a small batch's prompts of a layer without clusters
        {"name": "packed_prompt_4x72_dense", "path": "packed", "B": 4, "H": 72, "k": 72, "Tn": 1000, "prompts": 4, "page": 16,
         "cache": "bf16", "by_slot": False, "rot": 96, "layout": "pairs", "scaling": "base"},
        # the new tokens of a full batch, each with an adapter of its own
        {"name": "adapted_token_16x32", "path": "adapted", "B": 16, "H": 32, "k": 8, "Tn": 1, "D": 4096, "R": 16, "adapters": 16,
         "parts": "qk", "bare": False},
        # a few short blocks of a wide model, adapters of the queries alone, some rows without
        {"name": "adapted_block_8x72", "path": "adapted", "B": 8, "H": 72, "k": 16, "Tn": 37, "D": 9216, "R": 8, "adapters": 5,
         "parts": "q", "bare": True},
        # one prompt, a larger rank
        {"name": "adapted_prompt_1x52", "path": "adapted", "B": 1, "H": 52, "k": 16, "Tn": 1777, "D": 6656, "R": 64, "adapters": 3,
         "parts": "qk", "bare": False},
        # the prompts of a full batch: the largest call
        {"name": "adapted_prompt_16x32", "path": "adapted", "B": 16, "H": 32, "k": 8, "Tn": 2043, "D": 4096, "R": 16,
         "adapters": 8, "parts": "qk", "bare": False},
    ]


MOST_BYTES = 1.0e9                 # of a drawn case; the largest listed ones are at about this
MOST_FLOPS = 5.4e11


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _turning(rng):
    return {"rot": rng.choice([128, 128, 128, 96, 64, 32]), "layout": rng.choice(["halves", "pairs"]),
            "scaling": rng.choice(["none", "linear", "base", "turns"])}


def draw(rng: random.Random):
    while True:
        path = rng.choice(["place", "rotate", "rotate", "packed", "packed", "adapted", "adapted", "adapted"])
        H = rng.choice([16, 32, 52, 72])
        heads = {"H": H, "k": rng.choice([4, 8, 16, H])}
        page = rng.choice([8, 16, 24, 32, 64, 128])
        if path == "place":
            B = _log_int(rng, 1, 1024)
            case = {"path": path, "B": B, "T": _log_int(rng, 1, 8192), "Tn": _log_int(rng, 1, 4096),
                    "prompts": rng.choice([0, (B + 7) // 8, B]), "page": page, "short": rng.random() < 0.4}
        elif path == "rotate":
            case = {"path": path, "B": _log_int(rng, 1, 64), **heads, "Tn": _log_int(rng, 1, 4096),
                    "pos0": rng.choice([0, 5, rng.randrange(1, 1024)]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                    **_turning(rng), "far": rng.random() < 0.4}
        elif path == "packed":
            B = _log_int(rng, 1, 128)
            case = {"path": path, "B": B, **heads, "Tn": _log_int(rng, 1, 4096), "prompts": rng.choice([0, (B + 7) // 8, B]),
                    "page": page, "cache": rng.choice(["bf16", "bf16", "e4m3", "e4m3", "f32"]), "by_slot": rng.random() < 0.5,
                    **_turning(rng)}
        else:
            B = _log_int(rng, 1, 64)
            case = {"path": path, "B": B, **heads, "Tn": rng.choice([1, _log_int(rng, 1, 2048)]),
                    "D": rng.choice([1024, 2048, 4096, 6656, 9216, 64 * _log_int(rng, 8, 144)]), "R": rng.choice([8, 16, 16, 32, 64, 128]),
                    "adapters": rng.randint(1, B + 2), "parts": rng.choice(["qk", "qk", "q", "k"]), "bare": rng.random() < 0.3}
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


# ------------------------------------------------------------------------------------------------- inputs
def _counts(case):
    """New tokens of every row: the same for every seed, so that the work of a case does not hang on it."""
    B, p = case["B"], case["prompts"]
    n = np.ones(B, np.int64)
    n[:p] = np.maximum(1, np.ceil(case["Tn"] * (np.arange(p) + 1.0) / max(p, 1)))
    if case["path"] == "place" and B > 8:
        n[p:][7::8] = 0                                    # places without a request
    return n


def _pages_needed(lens, counts, page):
    return -(-(lens + counts) // page) - -(-lens // page)


def _maps(case, g):
    """Representatives of a partition of its own for every row: k different heads, ascending."""
    B, H, k = case["B"], case["H"], case["k"]
    rep = np.stack([np.sort(g.permutation(H)[:k]) for _ in range(B)]).astype(np.int32)
    return torch.from_numpy(rep).cuda()


def _frequencies(case):
    """Radians per position of every pair of a head's rotated part."""
    rot = case["rot"]
    i = np.arange(rot // 2, dtype=np.float64)
    f = THETA ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        f = f / 4.0
    elif case["scaling"] == "base":
        f = (THETA * 8.0 ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
    elif case["scaling"] == "turns":                       # slow ones divided, fast ones kept, by their turns over 2048 positions
        w = np.clip((2048.0 * f / (2.0 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = w * f + (1.0 - w) * f / 16.0
    return torch.from_numpy(f).cuda()


def _gain(case):
    return 1.25 if case["scaling"] == "turns" else 1.0


def _pool(g, shape, cache):
    """Pages that have been in use: values as a model's, or codes of every size and a scale for each row of them."""
    if cache != "e4m3":
        return torch.randn(shape, generator=g, device="cuda").to(TYPES[cache]), None
    x = torch.randn(shape, generator=g, device="cuda")
    x.mul_(150.0).clamp_(-LARGEST, LARGEST)
    return x.to(E4M3).view(torch.uint8), torch.rand(shape[:3], generator=g, device="cuda").add_(0.5).mul_(0.0065)


def prepare(case, seed):
    path, B = case["path"], case["B"]
    host = np.random.default_rng(int(seed))
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    empty = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": case}
    if path == "place":
        page, T = case["page"], case["T"]
        counts = host.permutation(_counts(case))
        lens = host.permutation(np.ceil(T * (np.arange(B) + 1.0) / B).astype(np.int64))
        blocks = -(-(T + case["Tn"]) // page)
        need, used = _pages_needed(lens, counts, page), -(-lens // page)
        free = int(need.sum()) * 3 // 4 if case["short"] else int(need.sum()) + 1 + B // 4
        n_pages = int(used.sum()) + free
        pages = host.permutation(n_pages)
        table = np.full((B, blocks), -1, np.int64)
        at = 0
        for b in range(B):
            table[b, :used[b]] = pages[at:at + used[b]]
            at += used[b]
        held = host.integers(0, n_pages, n_pages)          # (what the list holds above its top does not matter)
        held[:free] = pages[at:]
        N = int(counts.sum())
        N = -(-N // 16) * 16                               # a block of a size that a recorded step was made for
        s.update(page=page, counts=ints(counts), lens=ints(lens), table=ints(table), free=ints(held), n_free=ints([free]),
                 new_lens=empty(B), n_left=empty(1), granted=empty(B), offsets=empty(B + 1), rows=empty(N), positions=empty(N),
                 slots=empty(N))
        return s
    H, k = case["H"], case["k"]
    s["rep"] = _maps(case, host) if k < H else None
    if path == "adapted":
        Tn, W, R, n = case["Tn"], case["D"], case["R"], case["adapters"]
        new = lambda std, *shape: torch.randn(shape, generator=g, device="cuda").mul_(std).to(torch.bfloat16)  # noqa: E731
        if s["rep"] is None:
            s["rep"] = ints(np.tile(np.arange(H), (B, 1)))
        s["x"] = new(1.0, B, Tn, W)
        s["w"] = {p: new(W ** -0.5, H * D, W) for p in "qk"}
        s["a"] = {p: new(W ** -0.5, n, R, W) if p in case["parts"] else None for p in "qk"}
        s["b"] = {p: new(R ** -0.5, n, H * D, R) if p in case["parts"] else None for p in "qk"}
        ids = host.integers(0, n, B)
        if n >= B:
            ids = host.permutation(n)[:B]
        if case["bare"]:
            ids[host.random(B) < 0.4] = -1
        s["ids"] = ints(ids)
        s["scales"] = torch.from_numpy(host.uniform(0.25, 2.0, n).astype(np.float32)).cuda()
        s["q_out"] = torch.zeros((B, H, Tn, D), dtype=torch.bfloat16, device="cuda")
        s["k_out"] = torch.zeros((B, k, Tn, D), dtype=torch.bfloat16, device="cuda")
        return s
    s["freq"], s["gain"] = _frequencies(case), _gain(case)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)  # noqa: E731
    if path == "rotate":
        Tn, pos0, dt = case["Tn"], case["pos0"], TYPES[case["dtype"]]
        s["q"], s["k"] = new(B, H, Tn, D), new(B, k, Tn, D)
        s["q_out"] = torch.zeros((B, H, Tn, D), dtype=dt, device="cuda")
        s["k_out"] = torch.zeros((B, k, pos0 + Tn + 3, D), dtype=dt, device="cuda")
        s["positions"] = ints(host.integers(0, 1000000, (B, 1)) + np.arange(Tn)) if case["far"] else None
        return s
    page, dt = case["page"], TYPES[case["cache"]]
    counts = host.permutation(_counts(case))
    N = int(counts.sum())
    start = host.integers(0, 2048, B) * (counts == 1)      # (rows that decode have some tokens, prompts none)
    rows = np.repeat(np.arange(B), counts)
    pos = np.concatenate([np.arange(start[b], start[b] + counts[b]) for b in range(B)])
    # every row writes to the pages from its first new position's on; those before are not touched and not made
    first = start // page
    blocks = -(-(start + counts) // page) - first
    n_pages = int(blocks.sum()) + 1 + B // 2
    ids = host.permutation(n_pages)
    begin = np.concatenate([[0], np.cumsum(blocks)])
    s["rows"], s["positions"] = ints(rows), ints(pos)
    s["slots"] = ints(ids[begin[rows] + pos // page - first[rows]] * page + pos % page)
    s["q"], s["v"] = new(N, H, D), new(N, H, D)
    s["k"] = new(N, k if case["by_slot"] else H, D)
    s["q_out"] = torch.zeros((N, H, D), dtype=dt, device="cuda")
    s["k_pages"], s["k_scales"] = _pool(g, (n_pages, k, page, D), case["cache"])
    s["v_pages"], s["v_scales"] = _pool(g, (n_pages, H, page, D), case["cache"])
    return s


# ------------------------------------------------------------------------------------------------- plain form
def _plain_place(s):
    page, table = s["page"], s["table"]
    B, blocks = table.shape
    N, n_pages = s["slots"].shape[0], s["free"].shape[0]
    counts, lens, n_free = s["counts"].long().clamp(min=0), s["lens"].long().clamp(min=0), s["n_free"].long()
    ends = torch.cumsum(counts, 0)
    fits = (ends <= N) & (lens + counts <= blocks * page)
    held = (lens + page - 1) // page
    need = torch.where(fits, (lens + counts + page - 1) // page - held, torch.zeros_like(lens))
    upto = torch.cumsum(need, 0)
    granted = fits & ((need == 0) | (upto <= n_free))
    need, before = need * granted, upto - need
    taken = need.sum().reshape(1)
    # the new blocks of all rows one behind the other
    i = torch.arange(n_pages, device=table.device)
    row = torch.searchsorted(torch.cumsum(need, 0), i, right=True).clamp(max=B - 1)
    first = torch.cumsum(need, 0) - need
    block = held[row] + i - first[row]
    page_of = s["free"].long()[(n_free - 1 - before[row] - (i - first[row])).clamp(0, n_pages - 1)]
    put = i < taken
    flat = torch.where(put, row * blocks + block, torch.full_like(i, B * blocks))
    wide = torch.cat([table.flatten().long(), torch.zeros(1, dtype=torch.long, device=table.device)])
    wide[flat] = torch.where(put, page_of, torch.zeros_like(page_of))
    table = wide[:-1].reshape(B, blocks)
    # the tokens
    n = torch.arange(N, device=table.device)
    row = torch.searchsorted(ends, n, right=True)
    there = row < B
    row_at = row.clamp(max=B - 1)
    pos = torch.where(there, lens[row_at] + n - (ends - counts)[row_at], torch.zeros_like(n))
    at = table[row_at, (pos // page).clamp(max=blocks - 1)]
    ok = there & granted[row_at] & (at >= 0) & (at < n_pages)
    slots = torch.where(ok, at * page + pos % page, torch.full_like(n, -1))
    offsets = torch.cat([torch.zeros_like(ends[:1]), ends.clamp(max=N)])
    got = {"table": table, "new_lens": lens + counts * granted, "n_left": n_free - taken, "granted": granted, "offsets": offsets,
           "rows": torch.where(there, row, torch.full_like(row, -1)), "positions": pos, "slots": slots}
    return {name: t.to(torch.int32) for name, t in got.items()}


def _turned(x, angle, layout, gain):
    """x [...,128], angle [...,rot/2] (64 bits, as far positions need): the first `rot` elements turned, in 64 bits."""
    half = angle.shape[-1]
    x = x.double()
    c, s = torch.cos(angle) * gain, torch.sin(angle) * gain
    if layout == "halves":
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], -1).float()


def _plain_rotate(s):
    case, rep, q, k = s["case"], s["rep"], s["q"], s["k"]
    B, Tn, pos0 = case["B"], case["Tn"], case["pos0"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(pos0, pos0 + Tn, device="cuda").expand(B, Tn)
    angle = pos.double()[..., None] * s["freq"]
    turn = lambda x: _turned(x, angle[:, None], case["layout"], s["gain"]).to(x.dtype)  # noqa: E731
    if rep is None:
        s["q_out"].copy_(turn(q))
    else:
        at = rep.long()[:, :, None, None].expand(-1, -1, Tn, D)
        s["q_out"].scatter_(1, at, turn(torch.gather(q, 1, at)))
    s["k_out"][:, :, pos0:pos0 + Tn] = turn(k)
    return {"q": s["q_out"], "k": s["k_out"]}


def _stored(rows):
    """E4M3 codes and scales of 32-bit rows [...,128]."""
    amax = rows.abs().amax(-1, keepdim=True)
    largest = torch.full_like(amax, LARGEST)               # (a quotient with a number would be a product with its inverse)
    inv = torch.where(amax == 0, torch.zeros_like(amax), largest / amax)
    return (rows * inv).clamp(-LARGEST, LARGEST).to(E4M3).view(torch.uint8), (amax / largest).squeeze(-1)


def _write(pages, scales, rows, slots, page):
    """rows [N,streams,128], 32 bits, to their places."""
    at, slot = slots // page, slots % page
    if scales is None:
        pages[at, :, slot] = rows.to(pages.dtype)
    else:
        pages[at, :, slot], scales[at, :, slot] = _stored(rows)


def _held(s):
    """The pages as the values that they hold (codes as 8-bit floating point values, beside their scales)."""
    if s["k_scales"] is None:
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {"k_pages": s["k_pages"].view(E4M3), "v_pages": s["v_pages"].view(E4M3), "k_scales": s["k_scales"],
            "v_scales": s["v_scales"]}


def _plain_packed(s):
    case, rep, q, k = s["case"], s["rep"], s["q"], s["k"]
    angle = (s["positions"].double()[:, None] * s["freq"])[:, None]
    turn = lambda x: _turned(x, angle, case["layout"], s["gain"])  # noqa: E731
    if rep is None:
        s["q_out"].copy_(turn(q))
    else:
        at = rep.long()[s["rows"].long()][:, :, None].expand(-1, -1, D)
        s["q_out"].scatter_(1, at, turn(torch.gather(q, 1, at)).to(q.dtype))
        if not case["by_slot"]:
            k = torch.gather(k, 1, at)
    slots = s["slots"].long()
    _write(s["k_pages"], s["k_scales"], turn(k), slots, case["page"])
    _write(s["v_pages"], s["v_scales"], s["v"].float(), slots, case["page"])
    return {"q": s["q_out"], **_held(s)}


def _plain_adapted(s):
    case = s["case"]
    W, R = case["D"], case["R"]
    rep, ids = s["rep"].long(), s["ids"].long()
    there = (ids >= 0).float()
    ids = ids.clamp(min=0)
    scale = s["scales"][ids] * there
    for b in range(case["B"]):
        x = s["x"][b].float()
        for part, out in (("q", s["q_out"]), ("k", s["k_out"])):
            w = s["w"][part].view(-1, D, W)[rep[b]].reshape(-1, W)
            y = torch.matmul(x, w.float().t())
            if s["a"][part] is not None:
                t = torch.matmul(x, s["a"][part].index_select(0, ids[b:b + 1])[0].float().t()) * scale[b]
                up = s["b"][part].index_select(0, ids[b:b + 1])[0].view(-1, D, R)[rep[b]].reshape(-1, R)
                y = y + torch.matmul(t, up.float().t())
            y = y.view(x.shape[0], -1, D).transpose(0, 1).to(out.dtype)
            if part == "q":
                out[b, rep[b]] = y
            else:
                out[b] = y
    return {"q": s["q_out"], "k": s["k_out"]}


PLAIN = {"place": _plain_place, "rotate": _plain_rotate, "packed": _plain_packed, "adapted": _plain_adapted}


def run(s):
    path = s["case"]["path"]
    return _own(s, path) if own else PLAIN[path](s)


# ------------------------------------------------------------------------------------------------- the library
def _own(s, path):
    import paper_2403_08058_amd as C
    case = s["case"]
    if path == "place":
        if "workspace" not in s:                           # workspaces are kept from step to step, as a server does
            s["workspace"] = C.alloc_paged_place_workspace(case["B"])
        C.chai_paged_place_tokens(s["counts"], s["lens"], s["table"], s["free"], s["n_free"], s["page"], s["new_lens"], s["n_left"],
                                  s["granted"], s["offsets"], s["rows"], s["positions"], s["slots"], s["workspace"])
        return {n: s[n] for n in ("table", "new_lens", "n_left", "granted", "offsets", "rows", "positions", "slots")}
    if path == "adapted":
        if "workspace" not in s:
            s["workspace"] = C.alloc_adapted_workspace(case["B"], case["Tn"], case["R"])
        C.chai_project_qk_adapted(s["x"], s["w"]["q"], s["w"]["k"], s["rep"], s["ids"], s["a"]["q"], s["b"]["q"], s["a"]["k"],
                                  s["b"]["k"], s["scales"], s["q_out"], s["k_out"], 0, s["workspace"])
        return {"q": s["q_out"], "k": s["k_out"]}
    layout = C.CHAI_ROPE_PAIRS if case["layout"] == "pairs" else C.CHAI_ROPE_HALVES
    if path == "rotate":
        C.chai_rotate_qk(s["q"], s["k"], s["rep"], s["freq"], s["q_out"], s["k_out"], case["pos0"], positions=s["positions"],
                         layout=layout, gain=s["gain"])
        return {"q": s["q_out"], "k": s["k_out"]}
    C.chai_paged_append_packed(s["q"], s["k"], s["v"], s["rep"], s["rows"], s["positions"], s["slots"], s["freq"], s["q_out"],
                               s["k_pages"], s["v_pages"], k_scales=s["k_scales"], v_scales=s["v_scales"], layout=layout,
                               gain=s["gain"], k_by_slot=case["by_slot"])
    return {"q": s["q_out"], **_held(s)}


def work(case):
    """One pass's bytes, each input once and each output once; its multiplications and additions."""
    B = case["B"]
    if case["path"] == "place":
        page, counts = case["page"], _counts(case)
        N = -(-int(counts.sum()) // 16) * 16
        pages = int(np.ceil(counts / page).sum())          # taken from the list and written to the table, about
        return {"bytes": 4 * (2 * B + 3 * B + 2 + 1 + 3 * N + 2 * pages + B), "flops": 4 * N + 8 * B}
    H, k = case["H"], case["k"]
    maps = 4 * B * k if k < H else 0
    if case["path"] == "adapted":
        Tn, W, R, n = case["Tn"], case["D"], case["R"], min(case["adapters"], B)
        heads = H if k == H else H * (1.0 - (1.0 - k / H) ** B)                # in use, if the rows' maps are independent
        parts, tokens = len(case["parts"]), B * Tn
        weights = 2 * heads * 2 * D * W
        adapters = parts * n * R * (W + min(heads, k * B / n) * D) * 2
        return {"bytes": int(weights + adapters + tokens * W * 2 + tokens * k * 2 * D * 2 + maps + 8 * B),
                "flops": 2 * tokens * k * 2 * D * W + 2 * tokens * parts * R * (W + k * D)}
    turned = 3 * case["rot"] + case["rot"] // 2            # per row of 128: four products and two sums a pair
    if case["path"] == "rotate":
        width, tokens = {"f32": 4, "bf16": 2}[case["dtype"]], B * case["Tn"]
        return {"bytes": 2 * tokens * 2 * k * D * width + maps + (4 * tokens if case["far"] else 0) + 4 * case["rot"],
                "flops": tokens * 2 * k * turned}
    new, held = {"f32": (4, 512), "bf16": (2, 256), "e4m3": (2, 132)}[case["cache"]]
    N = int(_counts(case).sum())
    return {"bytes": N * (2 * k * D * new + (k + H) * (D * new + held) + 12) + maps + 4 * case["rot"], "flops": N * 2 * k * turned}


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_place(s):
    page = s["page"]
    table, free, n_free = s["table"].tolist(), s["free"].tolist(), int(s["n_free"])
    counts, lens, N, n_pages = s["counts"].tolist(), s["lens"].tolist(), len(s["slots"]), len(s["free"])
    got = {"new_lens": [], "granted": [], "offsets": [0], "rows": [], "positions": [], "slots": []}
    top, ended, open_ = n_free, 0, True
    for b, (n, count) in enumerate(zip(lens, counts)):
        ended += count
        new = list(range(-(-n // page), -(-(n + count) // page)))
        ok = ended <= N and n + count <= len(table[b]) * page
        if ok and new:
            if len(new) > top:
                open_ = False                              # first come, first served: nobody behind gets a page
            ok = open_
        if ok:
            for block in new:
                top -= 1
                table[b][block] = free[top]
        got["granted"].append(int(ok))
        got["new_lens"].append(n + count if ok else n)
        got["offsets"].append(min(ended, N))
        for i in range(count):
            if len(got["rows"]) < N:
                at = table[b][(n + i) // page] if ok else -1
                got["rows"].append(b)
                got["positions"].append(n + i)
                got["slots"].append(at * page + (n + i) % page if 0 <= at < n_pages else -1)
    rest = N - len(got["rows"])
    got["rows"] += [-1] * rest
    got["positions"] += [0] * rest
    got["slots"] += [-1] * rest
    got.update(table=table, n_left=[top])
    return {name: torch.tensor(got[name], dtype=torch.int32, device="cuda") for name in
            ("table", "new_lens", "n_left", "granted", "offsets", "rows", "positions", "slots")}


def _exact_turn(x, pos, s):
    """x [n,heads,128] at positions pos [n]: as products of complex numbers."""
    case, rot = s["case"], s["case"]["rot"]
    x = x.double()
    turn = torch.polar(torch.full_like(pos, s["gain"], dtype=torch.float64)[:, None].expand(-1, rot // 2).contiguous(),
                       pos.double()[:, None] * s["freq"][None])[:, None]
    part = x[..., :rot]
    part = part.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "halves" else part.unflatten(-1, (rot // 2, 2))
    part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
    if case["layout"] == "halves":
        part = part.transpose(-1, -2)
    return torch.cat([part.flatten(-2), x[..., rot:]], -1)


def _exact_codes(x):
    """The E4M3 values nearest to x * 448 / (largest of the row), ties to even, and the scale.  Rows are of 32 bits, and what is
    rounded to 8 is the product of 32-bit factors, as the codes are defined: those beside a tie would else go by its last bit."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    y = torch.where(top > 0, x * torch.full_like(top, LARGEST).div(top), 0.0).double()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, (top.double() / LARGEST)[..., 0]


def exact(case, seed):
    s = prepare(case, seed)
    path, B = case["path"], case["B"]
    if path == "place":
        return _exact_place(s)
    H, k = case["H"], case["k"]
    rep = s["rep"].tolist() if s["rep"] is not None else [list(range(H))] * B
    if path == "rotate":
        Tn, pos0 = case["Tn"], case["pos0"]
        q, keys = s["q_out"].double(), s["k_out"].double()
        for b in range(B):
            pos = s["positions"][b] if case["far"] else torch.arange(Tn, device="cuda") + pos0
            q[b, rep[b]] = _exact_turn(s["q"][b, rep[b]].transpose(0, 1), pos, s).transpose(0, 1)
            keys[b, :, pos0:pos0 + Tn] = _exact_turn(s["k"][b].transpose(0, 1), pos, s).transpose(0, 1)
        return {"q": q, "k": keys}
    if path == "packed":
        coded, page = s["k_scales"] is not None, case["page"]
        q = s["q_out"].double()
        held = {n: (s[n].view(E4M3) if coded else s[n]).double() for n in ("k_pages", "v_pages")}
        if coded:
            held.update({n: s[n].double() for n in ("k_scales", "v_scales")})
        for b in range(B):
            n = (s["rows"] == b).nonzero()[:, 0]
            heads, pos, slots = torch.tensor(rep[b], device="cuda"), s["positions"][n], s["slots"][n].long()
            q[n[:, None], heads[None]] = _exact_turn(s["q"][n][:, heads], pos, s)
            rows = {"k": _exact_turn(s["k"][n] if case["by_slot"] else s["k"][n][:, heads], pos, s), "v": s["v"][n].double()}
            for name, x in rows.items():
                if coded:
                    x, held[name + "_scales"][slots // page, :, slots % page] = _exact_codes(x)
                held[name + "_pages"][slots // page, :, slots % page] = x
        return {"q": q, **held}
    got = {"q": s["q_out"].double(), "k": s["k_out"].double()}
    for b, a in enumerate(s["ids"].tolist()):
        x = s["x"][b].double()
        for part in "qk":
            for j, head in enumerate(rep[b]):
                cols = slice(head * D, (head + 1) * D)
                y = x @ s["w"][part][cols].double().t().contiguous()
                if a >= 0 and s["a"][part] is not None:
                    t = x @ s["a"][part][a].double().t().contiguous()
                    y = y + float(s["scales"][a]) * (t @ s["b"][part][a, cols].double().t().contiguous())
                got[part][b, head if part == "q" else j] = y
    return got
