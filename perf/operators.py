"""The operators around a paged key/value cache of 8-bit codes, as a serving (and, for the rotation, a training) program calls them:

    rope        rotary positions of Q and K, and their gradient
    write       new tokens quantised into the cache
    attend      attention over the cache
    copy, fork, compact, free    the pages of the cache

    own                 False: run() computes the plain form below; True: it calls the library's entry points
    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) device tensors a program has in hand before the call
    run(state)          one call and its outputs
    work(case)          bytes and flops the call cannot do without
    exact(case, seed)   what run() returns, from the definition in 64 bits

The cache: a block is 16 tokens of one head of one page, and has a scale for K and one for V; a value is code * scale.  Codes of K lie as
[page, head, block, channel / 16, token, channel % 16], codes of V as [page, head, block, channel, token].
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
FORMATS = ("e4m3", "int8")
CODE_TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
# largest code, as (fraction in [0.5, 1), exponent)
LARGEST = {"e4m3": (448 / 512, 9), "int8": (127 / 128, 7)}
LEAST_EXPONENT = -100
HEAD_SIZES = (32, 64, 96, 128, 256)
PAGES = (16, 32, 64, 128, 256)


# ---- cases ------------------------------------------------------------------------------------------------------------------------------

def _rope(name, B, N, Hq, Hk, d, rot, layout="half", dtype="bf16", transpose=False, scaling="none", far=0):
    return {"name": name, "op": "rope", "B": B, "N": N, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "layout": layout, "dtype": dtype,
            "transpose": transpose, "scaling": scaling, "far": far}


def _write(name, B, Hkv, d, N, start, page, fmt, ragged=False):
    return {"name": name, "op": "write", "B": B, "Hkv": Hkv, "d": d, "N": N, "start": start, "page": page, "fmt": fmt, "ragged": ragged}


def _attend(name, B, H, Hkv, d, Nq, keys, page, fmt, mask=0, ragged=False):
    return {"name": name, "op": "attend", "B": B, "H": H, "Hkv": Hkv, "d": d, "Nq": Nq, "keys": keys, "page": page, "fmt": fmt, "mask": mask,
            "ragged": ragged}


def _pages(name, op, seqs, keys, Hkv, d, page, count, spare=64):
    return {"name": name, "op": op, "seqs": seqs, "keys": keys, "Hkv": Hkv, "d": d, "page": page, "count": count, "spare": spare}


def listed():
    return [
        # one new position of each request of a batch, far into its sequence
        _rope("rope_decode", 64, 1, 32, 8, 128, 128, scaling="bands", far=100000),
        # the gradient of the rotation of half of each head, as a training step of a few thousand positions meets it
        _rope("rope_grad_f32", 2, 4096, 16, 16, 128, 64, layout="interleaved", dtype="f32", transpose=True),
        # one new token of each request of a batch
        _write("write_decode", 64, 8, 128, 1, 4001, 64, "e4m3", ragged=True),
        # a chunk of each of a few prompts that are begun already
        _write("write_prompt", 4, 8, 128, 4096, 1000, 64, "int8"),
        # one request, one new position, a short cache: mostly latency
        _attend("attend_one_700", 1, 16, 16, 64, 1, 700, 16, "e4m3"),
        # one new position for each request of a batch, four query heads to a head of the cache, caches of different lengths
        _attend("attend_batch", 32, 32, 8, 128, 1, 4001, 64, "e4m3", mask=1, ragged=True),
        # one new position over a very long cache
        _attend("attend_64k", 1, 16, 16, 64, 1, 65536, 256, "int8", mask=1),
        # the next chunk of two long prompts
        _attend("attend_chunk", 2, 16, 4, 128, 2048, 16384, 64, "e4m3", mask=1, ragged=True),
        # pages listed by the program, moved between requests
        _pages("copy_200", "copy", 32, 4001, 8, 128, 64, 200, 256),
        # every request of a batch continued twice: full pages shared, the begun one copied
        _pages("fork_64", "fork", 64, 2001, 8, 128, 64, 64, 128),
        # half of the requests have ended: what is left moves to the front
        _pages("compact_half", "compact", 64, 2001, 8, 64, 64, 32),
        # requests that ended give their pages back, small pages, a large table
        _pages("free_16", "free", 256, 8001, 1, 32, 16, 16, 1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


MAX_BYTES, MAX_FLOPS = 2.0e8, 4.0e11   # of a drawn case


def draw(rng):
    while True:
        op = rng.choice(("rope", "rope", "write", "write", "attend", "attend", "attend", "attend", "copy", "fork", "compact", "free"))
        d, page, fmt = rng.choice((64, 64, 128, 128, 32, 96, 256)), rng.choice(PAGES), rng.choice(FORMATS)
        Hkv = rng.choice((1, 2, 4, 8, 8, 16))
        if op == "rope":
            N = _log_int(rng, 1, 16384)
            rot = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)))
            case = _rope("", _log_int(rng, 1, 128), N, Hkv * rng.choice((1, 2, 4, 5, 8)), Hkv, d, rot, rng.choice(("half", "interleaved")),
                         rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.3, rng.choice(("none", "linear", "base", "bands")),
                         rng.choice((0, 0, 5000, 1000000)))
        elif op == "write":
            N = rng.choice((1, 1, _log_int(rng, 2, 100), _log_int(rng, 100, 8192)))
            case = _write("", _log_int(rng, 1, 128), Hkv, d, N, _log_int(rng, 1, 20000) - 1, page, fmt, rng.random() < 0.5)
        elif op == "attend":
            keys = _log_int(rng, 1, 131072)
            Nq = min(keys, rng.choice((1, 1, 1, _log_int(rng, 2, 32), _log_int(rng, 32, 2048))))
            case = _attend("", _log_int(rng, 1, 128), Hkv * rng.choice((1, 1, 2, 4, 5, 8, 16)), Hkv, d, Nq, keys, page, fmt, rng.randrange(2),
                           rng.random() < 0.5)
        else:
            seqs = _log_int(rng, 2, 256)
            case = _pages("", op, seqs, _log_int(rng, 16, 20000), Hkv, d, page, max(1, int(seqs * rng.uniform(0.1, 0.9))), 32 + seqs)
            if op == "copy":
                case["count"] = _log_int(rng, 1, 300)
                case["spare"] = case["count"] + 32
        del case["name"]
        w = work(case)
        pool = 0
        if op not in ("rope",):
            held = sum(-(-n // page) for n in _held(case)) + case.get("spare", 8)
            pool = 2 * held * page * Hkv * d
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS and pool <= 1 << 30:
            if op == "attend" and case["B"] * case["H"] * case["Nq"] * case["keys"] * 4 > 4 << 30:
                continue
            return case


def _spread(n, count, ragged):
    """Lengths of `count` requests, the longest n; ragged ones lie anywhere between a tenth of it and all of it."""
    if not ragged:
        return [n] * count
    return [n if b == 0 else max(min(n, 1), int(n * (0.1 + 0.9 * ((0.37 + 0.6180339887 * b) % 1.0)))) for b in range(count)]


def _held(case):
    """Tokens of each request that its pages have room for."""
    if case["op"] == "write":
        return [n + case["N"] for n in _spread(case["start"], case["B"], case["ragged"])]
    if case["op"] == "attend":
        return _spread(case["keys"], case["B"], case["ragged"])
    return _spread(case["keys"], case["seqs"], True)


def _queries(case):
    """New positions of each request, at most its keys."""
    return [min(n, q) for n, q in zip(_held(case), _spread(case["Nq"], case["B"], case["ragged"] and case["Nq"] > 1))]


def _new_tokens(case):
    return _spread(case["N"], case["B"], case["ragged"] and case["N"] > 1)


def _visible(case):
    """Pairs of a query and a key it sees, over the batch."""
    total = 0
    for keys, q in zip(_held(case), _queries(case)):
        total += q * keys - (q * (q - 1) // 2 if case["mask"] else 0)
    return total


def work(case):
    op = case["op"]
    if op == "rope":
        size = case["B"] * case["N"] * (case["Hq"] + case["Hk"]) * case["d"]
        pairs = case["B"] * case["N"] * (case["Hq"] + case["Hk"]) * case["rot"] // 2
        return {"bytes": 2 * size * (2 if case["dtype"] == "bf16" else 4) + case["rot"] * 4 + case["B"] * case["N"] * 4, "flops": 6 * pairs}
    if op == "write":
        new = sum(_new_tokens(case)) * case["Hkv"] * case["d"] * 2
        blocks = sum(-(-(s + n) // BLOCK) - s // BLOCK for s, n in zip(_spread(case["start"], case["B"], case["ragged"]), _new_tokens(case)))
        return {"bytes": 3 * new + blocks * case["Hkv"] * 8, "flops": 2 * new}
    if op == "attend":
        keys = sum(_held(case)) * case["Hkv"]
        rows = sum(_queries(case)) * case["H"]
        return {"bytes": keys * case["d"] * 2 + keys // BLOCK * 8 + rows * case["d"] * 4, "flops": 4 * _visible(case) * case["H"] * case["d"]}
    page_bytes = 2 * case["Hkv"] * case["page"] * case["d"] + 2 * case["Hkv"] * case["page"] // BLOCK * 4
    held = [-(-n // case["page"]) for n in _held(case)]
    table = 4 * case["seqs"] * max(held)
    if op == "copy":
        return {"bytes": 2 * case["count"] * page_bytes + 8 * case["count"], "flops": 0}
    if op == "fork":
        forks = _forks(case)
        begun = sum(1 for p, _ in forks if _held(case)[p] % case["page"])
        return {"bytes": 2 * begun * page_bytes + 2 * 4 * len(forks) * max(held), "flops": 0}
    if op == "compact":
        return {"bytes": 2 * _moved(case) * page_bytes + 2 * table, "flops": 0}
    return {"bytes": table + 4 * (sum(held) + case["spare"]) + 8 * case["count"], "flops": 0}


def _forks(case):
    """(parent, child): the first `count` rows are parents, and as many empty rows follow the others."""
    return [(i, case["seqs"] + i) for i in range(case["count"])]


def _moved(case):
    """Pages that a compaction moves, for a pool of scattered pages: about this many lie behind the number of held ones."""
    held = [-(-n // case["page"]) for n in _held(case)]
    kept, everything = sum(held[case["count"]:]), sum(held) + case["spare"]
    return int(kept * (1 - kept / everything))


# ---- inputs -----------------------------------------------------------------------------------------------------------------------------

def _gen(seed, *what):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + sum((i + 1) * 7919 * w for i, w in enumerate(what))) % (1 << 62))
    return g


def _normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _frequencies(case):
    """Radians per position of each pair, in 64 bits: base 10000, and the scalings a model extended to 8 times its length is given."""
    n = case["rot"] // 2
    i = torch.arange(n, dtype=torch.float64)
    base, factor, original = 10000.0, 8.0, 4096.0
    kind = case["scaling"]
    if kind == "base" and case["rot"] > 2:
        base *= factor ** (case["rot"] / (case["rot"] - 2))
    f = base ** (-2.0 * i / case["rot"])
    if kind == "linear":
        f = f / factor
    elif kind == "bands":
        turns = original * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f


def _table(rows, page, n_pages, width, seed, empty=0):
    """A page table of scattered pages: rows with the pages that their tokens need, -1 behind them."""
    rng = np.random.RandomState((seed * 7 + 3) % (1 << 31))
    need = [-(-n // page) for n in rows]
    ids = rng.permutation(n_pages)[: sum(need)]
    table = np.full((len(rows) + empty, width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at : at + n]
        at += n
    return torch.from_numpy(table).cuda()


def _pool(n_pages, Hkv, page, d, fmt, g):
    """Codes and scales of a cache in use: normal values with a few strong channels, and blocks of different size."""
    def half(transposed):
        shape = (n_pages, Hkv, page // BLOCK, d // 16, 16, 16) if not transposed else (n_pages, Hkv, page // BLOCK, d, BLOCK)
        amplitude = torch.exp2(torch.randint(-4, 2, shape[:3], generator=g, device="cuda").float())
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
        strong = torch.where(torch.rand(d, generator=g, device="cuda") < 0.05, 4.0, 1.0).to(torch.bfloat16)
        x = x * (strong.view(d // 16, 1, 16) if not transposed else strong.view(d, 1))
        scale = torch.exp2(torch.ceil(torch.log2(x.abs().flatten(3).amax(-1).float() / (448.0 if fmt == "e4m3" else 127.0))))
        x = x / scale.view(*shape[:3], *([1] * (len(shape) - 3))).to(torch.bfloat16)
        codes = (x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.float().round().clamp(-127, 127).to(torch.int8)).view(torch.uint8)
        return codes.view(n_pages, Hkv, page, d), scale * amplitude
    k, ks = half(False)
    v, vs = half(True)
    return k, v, ks, vs


def _stale(state, rows):
    """Bytes behind each request's last token, as an earlier owner of the page may have left them."""
    page, d = state["page"], state["d"]
    lens = torch.tensor(rows, device="cuda")
    last = ((lens - 1).clamp(min=0) // BLOCK)
    ids = state["table"][torch.arange(len(rows), device="cuda"), last // (page // BLOCK)].long()
    inside = torch.arange(BLOCK, device="cuda")[None] + last[:, None] * BLOCK >= lens[:, None]
    blk = last % (page // BLOCK)
    for name, view in (("k", (d // 16, BLOCK, 16)), ("v", (d, BLOCK))):
        pool = state[name].view(*state[name].shape[:2], page // BLOCK, *view)
        now = pool[ids, :, blk]
        m = inside.view(-1, 1, 1, BLOCK, 1) if name == "k" else inside.view(-1, 1, 1, BLOCK)
        pool[ids, :, blk] = torch.where(m, torch.full_like(now, 0x7F), now)


def prepare(case, seed):
    op, g = case["op"], _gen(seed, 1)
    s = {"case": case, "op": op}
    if op == "rope":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["q"], s["k"] = (_normal((case["B"], h, case["N"], case["d"]), g, dtype) for h in (case["Hq"], case["Hk"]))
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["freqs"] = _frequencies(case).cuda()
        first = torch.randint(0, case["far"] + 1, (case["B"], 1), generator=g, device="cuda")
        s["positions"] = (first + torch.arange(case["N"], device="cuda")).to(torch.int32)
        s["magnitude"] = 1.0 if case["scaling"] != "bands" else 0.1 * math.log(8.0) + 1.0
        return s
    Hkv, d, page = case["Hkv"], case["d"], case["page"]
    rows = _held(case)
    fmt = case.get("fmt", "e4m3")
    n_pages = sum(-(-n // page) for n in rows) + case.get("spare", 8)
    width = max(-(-n // page) for n in rows) + (2 if op != "free" else 0)
    s["fmt"], s["page"], s["d"] = fmt, page, d
    s["table"] = _table(rows, page, n_pages, width, seed, case["count"] if op == "fork" else 0)
    s["k"], s["v"], s["k_scale"], s["v_scale"] = _pool(n_pages, Hkv, page, d, fmt, g)
    if op == "write":
        s["new_k"], s["new_v"] = (_normal((case["B"], Hkv, case["N"], d), g, torch.bfloat16) for _ in range(2))
        s["lens"] = torch.tensor(_spread(case["start"], case["B"], case["ragged"]), dtype=torch.int32, device="cuda")
        s["n_new"] = torch.tensor(_new_tokens(case), dtype=torch.int32, device="cuda")
    elif op == "attend":
        _stale(s, rows)
        s["q"] = _normal((case["B"], case["H"], case["Nq"], d), g, torch.bfloat16)
        s["out"] = torch.zeros_like(s["q"])
        s["lens"] = torch.tensor(rows, dtype=torch.int32, device="cuda")
        s["q_lens"] = torch.tensor(_queries(case), dtype=torch.int32, device="cuda")
        s["scale"] = d ** -0.5
    else:
        s["lens"] = torch.tensor(rows + [0] * (case["count"] if op == "fork" else 0), dtype=torch.int32, device="cuda")
        free = np.setdiff1d(np.arange(n_pages), s["table"].cpu().numpy().ravel())
        rng = np.random.RandomState((seed * 11 + 5) % (1 << 31))
        if op == "copy":
            s["src"] = torch.from_numpy(rng.choice(np.setdiff1d(np.arange(n_pages), free), case["count"]).astype(np.int32)).cuda()
            s["dst"] = torch.from_numpy(rng.permutation(free)[: case["count"]].astype(np.int32)).cuda()
        elif op == "fork":
            forks = _forks(case)
            s["parents"], s["children"] = (torch.tensor([f[i] for f in forks], dtype=torch.int32, device="cuda") for i in (0, 1))
            s["spares"] = torch.from_numpy(rng.permutation(free)[: len(forks)].astype(np.int32)).cuda()
        elif op == "compact":
            s["table"][: case["count"]] = -1
            s["new_table"] = torch.empty_like(s["table"])
            s["n_used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        else:
            s["seqs"] = torch.from_numpy(rng.permutation(case["seqs"])[: case["count"]].astype(np.int32)).cuda()
            s["unused"] = torch.empty(n_pages, dtype=torch.int32, device="cuda")
            s["n_unused"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2107_06419_amd as fa
        s["cache"] = fa.FlatCache8(s["k"], s["v"], s["k_scale"], s["v_scale"], fa.FLAT_CACHE8_E4M3 if fmt == "e4m3" else fa.FLAT_CACHE8_INT8)
        if op == "attend":
            nbytes = fa.flat_attn_fwd_cache8_workspace_bytes(case["B"], case["H"], Hkv, case["Nq"], width * page, d)
            s["workspace"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        elif op == "compact":
            s["workspace"] = torch.empty(fa.flat_attn_cache8_compact_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _cache_out(s):
    """The cache as it is: e4m3 and int8 codes as the numbers they stand for, and the scales."""
    t = CODE_TYPE[s["fmt"]]
    return {"k": s["k"].view(t), "v": s["v"].view(t), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _run_own(s):
    import paper_2107_06419_amd as fa
    op = s["op"]
    if op == "rope":
        fa.flat_attn_rope(s["q"], s["q_out"], s["k"], s["k_out"], s["freqs"], s["positions"],
                          layout=fa.FLAT_ROPE_HALF if s["case"]["layout"] == "half" else fa.FLAT_ROPE_INTERLEAVED, magnitude=s["magnitude"],
                          transpose=s["case"]["transpose"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "write":
        fa.flat_attn_cache8_write(s["cache"], s["new_k"], s["new_v"], s["table"], s["lens"], s["n_new"])
        return _cache_out(s)
    if op == "attend":
        fa.flat_attn_fwd_cache8(s["cache"], s["q"], s["out"], s["table"], s["lens"], s["scale"], s["case"]["mask"], s["q_lens"], s["workspace"])
        return s["out"]
    if op == "copy":
        fa.flat_attn_cache8_copy_pages(s["cache"], s["src"], s["dst"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "fork":
        fa.flat_attn_cache8_fork(s["cache"], s["table"], s["lens"], s["parents"], s["children"], s["spares"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "table": s["table"], "lens": s["lens"]}
    if op == "compact":
        fa.flat_attn_cache8_compact(s["cache"], s["table"], s["new_table"], s["n_used"], s["workspace"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "table": s["new_table"], "n_used": s["n_used"]}
    fa.flat_attn_cache8_free(s["table"], s["lens"], s["seqs"], s["unused"], s["n_unused"])
    return {"table": s["table"], "lens": s["lens"], "unused": s["unused"], "n_unused": s["n_unused"]}


def _run_plain(s):
    return {"rope": _plain_rope, "write": _plain_write, "attend": _plain_attend, "copy": _plain_copy, "fork": _plain_fork,
            "compact": _plain_compact, "free": _plain_free}[s["op"]](s)


def _pairs(x, rot, layout):
    """The two members of every pair, [..., rot / 2] each."""
    if layout == "half":
        return x[..., : rot // 2], x[..., rot // 2 : rot]
    return x[..., 0:rot:2], x[..., 1:rot:2]


def _plain_rope(s):
    case = s["case"]
    angle = s["positions"].double()[:, None, :, None] * s["freqs"]   # 64 bits: far positions
    c, n = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    n = -n if case["transpose"] else n

    def turned(x):
        f = x.float()
        a, b = _pairs(f, case["rot"], case["layout"])
        out = f.clone()
        ya, yb = _pairs(out, case["rot"], case["layout"])
        ya.copy_(a * c - b * n)
        yb.copy_(a * n + b * c)
        return out.to(x.dtype)
    return {"q": turned(s["q"]), "k": turned(s["k"])}


def _values(codes, fmt):
    return codes.view(CODE_TYPE[fmt]).float()


def _blocks_k(s):
    p, h, t, d = s["k"].shape
    return s["k"].view(p, h, t // BLOCK, d // 16, BLOCK, 16)


def _blocks_v(s):
    p, h, t, d = s["v"].shape
    return s["v"].view(p, h, t // BLOCK, d, BLOCK)


def _plain_write(s):
    case, fmt, page = s["case"], s["fmt"], s["page"]
    B, N, per = case["B"], case["N"], page // BLOCK
    lens, n_new = s["lens"].long(), s["n_new"].long()
    j = lens[:, None] // BLOCK + torch.arange(N // BLOCK + 2, device="cuda")                      # [B, blocks]
    pos = j[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")                               # [B, blocks, 16]
    src = pos - lens[:, None, None]
    new, old = (src >= 0) & (src < n_new[:, None, None]), src < 0
    at = (j // per).clamp(max=s["table"].shape[1] - 1)
    ids = torch.gather(s["table"].long(), 1, at)
    b, i = torch.nonzero(new.any(-1) & (j // per < s["table"].shape[1]) & (ids >= 0) & (ids < s["k"].shape[0]), as_tuple=True)
    ids, blk, new, old, src = ids[b, i], j[b, i] % per, new[b, i], old[b, i], src[b, i].clamp(0, N - 1)
    fraction, exponent = LARGEST[fmt]
    for name, pool, scales, x in (("k", _blocks_k(s), s["k_scale"], s["new_k"]), ("v", _blocks_v(s), s["v_scale"], s["new_v"])):
        x = x[b[:, None], :, src].permute(0, 2, 1, 3).float()                                      # [n, heads, 16, d]
        codes = pool[ids, :, blk]
        was = _values(codes, fmt)
        was = was.permute(0, 1, 3, 2, 4).flatten(3) if name == "k" else was.transpose(2, 3)
        keep, take = old[:, None, :, None], new[:, None, :, None]
        before = torch.where(old.any(-1)[:, None], scales[ids, :, blk], 0.0)
        x = torch.where(take, x, 0.0)
        f, e = torch.frexp(x.abs().amax((2, 3)))
        need = torch.exp2((e - exponent + (f > fraction)).clamp(min=LEAST_EXPONENT).float())
        scale = torch.maximum(torch.where(f > 0, need, 0.0), before)
        scale = torch.where(torch.isfinite(x).all(-1).all(-1), scale, float("nan"))
        by = torch.where(scale > 0, 1.0 / scale, 0.0)[..., None, None]
        q = torch.where(keep, was * before[..., None, None] * by, torch.where(take, x * by, 0.0))
        q = torch.where(by > 0, q, 0.0)
        q = (q.to(torch.float8_e4m3fn) if fmt == "e4m3" else q.round().to(torch.int8)).view(torch.uint8)
        pool[ids, :, blk] = q.unflatten(3, (-1, 16)).transpose(2, 3).contiguous() if name == "k" else q.transpose(2, 3).contiguous()
        scales[ids, :, blk] = scale
    return _cache_out(s)


def _plain_attend(s):
    case, fmt = s["case"], s["fmt"]
    B, H, Hkv, Nq, d = case["B"], case["H"], case["Hkv"], case["Nq"], case["d"]
    width = -(-case["keys"] // s["page"])
    ids = s["table"][:, :width].long()
    there = (ids >= 0) & (ids < s["k"].shape[0])
    ids = ids.clamp(0, s["k"].shape[0] - 1)
    L = width * s["page"]
    k = _values(_blocks_k(s)[ids], fmt) * s["k_scale"][ids][..., None, None, None]                 # [B, pages, heads, blocks, d/16, 16, 16]
    k = k.permute(0, 2, 1, 3, 5, 4, 6).reshape(B, Hkv, L, d)
    v = _values(_blocks_v(s)[ids], fmt) * s["v_scale"][ids][..., None, None]                       # [B, pages, heads, blocks, d, 16]
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, Hkv, L, d)
    j = torch.arange(L, device="cuda")
    seen = (j < s["lens"][:, None]) & there.repeat_interleave(s["page"], 1)                        # [B, L]
    k, v = (torch.where(seen[:, None, :, None], x, 0.0) for x in (k, v))
    i = torch.arange(Nq, device="cuda")
    mask = seen[:, None, :].expand(B, Nq, L)
    if case["mask"]:
        mask = mask & (j <= i[:, None] + (s["lens"] - s["q_lens"])[:, None, None])
    q = s["q"].float().reshape(B, Hkv, H // Hkv * Nq, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, H // Hkv, Nq, L) * s["scale"]
    x = torch.where(mask[:, None, None], x, float("-inf"))
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.view(B, Hkv, -1, L), v).view(B, Hkv, H // Hkv, Nq, d) / torch.where(total > 0, total, 1.0)
    out = out.reshape(B, H, Nq, d).to(torch.bfloat16)
    return torch.where((i < s["q_lens"][:, None])[:, None, :, None], out, s["out"])


def _whole_cache(s):
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_move(s, src, dst):
    s["k"][dst], s["v"][dst], s["k_scale"][dst], s["v_scale"][dst] = s["k"][src], s["v"][src], s["k_scale"][src], s["v_scale"][src]


def _plain_copy(s):
    _plain_move(s, s["src"].long(), s["dst"].long())
    return _whole_cache(s)


def _plain_fork(s):
    parents, children, spares, table, lens = s["parents"].long(), s["children"].long(), s["spares"], s["table"], s["lens"]
    n = lens[parents]
    full, begun = n // s["page"], n % s["page"] > 0
    j = torch.arange(table.shape[1], device="cuda")
    rows = torch.where(j < full[:, None], table[parents], -1)
    rows = torch.where((j == full[:, None]) & begun[:, None], spares[:, None], rows)
    last = table[parents, full.long().clamp(max=table.shape[1] - 1)]
    _plain_move(s, last[begun].long(), spares[begun].long())
    table[children] = rows
    lens[children] = n
    return {**_whole_cache(s), "table": table, "lens": lens}


def _plain_compact(s):
    table, n_pages = s["table"].long(), s["k"].shape[0]
    there = (table >= 0) & (table < n_pages)
    held = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    held[torch.where(there, table, n_pages)] = True
    held, ids = held[:n_pages], torch.arange(n_pages, device="cuda")
    used = held.sum()
    src, dst = torch.nonzero(held & (ids >= used)).flatten(), torch.nonzero(~held & (ids < used)).flatten()
    _plain_move(s, src, dst)
    ids[src] = dst
    new = torch.where(there, ids[table.clamp(0, n_pages - 1)], table).to(torch.int32)
    return {**_whole_cache(s), "table": new, "n_used": used.to(torch.int32).view(1)}


def _plain_free(s):
    table, n_pages, seqs = s["table"], s["unused"].shape[0], s["seqs"].long()
    table[seqs] = -1
    s["lens"][seqs] = 0
    held = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    held[torch.where((table >= 0) & (table < n_pages), table, n_pages).long()] = True
    ids = torch.arange(n_pages, device="cuda")
    order = torch.where(held[:n_pages], n_pages, ids).sort().values
    unused = torch.where(order < n_pages, order, -1).to(torch.int32)
    return {"table": table, "lens": s["lens"], "unused": unused, "n_unused": (~held[:n_pages]).sum().to(torch.int32).view(1)}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "rope":
        return _exact_rope(s)
    if case["op"] == "write":
        return _exact_write(s)
    if case["op"] == "attend":
        return _exact_attend(s)
    return None   # pages hold whole numbers, and scales that are copied


def _exact_rope(s):
    """Each pair as a complex number, times magnitude * e^(i angle)."""
    case = s["case"]
    half = case["rot"] // 2
    pos, f = s["positions"].double(), s["freqs"]
    angle = torch.remainder(pos.unsqueeze(-1) * f, 2 * math.pi) * (-1.0 if case["transpose"] else 1.0)
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle).unsqueeze(1)
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        first = x[..., : case["rot"]]
        z = first.unflatten(-1, (2, half)).transpose(-1, -2) if case["layout"] == "half" else first.unflatten(-1, (half, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        y = z.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else z.flatten(-2)
        out[name] = torch.cat([y, x[..., case["rot"] :]], -1)
    return out


def _grid(x, fmt):
    """x (64 bits) to the nearest code value, ties to the even one."""
    if fmt == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_write(s):
    """Request by request: the values its touched blocks hold are put together, scaled and rounded; everything else stays."""
    case, fmt, page = s["case"], s["fmt"], s["page"]
    largest = 448.0 if fmt == "e4m3" else 127.0
    t, per, d = CODE_TYPE[fmt], page // BLOCK, s["d"]
    out = {}
    for name in ("k", "v"):
        pool = s[name].view(t).double().view(*s[name].shape[:2], per, -1)
        pool = pool.unflatten(3, (d // 16, BLOCK, 16)).permute(0, 1, 2, 4, 3, 5).flatten(4) if name == "k" else pool.unflatten(3, (d, BLOCK)).transpose(3, 4)
        pool, scales = pool.contiguous(), s[name + "_scale"].double().clone()
        lens, news, table = s["lens"].tolist(), s["n_new"].tolist(), s["table"].cpu().numpy()
        for b in range(case["B"]):
            lo, hi = lens[b], lens[b] + news[b]
            if hi == lo:
                continue
            first, end = lo // BLOCK, -(-hi // BLOCK)
            ids = torch.from_numpy(table[b, np.arange(first, end) // per].astype(np.int64)).cuda()
            blk = torch.arange(first, end, device="cuda") % per
            kept, fresh = lo - first * BLOCK, s["new_" + name][b, :, : news[b]].double()
            held = torch.zeros(end - first, fresh.shape[0], BLOCK, d, dtype=torch.float64, device="cuda")
            flat = held.transpose(0, 1).reshape(fresh.shape[0], -1, d)
            flat[:, kept : kept + news[b]] = fresh
            held = flat.view(fresh.shape[0], end - first, BLOCK, d).transpose(0, 1).contiguous()
            most = held.abs().amax((2, 3)) / largest
            scale = torch.where(most > 0, torch.exp2(torch.ceil(torch.log2(most.clamp(min=1e-300)))), 0.0)
            if kept:
                before = scales[ids[0], :, blk[0]]
                held[0, :, :kept] = pool[ids[0], :, blk[0], :kept] * before[:, None, None]
                scale[0] = torch.maximum(scale[0], before)
            pool[ids, :, blk] = _grid(torch.where(scale > 0, 1 / scale, 0.0)[..., None, None] * held, fmt)
            scales[ids, :, blk] = scale
        codes = pool.unflatten(4, (d // 16, 16)).transpose(3, 4) if name == "k" else pool.transpose(3, 4)
        out[name], out[name + "_scale"] = codes.reshape(s[name].shape), scales
    return {k: out[k] for k in ("k", "v", "k_scale", "v_scale")}


def _exact_attend(s):
    """Request by request and head by head, over the keys that the request has."""
    case, page, d = s["case"], s["page"], s["d"]
    t, G, per = CODE_TYPE[s["fmt"]], case["H"] // case["Hkv"], page // BLOCK
    if 4.0 * _visible(case) * case["H"] * d > 2e12:
        return None
    out = s["out"].double()
    lens, q_lens, table = s["lens"].tolist(), s["q_lens"].tolist(), s["table"].long()
    for b in range(case["B"]):
        n, rows = lens[b], q_lens[b]
        ids = table[b, : -(-n // page)]
        hidden = torch.zeros(rows, n, dtype=torch.bool, device="cuda")
        if case["mask"]:
            hidden = torch.ones_like(hidden).triu(n - rows + 1)
        for h in range(case["Hkv"]):
            k = s["k"][ids, h].view(t).double().view(-1, per, d // 16, BLOCK, 16).transpose(2, 3).reshape(-1, BLOCK, d)
            v = s["v"][ids, h].view(t).double().view(-1, d, BLOCK).transpose(1, 2)
            k, v = ((x * sc[ids, h].double().view(-1, 1, 1)).reshape(-1, d)[:n].contiguous() for x, sc in ((k, s["k_scale"]), (v, s["v_scale"])))
            x = torch.matmul(s["q"][b, h * G : (h + 1) * G, :rows].double(), k.t().contiguous()) * s["scale"]
            p = torch.softmax(x.masked_fill(hidden, float("-inf")), -1)
            out[b, h * G : (h + 1) * G, :rows] = torch.matmul(p, v)
    return out
