"""The serving operators on bf16 pages, as cases that a measuring program runs.

Four operators, each in plain torch (``own`` false) and through the library's entry points (``own`` true):

  append     new K and V rows into a paged bf16 cache, rotated to their positions on the way; Q rotated in the same pass
             (kvp_append)
  attention  new rows against that cache: one token a sequence, a few, a chunk of a prompt or a whole one (kvp_attention)
  window     the same where a row sees the last ``window`` positions and the first ``sinks`` only (kvp_set_layer_window)
  copy       pages copied to others in the pools of every producer, of the bf16 or of the 8-bit cache (kvp_copy_pages,
             kvp_copy_pages_fp8)

Fields of a case: ``op``; query heads ``a``, K/V heads ``g``; append, attention and window: sequences ``B``, shortest and
longest cached context ``lo``, ``hi``, fewest and most new tokens of a sequence ``new_lo``, ``new_hi``, and ``window`` (0:
none) with ``sinks``; copy: pages copied ``n``, ``producers``, and whether the pools are 8-bit ones, ``fp8``.

The bf16 cache: pages of 64 positions, K [g][page][64][128], V [g][page][128][64] (the positions of one dimension side by
side).  The 8-bit one: K codes [g][page][64][128], V codes [g][page][4][128][16], fp32 scales [g][page][2][4].
"""
import math

import torch

own = False

D, PAGE = 128, 64
BASE = 10000.0


def _case(name, op, a=32, g=8, B=0, lo=0, hi=0, new_lo=1, new_hi=1, window=0, sinks=0, n=0, producers=0, fp8=False):
    return dict(name=name, op=op, a=a, g=g, B=B, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, window=window, sinks=sinks,
                n=n, producers=producers, fp8=fp8)


def listed():
    return [
        # A few users' next tokens: the launch and some rows.
        _case("append-8", "append", 32, 8, 8, 301, 9001),
        # Chunks of prompts of odd lengths behind cached prefixes.
        _case("append-chunks", "append", 64, 8, 7, 5, 2000, 33, 700),
        # One user's chat turn.
        _case("attn-1", "attention", 32, 8, 1, 977, 977),
        # A serving batch of long contexts, one of its layers.
        _case("attn-64-16k", "attention", 32, 8, 64, 16384, 16384),
        # A few proposed tokens a sequence to be checked at once.
        _case("attn-verify", "attention", 32, 8, 16, 1500, 8000, 4, 4),
        # Prompts behind cached prefixes, odd lengths throughout.
        _case("attn-chunks", "attention", 32, 8, 3, 700, 5000, 333, 1001),
        # The prompts of the benchmark's pipeline-stage share.
        _case("attn-prompt", "attention", 16, 8, 4, 0, 0, 4096, 4096),
        # One token of a windowed layer far into a conversation.
        _case("window-1", "window", 32, 8, 1, 9001, 9001, window=1000, sinks=4),
        # A batch of such tokens; contexts of mixed lengths, of which the window and the first tokens are held.
        _case("window-64", "window", 32, 8, 64, 3000, 40000, window=4096, sinks=4),
        # Chunks of long prompts through a windowed layer.
        _case("window-chunks", "window", 32, 8, 3, 2500, 12000, 700, 2049, window=2048, sinks=4),
        # Sequences that were forked write on: each gets its own copy of the page that it shared (8-bit pools).
        _case("copy-fork", "copy", 32, 8, n=5, producers=4, fp8=True),
        # A pool with holes is compacted.
        _case("copy-compact", "copy", 32, 8, n=1501, producers=4),
    ]


HEADS = [(8, 4), (16, 8), (16, 16), (32, 8), (32, 8), (40, 8), (64, 8), (16, 1), (12, 4), (5, 1)]


def _loguniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges, costing no more than the largest of them."""
    limit = max(_cost(c) for c in listed()) * 0.9
    while True:
        c = _draw(rng)
        if _cost(c) <= limit and _room(c) <= 3e9 and c["B"] * c["g"] * (c["hi"] + c["new_hi"]) <= 3e7:
            return c


def _draw(rng):
    op = rng.choice(["append", "append", "attention", "attention", "attention", "window", "window", "window", "copy"])
    a, g = rng.choice(HEADS)
    c = _case("", op, a, g)
    del c["name"]
    if op == "copy":
        c["n"], c["producers"], c["fp8"] = _loguniform(rng, 1, 1500), _loguniform(rng, 1, 8), rng.random() < 0.5
        return c
    c["hi"] = _loguniform(rng, 1, 60000) if rng.random() < 0.85 else 0
    c["lo"] = int(c["hi"] * rng.choice([0.0, 0.1, 0.5, 1.0]))
    kind = rng.choice(["one", "one", "few", "chunk", "chunk"])
    if kind == "one":
        c["B"] = _loguniform(rng, 1, 100)
    elif kind == "few":
        c["B"], c["new_hi"] = _loguniform(rng, 1, 40), rng.randint(2, 12)
        c["new_lo"] = rng.randint(1, c["new_hi"])
    else:
        c["B"], c["new_hi"] = _loguniform(rng, 1, 6), _loguniform(rng, 13, 4000)
        c["new_lo"] = max(1, int(c["new_hi"] * rng.choice([0.05, 0.5, 1.0])))
    if op == "window":
        c["window"], c["sinks"] = _loguniform(rng, 1, 8192), rng.choice([0, 0, 1, 4, 4, 64, 100])
    return c


def _cost(c):
    """Rough microseconds of a pass."""
    w = work(c)
    return 10.0 + w["flops"] / 6e8 + w["bytes"] / 5e6


def _room(c):
    """Scores of the plain form's attention."""
    return 0 if c["op"] not in ("attention", "window") else c["B"] * c["a"] * c["new_hi"] * (c["hi"] + c["new_hi"])


def _lens(c, seed=0):
    """Cached and new tokens of every sequence: evenly over their ranges, the longest contexts with the fewest new ones, in an
    order that the seed gives."""
    i = torch.randperm(c["B"], generator=torch.Generator().manual_seed(seed)).tolist()
    last = max(1, c["B"] - 1)
    return [c["lo"] + (c["hi"] - c["lo"]) * x // last for x in i], [c["new_hi"] - (c["new_hi"] - c["new_lo"]) * x // last for x in i]


def work(case):
    """Each input read once, each output written once: of the cache the positions that some row sees.  FLOPs: the products,
    pairs a row may see only; append: the rotation."""
    c = case
    nq, nkv = c["a"] * D, c["g"] * D
    if c["op"] == "copy":
        page = c["g"] * (2 * PAGE * D + 32) if c["fp8"] else c["g"] * 4 * PAGE * D
        return {"bytes": 2 * c["n"] * page * c["producers"], "flops": 0}
    lens, new = _lens(c)
    rows = sum(new)
    if c["op"] == "append":
        return {"bytes": rows * (4 * nq + 8 * nkv), "flops": 3 * rows * (nq + nkv)}
    W, S = c["window"] or 1 << 40, c["sinks"]
    held = pairs = 0
    for n, t in zip(lens, new):
        first = max(0, n - W + 1)                   # behind it the first tokens only
        held += n + t - first + min(first, S)
        pairs += sum(min(p + 1, W) + min(S, max(0, p + 1 - W)) for p in range(n, n + t))
    return {"bytes": 4 * rows * nq + 4 * held * nkv, "flops": 4 * c["a"] * D * pairs}


# ---- inputs ------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=dev).normal_(0.0, 1.0, generator=gen)

    return _prepare_copy(c, dev, gen, normal) if c["op"] == "copy" else _prepare_rows(c, int(seed), dev, gen, normal)


def _prepare_copy(c, dev, gen, normal):
    g, n = c["g"], c["n"]
    n_pages = 2 * n + 3
    s = {"case": c, "pools": []}
    for _ in range(c["producers"]):
        if c["fp8"]:
            codes = [torch.randint(0, 255, (g, n_pages, PAGE * D), dtype=torch.uint8, device=dev, generator=gen) for _ in range(2)]
            for t in codes:
                t[(t & 127) == 127] = 0             # no NaN codes
            scales = torch.exp2(torch.randint(-12, -4, (g, n_pages, 2, 4), device=dev, generator=gen).float())
            s["pools"].append((codes[0].view(g, n_pages, PAGE, D), codes[1].view(g, n_pages, 4, D, 16), scales))
        else:
            s["pools"].append((normal(g, n_pages, PAGE, D), normal(g, n_pages, D, PAGE)))
    order = torch.randperm(n_pages, generator=gen, device=dev).int()
    s["src"], s["dst"] = order[:n].contiguous(), order[n: 2 * n].contiguous()
    if own:
        from paper_2608_15943_amd import binding as kb
        P = c["producers"]
        m = kb.Model(P, c["a"] * D, c["a"], g, D, kb.KVP_DTYPE_BF16, list(range(P)), max_batch=1, max_seq=1, kv_capacity=PAGE)
        for l, pool in enumerate(s["pools"]):
            (m.kvp_set_kv_pool_fp8 if c["fp8"] else m.kvp_set_kv_pool)(l, *(t.data_ptr() for t in pool), n_pages)
        s["m"] = m
    return s


def _prepare_rows(c, seed, dev, gen, normal):
    a, g, B = c["a"], c["g"], c["B"]
    s = {"case": c}
    lens, new = _lens(c, seed)
    need = torch.tensor([(n + t + PAGE - 1) // PAGE for n, t in zip(lens, new)], device=dev)
    stride, rows = int(need.max()), sum(new)
    s["len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["cu"] = torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device=dev)
    # A page for each 64 positions of a sequence; those that lie wholly behind every row's window are not held any more.
    j = torch.arange(stride, device=dev)
    held = j < need[:, None]
    if c["window"]:
        held &= (PAGE * j + PAGE - 1 > s["len"][:, None] - c["window"]) | (PAGE * j < c["sinks"])
    n_pages = int(held.sum()) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev).int()
    pages = torch.full((B, stride), -1, dtype=torch.int32, device=dev)
    pages[held] = order[: n_pages - 3]
    s["pages"], s["n_pages"], s["stride"], s["rows"] = pages, n_pages, stride, rows
    s["max_new"], s["max_pos"] = max(new), max(n + t - 1 for n, t in zip(lens, new))
    # Keys have dimensions that are larger than others in every token; values do not.
    s["kc"], s["vc"] = normal(g, n_pages, PAGE, D), normal(g, n_pages, D, PAGE)
    s["kc"] *= torch.exp(0.5 * normal(g, 1, 1, D, dtype=torch.float32)).bfloat16()
    s["qkv"] = normal(rows, (a + 2 * g) * D)        # what a fused projection leaves: rows of Q | K | V
    s["q"] = torch.zeros(rows, a * D, dtype=torch.bfloat16, device=dev)
    if c["op"] != "append":
        s["q"].copy_(s["qkv"][:, : a * D])
        s["out"] = torch.zeros_like(s["q"])
        del s["qkv"]
    if own:
        from paper_2608_15943_amd import binding as kb
        m = kb.Model(1, a * D, a, g, D, kb.KVP_DTYPE_BF16, [0], max_batch=B, max_seq=s["max_new"],
                     kv_capacity=(s["max_new"] + PAGE - 1) // PAGE * PAGE, rope_base=BASE)
        m.kvp_set_kv_pool(0, s["kc"].data_ptr(), s["vc"].data_ptr(), n_pages)
        if c["window"]:
            m.kvp_set_layer_window(0, c["window"], c["sinks"])
        s["m"] = m
        s["r"] = kb.kvp_rows(0 if c["new_hi"] == 1 else s["cu"].data_ptr(), s["len"].data_ptr(), pages.data_ptr(), stride, B,
                             rows, s["max_new"], s["max_pos"])
        if c["op"] != "append":
            s["n"] = m.kvp_workspace_size(kb.KVP_PHASE_STEP, B, rows)
            s["ws"] = torch.empty(s["n"], dtype=torch.uint8, device=dev)
    return s


# ---- a pass ------------------------------------------------------------------------------------

def run(state):
    s = state
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"append": _append, "attention": _attention, "window": _attention, "copy": _copy}[c["op"]](s, c)


def _run_own(s, c):
    st = torch.cuda.current_stream().cuda_stream
    m = s["m"]
    if c["op"] == "copy":
        (m.kvp_copy_pages_fp8 if c["fp8"] else m.kvp_copy_pages)(s["src"].data_ptr(), s["dst"].data_ptr(), c["n"], st)
        return _pools(s, c)
    if c["op"] == "append":
        q, ld = s["qkv"].data_ptr(), s["qkv"].shape[1]
        k = q + 2 * c["a"] * D
        m.kvp_append(0, q, k, k + 2 * c["g"] * D, ld, s["r"], s["q"].data_ptr(), st)
        return {"q": s["q"], "k": s["kc"], "v": s["vc"]}
    m.kvp_attention(0, s["q"].data_ptr(), s["r"], s["out"].data_ptr(), s["ws"].data_ptr(), s["n"], st)
    return {"out": s["out"]}


def _pools(s, c):
    """Every producer's pools, 8-bit codes as the numbers that they stand for."""
    if c["fp8"]:
        return [(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), sc) for k, v, sc in s["pools"]]
    return s["pools"]


def _copy(s, c):
    src, dst = s["src"].long(), s["dst"].long()
    for pool in s["pools"]:
        for t in pool:
            t[:, dst] = t[:, src]
    return _pools(s, c)


def _rows(s):
    """Sequence and position of every new row."""
    i = torch.arange(s["rows"], device=s["cu"].device)
    b = torch.searchsorted(s["cu"][1:].contiguous(), i.int(), right=True)
    return b, s["len"].long()[b] + i - s["cu"].long()[b]


def _append(s, c):
    a, g, rows = c["a"], c["g"], s["rows"]
    b, pos = _rows(s)
    x = s["qkv"].float().view(rows, a + 2 * g, D)
    # Angles in 64 bits: far positions.
    th = torch.pow(torch.tensor(BASE, dtype=torch.float64, device=x.device),
                   -torch.arange(D // 2, dtype=torch.float64, device=x.device) / (D // 2))
    ang = pos.double()[:, None] * th
    co, si = ang.cos().float()[:, None], ang.sin().float()[:, None]
    x1, x2 = x[:, : a + g, : D // 2], x[:, : a + g, D // 2:]
    y = torch.cat([x1 * co - x2 * si, x2 * co + x1 * si], -1)
    s["q"].copy_(y[:, :a].reshape(rows, a * D))
    page = s["pages"].long()[b, pos // PAGE]
    s["kc"][:, page, pos % PAGE] = y[:, a:].to(torch.bfloat16).transpose(0, 1)
    s["vc"].transpose(2, 3)[:, page, pos % PAGE] = x[:, a + g:].to(torch.bfloat16).transpose(0, 1)
    return {"q": s["q"], "k": s["kc"], "v": s["vc"]}


def _attention(s, c):
    a, g, B, T = c["a"], c["g"], c["B"], s["max_new"]
    r, n = a // g, s["stride"] * PAGE
    pages = s["pages"].long().clamp_min(0)
    k = s["kc"][:, pages].float().view(g, B, n, D)
    v = s["vc"][:, pages].float().transpose(3, 4).reshape(g, B, n, D)
    t = torch.arange(T, device=k.device)
    row = (s["cu"].long()[:-1, None] + t).clamp_max(s["rows"] - 1)                     # [B][T]
    q = s["q"].float()[row].view(B, T, g, r, D).permute(2, 0, 1, 3, 4).reshape(g, B, T * r, D)
    p = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    at = (s["len"].long()[:, None] + t)[..., None]                                     # [B][T][1]
    j = torch.arange(n, device=k.device)
    seen = j <= at
    if c["window"]:
        seen &= (j > at - c["window"]) | (j < c["sinks"])
    p = p.view(g, B, T, r, n).masked_fill_(~seen[None, :, :, None], -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True))
    o = torch.matmul(p.view(g, B, T * r, n), v).view(g, B, T, r, D) / p.sum(-1)[..., None]
    o = o.permute(1, 2, 0, 3, 4).reshape(B * T, a * D)
    # Back to rows: those past a sequence's own go nowhere.
    b, pos = _rows(s)
    s["out"].copy_(o[b * T + pos - s["len"].long()[b]])
    return {"out": s["out"]}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "copy":
        return None                                 # nothing is computed
    s = prepare(c, seed)
    a, g, B = c["a"], c["g"], c["B"]
    lens, cu = s["len"].tolist(), s["cu"].tolist()
    if c["op"] == "append":
        q64 = torch.zeros(s["rows"], a * D, dtype=torch.float64, device="cuda")
        k64, v64 = s["kc"].double(), s["vc"].double()
        i = torch.arange(D // 2, dtype=torch.float64, device="cuda")
        freq = torch.exp(-i * (math.log(BASE) / (D // 2)))
        for b in range(B):
            n, T = lens[b], cu[b + 1] - cu[b]
            x = s["qkv"][cu[b]: cu[b + 1]].double().view(T, a + 2 * g, D)
            pos = torch.arange(n, n + T, device="cuda")
            # Pairs of the two halves as complex numbers, times exp(i angle).
            z = torch.complex(x[:, : a + g, : D // 2].contiguous(), x[:, : a + g, D // 2:].contiguous())
            ang = pos.double()[:, None] * freq
            z = z * torch.polar(torch.ones_like(ang), ang)[:, None]
            y = torch.cat([z.real, z.imag], -1)
            q64[cu[b]: cu[b + 1]] = y[:, :a].reshape(T, a * D)
            at = s["pages"][b].long()[pos // PAGE] * PAGE + pos % PAGE
            k64.view(g, -1, D)[:, at] = y[:, a:].transpose(0, 1)
            v64[:, at // PAGE, :, at % PAGE] = x[:, a + g:]
        return {"q": q64, "k": k64, "v": v64}
    r = a // g
    out = torch.zeros(s["rows"], a * D, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, T = lens[b], cu[b + 1] - cu[b]
        # The positions that some row sees, and whether a row does.
        pos = torch.arange(n + T, device="cuda")
        if c["window"]:
            pos = pos[(pos > n - c["window"]) | (pos < c["sinks"])]
        at = torch.arange(n, n + T, device="cuda")[:, None]
        hid = pos[None] > at
        if c["window"]:
            hid |= (pos[None] + c["window"] <= at) & (pos[None] >= c["sinks"])
        pg = s["pages"][b].long()[pos // PAGE]
        for h in range(g):
            k = s["kc"][h, pg, pos % PAGE].double()
            v = s["vc"][h, pg, :, pos % PAGE].double()
            for j in range(h * r, h * r + r):
                q = s["q"][cu[b]: cu[b + 1], j * D: (j + 1) * D].double()
                p = torch.softmax((q @ k.T / math.sqrt(D)).masked_fill(hid, -math.inf), -1)
                out[cu[b]: cu[b + 1], j * D: (j + 1) * D] = p @ v
    return {"out": out}
