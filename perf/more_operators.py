"""Cases of the quantised paged caches: the plain forms in torch and the calls a user makes.

A decoding server keeps compressed caches in pages (see operators.py for tables and lengths).  Here a pool holds 4 or 8 bits
per element: uint8 [n_pages][n_kv_heads][page_bytes], a page of a head being its rows' codes [page_size][head_dim * bits / 8]
and then [page_size][2][head_dim / 64] bf16, the step and the lowest value of every 64 dimensions of a row.  The codes of a
row lie in units of eight dimensions, the first units of all groups, then the second ones, and so on; inside a unit in order, from
the lowest bits up.

  store   compacted rows into quantised pages with the key bounds of every page, and all of them read back
  load    rows of quantised pages read back into dense rows
  append  rotary positions with three axes on queries and keys, the new rows quantised into their slots and read back
  attend  attention of one new token per sequence over its quantised pages, or over chosen ones of them
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 64                                              # dimensions that share a step and a lowest value
LEAST = 2.0 ** -126                                     # the smallest step


# ------------------------------------------------------------------------------------------------ cases

def listed():
    heads = dict(n_q_heads=28, n_kv_heads=4, head_dim=128, dtype="bf16")     # the long-video shape
    return [
        # a tiny fp32 prompt of two layers into 8-bit pages and back
        dict(name="store_tiny_f32_8", kind="store", n_q_heads=4, n_kv_heads=4, head_dim=64, dtype="f32", bits=8, page_size=32,
             n_seqs=2, capacity=1024, len_lo=201, len_hi=311),
        # every layer of a compressed 19K-token video prompt
        dict(name="store_video_19k_4", kind="store", bits=4, page_size=16, n_seqs=28, capacity=18944, len_lo=190, len_hi=18944,
             **heads),
        # the last rows of one request's 28 layers, to hand them on
        dict(name="load_tail_4", kind="load", bits=4, page_size=16, n_seqs=28, len_lo=36, len_hi=2842, tail=33, **heads),
        # 64 requests of one layer read back whole
        dict(name="load_batch_8", kind="load", bits=8, page_size=32, n_seqs=64, len_lo=36, len_hi=18944, tail=0, **heads),
        # one decoding step of 64 requests at far positions
        dict(name="append_step_4", kind="append", bits=4, page_size=16, n_seqs=64, len_lo=36, len_hi=2842, grow=1, pos="step", axis_t=16,
             axis_h=24, axis_w=24, order=0, pairing=0, theta=1e6, pad=0, **heads),
        # a whole 19K-token video prompt, ragged last page, some padding rows
        dict(name="append_video_19k_4", kind="append", bits=4, page_size=32, n_seqs=1, len_lo=0, len_hi=0, grow=18944, pos="video",
             axis_t=24, axis_h=20, axis_w=20, order=1, pairing=0, theta=5e6, pad=7, **heads),
        # one request with a short compressed cache: nothing but latency
        dict(name="attend_one_short_4", kind="attend", bits=4, page_size=16, n_seqs=1, len_lo=947, len_hi=947, empty=0, keep=0, **heads),
        # one request, full 128K cache: the split over the length
        dict(name="attend_one_128k_4", kind="attend", bits=4, page_size=64, n_seqs=1, len_lo=129072, len_hi=129072, empty=0,
             keep=0, **heads),
        # 192 requests of one layer, compressed to very different lengths, two slots of the batch unused
        dict(name="attend_batch_4", kind="attend", bits=4, page_size=16, n_seqs=192, len_lo=36, len_hi=18944, empty=2, keep=0,
             **heads),
        # ten requests up to 32K, one query head per KV head, 8 bits
        dict(name="attend_batch_8", kind="attend", bits=8, n_q_heads=32, n_kv_heads=32, head_dim=128, dtype="bf16", page_size=32,
             n_seqs=10, len_lo=517, len_hi=32768, empty=0, keep=0),
        # small fp32 batch
        dict(name="attend_f32_4", kind="attend", n_q_heads=12, n_kv_heads=4, head_dim=64, dtype="f32", bits=4, page_size=32,
             n_seqs=9, len_lo=1, len_hi=1024, empty=1, keep=0),
        # sixteen requests up to 32K, about an eighth of the pages of each chosen
        dict(name="attend_chosen_4", kind="attend", bits=4, page_size=32, n_seqs=16, len_lo=517, len_hi=32768, empty=0, keep=128,
             **heads),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "load", "append", "attend", "attend", "attend"])
    hkv, group = rng.choice([(4, 7), (4, 7), (32, 1), (8, 4), (8, 8), (2, 3), (1, 16), (2, 12), (4, 1)])
    dim = rng.choice([64, 128, 128, 128, 256])
    s = dict(kind=kind, page_size=rng.choice([16, 16, 32, 64, 128]), bits=rng.choice([4, 4, 8]), n_q_heads=hkv * group,
             n_kv_heads=hkv, head_dim=dim, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    es = 4 if s["dtype"] == "f32" else 2
    row = hkv * dim * es * 2
    if kind == "append":
        half = dim // 2
        a = rng.randint(1, half // 4)
        s.update(order=rng.randint(0, 1), axis_t=half - 2 * a, axis_h=a, axis_w=a, pairing=rng.randint(0, 1),
                 theta=rng.choice([1e4, 1e6]), pad=rng.randint(0, 3))
        most = max(2, 90_000_000 // (row * (1 + group)) // es)
        if rng.random() < 0.5:
            s.update(n_seqs=_log(rng, 1, min(200, most)), len_lo=rng.randint(0, 60), len_hi=_log(rng, 64, 2000),
                     grow=rng.choice([1, 1, 1, 3]), pos="step")
        else:
            s.update(n_seqs=1, len_lo=0, len_hi=0, grow=_log(rng, 2, min(9000, most)), pos="video")
        return s
    n = _log(rng, 1, 100)
    lo = rng.randint(1, 40)
    hi = _log(rng, 64, max(65, min(130_000, 120_000_000 // row // n)))
    s.update(n_seqs=n, len_lo=lo, len_hi=hi)
    if kind == "store":
        s["capacity"] = hi + rng.randint(0, 50)
    elif kind == "load":
        s["tail"] = rng.choice([0, 0, rng.randint(1, 100)])
    else:
        s["empty"] = rng.randint(0, min(2, n - 1))
        s["keep"] = rng.choice([0, 0, rng.randint(1, max(1, hi // s["page_size"] // 2))])
    return s


def _lens(case):
    """The sequences' lengths, spread evenly over the logarithm; prepare() hands them out in an order of the seed."""
    n, lo, hi = case["n_seqs"], case["len_lo"], max(case["len_lo"], case["len_hi"])
    lens = [hi if n == 1 else int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** (i / (n - 1)))) - 1 for i in range(n)]
    return [0] * case.get("empty", 0) + lens[case.get("empty", 0):]


def _pages(n, page):
    return -(-n // page)


def _row_bytes(case):
    """Of one head: codes, and with them steps and lowest values."""
    d = case["head_dim"]
    return d * case["bits"] // 8, d * case["bits"] // 8 + 4 * (d // GROUP)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    held = 2 * hkv * _row_bytes(case)[1]                # keys and values of a row in the pools, and as they are
    plain = 2 * hkv * d * es
    lens, p = _lens(case), case["page_size"]
    if case["kind"] == "append":
        t = case["n_seqs"] * case["grow"]
        return {"bytes": t * (2 * hq * d * es + 2 * plain + 2 * held + 12 + 8), "flops": t * d * (6 * hq + 14 * hkv)}
    rows, pages = sum(lens), sum(_pages(n, p) for n in lens)
    if case["kind"] == "store":
        return {"bytes": rows * 2 * (plain + held) + pages * hkv * 2 * d * es, "flops": 14 * rows * hkv * d}
    if case["kind"] == "load":
        rows = sum(min(n, case["tail"] or n) for n in lens)
        return {"bytes": rows * (plain + held), "flops": 4 * rows * hkv * d}
    if case["keep"]:
        rows = sum(min(n, case["keep"] * p) for n in lens)
        pages = sum(min(_pages(n, p), case["keep"]) for n in lens)
    return {"bytes": rows * held + 2 * len(lens) * hq * d * es + 4 * pages * (1 + (hkv if case["keep"] else 0)),
            "flops": 4 * rows * hq * d}


# ----------------------------------------------------------------------------------------------- inputs

def _normal(gen, shape, dtype, mean=0.0, std=1.0):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    return x.normal_(mean, std, generator=gen).to(dtype)


def _table(gen, lens, page, slack):
    """Pages handed out in a shuffled order, as in a pool in use: (table, pages in the pool)."""
    counts = torch.tensor([_pages(n, page) for n in lens], dtype=torch.int64, device="cuda")
    total = int(counts.sum()) + slack
    perm = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    at = torch.arange(max(1, int(counts.max())), device="cuda")[None, :]
    start = (counts.cumsum(0) - counts)[:, None]
    table = torch.where(at < counts[:, None], perm[(start + at).clamp(max=total - 1)], -1)
    return table.to(torch.int32).contiguous(), total


def _pool(gen, case, n_pages, mean):
    """A pool of rows as a model leaves them (neighbouring rows alike, some dimensions far larger than others), quantised."""
    hkv, p, d = case["n_kv_heads"], case["page_size"], case["head_dim"]
    pool = torch.empty((n_pages, hkv, p * _row_bytes(case)[1]), dtype=torch.uint8, device="cuda")
    wide = torch.exp(_normal(gen, (hkv, 1, d), torch.float32, 0.0, 0.5))
    for at in range(0, n_pages, 4096):                  # a part at a time: the rows in 32 bits take eight times the pool
        n = min(4096, n_pages - at)
        rows = _normal(gen, (n, hkv, p, d), torch.float32, mean, 0.7)
        rows += _normal(gen, (n, hkv, 1, d), torch.float32, 0.0, 0.7)
        pool[at:at + n] = _pack(case, *_encode((rows * wide).to(DTYPES[case["dtype"]]).float(), case["bits"]))
    return pool


def prepare(case, seed):
    case = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    dtype, hq, hkv, d, p = DTYPES[case["dtype"]], case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["page_size"]
    kind = case["kind"]
    temperature = 0.5 + 1.5 * rng.random()
    lens = _lens(case)
    rng.shuffle(lens)
    before = list(lens)
    if kind == "append":
        lens = [n + case["grow"] for n in lens]
    elif kind == "load":
        before = [max(0, n - case["tail"]) if case["tail"] else 0 for n in lens]
    n = len(lens)
    table, n_pages = _table(gen, lens, p, slack=3)
    i32 = dict(dtype=torch.int32, device="cuda")
    st = {"case": case, "table": table, "lens": torch.tensor(lens, **i32), "lens_from": torch.tensor(before, **i32)}

    def zeros(*shape, dtype=dtype):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    page_bytes = p * _row_bytes(case)[1]
    if kind in ("store", "append"):
        st["k_pages"], st["v_pages"] = (zeros(n_pages, hkv, page_bytes, dtype=torch.uint8) for _ in range(2))
    else:
        st["k_pages"], st["v_pages"] = _pool(gen, case, n_pages, 0.5), _pool(gen, case, n_pages, 0.2)
    if kind == "store":
        cap = case["capacity"]
        wide = torch.exp(_normal(gen, (1, hkv, 1, d), torch.float32, 0.0, 0.5))
        st["k"] = _normal(gen, (n, hkv, cap, d), torch.float32, 0.5).mul_(wide).to(dtype)
        st["v"] = _normal(gen, (n, hkv, cap, d), dtype, 0.2)
        st["bounds"] = zeros(n_pages, hkv, 2, d)
        st["lens_from"] = None
        st["k_back"], st["v_back"] = zeros(n, hkv, cap, d), zeros(n, hkv, cap, d)
    elif kind == "load":
        cap = max(1, max(b - a for a, b in zip(before, lens)))
        st["k_back"], st["v_back"] = zeros(n, hkv, cap, d), zeros(n, hkv, cap, d)
    elif kind == "append":
        grow, pad = case["grow"], case["pad"]
        t = n * grow + pad
        row = st["lens_from"].long()[:, None] + torch.arange(grow, device="cuda")
        slots = table.long().gather(1, row // p) * p + row % p
        st["slots"] = torch.cat([slots.flatten(), torch.full((pad,), -1, dtype=torch.int64, device="cuda")])
        if case["pos"] == "video":
            frame, side, text = 144, 12, 64
            at = (torch.arange(t, device="cuda") - text).clamp(min=0)
            pos = torch.stack([text + at // frame, text + at % frame // side, text + at % side])
            pos = torch.where(torch.arange(t, device="cuda") < text, torch.arange(t, device="cuda"), pos)
        else:
            pos = torch.randint(0, 130_000, (1, t), generator=gen, device="cuda").expand(3, t)
        # queries, keys and values are slices of one projection's rows, as a model hands them over
        qkv = _normal(gen, (t, hq + 2 * hkv, d), dtype, 0.0, temperature)
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], positions=pos.to(torch.int32).contiguous(),
                  q_out=zeros(t, hq, d), k_back=zeros(n, hkv, grow, d), v_back=zeros(n, hkv, grow, d))
    else:
        st.update(q=_normal(gen, (n, hq, d), dtype, 0.0, temperature), out=zeros(n, hq, d), lse=zeros(n, hq, dtype=torch.float32),
                  sel=None)
        if case["keep"]:
            # chosen by another call: some pages of every sequence and KV head, in ascending order
            count = ((st["lens"] + p - 1) // p).long()[:, None, None]
            rank = torch.rand((n, hkv, table.shape[1]), generator=gen, device="cuda")
            rank = torch.where(torch.arange(table.shape[1], device="cuda") < count, rank, 2.0)
            k = min(case["keep"], table.shape[1])
            sel = torch.argsort(rank, -1)[..., :k]
            sel = torch.where(torch.arange(k, device="cuda") < count, sel, 1 << 30).sort(-1).values
            st["sel"] = torch.full((n, hkv, case["keep"]), -1, **i32)
            st["sel"][..., :k] = torch.where(sel < 1 << 30, sel, -1).to(torch.int32)
    if own:
        from paper_2502_17599_b200 import binding
        rope = {}
        if kind == "append":
            rope = dict(rope_theta=case["theta"], rope_sections=(case["axis_t"], case["axis_h"], case["axis_w"]),
                        rope_order=case["order"], rope_pairing=case["pairing"])
        st["pages"] = binding.Pages(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=case["dtype"], page_size=p, n_pages=n_pages,
                                    max_seqs=n, max_seq_pages=table.shape[1], cache_bits=case["bits"], **rope)
    return st


# ----------------------------------------------------------------------------- the framework's operators

def _run_own(s):
    pages, kind = s["pages"], s["case"]["kind"]
    if kind == "attend":
        pages.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["out"], s["lse"], sel=s["sel"])
        return
    if kind == "store":
        pages.page_store(s["k"], s["v"], s["lens"], s["table"], s["k_pages"], s["v_pages"], s["bounds"])
    elif kind == "append":
        pages.rope_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"], s["k_pages"], s["v_pages"])
    pages.page_load(s["k_pages"], s["v_pages"], s["table"], s["lens"], s["k_back"], s["v_back"], lens_from=s["lens_from"])


def _outputs(s):
    names = {"store": ("k_back", "v_back", "bounds"), "load": ("k_back", "v_back"), "append": ("q_out", "k_back", "v_back"),
             "attend": ("out", "lse")}
    return {n: s[n] for n in names[s["case"]["kind"]]}


# --------------------------------------------------------------------------------------------- plain forms

def run(state):
    if own:
        _run_own(state)
    else:
        {"store": _store, "load": _load, "append": _append, "attend": _attend}[state["case"]["kind"]](state)
    return _outputs(state)


def _to_bf16(x, up):
    """fp32 values rounded up or down to those of a bf16 (cutting a number's lower half moves it towards zero)."""
    cut = (x.view(torch.int32) & -65536).view(torch.float32)
    away = ((x.view(torch.int32) & -65536) + 65536).view(torch.float32)
    return torch.where(cut == x, x, torch.where((x > 0) == up, away, cut))


def _encode(x, bits):
    """fp32 rows [..., head_dim] -> codes uint8 [..., groups, 64], steps and lowest values fp32 [..., groups].  A code is what these
    fp32 operations give: next to a border another order of them would give another one."""
    x = x.unflatten(-1, (-1, GROUP))
    top = x.amax(-1)
    low = _to_bf16(x.amin(-1), up=False)
    levels = (1 << bits) - 1
    step = _to_bf16((top - low) * (1.0 / levels), up=True).clamp(min=LEAST)
    code = torch.round((x - low[..., None]) * (1.0 / step)[..., None])
    return code.to(torch.uint8), step, low


def _pack(case, code, step, low):
    """[pages, heads, page_size, ...] of _encode -> the pool's bytes [pages, heads, page_bytes]."""
    unit = code.unflatten(-1, (8, 8)).transpose(-3, -2).flatten(-3)              # [..., 8, groups, 8]
    if case["bits"] == 4:
        unit = unit[..., 0::2] | unit[..., 1::2] << 4
    more = torch.stack([step, low], -2).to(torch.bfloat16).flatten(-2)
    return torch.cat([unit.flatten(-2), more.contiguous().view(torch.uint8).flatten(-2)], -1)


def _unpack(case, pool):
    """The pool's pages [..., page_bytes] -> values fp32 [..., page_size, head_dim]."""
    p, groups, bits = case["page_size"], case["head_dim"] // GROUP, case["bits"]
    codes = p * _row_bytes(case)[0]
    unit, more = pool[..., :codes].unflatten(-1, (p, -1)), pool[..., codes:].contiguous().view(torch.bfloat16).float()
    if bits == 4:
        unit = torch.stack([unit & 15, unit >> 4], -1).flatten(-2)
    code = unit.unflatten(-1, (8, groups, 8)).transpose(-3, -2).flatten(-2).float()        # [..., p, groups, 64]
    more = more.unflatten(-1, (p, 2, groups))
    return (more[..., 1, :, None] + more[..., 0, :, None] * code).flatten(-2)


def _put(s, rows, pool, seq, pos):
    """Rows [x][heads][head_dim] into the pool as rows `pos` of the sequences `seq`."""
    c, p = s["case"], s["case"]["page_size"]
    code, step, low = _encode(rows.float(), c["bits"])
    page = s["table"].long()[seq, pos // p]
    one = _pack(dict(c, page_size=1), code[:, :, None], step[:, :, None], low[:, :, None])     # each row as a page of one
    codes, both = _row_bytes(c)
    more = both - codes
    n_pages, hkv = pool.shape[:2]
    pool[:, :, :p * codes].view(n_pages, hkv, p, codes)[page, :, pos % p] = one[..., :codes]
    pool[:, :, p * codes:].unflatten(-1, (p, more))[page, :, pos % p] = one[..., codes:]


def _get(s, pool, back):
    """Rows [lens_from, lens) of every sequence from the pool, the first of them to row 0."""
    c, p = s["case"], s["case"]["page_size"]
    first = torch.zeros_like(s["lens"]) if s["lens_from"] is None else s["lens_from"]
    count = (s["lens"] - first).long()
    at = torch.arange(back.shape[2], device=back.device)[None, :]
    seq, to = (at < count[:, None]).nonzero(as_tuple=True)
    pos = to + first.long()[seq]
    page = s["table"].long()[seq, pos // p]
    codes, both = _row_bytes(c)
    n_pages, hkv = pool.shape[:2]
    unit = pool[:, :, :p * codes].unflatten(-1, (p, codes))[page, :, pos % p]
    more = pool[:, :, p * codes:].unflatten(-1, (p, both - codes))[page, :, pos % p]
    rows = _unpack(dict(c, page_size=1), torch.cat([unit, more], -1))[:, :, 0]
    back[seq, :, to] = rows.to(back.dtype)


def _load(s):
    _get(s, s["k_pages"], s["k_back"])
    _get(s, s["v_pages"], s["v_back"])


def _store(s):
    p, table, lens = s["case"]["page_size"], s["table"].long(), s["lens"].long()
    row = torch.arange(s["k"].shape[2], device=table.device)[None, :]
    seq, pos = (row < lens[:, None]).nonzero(as_tuple=True)
    for src, pool in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
        _put(s, src[seq, :, pos], pool, seq, pos)
    _load(s)
    # bounds of every page, of the keys as they are read back
    at = torch.arange(table.shape[1], device=table.device)[None, :]
    seq, col = (at * p < lens[:, None]).nonzero(as_tuple=True)
    page = table[seq, col]
    keys = _unpack(s["case"], s["k_pages"][page]).to(s["bounds"].dtype)          # [pages in use][Hkv][page_size][D]
    live = (torch.arange(p, device=table.device)[None, :] < (lens[seq] - col * p)[:, None])[:, None, :, None]
    s["bounds"][page] = torch.stack([torch.where(live, keys, math.inf).amin(2), torch.where(live, keys, -math.inf).amax(2)], 2)


def _axes(case, device):
    """Axis (0 time, 1 height, 2 width) of every frequency: in runs, or dealt out in turn while the later axes last."""
    t, h, w = case["axis_t"], case["axis_h"], case["axis_w"]
    i = torch.arange(t + h + w, device=device)
    if case["order"] == 0:
        return (i >= t).long() + (i >= t + h).long()
    return torch.where((i % 3 == 1) & (i < 3 * h), 1, torch.where((i % 3 == 2) & (i < 3 * w), 2, 0))


def _append(s):
    c = s["case"]
    pos = s["positions"].double()                       # angles of far positions need 64 bits
    half = c["axis_t"] + c["axis_h"] + c["axis_w"]
    freq = torch.pow(torch.tensor(c["theta"], dtype=torch.float64, device=pos.device),
                     -torch.arange(half, device=pos.device, dtype=torch.float64) / half)
    angle = pos[_axes(c, pos.device)].T * freq          # [tokens][half]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x):
        x, dtype = x.float(), x.dtype
        if c["pairing"] == 0:
            a, b = x[..., :half], x[..., half:2 * half]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)
        else:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y = torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * half:]], -1)
        return y.to(dtype)

    live = s["slots"] >= 0
    s["q_out"][live] = turn(s["q"])[live]
    seq = torch.arange(c["n_seqs"], device=pos.device).repeat_interleave(c["grow"])
    row = s["lens_from"].long()[seq] + torch.arange(c["grow"], device=pos.device).repeat(c["n_seqs"])
    _put(s, turn(s["k"])[live], s["k_pages"], seq, row)
    _put(s, s["v"][live], s["v_pages"], seq, row)
    _load(s)


def _attend(s):
    c, p = s["case"], s["case"]["page_size"]
    table, lens = s["table"].long(), s["lens"].long()
    n, width = table.shape
    hkv, d = c["n_kv_heads"], c["head_dim"]
    rows = torch.arange(p, device=table.device)
    if s["sel"] is None:
        page = table.clamp(min=0)[:, None].expand(n, hkv, width)
        first = (torch.arange(width, device=table.device) * p).expand(n, hkv, width)
    else:
        col = s["sel"].long()
        page = table.clamp(min=0)[:, None].expand(n, hkv, width).gather(2, col.clamp(min=0))
        first = torch.where(col >= 0, col * p, 1 << 40)
    live = (first[..., None] + rows < lens[:, None, None, None]).flatten(2)      # [n][Hkv][rows]
    head = torch.arange(hkv, device=table.device)[None, :, None]
    keys = _unpack(c, s["k_pages"][page, head]).flatten(2, 3)
    q = s["q"].float().view(n, hkv, -1, d)
    logits = torch.matmul(q, keys.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    del keys
    logits = torch.where(live[:, :, None], logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    e = torch.where(live[:, :, None], torch.exp(logits - torch.where(top == -math.inf, 0.0, top)), 0.0)
    z = e.sum(-1, keepdim=True)
    values = torch.where(live[..., None], _unpack(c, s["v_pages"][page, head]).flatten(2, 3), 0.0)
    out = torch.matmul(e, values) / torch.where(z > 0, z, 1.0)
    s["out"].copy_(out.view(n, hkv * q.shape[2], d))
    s["lse"].copy_((top + torch.log(z)).view(n, -1))


# --------------------------------------------------------------------------------- the definition in 64 bits

def _place(case):
    """Of every dimension of a row: (byte of the codes, lowest bit in it)."""
    d, bits = case["head_dim"], case["bits"]
    groups, place = d // GROUP, []
    for x in range(d):
        g, i, e = x // GROUP, x % GROUP // 8, x % 8
        bit = ((i * groups + g) * 8 + e) * bits
        place.append((bit // 8, bit % 8))
    return place


def _exact_rows(case, pool, page, row):
    """Rows (page[x], every head, row[x]) of a pool in 64 bits [x][heads][head_dim]."""
    d, p, bits = case["head_dim"], case["page_size"], case["bits"]
    codes = d * bits // 8
    at = torch.tensor(_place(case), device="cuda")
    data = pool[page]                                                            # [x][heads][page_bytes]
    byte = (row[:, None] * codes + at[:, 0])[:, None].expand(-1, data.shape[1], -1)
    code = (data.gather(2, byte).long() >> at[:, 1]) % (1 << bits)
    half = torch.arange(2 * (d // GROUP), device="cuda") * 2
    byte = (p * codes + row[:, None] * 4 * (d // GROUP) + half)[:, None].expand(-1, data.shape[1], -1)
    word = data.gather(2, byte).int() << 16 | data.gather(2, byte + 1).int() << 24
    more = word.view(torch.float32).double()
    group = torch.arange(d, device="cuda") // GROUP
    return more[..., d // GROUP + group] + more[..., group] * code


def _held(x, bits):
    """What rows [..., head_dim] of the cache's own type read back as, in 64 bits.  Steps and codes go by fp32 arithmetic: that is
    part of their definition."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    levels = 2 ** bits - 1
    for g in range(0, x.shape[-1], GROUP):
        y = x[..., g:g + GROUP].to(torch.float32)
        low = y.min(-1, keepdim=True).values
        near = low.to(torch.bfloat16)
        below = torch.nextafter(near, torch.full_like(near, -math.inf))
        low = torch.where(near.float() > low, below, near).float()
        step = (y.max(-1, keepdim=True).values - low) * torch.tensor(1.0 / levels, dtype=torch.float32, device=x.device)
        near = step.to(torch.bfloat16)
        above = torch.nextafter(near, torch.full_like(near, math.inf))
        step = torch.where(near.float() < step, above, near).float().clamp(min=LEAST)
        code = ((y - low) * step.reciprocal()).round().double()
        out[..., g:g + GROUP] = low.double() + step.double() * code
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind, p = case["kind"], case["page_size"]
    lens = s["lens"].cpu().tolist()
    first = [0] * len(lens) if s["lens_from"] is None else s["lens_from"].cpu().tolist()
    if kind == "append":
        return _exact_append(s, case)
    if kind in ("store", "load"):
        k_back, v_back = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s["k_back"], s["v_back"]))
    if kind == "load":
        for i, m in enumerate(lens):
            row = torch.arange(first[i], m, device="cuda")
            page = s["table"][i, row // p].long()
            for pool, back in ((s["k_pages"], k_back), (s["v_pages"], v_back)):
                back[i, :, :m - first[i]] = _exact_rows(case, pool, page, row % p).transpose(0, 1)
        return {"k_back": k_back, "v_back": v_back}
    if kind == "store":
        bounds = torch.zeros(s["bounds"].shape, dtype=torch.float64, device="cuda")
        for i, m in enumerate(lens):
            k_back[i, :, :m] = _held(s["k"][i, :, :m], case["bits"])
            v_back[i, :, :m] = _held(s["v"][i, :, :m], case["bits"])
            for c0, page in enumerate(s["table"][i, :_pages(m, p)].tolist()):
                rows = k_back[i, :, c0 * p:min(m, c0 * p + p)]
                bounds[page] = torch.stack([rows.amin(1), rows.amax(1)], 1)
        return {"k_back": k_back, "v_back": v_back, "bounds": bounds}
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    group = hq // hkv
    out = torch.zeros((len(lens), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((len(lens), hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, m in enumerate(lens):
        if m == 0:
            continue
        for g in range(hkv):
            row = torch.arange(m, device="cuda")
            if s["sel"] is not None:
                row = row[torch.isin(row // p, s["sel"][i, g])]
            page = s["table"][i, row // p].long()
            k = _exact_rows(case, s["k_pages"][:, g:g + 1], page, row % p)[:, 0]
            v = _exact_rows(case, s["v_pages"][:, g:g + 1], page, row % p)[:, 0]
            logits = (s["q"][i, g * group:(g + 1) * group].double() @ k.T) / math.sqrt(d)
            norm = torch.logsumexp(logits, -1)
            lse[i, g * group:(g + 1) * group] = norm
            out[i, g * group:(g + 1) * group] = torch.exp(logits - norm[:, None]) @ v
    return {"out": out, "lse": lse}


def _exact_append(s, case):
    t, h, w = case["axis_t"], case["axis_h"], case["axis_w"]
    half = t + h + w
    if case["order"] == 0:
        axis = [0] * t + [1] * h + [2] * w
    else:
        axis = [0] * half
        for a, n in ((1, h), (2, w)):
            for i in range(a, min(half, 3 * n), 3):
                axis[i] = a
    angle = torch.stack([s["positions"][axis[i]].double() * case["theta"] ** (-i / half) for i in range(half)], 1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]          # e^(i angle)

    def turn(x):
        x = x.double().clone()
        a = slice(0, half) if case["pairing"] == 0 else slice(0, 2 * half, 2)
        b = slice(half, 2 * half) if case["pairing"] == 0 else slice(1, 2 * half, 2)
        z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * unit
        x[..., a], x[..., b] = z.real, z.imag
        return x

    dtype, n, grow = DTYPES[case["dtype"]], case["n_seqs"], case["grow"]
    q_out = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
    q_out[:n * grow] = turn(s["q"])[:n * grow]
    rows = [x[:n * grow].unflatten(0, (n, grow)).transpose(1, 2) for x in (turn(s["k"]).to(dtype), s["v"])]
    # a key rounded to 32 bits may fall on the other side of a border between codes: one code in 10^5 is another one
    k_back = _held(rows[0], case["bits"]) if case["dtype"] == "bf16" else None
    return {"q_out": q_out, "k_back": k_back, "v_back": _held(rows[1], case["bits"])}
