"""Cases of the paged-cache operators: the plain forms in torch and the calls a user makes.

A decoding server keeps the caches of many prompts, compressed layer by layer to lengths of their own, in one pool of
pages per tensor: `k_pages`, `v_pages` [n_pages][n_kv_heads][page_size][head_dim].  A "sequence" is one layer of one
request; `table` [n_seqs][max_seq_pages] holds its pages in order and `lens` its row count.

  tables  page tables, slot maps and the free list moved from one set of lengths to the next
  store   compacted rows [n_seqs][n_kv_heads][capacity][head_dim] into the pages, and the key bounds of every page
  append  rotary positions with three axes on queries and keys, keys and values into their slots
  attend  attention of one new token per sequence over its pages
  sparse  the same over the pages whose key bounds promise the most, chosen per sequence and KV head
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases

def listed():
    heads = dict(n_q_heads=28, n_kv_heads=4, head_dim=128, dtype="bf16")     # the long-video shape
    return [
        # one decoding step of 64 requests x 28 layers: one token each, a few requests leave and a few arrive
        dict(name="tables_step", kind="tables", page_size=16, n_seqs=1792, len_lo=36, len_hi=2842, grow=1, ends=28,
             starts=28, pad=11),
        # sixteen compressed prompts admitted at once, while twelve others leave
        dict(name="tables_prompts", kind="tables", page_size=16, n_seqs=784, len_lo=33, len_hi=18944, grow=0, ends=336,
             starts=448, pad=300),
        # a tiny fp32 prompt of two layers into pages
        dict(name="store_tiny_f32", kind="store", n_q_heads=4, n_kv_heads=4, head_dim=64, dtype="f32", page_size=32,
             n_seqs=2, capacity=1024, len_lo=201, len_hi=311),
        # every layer of a compressed 19K-token video prompt
        dict(name="store_video_19k", kind="store", page_size=16, n_seqs=28, capacity=18944, len_lo=190, len_hi=18944,
             **heads),
        # one step of 64 requests at far positions
        dict(name="append_step", kind="append", page_size=16, n_tokens=64, pos="step", axis_t=16, axis_h=24, axis_w=24, order=0,
             pairing=0, theta=1e6, pad=0, **heads),
        # a whole 19K-token video prompt, ragged last page, some padding rows
        dict(name="append_video_19k", kind="append", page_size=32, n_tokens=18951, pos="video", axis_t=24, axis_h=20,
             axis_w=20, order=1, pairing=0, theta=5e6, pad=7, **heads),
        # one request with a short compressed cache: nothing but latency
        dict(name="attend_one_short", kind="attend", page_size=16, n_seqs=1, len_lo=947, len_hi=947, empty=0, **heads),
        # one request, full 128K cache: the split over the length
        dict(name="attend_one_128k", kind="attend", page_size=64, n_seqs=1, len_lo=129072, len_hi=129072, empty=0, **heads),
        # 64 requests of one layer, compressed to very different lengths, two slots of the batch unused
        dict(name="attend_batch_ragged", kind="attend", page_size=16, n_seqs=64, len_lo=36, len_hi=18944, empty=2, **heads),
        # small fp32 batch, one query head per KV head
        dict(name="attend_f32", kind="attend", n_q_heads=4, n_kv_heads=4, head_dim=64, dtype="f32", page_size=32,
             n_seqs=9, len_lo=1, len_hi=1024, empty=1),
        # one request, 128K cache, about 5 % of its pages attended
        dict(name="sparse_one_128k", kind="sparse", page_size=16, n_seqs=1, len_lo=129072, len_hi=129072, keep=404,
             first=4, last=16, **heads),
        # ten requests up to 32K, one query head per KV head, at most 3,264 rows of each attended
        dict(name="sparse_batch_32k", kind="sparse", n_q_heads=32, n_kv_heads=32, head_dim=128, dtype="bf16",
             page_size=32, n_seqs=10, len_lo=517, len_hi=32768, keep=102, first=1, last=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _shape(rng):
    hkv, group = rng.choice([(4, 7), (4, 7), (32, 1), (8, 4), (8, 8), (2, 3), (1, 16), (4, 1)])
    dim = rng.choice([64, 128, 128, 128, 256])
    return dict(n_q_heads=hkv * group, n_kv_heads=hkv, head_dim=dim, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))


def draw(rng):
    kind = rng.choice(["tables", "store", "append", "attend", "attend", "sparse"])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind == "tables":
        n = _log(rng, 1, 2000)
        ends, starts = rng.randint(0, n // 3), rng.randint(0, n // 3)
        return dict(kind=kind, page_size=page, n_seqs=n, len_lo=rng.randint(1, 60), len_hi=_log(rng, 64, 9000),
                    grow=rng.choice([0, 1, 1, 5, rng.randint(1, 700)]), ends=ends, starts=starts, pad=rng.randint(0, 99))
    s = _shape(rng)
    row = s["n_kv_heads"] * s["head_dim"] * (4 if s["dtype"] == "f32" else 2) * 2
    if kind == "append":
        t = _log(rng, 1, max(1, min(9000, 90_000_000 // (row * (1 + s["n_q_heads"] // s["n_kv_heads"])))))
        half = s["head_dim"] // 2
        a = rng.randint(1, half // 4)
        return dict(kind=kind, page_size=page, n_tokens=t, pos=rng.choice(["step", "video"]), order=rng.randint(0, 1),
                    axis_t=half - 2 * a, axis_h=a, axis_w=a, pairing=rng.randint(0, 1), theta=rng.choice([1e4, 1e6]),
                    pad=rng.randint(0, 3), **s)
    rows = 120_000_000 // row
    n = _log(rng, 1, 100)
    lo = rng.randint(1, 40)
    hi = _log(rng, 64, max(65, min(130_000, rows // n)))
    case = dict(kind=kind, page_size=page, n_seqs=n, len_lo=lo, len_hi=hi, **s)
    if kind == "store":
        case["capacity"] = hi + rng.randint(0, 50)
    elif kind == "attend":
        case["empty"] = rng.randint(0, min(2, n - 1))
    else:
        case["first"], case["last"] = rng.randint(0, 2), rng.randint(1, 3)
        case["keep"] = case["first"] + case["last"] + rng.randint(1, max(1, hi // page // 3))
    return case


def _lens(case):
    """The sequences' lengths, spread evenly over the logarithm; prepare() hands them out in an order of the seed."""
    n, lo, hi = case["n_seqs"], case["len_lo"], max(case["len_lo"], case["len_hi"])
    lens = [hi if n == 1 else int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [0] * case.get("empty", 0) + lens[case.get("empty", 0):]


def _steps(case):
    """(old, new) lengths of a tables case: those who leave, those who arrive, those who grow."""
    lens = _lens(case)
    every = max(1, case["n_seqs"] // max(1, case["ends"] + case["starts"]))
    out, ends, starts = [], case["ends"], case["starts"]
    for i, n in enumerate(lens):
        turn = i % every == 0
        if turn and ends and (ends >= starts or not starts):
            out.append((n, 0))
            ends -= 1
        elif turn and starts:
            out.append((0, n))
            starts -= 1
        else:
            out.append((n, n + case["grow"]))
    return out


def _pages(n, page):
    return -(-n // page)


def work(case):
    if case["kind"] == "tables":
        steps, p = _steps(case), case["page_size"]
        pops = sum(max(0, _pages(b, p) - _pages(a, p)) for a, b in steps)
        drops = sum(max(0, _pages(a, p) - _pages(b, p)) for a, b in steps)
        fresh = sum(max(0, b - a) for a, b in steps) + case["pad"]
        return {"bytes": 8 * len(steps) + 8 * pops + 4 * drops + 8 * fresh + 4 * (len(steps) + 1) + 4 * max(0, drops - pops),
                "flops": 0}
    es = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        t = case["n_tokens"]
        return {"bytes": t * d * es * (2 * hq + 4 * hkv) + t * (12 + 8), "flops": t * d * 3 * (hq + hkv)}
    lens, p = _lens(case), case["page_size"]
    rows, pages = sum(lens), sum(_pages(n, p) for n in lens)
    bound = hkv * 2 * d * es
    if case["kind"] == "store":
        return {"bytes": 4 * rows * hkv * d * es + pages * bound, "flops": 2 * rows * hkv * d}
    n = len(lens)
    io = n * hq * d * es * 2
    if case["kind"] == "attend":
        return {"bytes": 2 * rows * hkv * d * es + io + 4 * pages, "flops": 4 * rows * hq * d}
    kept = [min(_pages(m, p), case["keep"]) for m in lens]
    kept_rows = sum(m if _pages(m, p) <= k else k * p - (_pages(m, p) * p - m) for m, k in zip(lens, kept))
    return {"bytes": pages * bound + n * hkv * p * d * es + 2 * kept_rows * hkv * d * es + io + 4 * hkv * sum(kept) + 4 * pages,
            "flops": 2 * pages * hq * d + 4 * kept_rows * hq * d}


# ----------------------------------------------------------------------------------------------- inputs

def _normal(gen, shape, dtype, mean=0.0, std=1.0):
    x = torch.empty(shape, dtype=torch.float32, device="cuda")
    return x.normal_(mean, std, generator=gen).to(dtype)


def _table(gen, lens, page, slack=0, width=None):
    """Pages handed out in a shuffled order, as in a pool in use: (table, pages in the pool, pages in use)."""
    counts = torch.tensor([_pages(n, page) for n in lens], dtype=torch.int64, device="cuda")
    used = int(counts.sum())
    perm = torch.randperm(used + slack, generator=gen, device="cuda").to(torch.int32)
    width = width or max(1, int(counts.max()))
    at = torch.arange(width, device="cuda")[None, :]
    start = (counts.cumsum(0) - counts)[:, None]
    table = torch.where(at < counts[:, None], perm[(start + at).clamp(max=max(0, used + slack - 1))], -1)
    return table.to(torch.int32).contiguous(), perm, used


def prepare(case, seed):
    case = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    st = {"case": case, "kind": case["kind"]}
    p = case["page_size"]
    if case["kind"] == "tables":
        steps = _steps(case)
        rng.shuffle(steps)
        old, new = [a for a, _ in steps], [b for _, b in steps]
        fresh = sum(max(0, b - a) for a, b in steps)
        width = max(1, max(_pages(max(a, b), p) for a, b in steps))
        room = sum(max(0, _pages(b, p) - _pages(a, p)) for a, b in steps) + 64
        table, perm, used = _table(gen, old, p, slack=room, width=width)
        i32 = dict(dtype=torch.int32, device="cuda")
        st.update(table=table, free_pages=perm, free_top=torch.tensor([used], **i32), free_top_out=torch.zeros(1, **i32),
                  lens=torch.tensor(old, **i32), new_lens=torch.tensor(new, **i32), cu_new=torch.zeros(len(old) + 1, **i32),
                  slots=torch.empty(fresh + case["pad"], dtype=torch.int64, device="cuda"))
        if own:
            st["pages"] = _handle(case, n_pages=perm.numel(), max_seqs=len(old), max_seq_pages=width, n_q_heads=1,
                                  n_kv_heads=1, head_dim=128, dtype="bf16")
        return st

    dtype, hq, hkv, d = DTYPES[case["dtype"]], case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    temperature = 0.5 + 2.5 * rng.random()
    if case["kind"] == "append":
        t, real = case["n_tokens"], case["n_tokens"] - min(case["pad"], case["n_tokens"] - 1)
        # the slots of `real` rows: whole pages in a shuffled order for a prompt, one row of a page each for a step
        if case["pos"] == "video":
            order = torch.randperm(_pages(real, p), generator=gen, device="cuda")
            row = torch.arange(real, device="cuda")
            slots, n_pages = order[row // p] * p + row % p, order.numel()
            frame, side = 144, 12
            text = min(64, real)
            at = (torch.arange(t, device="cuda") - text).clamp(min=0)
            pos = torch.stack([text + at // frame, text + at % frame // side, text + at % side])
            pos = torch.where(torch.arange(t, device="cuda") < text, torch.arange(t, device="cuda"), pos)
        else:
            n_pages = real + 3
            slots = torch.randperm(n_pages, generator=gen, device="cuda")[:real] * p
            slots = slots + torch.randint(0, p, (real,), generator=gen, device="cuda")
            pos = torch.randint(0, 130_000, (1, t), generator=gen, device="cuda").expand(3, t)
        slots = torch.cat([slots, torch.full((t - real,), -1, dtype=torch.int64, device="cuda")])
        # queries, keys and values are slices of one projection's rows, as a model hands them over
        qkv = _normal(gen, (t, hq + 2 * hkv, d), dtype, 0.0, temperature)
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], positions=pos.to(torch.int32).contiguous(),
                  slots=slots, q_out=torch.zeros((t, hq, d), dtype=dtype, device="cuda"),
                  k_pages=torch.zeros((n_pages, hkv, p, d), dtype=dtype, device="cuda"),
                  v_pages=torch.zeros((n_pages, hkv, p, d), dtype=dtype, device="cuda"))
        if own:
            st["pages"] = _handle(case, n_pages=n_pages, max_seqs=1, max_seq_pages=1, rope_theta=case["theta"],
                                  rope_sections=(case["axis_t"], case["axis_h"], case["axis_w"]), rope_order=case["order"],
                                  rope_pairing=case["pairing"])
        return st

    lens = _lens(case)
    rng.shuffle(lens)
    table, perm, used = _table(gen, lens, p, slack=3)
    n, n_pages = len(lens), perm.numel()
    st.update(table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if case["kind"] == "store":
        st.update(k=_normal(gen, (n, hkv, case["capacity"], d), dtype, 0.5), v=_normal(gen, (n, hkv, case["capacity"], d), dtype, 0.5),
                  k_pages=torch.zeros((n_pages, hkv, p, d), dtype=dtype, device="cuda"),
                  v_pages=torch.zeros((n_pages, hkv, p, d), dtype=dtype, device="cuda"),
                  bounds=torch.zeros((n_pages, hkv, 2, d), dtype=dtype, device="cuda"))
    else:
        # neighbouring rows resemble one another, as frames do: a page has a part of its own and one in common
        own_part = _normal(gen, (n_pages, hkv, p, d), torch.float32, 0.5, 0.7)
        st["k_pages"] = own_part.add_(_normal(gen, (n_pages, hkv, 1, d), torch.float32, 0.0, 0.7)).to(dtype)
        del own_part
        st["v_pages"] = _normal(gen, (n_pages, hkv, p, d), dtype, 0.5)
        st["q"] = _normal(gen, (n, hq, d), dtype, 0.0, temperature)
        st["out"] = torch.zeros((n, hq, d), dtype=dtype, device="cuda")
        st["lse"] = torch.zeros((n, hq), dtype=torch.float32, device="cuda")
        if case["kind"] == "sparse":
            # the bounds of every page but the last one's newest row are already there
            st["lens_before"] = (st["lens"] - 1).clamp(min=0)
            live = _live_rows(table, st["lens_before"], n_pages, p)
            k = st["k_pages"]
            lo = torch.where(live[:, None, :, None], k, math.inf).amin(2)
            hi = torch.where(live[:, None, :, None], k, -math.inf).amax(2)
            st["bounds"] = torch.where(live.any(1)[:, None, None, None], torch.stack([lo, hi], 2), 0).to(dtype).contiguous()
            st["sel"] = torch.full((n, hkv, case["keep"]), -1, dtype=torch.int32, device="cuda")
    if own:
        st["pages"] = _handle(case, n_pages=n_pages, max_seqs=n, max_seq_pages=table.shape[1])
    return st


def _live_rows(table, lens, n_pages, p):
    """bool [n_pages][p]: the rows of the pool that belong to a sequence."""
    at = torch.arange(table.shape[1], device="cuda")[None, :]
    rows = (lens[:, None] - at * p).clamp(0, p)
    count = torch.zeros(n_pages, dtype=torch.int64, device="cuda")
    count.index_add_(0, table.clamp(min=0).long().flatten(), torch.where(table >= 0, rows, 0).long().flatten())
    return torch.arange(p, device="cuda")[None, :] < count[:, None]


# ----------------------------------------------------------------------------- the framework's operators

def _handle(case, **more):
    from paper_2502_17599_b200 import binding
    geometry = {k: case[k] for k in ("n_q_heads", "n_kv_heads", "head_dim", "dtype", "page_size") if k in case}
    return binding.Pages(**{**geometry, **more})


def _run_own(s):
    pages, kind = s["pages"], s["kind"]
    if kind == "tables":
        pages.page_tables(s["lens"], s["new_lens"], s["free_pages"], s["free_top"], s["free_top_out"], s["table"],
                          s["cu_new"], s["slots"])
    elif kind == "store":
        pages.page_store(s["k"], s["v"], s["lens"], s["table"], s["k_pages"], s["v_pages"], s["bounds"])
    elif kind == "append":
        pages.rope_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"], s["k_pages"], s["v_pages"])
    elif kind == "attend":
        pages.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["out"], s["lse"])
    else:
        c = s["case"]
        pages.page_bounds(s["k_pages"], s["table"], s["lens_before"], s["lens"], s["bounds"])
        pages.select_pages(s["q"], s["bounds"], s["table"], s["lens"], c["first"], c["last"], s["sel"])
        pages.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["out"], s["lse"], sel=s["sel"])
    return _outputs(s)


def _outputs(s):
    names = {"tables": ("table", "free_pages", "free_top_out", "cu_new", "slots"), "store": ("k_pages", "v_pages", "bounds"),
             "append": ("q_out", "k_pages", "v_pages"), "attend": ("out", "lse"), "sparse": ("bounds", "sel", "out", "lse")}
    return {n: s[n] for n in names[s["kind"]]}


# --------------------------------------------------------------------------------------------- plain forms

def run(state):
    if own:
        return _run_own(state)
    {"tables": _tables, "store": _store, "append": _append, "attend": _attend, "sparse": _sparse}[state["kind"]](state)
    return _outputs(state)


def _tables(s):
    p, table, free = s["case"]["page_size"], s["table"], s["free_pages"]
    old, new, top = s["lens"].long(), s["new_lens"].long(), s["free_top"].long()
    n, width = table.shape
    have, need = (old + p - 1) // p, (new + p - 1) // p
    grow, drop = (need - have).clamp(min=0), (have - need).clamp(min=0)
    grow_end, drop_end = grow.cumsum(0), drop.cumsum(0)
    pops, pushes = grow_end[-1], drop_end[-1]
    at = torch.arange(width, device=table.device)[None, :]
    # pages given back, in the order of the sequences and of the pages in each
    all_pushed = torch.full((n * width + 1,), -1, dtype=torch.int64, device=table.device)
    goes = (at >= need[:, None]) & (at < have[:, None])
    rank = torch.where(goes, (drop_end - drop)[:, None] + at - need[:, None], n * width)
    all_pushed.scatter_(0, rank.flatten(), table.long().flatten())
    # pages taken: first those just given back, then the top of the free list
    comes = (at >= have[:, None]) & (at < need[:, None])
    j = torch.where(comes, (grow_end - grow)[:, None] + at - have[:, None], 0)
    from_list = free.long()[(top + j - pushes).clamp(0, free.numel() - 1)]
    taken = torch.where(j < pushes, all_pushed[j.clamp(max=n * width)], from_list)
    # what is left of the given pages goes on the list, below its top
    idx = torch.arange(free.numel(), device=table.device)
    r = pops + top - 1 - idx
    back = (idx < top) & (r >= pops) & (r < pushes)
    new_free = torch.where(back, all_pushed[r.clamp(0, n * width)], free.long())
    table.copy_(torch.where(comes, taken, table.long()))
    free.copy_(new_free)
    s["free_top_out"].copy_(top + pops - pushes)
    # slots of the new rows
    fresh = (new - old).clamp(min=0)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=table.device), fresh.cumsum(0)])
    s["cu_new"].copy_(cu)
    tok = torch.arange(s["slots"].numel(), device=table.device)
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True).clamp(max=n - 1)
    row = tok - cu[seq] + old[seq]
    page = table.long()[seq, (row // p).clamp(0, width - 1)]
    s["slots"].copy_(torch.where(tok < cu[-1], page * p + row % p, -1))


def _bounds_of(k, live):
    lo = torch.where(live[..., None, :, None], k, math.inf).amin(-2)
    hi = torch.where(live[..., None, :, None], k, -math.inf).amax(-2)
    return torch.stack([lo, hi], -2)


def _store(s):
    p, table, lens = s["case"]["page_size"], s["table"].long(), s["lens"].long()
    cap = s["k"].shape[2]
    row = torch.arange(cap, device=table.device)[None, :]
    live = row < lens[:, None]
    seq, pos = live.nonzero(as_tuple=True)
    page = table[seq, pos // p]
    for src, dst in ((s["k"], s["k_pages"]), (s["v"], s["v_pages"])):
        dst[page, :, pos % p] = src[seq, :, pos]
    at = torch.arange(table.shape[1], device=table.device)[None, :]
    seq, col = (at * p < lens[:, None]).nonzero(as_tuple=True)
    page = table[seq, col]
    live = torch.arange(p, device=table.device)[None, :] < (lens[seq] - col * p)[:, None]
    s["bounds"][page] = _bounds_of(s["k_pages"][page], live)


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
    page, row = s["slots"][live] // c["page_size"], s["slots"][live] % c["page_size"]
    s["q_out"][live] = turn(s["q"])[live]
    s["k_pages"][page, :, row] = turn(s["k"])[live]
    s["v_pages"][page, :, row] = s["v"][live]


def _softmax_rows(s, keys, values, live):
    """keys, values [n][Hkv][rows][D], live [n][Hkv or 1][rows]."""
    n, hkv, _, d = keys.shape
    q = s["q"].float().view(n, hkv, -1, d)
    logits = torch.matmul(q, keys.float().transpose(-1, -2)) * (1.0 / math.sqrt(d))
    logits = torch.where(live[:, :, None], logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    e = torch.where(live[:, :, None], torch.exp(logits - torch.where(top == -math.inf, 0.0, top)), 0.0)
    z = e.sum(-1, keepdim=True)
    values = torch.where(live[..., None], values.float(), 0.0)
    out = torch.matmul(e, values) / torch.where(z > 0, z, 1.0)
    s["out"].copy_(out.view(n, hkv * q.shape[2], d))
    s["lse"].copy_((top + torch.log(z)).view(n, -1))


def _attend(s):
    p, table, lens = s["case"]["page_size"], s["table"].long(), s["lens"].long()
    n, width = table.shape
    page = table.clamp(min=0)
    rows = torch.arange(width * p, device=table.device)
    live = (rows[None, :] < lens[:, None])[:, None]
    hkv, d = s["k_pages"].shape[1], s["k_pages"].shape[3]
    keys = s["k_pages"][page].transpose(1, 2).reshape(n, hkv, width * p, d)
    values = s["v_pages"][page].transpose(1, 2).reshape(n, hkv, width * p, d)
    _softmax_rows(s, keys, values, live)


def _sparse(s):
    c, table, lens = s["case"], s["table"].long(), s["lens"].long()
    p, keep = c["page_size"], c["keep"]
    n, width = table.shape
    hkv, d = s["k_pages"].shape[1], s["k_pages"].shape[3]
    # the newest row changes its page's bounds
    last = ((lens - 1).clamp(min=0) // p)
    page = table[torch.arange(n, device=table.device), last][lens > 0]
    live = torch.arange(p, device=table.device)[None, :] < (lens - last * p)[lens > 0][:, None]
    s["bounds"][page] = _bounds_of(s["k_pages"][page], live)
    # score of a page: the largest logit its key bounds allow, in 64 bits because the order of two pages may hang on it
    b = s["bounds"][table.clamp(min=0)]                                          # [n][width][Hkv][2][D]
    q = s["q"].view(n, 1, hkv, -1, d)
    best = torch.where(q >= 0, b[:, :, :, 1:2], b[:, :, :, 0:1])
    score = (q.double() * best).sum(-1).amax(-1).float().transpose(1, 2)         # [n][Hkv][width]
    col = torch.arange(width, device=table.device)[None, :]
    count = (lens + p - 1) // p
    forced = (col < c["first"]) | (col >= (count - c["last"])[:, None])
    score = torch.where(forced[:, None], math.inf, score)
    score = torch.where((col < count[:, None])[:, None], score, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices
    k = min(keep, width)
    taken = count.clamp(max=k)
    slot = torch.arange(k, device=table.device)
    order = torch.where(slot < taken[:, None, None], order[..., :k], width)
    order = torch.sort(order, dim=-1).values
    s["sel"][..., :k] = torch.where(order < width, order, s["sel"][..., :k].long()).to(torch.int32)
    # attention over the rows of those pages
    chosen = table.clamp(min=0)[:, None].expand(n, hkv, width).gather(2, order.clamp(max=width - 1))
    head = torch.arange(hkv, device=table.device)[None, :, None]
    keys = s["k_pages"][chosen, head].flatten(2, 3)
    values = s["v_pages"][chosen, head].flatten(2, 3)
    row = order[..., None] * p + torch.arange(p, device=table.device)
    live = ((row < lens[:, None, None, None]) & (order < width)[..., None]).flatten(2)
    _softmax_rows(s, keys, values, live)


# --------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind, p = case["kind"], case["page_size"]
    if kind == "tables":
        return None                                     # whole numbers only
    if kind == "append":
        return _exact_append(s, case)
    table, lens = s["table"].cpu().tolist(), s["lens"].cpu().tolist()
    if kind == "store":
        k_pages, v_pages, bounds = (torch.zeros(x.shape, dtype=torch.float64, device="cuda")
                                    for x in (s["k_pages"], s["v_pages"], s["bounds"]))
        for i, m in enumerate(lens):
            for c0 in range(_pages(m, p)):
                rows = slice(c0 * p, min(m, c0 * p + p))
                at = table[i][c0]
                k_pages[at, :, :rows.stop - rows.start] = s["k"][i, :, rows]
                v_pages[at, :, :rows.stop - rows.start] = s["v"][i, :, rows]
                bounds[at, :, 0], bounds[at, :, 1] = s["k"][i, :, rows].amin(1), s["k"][i, :, rows].amax(1)
        return {"k_pages": k_pages, "v_pages": v_pages, "bounds": bounds}
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    group = hq // hkv
    out = torch.zeros((len(lens), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((len(lens), hq), -math.inf, dtype=torch.float64, device="cuda")
    if kind == "sparse":
        bounds = s["bounds"].double()
    for i, m in enumerate(lens):
        if m == 0:
            continue
        n_pages = _pages(m, p)
        pages = s["table"][i, :n_pages].long()
        if kind == "sparse":
            tail = m - (n_pages - 1) * p
            rows = s["k_pages"][pages[-1], :, :tail].double()
            bounds[pages[-1], :, 0], bounds[pages[-1], :, 1] = rows.min(1).values, rows.max(1).values
        for g in range(hkv):
            q = s["q"][i, g * group:(g + 1) * group].double()
            idx = torch.arange(n_pages, device="cuda")
            if kind == "sparse":
                b = bounds[pages, g]
                promise = torch.maximum(q[:, None] * b[None, :, 0], q[:, None] * b[None, :, 1]).sum(-1).max(0).values
                promise = promise.float()
                promise[:case["first"]] = math.inf
                promise[max(0, n_pages - case["last"]):] = math.inf
                idx = torch.argsort(promise, descending=True, stable=True)[:case["keep"]].sort().values
            k = s["k_pages"][pages[idx], g].double().reshape(-1, d)
            v = s["v_pages"][pages[idx], g].double().reshape(-1, d)
            real = (idx[:, None] * p + torch.arange(p, device="cuda")[None, :]).flatten() < m
            logits = (q @ k[real].T) / math.sqrt(d)
            norm = torch.logsumexp(logits, -1)
            lse[i, g * group:(g + 1) * group] = norm
            out[i, g * group:(g + 1) * group] = torch.exp(logits - norm[:, None]) @ v[real]
    if kind == "attend":
        return {"out": out, "lse": lse}
    return {"bounds": bounds, "sel": None, "out": out, "lse": lse}


def _exact_append(s, case):
    t, h, w = case["axis_t"], case["axis_h"], case["axis_w"]
    half, p = t + h + w, case["page_size"]
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
        first = slice(0, half) if case["pairing"] == 0 else slice(0, 2 * half, 2)
        second = slice(half, 2 * half) if case["pairing"] == 0 else slice(1, 2 * half, 2)
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * unit
        x[..., first], x[..., second] = z.real, z.imag
        return x

    q, k, v = turn(s["q"]), turn(s["k"]), s["v"].double()
    q_out, k_pages, v_pages = (torch.zeros(x.shape, dtype=torch.float64, device="cuda")
                               for x in (s["q_out"], s["k_pages"], s["v_pages"]))
    rows = [i for i, x in enumerate(s["slots"].cpu().tolist()) if x >= 0]
    at = s["slots"][rows]
    q_out[rows] = q[rows]
    k_pages[at // p, :, at % p] = k[rows]
    v_pages[at // p, :, at % p] = v[rows]
    return {"q_out": q_out, "k_pages": k_pages, "v_pages": v_pages}
