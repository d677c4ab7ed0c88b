"""Operators around the target's cache, as calls that can be measured.

Three operators of the serving path beside the verification attention:

    rope     rotary positions with one to four axes (text; height and width of
             patches; time, height and width of video tokens), forward and
             inverse (the gradient, and taking a cached key's rotation back)
    append   new keys and values rotated and written into the cache (contiguous
             or 16-token pages), their queries rotated beside them
    shared   attention of drafted blocks of sequences that share long prefixes:
             a prefix is read once for all sequences of its group

Each case is computed in its plain form (elementary torch operations, 32 bits,
64 for the angles) or, with ``own`` set, by the library's entry points.
``exact`` states the same results in 64 bits.
"""

import math
import random

import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases

def rope_case(name, T, H, D, sections, dtype, theta=10000.0, per_axis=False, inverse=False, far=0, gap=0):
    return dict(name=name, op="rope", T=T, H=H, D=D, sections=sections, dtype=dtype, theta=theta, per_axis=per_axis,
                inverse=inverse, far=far, gap=gap)


def append_case(name, B, T, Hq, Hkv, D, sections, src, dtype, paged, ragged, past, theta=10000.0, video=False):
    return dict(name=name, op="append", B=B, T=T, Hq=Hq, Hkv=Hkv, D=D, sections=sections, src=src, dtype=dtype,
                paged=paged, ragged=ragged, past=past, theta=theta, video=video)


def shared_case(name, B, k, Hq, Hkv, D, G, prefix, suffix, dtype, out, paged):
    return dict(name=name, op="shared", B=B, k=k, Hq=Hq, Hkv=Hkv, D=D, G=G, prefix=prefix, suffix=suffix, dtype=dtype,
                out=out, paged=paged)


def listed():
    return [
        # one block of 8 video-model positions, queries and keys of a layer: latency
        rope_case("rope_block", 8, 32, 128, "16,24,24", "bf16", theta=1e6, far=6520),
        # a video prompt's rows of one layer (28 query and 4 key heads), a view of the fused projection
        rope_case("rope_video", 6272, 32, 128, "16,24,24", "bf16", theta=1e6, gap=512),
        # the gradient of the patches' rotation in a vision encoder, two axes
        rope_case("rope_patches_grad", 20736, 16, 80, "20,20", "f32", per_axis=True, inverse=True),
        # the drafted blocks of 16 sequences, straight from the fp32 projection into the pages
        append_case("append_block", 16, 96, 32, 8, 128, "64", "f32", "bf16", True, False, 16000),
        # four video prompts of different lengths into pages
        append_case("append_video", 4, 26111, 28, 4, 128, "16,24,24", "bf16", "bf16", True, True, 300, 1e6, True),
        # a long prompt into a contiguous cache
        append_case("append_long", 1, 65536, 64, 8, 128, "64", "bf16", "bf16", False, False, 0, 1e6),
        # fp32 cache of the small workload, all of it
        append_case("append_f32", 3, 1824, 4, 1, 64, "32", "f32", "f32", False, False, 17),
        # next tokens of four answers about one image: few rows, latency
        shared_case("shared_tokens", 4, 1, 32, 32, 128, 1, 1136, 64, "bf16", "f32", False),
        # 16 requests about the same document in pages, drafted blocks of 6
        shared_case("shared_paged", 16, 6, 32, 8, 128, 1, 16001, 700, "bf16", "f32", True),
        # three videos with 24 questions between them, drafted blocks of 8
        shared_case("shared_groups", 24, 8, 28, 4, 128, 3, 6528, 515, "bf16", "bf16", True),
        # 16 answers about one long video, the largest
        shared_case("shared_long", 16, 8, 64, 8, 128, 1, 65500, 300, "bf16", "bf16", False),
        # fp32 cache of the small workload
        shared_case("shared_f32", 5, 4, 4, 1, 64, 2, 608, 60, "f32", "f32", False),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((28, 4), (32, 32), (32, 8), (64, 8), (8, 2), (4, 1), (12, 4))


def draw(rng):
    op = rng.choice(("rope", "append", "append", "shared", "shared", "shared"))
    if op == "rope":
        D, sections, per_axis = rng.choice(((128, "16,24,24", False), (128, "64", False), (80, "20,20", True),
                                            (64, "16,16", True), (64, "32", False), (128, "8,12,12", False),
                                            (72, "12,12,12", True)))
        H = rng.choice((1, 5, 12, 16, 32, 36, 40))
        T = log_int(rng, 1, 65536)
        dtype = rng.choice(("bf16", "bf16", "f32"))
        T = max(1, min(T, (1 << 28) // (H * D)))
        return {k: v for k, v in rope_case("", T, H, D, sections, dtype, rng.choice((1e4, 5e5, 1e6)), per_axis,
                                           rng.random() < 0.3, rng.choice((0, 0, 100000)),
                                           rng.choice((0, 8, 512))).items() if k != "name"}
    Hq, Hkv = rng.choice(HEADS)
    D = rng.choice((64, 128, 128))
    if op == "append":
        video = rng.random() < 0.4
        sections = {(128, True): "16,24,24", (64, True): "8,12,12"}.get((D, video), str(D // 2))
        src, dtype = rng.choice((("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")))
        B = rng.randint(1, 32)
        paged = rng.random() < 0.6
        ragged = paged and rng.random() < 0.6
        if ragged:
            T = log_int(rng, B, 65536)
        else:
            T = B * log_int(rng, 1, max(1, 65536 // B))
        bytes_each = sum(2 if t == "bf16" else 4 for t in (src, dtype))
        while T * (Hq + 2 * Hkv) * D * bytes_each > 65536 * 80 * 128 * 4:
            T = max(B, T // 2 // B * B)
        return {k: v for k, v in append_case("", B, T, Hq, Hkv, D, sections, src, dtype, paged, ragged,
                                             rng.choice((0, 5, 100, 3001)), rng.choice((1e4, 1e6)),
                                             video).items() if k != "name"}
    f32 = rng.random() < 0.15
    B = rng.randint(2, 6) if f32 else log_int(rng, 2, 64)
    k = rng.choice((1, 4)) if f32 else rng.choice((1, 1, 3, 5, 6, 8))
    if f32:
        Hq, Hkv = rng.choice(((4, 1), (8, 2), (12, 4)))
    G = rng.choice((1, 1, min(2, B), min(3, B), min(5, B)))
    prefix = log_int(rng, 40, 2000) if f32 else log_int(rng, 100, 65536)
    while B * k * Hq * prefix > 16 * 8 * 64 * 65500 or (not f32 and G * prefix * Hkv > 1 << 21):
        prefix = prefix // 2 + rng.randint(1, 30)
    return {k_: v for k_, v in shared_case("", B, k, Hq, Hkv, D, G, prefix, max(k, log_int(rng, 16, 1000)),
                                           "f32" if f32 else "bf16", "f32" if f32 else rng.choice(("f32", "bf16")),
                                           rng.random() < 0.5).items() if k_ != "name"}


# ------------------------------------------------------------------ inputs

def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def parse(sections):
    return [int(s) for s in sections.split(",")]


def grid_positions(rows, axes, start):
    """Positions of `rows` tokens from `start` on: text (all axes alike), a
    patch grid (height, width) or a video grid (time, height, width)."""
    i = torch.arange(rows, device="cuda")
    if axes == 1:
        p = [i]
    else:
        side = max(1, int(math.sqrt(rows / (8 if axes == 3 else 1))))
        p = [(i // side) % side, i % side]
        if axes == 3:
            p = [i // (side * side)] + p
    return torch.stack(p).to(torch.int32) + start


def append_rows(case):
    """First row of each sequence (its pieces of T rows differ, some may be
    empty) and the positions that its cache holds already."""
    B, T = case["B"], case["T"]
    r = random.Random(T * 64 + B)
    past = [r.randint(0, case["past"]) for _ in range(B)]
    if not case["ragged"]:
        return list(range(0, T + 1, T // B)), past
    return [0] + sorted(r.randint(0, T) for _ in range(B - 1)) + [T], past


def group_sizes(case):
    """Sequences of each group: different ones, at least one each."""
    B, G = case["B"], case["G"]
    total = G * (G + 1) // 2
    sizes = [max(1, B * (g + 1) // total) for g in range(G)]
    sizes[-1] += B - sum(sizes)
    while sizes[-1] < 1:
        i = max(range(G), key=lambda g: sizes[g])
        sizes[i] -= 1
        sizes[-1] += 1
    return sizes


def prefix_lengths(case):
    return [max(1, case["prefix"] - 37 * g) for g in range(case["G"])]


def suffix_lengths(case):
    lo, hi = case["k"], case["suffix"]
    return [lo + (b * 7919 + 13) % (hi - lo + 1) for b in range(case["B"])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    D = case["D"]
    s = {"case": case}
    if case["op"] == "rope":
        T, H = case["T"], case["H"]
        secs = parse(case["sections"])
        buf = normal(gen, (T, H * D + case["gap"]), dt)
        s["x"] = buf[:, :H * D].view(T, H, D)
        s["pos"] = grid_positions(T, len(secs), case["far"] + seed % 7)
        s["sections"] = secs
        return s
    Hq, Hkv, B = case["Hq"], case["Hkv"], case["B"]
    if case["op"] == "append":
        T = case["T"]
        secs = parse(case["sections"])
        qkv = normal(gen, (T, (Hq + 2 * Hkv) * D), DTYPES[case["src"]])
        s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        s["v"] = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        start, past = append_rows(case)
        lens = [past[b] + start[b + 1] - start[b] for b in range(B)]
        s["sections"] = secs
        s["row_start"] = int32(start) if case["ragged"] else None
        s["kv_len"] = int32(lens)
        s["pos"] = grid_positions(T, len(secs), 0) if case["video"] else None
        s["page_table"] = None
        if case["paged"]:
            pages = [max(1, -(-n // PAGE)) for n in lens]
            s["k_cache"], s["v_cache"] = (normal(gen, (sum(pages) + 3, Hkv, PAGE, D), dt) for _ in range(2))
            s["page_table"] = random_table(gen, pages, sum(pages) + 3)
        else:
            s["k_cache"], s["v_cache"] = (normal(gen, (B, max(lens) + 5, Hkv, D), dt) for _ in range(2))
        return s
    G, k = case["G"], case["k"]
    sizes, plens, slens = group_sizes(case), prefix_lengths(case), suffix_lengths(case)
    s["q"] = normal(gen, (B, k, Hq, D), dt)
    s["prefix_len"], s["kv_len"] = int32(plens), int32(slens)
    s["sizes"] = sizes
    s["group_start"] = int32([sum(sizes[:g]) for g in range(G + 1)])
    s["k_prefix"] = s["v_prefix"] = s["prefix_table"] = s["page_table"] = None
    if case["paged"]:
        pp, sp = [-(-n // PAGE) for n in plens], [-(-n // PAGE) for n in slens]
        pool = sum(pp) + sum(sp) + 2
        s["k_cache"], s["v_cache"] = (normal(gen, (pool, Hkv, PAGE, D), dt) for _ in range(2))
        both = random_table(gen, pp + sp, pool)
        s["prefix_table"] = both[:G, :max(pp)].contiguous()
        s["page_table"] = both[G:, :max(sp)].contiguous()
    else:
        s["k_cache"], s["v_cache"] = (normal(gen, (B, max(slens), Hkv, D), dt) for _ in range(2))
        s["k_prefix"], s["v_prefix"] = (normal(gen, (G, max(plens), Hkv, D), dt) for _ in range(2))
    return s


def random_table(gen, pages, pool):
    """Each row's pages, at random places of a pool; unused entries are 0."""
    perm = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
    widest = max(pages)
    first = torch.tensor([sum(pages[:i]) for i in range(len(pages))], device="cuda")[:, None]
    col = torch.arange(widest, device="cuda")[None, :]
    used = col < torch.tensor(pages, device="cuda")[:, None]
    return torch.where(used, perm[torch.where(used, first + col, 0)], 0).to(torch.int32).contiguous()


# ------------------------------------------------------------- plain forms

def angles(pos, sections, theta, per_axis):
    """[T, pairs] angles in 64 bits: pair i of axis a turns by pos[a] times
    theta^(-i / pairs), i counted over all axes or within the axis."""
    axis = torch.repeat_interleave(torch.arange(len(sections), device="cuda"), torch.tensor(sections, device="cuda"))
    pairs = sum(sections)
    if per_axis:
        n = torch.tensor(sections, device="cuda", dtype=torch.float64)[axis]
        first = torch.tensor([sum(sections[:a]) for a in range(len(sections))], device="cuda")[axis]
        e = (torch.arange(pairs, device="cuda") - first) / n
    else:
        e = torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs
    return pos.double()[axis].T * theta ** -e


def rotate(x, ang, sign=1.0):
    """x [T, H, D] in 32 bits, its first 2 pairs channels turned by ang [T, pairs]."""
    n = ang.shape[1]
    c, s = ang.cos().float()[:, None], (sign * ang.sin()).float()[:, None]
    x = x.float()
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat((a * c - b * s, a * s + b * c, x[..., 2 * n:]), -1)


def plain_append(st):
    case = st["case"]
    T, B = case["T"], case["B"]
    t = torch.arange(T, device="cuda")
    start = st["row_start"].long() if st["row_start"] is not None else torch.arange(B + 1, device="cuda") * (T // B)
    b = (t[:, None] >= start[None, 1:]).sum(1)
    p = st["kv_len"].long()[b] - start[b + 1] + t
    pos = st["pos"] if st["pos"] is not None else p.expand(len(st["sections"]), T)
    ang = angles(pos, st["sections"], case["theta"], False)
    dt = DTYPES[case["dtype"]]
    q, k, v = rotate(st["q"], ang).to(dt), rotate(st["k"], ang).to(dt), st["v"].to(dt)
    if st["page_table"] is not None:
        page = st["page_table"].long()[b, p // PAGE]
        st["k_cache"][page, :, p % PAGE] = k
        st["v_cache"][page, :, p % PAGE] = v
    else:
        st["k_cache"][b, p] = k
        st["v_cache"][b, p] = v
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def rows_of(cache, table):
    """Keys or values [n, Hkv, capacity, D] of a contiguous cache or of pages."""
    if table is None:
        return cache.float().transpose(1, 2).contiguous()
    n, pages = table.shape
    Hkv, D = cache.shape[1], cache.shape[3]
    got = cache[table.long()].float().transpose(1, 2).contiguous()
    return got.view(n, Hkv, pages * PAGE, D)


def plain_shared(st):
    case = st["case"]
    B, k, Hq, Hkv, D, G = (case[n] for n in ("B", "k", "Hq", "Hkv", "D", "G"))
    g = Hq // Hkv
    paged = st["page_table"] is not None
    q = st["q"].float().view(B, k, Hkv, g, D).transpose(1, 2).reshape(B, Hkv, k * g, D) / math.sqrt(D)
    # a group's sequences side by side: [G, most, ...], rows past a group's end are not used
    most = max(st["sizes"])
    start = st["group_start"].long()
    seq = start[:G, None] + torch.arange(most, device="cuda")
    used = seq < start[1:, None]
    seq = seq.clamp(max=B - 1)
    kp = rows_of(st["k_cache"] if paged else st["k_prefix"], st["prefix_table"])
    vp = rows_of(st["v_cache"] if paged else st["v_prefix"], st["prefix_table"])
    ks, vs = rows_of(st["k_cache"], st["page_table"]), rows_of(st["v_cache"], st["page_table"])
    qg = q[seq].transpose(1, 2).reshape(G, Hkv, most * k * g, D)
    sp = qg @ kp.transpose(2, 3).contiguous()
    ss = q @ ks.transpose(2, 3).contiguous()
    past = torch.arange(sp.shape[-1], device="cuda") >= st["prefix_len"][:, None]
    sp.masked_fill_(past[:, None, None], -math.inf)
    j = torch.arange(k * g, device="cuda") // g
    last = st["kv_len"][:, None] - k + j
    unseen = torch.arange(ss.shape[-1], device="cuda") > last[..., None]
    ss.masked_fill_(unseen[:, None], -math.inf)
    back = used.nonzero()                       # (group, place) of each sequence, in order

    def by_sequence(x):
        return x.view(G, Hkv, most, k * g, -1).transpose(1, 2)[back[:, 0], back[:, 1]]

    def by_group(x):
        return x[seq].transpose(1, 2).reshape(G, Hkv, most * k * g, -1)

    m = torch.maximum(by_sequence(sp.amax(-1, keepdim=True)), ss.amax(-1, keepdim=True))
    sp.sub_(by_group(m)).exp_()
    ss.sub_(m).exp_()
    total = by_sequence(sp.sum(-1, keepdim=True)) + ss.sum(-1, keepdim=True)
    out = (by_sequence(sp @ vp) + ss @ vs) / total
    lse = m + total.log()
    out = out.view(B, Hkv, k, g, D).transpose(1, 2).reshape(B, k, Hq, D).to(DTYPES[case["out"]])
    return {"out": out, "lse": lse.view(B, Hkv, k, g).transpose(1, 2).reshape(B, k, Hq)}


# ------------------------------------------------------------- entry points

def own_call(st):
    import paper_2505_12728_amd as sd
    case = st["case"]
    if case["op"] == "rope":
        return sd.sd_rope(st["x"], st["pos"], case["theta"], sections=st["sections"], per_axis=case["per_axis"],
                          inverse=case["inverse"])
    if case["op"] == "append":
        q = sd.sd_kv_append(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["kv_len"], case["theta"],
                            pos=st["pos"], sections=st["sections"], row_start=st["row_start"],
                            page_table=st["page_table"])
        return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    out, lse = sd.sd_verify_shared(st["q"], st["k_cache"], st["v_cache"], st["kv_len"], st["prefix_len"],
                                   k_prefix=st["k_prefix"], v_prefix=st["v_prefix"],
                                   prefix_table=st["prefix_table"], group_start=st["group_start"],
                                   page_table=st["page_table"], out_dtype=DTYPES[case["out"]])
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return own_call(state)
    case = state["case"]
    if case["op"] == "rope":
        ang = angles(state["pos"], state["sections"], case["theta"], case["per_axis"])
        return rotate(state["x"], ang, -1.0 if case["inverse"] else 1.0).to(DTYPES[case["dtype"]])
    return plain_append(state) if case["op"] == "append" else plain_shared(state)


# ------------------------------------------------------------------- work

def work(case):
    size = {"bf16": 2, "f32": 4}
    es, D = size[case["dtype"]], case["D"]
    if case["op"] == "rope":
        n = case["T"] * case["H"] * D
        axes = len(parse(case["sections"]))
        return {"bytes": 2 * n * es + 4 * axes * case["T"], "flops": 3 * n}
    Hq, Hkv, B = case["Hq"], case["Hkv"], case["B"]
    if case["op"] == "append":
        n = case["T"] * (Hq + 2 * Hkv) * D
        axes = len(parse(case["sections"])) if case["video"] else 0
        return {"bytes": n * (size[case["src"]] + es) + 4 * axes * case["T"] + 8 * B, "flops": 3 * n}
    k, rows = case["k"], case["k"] * Hq
    keys = sum(prefix_lengths(case)) + sum(suffix_lengths(case))
    seen = sum(n * m for n, m in zip(prefix_lengths(case), group_sizes(case))) + sum(suffix_lengths(case))
    return {"bytes": 2 * keys * Hkv * D * es + B * rows * (D * (es + size[case["out"]]) + 4),
            "flops": 4 * D * rows * seen}


# ------------------------------------------------------------------ exact

def turn64(x, pos, sections, theta, per_axis, sign):
    """Rotation of x [T, H, D] in 64 bits, as a product of complex numbers."""
    turns = []
    for a, n in enumerate(sections):
        i = torch.arange(n, device="cuda", dtype=torch.float64)
        e = i / n if per_axis else (i + sum(sections[:a])) / sum(sections)
        turns.append(pos[a].double()[:, None] * torch.exp(-math.log(theta) * e))
    ang = sign * torch.cat(turns, 1)
    n = ang.shape[1]
    x = x.double()
    z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * torch.polar(
        torch.ones_like(ang), ang)[:, None]
    return torch.cat((z.real, z.imag, x[..., 2 * n:]), -1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return turn64(st["x"], st["pos"], st["sections"], case["theta"], case["per_axis"],
                      -1.0 if case["inverse"] else 1.0)
    if case["op"] == "append":
        T, B = case["T"], case["B"]
        start = st["row_start"].tolist() if st["row_start"] is not None else list(range(0, T + 1, T // B))
        lens = st["kv_len"].tolist()
        places = torch.cat([torch.arange(lens[b] - start[b + 1] + start[b], lens[b]) for b in range(B)]).cuda()
        pos = st["pos"] if st["pos"] is not None else [places] * len(st["sections"])
        args = (pos, st["sections"], case["theta"], False, 1.0)
        q, k, v = turn64(st["q"], *args), turn64(st["k"], *args), st["v"].double()
        kc, vc = st["k_cache"].double(), st["v_cache"].double()
        for b in range(B):
            p, rows = places[start[b]:start[b + 1]], slice(start[b], start[b + 1])
            if st["page_table"] is None:
                kc[b, p], vc[b, p] = k[rows], v[rows]
            else:
                page = st["page_table"][b].long()[p // PAGE]
                kc[page, :, p % PAGE], vc[page, :, p % PAGE] = k[rows], v[rows]
        return {"q": q, "k_cache": kc, "v_cache": vc}
    B, k, Hq, Hkv, D = (case[n] for n in ("B", "k", "Hq", "Hkv", "D"))
    g = Hq // Hkv
    plens, slens = prefix_lengths(case), suffix_lengths(case)
    out = torch.empty(B, k, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, k, Hq, dtype=torch.float64, device="cuda")

    def keys(cache, row, table, length, h):
        if table is None:
            return cache[row, :length, h].double()
        return cache[table[row].long(), h].reshape(-1, D)[:length].double()

    b = 0
    for grp, size in enumerate(group_sizes(case)):
        for h in range(Hkv):
            pk, pv = (keys(st[c + ("_prefix" if st[c + "_prefix"] is not None else "_cache")], grp,
                           st["prefix_table"], plens[grp], h) for c in "kv")
            for i in range(b, b + size):
                sk, sv = (keys(st[c + "_cache"], i, st["page_table"], slens[i], h) for c in "kv")
                x = st["q"][i, :, h * g:(h + 1) * g].double().reshape(k * g, D)
                z = torch.cat((x @ pk.T, x @ sk.T), 1) / math.sqrt(D)
                j = torch.arange(k * g, device="cuda")[:, None] // g
                t = torch.arange(z.shape[1], device="cuda")[None, :] - plens[grp]
                z[t > slens[i] - k + j] = -math.inf
                w = torch.softmax(z, 1)
                out[i, :, h * g:(h + 1) * g] = (w[:, :plens[grp]] @ pv + w[:, plens[grp]:] @ sv).view(k, g, D)
                lse[i, :, h * g:(h + 1) * g] = torch.logsumexp(z, 1).view(k, g)
        b += size
    return {"out": out, "lse": lse}
