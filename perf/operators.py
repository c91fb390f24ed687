"""The paged key-value cache operators as measured calls.

A program that keeps a history longer than one prompt (the frames and actions
of many control steps, many robots whose histories differ in length) keeps its
keys and values in pages.  Per layer it makes three calls: it appends the new
rows' keys and values, normalised and rotated, to the pages (`append`); it
attends from one new token per sequence (`decode`); it attends from the rows
of a prompt, all of them or the recomputed ones (`prefill`).

`run` computes a case by these calls where `own` is true and otherwise in
plain torch operations in 32 bits (angles in 64).

Pages: K [pages][kv heads][page][head dim], V [pages][kv heads][head dim][page];
slot j of sequence s is in page table[s][j // page] at j % page.  A row sees
slot j iff j <= last and (window == 0 or j > last - window or j < sinks); a row
that sees nothing has an output of zeros.
"""
import math

import torch

own = False

ROPE_THETA = 10000.0
RMS_EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
# query heads, key-value heads, head dimension
LAYOUTS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (8, 1, 128), (12, 12, 64), (16, 2, 64), (4, 4, 64)]


def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", heads=32, kv=8, dh=128, page=16, seqs=1, idle=0, len_lo=1, len_hi=1, new_lo=1,
             new_hi=1, keep=1000, window=0, sinks=0, axes=1, rot=128, norm=False, fused=False)
    c.update(kw)
    return c


def listed():
    return [
        # one robot, one new token of a grouped-head layer: nothing but latency
        _case("append", name="append_1", len_lo=277, len_hi=277, norm=True),
        # 64 robots, one new token each, video positions, half of each head rotated
        _case("append", name="append_64", dtype="fp16", seqs=64, page=32, len_lo=500, len_hi=4000, norm=True, axes=3,
              rot=64, fused=True),
        # 16 episodes of the 7B decoder at 50% reuse: 148 of 276 prompt rows each, cut from the fused projection
        _case("append", name="append_16x148_7b", heads=32, kv=32, seqs=16, len_lo=276, len_hi=276, new_lo=276,
              new_hi=276, keep=537, fused=True),
        # the largest: a long video prompt for each of four sequences, of ragged lengths
        _case("append", name="append_video_16k", seqs=4, page=64, len_lo=2500, len_hi=8000, new_lo=2500, new_hi=8000,
              norm=True, axes=3, fused=True),
        # one robot with the 7B prompt cached, its last action token
        _case("decode", name="decode_1x282_7b", heads=32, kv=32, len_lo=282, len_hi=282),
        # 16 robots with two cameras and an action chunk each (589 slots and more), three slots of the batch idle
        _case("decode", name="decode_16_7b", heads=32, kv=32, seqs=16, idle=3, len_lo=500, len_hi=900),
        # one robot with a very long history: the work of few rows is split over the length
        _case("decode", name="decode_1x128k", page=64, len_lo=131072, len_hi=131072),
        # 64 sequences from a few tokens to 16 thousand
        _case("decode", name="decode_64_ragged", dtype="fp16", heads=64, page=32, seqs=64, len_lo=5, len_hi=16384),
        # long streams that see the latest 1000 tokens and the first 4
        _case("decode", name="decode_32_window", heads=28, kv=4, seqs=32, len_lo=700, len_hi=20000, window=1000,
              sinks=4),
        # one control step of a 7B layer at 50% reuse: 148 recomputed rows over 276 slots
        _case("prefill", name="prefill_148_7b", heads=32, kv=32, len_lo=276, len_hi=276, new_lo=276, new_hi=276,
              keep=537),
        # a long prompt: the matrix products bound it
        _case("prefill", name="prefill_8k", page=64, len_lo=8192, len_hi=8192, new_lo=8192, new_hi=8192),
        # chunks of ragged prompts behind cached prefixes, with a window and first tokens, heads of 64
        _case("prefill", name="prefill_16_window", dtype="fp16", heads=16, kv=2, dh=64, rot=64, seqs=16, len_lo=37,
              len_hi=7000, new_lo=20, new_hi=1100, window=500, sinks=8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["append", "decode", "prefill"])
    while True:
        heads, kv, dh = rng.choice(LAYOUTS)
        c = _case(kind, dtype=rng.choice(["bf16", "fp16"]), heads=heads, kv=kv, dh=dh, page=rng.choice([16, 32, 64, 128]),
                  seqs=_log(rng, 1, 128), rot=dh, fused=rng.random() < 0.5)
        c["len_hi"] = _log(rng, 1, {"append": 16384, "decode": 131072, "prefill": 32768}[kind])
        c["len_lo"] = rng.choice([c["len_hi"], _log(rng, 1, c["len_hi"])])
        if kind == "append":
            c["norm"], c["axes"], c["rot"] = rng.random() < 0.5, rng.choice([1, 3]), rng.choice([dh, dh, dh // 2])
        else:
            c["idle"] = rng.choice([0, 0, 1, c["seqs"] // 4])
            if c["idle"] >= c["seqs"]:
                c["idle"] = 0
            if rng.random() < 0.4:
                c["window"], c["sinks"] = _log(rng, 1, 4096), rng.choice([0, 1, 4, 64])
        if kind != "decode" and rng.random() < 0.8:
            c["new_hi"] = _log(rng, 1, c["len_hi"])
            c["new_lo"] = rng.choice([c["new_hi"], _log(rng, 1, c["new_hi"])])
            c["keep"] = rng.choice([1000, 1000, rng.randint(100, 999)])
        w = work(c)
        # the plain forms work on padded batches: what they hold is bounded as well
        padded = c["seqs"] * c["len_hi"] * kv * dh
        scores = c["seqs"] * c["heads"] * (c["new_hi"] if kind == "prefill" else 1) * c["len_hi"]
        if w["bytes"] <= 5e8 and w["flops"] <= 5.5e11 and padded <= 1.1e9 and scores <= 2.2e9:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly on a logarithmic scale."""
    if n == 1:
        return [hi]
    return [max(lo, min(hi, round(lo * (hi / lo) ** (i / (n - 1))))) for i in range(n)]


def _rows(c):
    """For each sequence its length and the slots of its rows (evenly spread over its newest slots)."""
    n = c["seqs"] - c["idle"]
    got = []
    for length, new in zip(_spread(c["len_lo"], c["len_hi"], n), _spread(c["new_lo"], c["new_hi"], n)):
        new = min(new, length)
        rows = max(1, new * c["keep"] // 1000)
        got.append((length, [length - new + (k + 1) * new // rows - 1 for k in range(rows)]))
    return got + [(0, [])] * c["idle"]


def _seen(c, last):
    """How many slots a row sees whose last slot is `last`."""
    if c["window"] == 0 or last < c["window"]:
        return last + 1
    return c["window"] + min(c["sinks"], last + 1 - c["window"])


def _angles(c, positions):
    """Angles in 64 bits, [rows][pairs]: pair i turns by position * theta^(-2 i / rot) of its axis."""
    pairs = c["rot"] // 2
    axis = torch.tensor([a for a, n in enumerate(_pairs(c)) for _ in range(n)], device=positions.device)
    freq = ROPE_THETA ** (-2.0 * torch.arange(pairs, device=positions.device, dtype=torch.float64) / c["rot"])
    return positions[axis].T.double() * freq


def _pairs(c):
    """Rotated pairs of each axis."""
    n = c["rot"] // 2
    return (n,) if c["axes"] == 1 else (n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2)


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    t = TYPES[c["dtype"]]
    order = torch.randperm(c["seqs"], generator=g, device=dev).tolist()
    rows = _rows(c)
    rows = [rows[i] for i in order]
    used = [-(-length // c["page"]) for length, _ in rows]
    most = max(used) + 1
    n_pages = sum(used) + 3
    ids = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    cut = torch.zeros(c["seqs"], dtype=torch.int64)
    cut[1:] = torch.tensor(used[:-1], dtype=torch.int64).cumsum(0)
    column = torch.arange(most, device=dev)
    held = column < torch.tensor(used, device=dev)[:, None]
    at = (cut.to(dev)[:, None] + column).clamp_(max=n_pages - 1)
    s = {"case": c, "page_table": torch.where(held, ids[at], -1).contiguous()}
    s["k_pages"] = torch.randn(n_pages, c["kv"], c["page"], c["dh"], generator=g, device=dev, dtype=t)
    s["v_pages"] = torch.randn(n_pages, c["kv"], c["dh"], c["page"], generator=g, device=dev, dtype=t)
    count = [len(r) for _, r in rows]
    s["longest"], s["most_rows"] = max(length for length, _ in rows), max(count)
    s["lengths"] = torch.tensor([length for length, _ in rows], dtype=torch.int32).to(dev)
    if c["kind"] == "decode":
        s["q"] = torch.randn(c["seqs"], c["heads"], c["dh"], generator=g, device=dev).mul_(2).to(t)
        return s
    n = sum(count)
    s["row_seq"] = torch.tensor([i for i, k in enumerate(count) for _ in range(k)], dtype=torch.int32).to(dev)
    s["row_slot"] = torch.tensor([j for _, r in rows for j in r], dtype=torch.int32).to(dev)
    begin = torch.zeros(c["seqs"] + 1, dtype=torch.int32)
    begin[1:] = torch.tensor(count, dtype=torch.int32).cumsum(0)
    s["row_begin"] = begin.to(dev)
    if c["kind"] == "prefill":
        s["q"] = torch.randn(n, c["heads"], c["dh"], generator=g, device=dev).mul_(2).to(t)
        return s
    if c["fused"]:  # views of the fused projection's rows
        qkv = torch.randn(n, c["heads"] + 2 * c["kv"], c["dh"], generator=g, device=dev, dtype=t)
        s["q"], s["k"], s["v"] = qkv.split([c["heads"], c["kv"], c["kv"]], dim=1)
    else:
        s["q"], s["k"], s["v"] = (torch.randn(n, h, c["dh"], generator=g, device=dev, dtype=t)
                                  for h in (c["heads"], c["kv"], c["kv"]))
    if c["norm"]:
        s["q_norm"], s["k_norm"] = (torch.randn(c["dh"], generator=g, device=dev).mul_(0.1).add_(1).to(t)
                                    for _ in range(2))
    if c["axes"] == 3:  # frames of 16 x 16 patches, the first frame far from the start of the recording
        far = int(torch.randint(1000, 100000, (), generator=g, device=dev))
        j = s["row_slot"]
        s["positions"] = torch.stack([far + j // 256, j % 256 // 16, j % 16]).contiguous()
    return s


def _normed(x, w):
    if w is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + RMS_EPS) * w.float()


def _rotated(x, cos, sin):
    n = cos.shape[-1]
    a, b, rest = x[..., :n], x[..., n:2 * n], x[..., 2 * n:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], dim=-1)


def _plain_append(s, c):
    j = s["row_slot"]
    angle = _angles(c, s["positions"] if "positions" in s else j[None])
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _rotated(_normed(s["q"].float(), s.get("q_norm")), cos, sin).to(s["q"].dtype)
    k = _rotated(_normed(s["k"].float(), s.get("k_norm")), cos, sin).to(s["k"].dtype)
    page = s["page_table"][s["row_seq"].long(), (j // c["page"]).long()].long()
    s["k_pages"][page, :, (j % c["page"]).long()] = k
    s["v_pages"][page, :, :, (j % c["page"]).long()] = s["v"]
    return q, s["k_pages"], s["v_pages"]


def _plain_attend(s, c, q, last):
    """q [seqs][rows][heads][dh], last [seqs][rows] (-1: sees nothing), padded; the same shape back."""
    n, rows, heads, dh = q.shape
    columns = -(-s["longest"] // c["page"])
    table = s["page_table"][:, :columns].long().clamp(min=0)
    k = s["k_pages"][table].permute(0, 2, 1, 3, 4).reshape(n, c["kv"], columns * c["page"], dh).float()
    v = s["v_pages"][table].permute(0, 2, 1, 4, 3).reshape(n, c["kv"], columns * c["page"], dh).float()
    q = q.float().reshape(n, rows, c["kv"], heads // c["kv"], dh).permute(0, 2, 3, 1, 4).reshape(n, c["kv"], -1, dh)
    slot = torch.arange(columns * c["page"], device=q.device)
    seen = slot <= last[..., None]
    if c["window"]:
        seen = seen & ((slot > last[..., None] - c["window"]) | (slot < c["sinks"]))
    scores = (q @ k.transpose(-1, -2)).view(n, c["kv"], heads // c["kv"], rows, -1).mul_(1 / math.sqrt(dh))
    scores = scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True).view(n, c["kv"], -1, 1)
    o = p.view(n, c["kv"], -1, columns * c["page"]) @ v
    o = torch.where(total > 0, o / total, 0).to(s["q"].dtype)
    return o.view(n, c["kv"], heads // c["kv"], rows, dh).permute(0, 3, 1, 2, 4).reshape(n, rows, heads, dh)


def _plain_prefill(s, c):
    begin = s["row_begin"].long()
    place = begin[:-1, None] + torch.arange(s["most_rows"], device=begin.device)
    held = place < begin[1:, None]
    place = place.clamp(max=s["q"].shape[0] - 1)
    last = torch.where(held, s["row_slot"][place], -1)
    o = _plain_attend(s, c, s["q"][place], last)
    seq = s["row_seq"].long()
    return o[seq, torch.arange(seq.shape[0], device=seq.device) - begin[seq]]


def run(state):
    c = state["case"]
    if own:
        from paper_2608_10824_amd.paged import PagedCache
        cache = PagedCache(state["k_pages"], state["v_pages"], state["page_table"])
        if c["kind"] == "append":
            q = cache.append(state["q"], state["k"], state["v"], state["row_seq"], state["row_slot"],
                             positions=state.get("positions"), rope_pairs=_pairs(c), rope_theta=ROPE_THETA,
                             q_norm=state.get("q_norm"), k_norm=state.get("k_norm"), rms_eps=RMS_EPS)
            return q, state["k_pages"], state["v_pages"]
        if c["kind"] == "decode":
            return cache.decode(state["q"], state["lengths"], window=c["window"], sinks=c["sinks"])
        return cache.prefill(state["q"], state["row_slot"], state["row_begin"], window=c["window"], sinks=c["sinks"])
    if c["kind"] == "append":
        return _plain_append(state, c)
    if c["kind"] == "decode":
        return _plain_attend(state, c, state["q"][:, None], state["lengths"][:, None] - 1)[:, 0]
    return _plain_prefill(state, c)


def work(case):
    c = case
    rows = _rows(c)
    n = sum(len(r) for _, r in rows) if c["kind"] != "decode" else c["seqs"]
    width = 2 * c["dh"]  # bytes of one head of one row
    if c["kind"] == "append":  # q, k, v in and out once; three flops for a value's norm, three for its rotation
        lists = n * 4 * (2 + (3 if c["axes"] == 3 else 0))
        values = n * c["dh"] * (c["heads"] + c["kv"])
        return {"bytes": 2 * n * (c["heads"] + 2 * c["kv"]) * width + lists, "flops": 6 * values}
    pairs = held = 0
    for length, slots in rows:
        if c["kind"] == "decode":
            slots = [length - 1] if length else []
        if not slots:
            continue
        pairs += sum(_seen(c, j) for j in slots)
        # slots that one row at least sees
        first = max(0, slots[0] - c["window"] + 1) if c["window"] else 0
        held += slots[-1] + 1 - first + min(c["sinks"], first)
    return {"bytes": 2 * n * c["heads"] * width + 2 * held * c["kv"] * width, "flops": 4 * c["dh"] * c["heads"] * pairs}


def _exact_append(s, c):
    rows = s["q"].shape[0]
    j = s["row_slot"].long()
    where = s["positions"].double() if "positions" in s else j[None].double()
    pairs = c["rot"] // 2
    step = torch.exp(-math.log(ROPE_THETA) / pairs * torch.arange(pairs, device=j.device, dtype=torch.float64))
    turn = torch.cat([torch.outer(where[a], f) for a, f in enumerate(step.split(_pairs(c)))], dim=1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def made(x, w):
        x = x.double()
        if w is not None:
            x = x / ((x * x).sum(-1, keepdim=True) / c["dh"] + RMS_EPS).sqrt() * w.double()
        z = torch.complex(x[..., :pairs].contiguous(), x[..., pairs:2 * pairs].contiguous()) * turn
        x[..., :pairs], x[..., pairs:2 * pairs] = z.real, z.imag
        return x

    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    flat = (s["page_table"].long()[s["row_seq"].long(), j // c["page"]] * c["kv"])[:, None] + torch.arange(
        c["kv"], device=j.device)
    flat = flat.view(-1)
    off = (j % c["page"]).repeat_interleave(c["kv"])
    k_pages.view(-1, c["page"], c["dh"])[flat, off] = made(s["k"], s.get("k_norm")).reshape(rows * c["kv"], -1)
    v_pages.view(-1, c["dh"], c["page"])[flat, :, off] = s["v"].double().reshape(rows * c["kv"], -1)
    return made(s["q"], s.get("q_norm")), k_pages, v_pages


def _exact_attend(s, c):
    lengths, table = s["lengths"].tolist(), s["page_table"].tolist()
    n = c["seqs"]
    if c["kind"] == "decode":
        begin, lasts = list(range(n + 1)), s["lengths"].long() - 1
    else:
        begin, lasts = s["row_begin"].tolist(), s["row_slot"].long()
    group = c["heads"] // c["kv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    for i in range(n):
        if begin[i] == begin[i + 1] or lengths[i] == 0:
            continue
        pages = torch.tensor(table[i][:-(-lengths[i] // c["page"])], device=out.device)
        last = lasts[begin[i]:begin[i + 1], None]
        slot = torch.arange(lengths[i], device=out.device)[None]
        hidden = slot > last
        if c["window"]:
            hidden |= (slot <= last - c["window"]) & (slot >= c["sinks"])
        for h in range(c["kv"]):
            k = s["k_pages"][pages, h].reshape(-1, c["dh"])[:lengths[i]].double()
            v = s["v_pages"][pages, h].transpose(1, 2).reshape(-1, c["dh"])[:lengths[i]].double()
            for a in range(h * group, (h + 1) * group):
                z = s["q"][begin[i]:begin[i + 1], a].double() @ k.T / c["dh"] ** 0.5
                z[hidden] = -math.inf
                out[begin[i]:begin[i + 1], a] = torch.softmax(z, 1) @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s, s["case"]) if case["kind"] == "append" else _exact_attend(s, s["case"])
