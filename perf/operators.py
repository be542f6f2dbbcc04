"""The operators on the K/V cache, as cases to time.

  append   rv_cache_append and rv_cache_read: query and key rows of a projection
           are normalised for each head (models that have such norms) and
           rotated to their positions, keys and values go to the cache, and the
           cached rows are read back as a program that keeps them elsewhere too
           (a second tier, another process) does.
  copy     rv_cache_copy: sequences of the cache are copied to other slots in
           one step, all layers: a prompt to its continuations, the survivors of
           a batch to its front, the beams of a step to their new order.
  attend   rv_cache_attend: attention of query rows over a layer of the cache,
           where all sequences may continue one prompt that the cache holds
           once (rv_cache_fork).

With `own` false the same is computed with elementary torch operations on plain
tensors.  A bf16 model's cache holds a value as the pair hi = bf16(x),
lo = bf16(x - hi); an fp32 model's holds it as it is.

Head counts are those of the model shapes of `workload`; draws take others too.
"""
import math

import numpy as np
import torch

own = False

EPS, BASE = 1e-5, 10000.0
TILE = 64  # positions in a tile of the cache

# query heads, kv heads, head_dim, type
HEADS = {
    "tiny": (4, 4, 64, "f32"),
    "tiny-gqa": (8, 2, 32, "bf16"),
    "1b": (32, 8, 64, "bf16"),
    "8b": (32, 8, 128, "bf16"),
    "14b": (40, 8, 128, "bf16"),
    "70b": (64, 8, 128, "bf16"),
    "f32-wide": (8, 2, 128, "f32"),
}
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


def _append(name, heads, io, batch, rows_lo, rows_hi, pos_lo, pos_hi, norm):
    return {"name": name, "kind": "append", "heads": heads, "io": io, "batch": batch, "rows_lo": rows_lo,
            "rows_hi": rows_hi, "pos_lo": pos_lo, "pos_hi": pos_hi, "norm": norm}


def _copy(name, heads, layers, batch, lo, hi, how):
    return {"name": name, "kind": "copy", "heads": heads, "layers": layers, "batch": batch, "len_lo": lo,
            "len_hi": hi, "how": how}


def _attend(name, heads, io, batch, shared, own_lo, own_hi, rows_lo, rows_hi):
    return {"name": name, "kind": "attend", "heads": heads, "io": io, "batch": batch, "shared": shared,
            "own_lo": own_lo, "own_hi": own_hi, "rows_lo": rows_lo, "rows_hi": rows_hi}


def listed():
    return [
        # one verify block of the small fp32 model: all launch latency
        _append("append-tiny-f32", "tiny", "f32", 1, 21, 21, 127, 127, False),
        # a verify block of four sequences, a model with norms of queries and keys
        _append("append-14b-block", "14b", "f32", 4, 43, 43, 2000, 2047, True),
        # ragged prompts of a batch, rows in bf16 as a bf16 projection gives them
        _append("append-8b-prompts", "8b", "bf16", 6, 300, 1100, 0, 0, True),
        # two short sequences exchanged, the small fp32 model
        _copy("copy-tiny-swap", "tiny", 2, 2, 30, 100, "reorder"),
        # one prompt to the three other slots of a draft model's cache, all its layers
        _copy("copy-1b-fan", "1b", 16, 4, 301, 301, "fan"),
        # sixteen ragged sequences in a new order (beams), eight layers of the 8B shape
        _copy("copy-8b-reorder", "8b", 8, 16, 512, 2048, "reorder"),
        # the small fp32 model: four verify blocks after one prompt
        _attend("attend-tiny-f32", "tiny", "f32", 4, 128, 22, 60, 21, 21),
        # one decode step of one user, nothing to share
        _attend("attend-8b-one", "8b", "f32", 1, 0, 1024, 1024, 1, 1),
        # a draft model's ragged steps of sixteen users, nothing to share
        _attend("attend-1b-ragged", "1b", "bf16", 16, 0, 300, 1900, 1, 9),
        # thirty-two continuations of one prompt, a decode step each
        _attend("attend-8b-decode", "8b", "bf16", 32, 4001, 1, 600, 1, 1),
        # sixteen continuations of one prompt, a verify block each
        _attend("attend-8b-verify", "8b", "f32", 16, 2048, 40, 500, 31, 31),
        # sixty-four continuations of a long document, a decode step each
        _attend("attend-70b-document", "70b", "f32", 64, 32768, 16, 2000, 1, 1),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "copy", "attend", "attend"])
    heads = rng.choice(list(HEADS))
    if kind == "append":
        batch = _logint(rng, 1, 64)
        hi = _logint(rng, 1, max(1, 1200 // batch))
        lo = rng.randint(max(1, hi // 3), hi)
        pos = _logint(rng, 1, 8000)
        case = _append("", heads, rng.choice(["f32", "bf16"]), batch, lo, hi, rng.randint(0, pos), pos,
                       rng.random() < 0.5)
    elif kind == "copy":
        batch = _logint(rng, 2, 16)
        hi = _logint(rng, 20, 2000)
        case = _copy("", heads, rng.randint(1, 4), batch, rng.randint(2, hi), hi,
                     rng.choice(["reorder", "fan", "front"]))
    else:
        batch = _logint(rng, 1, 48)
        rows = _logint(rng, 1, 60)
        shared = _logint(rng, 30, 16000) if rng.random() < 0.75 else 0
        hi = _logint(rng, rows, 1500)
        case = _attend("", heads, rng.choice(["f32", "bf16"]), batch, shared, rng.randint(rows, max(rows, hi)), hi,
                       rng.randint(1, rows), rows)
        # scores of the plain form, and the work, stay below the largest listed case's
        while batch * rows * HEADS[heads][0] * (shared + hi) > 10 ** 8:
            batch = case["batch"] = max(1, batch // 2)
            if batch == 1:
                shared = case["shared"] = shared // 2
    del case["name"]
    return case


# ------------------------------------------------------------------- inputs

def _dims(case):
    return HEADS[case["heads"]]


def _lens(key, lo, hi, n):
    """n whole numbers in [lo, hi], the first of them hi: a case's sizes, the same for every seed."""
    g = np.random.default_rng([key, lo, hi, n])
    v = g.integers(lo, hi + 1, size=n).astype(np.int32)
    v[0] = hi
    return v


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pair(x):
    hi = x.to(torch.bfloat16)
    return hi, (x - hi.float()).to(torch.bfloat16)


def _moves(case):
    """The slots that a copy reads and writes, and the committed tokens each brings."""
    B = case["batch"]
    g = np.random.default_rng([3, B])
    lens = _lens(4, case["len_lo"], case["len_hi"], B)
    if case["how"] == "fan":
        src, dst = np.zeros(B - 1, np.int32), np.arange(1, B, dtype=np.int32)
    elif case["how"] == "front":  # every second sequence lives on
        src = np.arange(1, B, 2, dtype=np.int32)
        dst = np.arange(len(src), dtype=np.int32)
    else:  # a new order in which some continue twice and some not at all
        dst = np.arange(B, dtype=np.int32)
        src = ((dst + 1) % B).astype(np.int32)
        twice = g.integers(0, B, size=B // 4)
        src[twice] = g.integers(0, B, size=B // 4)
    return src, dst, lens[src]


def _append_inputs(case, seed):
    hq, hkv, hd, _ = _dims(case)
    B = case["batch"]
    rows = _lens(1, case["rows_lo"], case["rows_hi"], B)
    pos = _lens(2, case["pos_lo"], case["pos_hi"], B)
    g = _generator(seed)
    qkv = torch.randn((int(rows.sum()), (hq + 2 * hkv) * hd), generator=g, device="cuda").to(IO[case["io"]])
    gains = 1 + 0.1 * torch.randn((2, hd), generator=g, device="cuda") if case["norm"] else None
    return rows, pos, qkv, gains


def _attend_inputs(case, seed):
    """Values of K and V: the prompt's [2][hkv][shared][hd], the sequences' own [2][B][hkv][longest][hd]."""
    hq, hkv, hd, dtype = _dims(case)
    B = case["batch"]
    rows = _lens(1, case["rows_lo"], case["rows_hi"], B)
    tail = np.maximum(_lens(2, case["own_lo"], case["own_hi"], B), rows)
    g = _generator(seed)
    q = torch.randn((int(rows.sum()), hq * hd), generator=g, device="cuda").to(IO[case["io"]])
    prompt = torch.randn((2, hkv, case["shared"], hd), generator=g, device="cuda")
    mine = torch.randn((2, B, hkv, int(tail.max()), hd), generator=g, device="cuda")
    if dtype == "bf16":  # the values that pairs can hold
        prompt = torch.stack([p.float() for p in _pair(prompt)]).sum(0)
        mine = torch.stack([p.float() for p in _pair(mine)]).sum(0)
    return rows, tail, q, prompt, mine


# ------------------------------------------------------------------- the library's handles

class _Cache:
    """A cache of one layer stack and the model that it belongs to, as a program holds them."""

    def __init__(self, heads, layers, batch, max_len, max_rows):
        import paper_2505_18629_amd as rv
        hq, hkv, hd, dtype = heads
        self.rv = rv
        cfg = rv.rv_config(layers, 256, hq, hkv, hd, 128, 16, rv.RV_BF16 if dtype == "bf16" else rv.RV_F32, EPS, BASE,
                           0.02)
        self.weights = torch.empty(rv.rv_model_bytes(cfg), dtype=torch.uint8, device="cuda")
        self.model = rv.rv_init_weights(cfg, 0, self.weights)
        self.buf = torch.empty(rv.rv_cache_bytes(self.model, batch, max_len, max_rows, 1), dtype=torch.uint8,
                               device="cuda")
        torch.cuda.synchronize()
        self.handle = rv.rv_cache_create(self.model, batch, max_len, max_rows, 1, self.buf)

    def span(self, which, dtype):
        at, n = self.rv.rv_debug_cache_span(self.handle, which)
        return self.buf[at:at + n].view(dtype)

    def __del__(self):
        if getattr(self, "handle", None):
            self.rv.rv_cache_free(self.handle)
        if getattr(self, "model", None):
            self.rv.rv_model_free(self.model)


# ------------------------------------------------------------------- prepare

def prepare(case, seed):
    return {"append": _prepare_append, "copy": _prepare_copy, "attend": _prepare_attend}[case["kind"]](case, seed)


def _prepare_append(case, seed):
    hq, hkv, hd, dtype = heads = _dims(case)
    rows, pos, qkv, gains = _append_inputs(case, seed)
    M, B = len(qkv), case["batch"]
    io = IO[case["io"]]
    s = {"kind": "append", "heads": heads, "pos": pos, "rows": rows, "gains": gains,
         "q": qkv[:, :hq * hd], "k": qkv[:, hq * hd:(hq + hkv) * hd], "v": qkv[:, (hq + hkv) * hd:]}
    if own:
        s["cache"] = _Cache(heads, 1, B, int((pos + rows).max()), int(rows.max()))
        s["q_out"] = torch.empty((M, hq * hd), dtype=io, device="cuda")
        s["k_out"], s["v_out"] = (torch.empty((M, hkv * hd), dtype=io, device="cuda") for _ in range(2))
        return s
    seq = np.repeat(np.arange(B), rows)
    at = np.concatenate([p + np.arange(r) for p, r in zip(pos, rows)])
    s["seq"], s["at"] = torch.from_numpy(seq).cuda(), torch.from_numpy(at.astype(np.int64)).cuda()
    shape = (2, B, int((pos + rows).max()), hkv * hd)
    s["hi"] = torch.zeros(shape, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    s["lo"] = torch.zeros_like(s["hi"]) if dtype == "bf16" else None
    return s


def _prepare_copy(case, seed):
    hq, hkv, hd, dtype = heads = _dims(case)
    B, layers = case["batch"], case["layers"]
    src, dst, lens = _moves(case)
    max_len = case["len_hi"] + 1
    kv_len = -(-max_len // TILE) * TILE
    elem = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = (layers, B, hkv, kv_len * hd)
    s = {"kind": "copy", "src": src, "dst": dst, "lens": lens, "tile": TILE * hd}
    if own:
        s["cache"] = c = _Cache(heads, layers, B, max_len, 1)
        names = [c.rv.RV_SPAN_K, c.rv.RV_SPAN_V] + ([c.rv.RV_SPAN_K_LO, c.rv.RV_SPAN_V_LO] if dtype == "bf16" else [])
        s["planes"] = [c.span(w, elem).view(shape) for w in names]
        s["ids"] = c.span(c.rv.RV_SPAN_IDS, torch.int32).view(B, max_len)
    else:
        s["planes"] = [torch.empty(shape, dtype=elem, device="cuda") for _ in range(4 if dtype == "bf16" else 2)]
        s["ids"] = torch.empty((B, max_len), dtype=torch.int32, device="cuda")
    g = _generator(seed)
    for p in s["planes"]:
        for layer in p:
            layer.normal_(generator=g)
    s["ids"].copy_(torch.randint(0, 1 << 17, (B, max_len), generator=g, device="cuda"))
    return s


def _prepare_attend(case, seed):
    hq, hkv, hd, dtype = heads = _dims(case)
    B, shared = case["batch"], case["shared"]
    rows, tail, q, prompt, mine = _attend_inputs(case, seed)
    pos = (shared + tail - rows).astype(np.int32)
    s = {"kind": "attend", "heads": heads, "pos": pos, "rows": rows, "tail": tail, "shared": shared, "q": q}
    if own:
        s["cache"] = c = _Cache(heads, 1, B, shared + int(tail.max()), max(int(rows.max()), 1))
        rv, zero = c.rv, np.zeros(B, np.int32)

        def write(at, n, kv):  # kv: [2][rows][hkv * hd]
            rv.rv_cache_append(c.handle, 0, at, n, None, kv[0], kv[1], None, rotate=False)

        if shared:
            first = zero.copy()
            first[0] = shared
            write(zero, first, prompt.transpose(1, 2).reshape(2, shared, hkv * hd))
            if B > 1:
                rv.rv_cache_fork(c.handle, 0, shared + 1, np.arange(1, B, dtype=np.int32))
        t = mine.transpose(2, 3).reshape(2, B, -1, hkv * hd)
        write(zero + shared, tail, torch.cat([t[:, b, :n] for b, n in enumerate(tail)], 1))
        s["out"] = torch.empty_like(q)
        return s
    # the rows of the batch as a rectangle, and the keys of its own that a row may see
    R = int(rows.max())
    at = np.zeros((B, R), np.int64)
    seen = np.zeros((B, R), np.int64)
    row0 = np.cumsum(rows) - rows
    for b in range(B):
        at[b, :rows[b]] = row0[b] + np.arange(rows[b])
        seen[b, :rows[b]] = tail[b] - rows[b] + 1 + np.arange(rows[b])
        seen[b, rows[b]:] = 1
    s["at"], s["seen"] = torch.from_numpy(at).cuda(), torch.from_numpy(seen).cuda()
    s["valid"] = torch.from_numpy(np.arange(R)[None, :] < rows[:, None]).cuda()
    if dtype == "bf16":
        s["prompt"], s["mine"] = _pair(prompt), _pair(mine)
    else:
        s["prompt"], s["mine"] = (prompt,), (mine,)
    return s


# ------------------------------------------------------------------- run

def run(s):
    if own:
        return {"append": _own_append, "copy": _own_copy, "attend": _own_attend}[s["kind"]](s)
    return {"append": _plain_append, "copy": _plain_copy, "attend": _plain_attend}[s["kind"]](s)


def _own_append(s):
    c, gains = s["cache"], s["gains"]
    c.rv.rv_cache_append(c.handle, 0, s["pos"], s["rows"], s["q"], s["k"], s["v"], s["q_out"],
                         q_gain=None if gains is None else gains[0], k_gain=None if gains is None else gains[1])
    c.rv.rv_cache_read(c.handle, 0, s["pos"], s["rows"], s["k_out"], s["v_out"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_copy(s):
    c = s["cache"]
    c.rv.rv_cache_copy(c.handle, s["src"], s["dst"], s["lens"])
    return {"planes": s["planes"], "ids": s["ids"]}


def _own_attend(s):
    c = s["cache"]
    c.rv.rv_cache_attend(c.handle, 0, s["pos"], s["rows"], s["q"], s["out"])
    return s["out"]


def _plain_append(s):
    hq, hkv, hd, dtype = s["heads"]
    half = hd // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    angle = s["at"].double()[:, None] * torch.pow(torch.tensor(BASE, device="cuda", dtype=torch.float64), -2 * i / hd)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(x, n, gain):
        x = x.float().view(-1, n, hd)
        if gain is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).reshape(-1, n * hd)

    gains = s["gains"] if s["gains"] is not None else (None, None)
    q = turn(s["q"], hq, gains[0]).to(s["q"].dtype)
    out = [q]
    for j, x in enumerate((turn(s["k"], hkv, gains[1]), s["v"].float())):
        if dtype == "bf16":
            s["hi"][j][s["seq"], s["at"]], s["lo"][j][s["seq"], s["at"]] = _pair(x)
            x = s["hi"][j][s["seq"], s["at"]].float() + s["lo"][j][s["seq"], s["at"]].float()
        else:
            s["hi"][j][s["seq"], s["at"]] = x
            x = s["hi"][j][s["seq"], s["at"]]
        out.append(x.to(q.dtype))
    return {"q": out[0], "k": out[1], "v": out[2]}


def _plain_copy(s):
    # what is read is read before anything is written
    for p in s["planes"]:
        got = [p[:, a, :, :-(-(int(n) - 1) // TILE) * s["tile"]].clone() for a, n in zip(s["src"], s["lens"])]
        for b, x in zip(s["dst"], got):
            p[:, b, :, :x.shape[-1]] = x
    got = [s["ids"][a, :int(n)].clone() for a, n in zip(s["src"], s["lens"])]
    for b, x in zip(s["dst"], got):
        s["ids"][b, :len(x)] = x
    return {"planes": s["planes"], "ids": s["ids"]}


def _plain_attend(s):
    hq, hkv, hd, _ = s["heads"]
    B, R = s["at"].shape
    G, shared = hq // hkv, s["shared"]
    prompt, mine = (sum(p.float() for p in x) for x in (s["prompt"], s["mine"]))
    # queries [hkv][B][R * G][hd]
    q = s["q"].float()[s["at"]].view(B, R, hkv, G, hd).permute(2, 0, 1, 3, 4).reshape(hkv, B, R * G, hd) / math.sqrt(hd)
    score = torch.matmul(q.transpose(0, 1), mine[0].transpose(-1, -2).contiguous()).view(B, hkv, R, G, -1)
    hidden = torch.arange(mine.shape[-2], device="cuda") >= s["seen"][..., None]
    score = score.masked_fill(hidden[:, None, :, None], -math.inf).view(B, hkv, R * G, -1)
    top = score.amax(-1, keepdim=True)
    if shared:
        first = torch.matmul(q.reshape(hkv, B * R * G, hd), prompt[0].transpose(-1, -2).contiguous())
        first = first.view(hkv, B, R * G, shared).transpose(0, 1)
        top = torch.maximum(top, first.amax(-1, keepdim=True))
        first = torch.exp(first - top)
    score = torch.exp(score - top)
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score, mine[1])
    if shared:
        total = total + first.sum(-1, keepdim=True)
        back = first.transpose(0, 1).reshape(hkv, B * R * G, shared)
        out = out + torch.matmul(back, prompt[1]).view(hkv, B, R * G, hd).transpose(0, 1)
    out = (out / total).view(B, hkv, R, G, hd).transpose(1, 2).reshape(B, R, hq * hd)
    return out[s["valid"]].to(s["q"].dtype)


# ------------------------------------------------------------------- work

def work(case):
    hq, hkv, hd, dtype = _dims(case)
    io = 4 if case.get("io") == "f32" else 2
    if case["kind"] == "append":
        rows = int(_lens(1, case["rows_lo"], case["rows_hi"], case["batch"]).sum())
        io_bytes = rows * hd * io * ((hq + 2 * hkv) + hq + 2 * hkv)   # rows in; q, and K and V read back, out
        kv_bytes = rows * hd * 4 * 2 * hkv                            # 4 bytes an element in either type
        return {"bytes": io_bytes + kv_bytes, "flops": rows * hd * (hq + hkv) * (7 if case["norm"] else 3)}
    if case["kind"] == "copy":
        src, dst, lens = _moves(case)
        tiles = -(-(lens - 1) // TILE)
        read = {}
        for a, b, n in zip(src, dst, tiles):
            if a != b:
                read[a] = max(read.get(a, 0), int(n))
        written = int(sum(n for a, b, n in zip(src, dst, tiles) if a != b))
        tile = case["layers"] * 2 * hkv * TILE * hd * 4
        return {"bytes": (sum(read.values()) + written) * tile + 8 * int(lens.sum()), "flops": 0}
    rows = _lens(1, case["rows_lo"], case["rows_hi"], case["batch"])
    tail = np.maximum(_lens(2, case["own_lo"], case["own_hi"], case["batch"]), rows)
    keys = float((rows * (case["shared"] + tail - rows) + rows * (rows + 1.0) / 2).sum())
    return {"bytes": 2 * int(rows.sum()) * hq * hd * io + 8 * hkv * hd * (case["shared"] + int(tail.sum())),
            "flops": 4 * hd * hq * keys}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    return {"append": _exact_append, "copy": _exact_copy, "attend": _exact_attend}[case["kind"]](case, seed)


def _exact_append(case, seed):
    hq, hkv, hd, _ = _dims(case)
    rows, pos, qkv, gains = _append_inputs(case, seed)
    x = qkv.double().view(len(qkv), hq + 2 * hkv, hd)
    row0 = np.cumsum(rows) - rows
    for b in range(case["batch"]):
        part = x[row0[b]:row0[b] + rows[b]]
        for first, n, which in ((0, hq, 0), (hq, hkv, 1)):
            y = part[:, first:first + n]
            if gains is not None:
                y = y * gains[which].double() * (y.square().sum(-1, keepdim=True) / hd + EPS).rsqrt()
            # dims i and i + hd/2 are the two parts of a complex number, turned by the position's angle
            z = torch.complex(y[..., :hd // 2].contiguous(), y[..., hd // 2:].contiguous())
            p = torch.arange(int(rows[b]), device="cuda", dtype=torch.float64) + int(pos[b])
            rate = torch.exp(-math.log(BASE) * 2 / hd * torch.arange(hd // 2, device="cuda", dtype=torch.float64))
            angle = p[:, None, None] * rate
            z = z * torch.polar(torch.ones_like(angle), angle)
            part[:, first:first + n] = torch.cat([z.real, z.imag], -1)
    x = x.reshape(len(qkv), -1)
    return {"q": x[:, :hq * hd], "k": x[:, hq * hd:(hq + hkv) * hd], "v": x[:, (hq + hkv) * hd:]}


def _exact_copy(case, seed):
    global own
    was, own = own, False
    try:
        s = _prepare_copy(case, seed)
    finally:
        own = was
    src, dst, lens = _moves(case)
    planes = []
    for p in s["planes"]:
        before, after = p, p.clone()
        per = p.shape[-1] // (s["tile"] // TILE)  # positions a slot holds
        view = (p.shape[0], p.shape[1], p.shape[2], per // TILE, -1)
        for a, b, n in zip(src, dst, lens):
            for t in range((int(n) - 1 + TILE - 1) // TILE):
                after.view(view)[:, b, :, t] = before.view(view)[:, a, :, t]
        planes.append(after)
    ids = s["ids"].clone()
    for a, b, n in zip(src, dst, lens):
        ids[b, :n] = s["ids"][a, :n]
    return {"planes": planes, "ids": ids}


def _exact_attend(case, seed):
    hq, hkv, hd, _ = _dims(case)
    rows, tail, q, prompt, mine = _attend_inputs(case, seed)
    G, shared = hq // hkv, case["shared"]
    out = torch.empty((len(q), hkv, G, hd), dtype=torch.float64, device="cuda")
    row = 0
    for b in range(case["batch"]):
        n, own_keys = int(rows[b]), int(tail[b])
        x = q[row:row + n].double().view(n, hkv, G, hd)
        mask = torch.ones((n, shared + own_keys), dtype=torch.bool, device="cuda").tril(shared + own_keys - n)
        for h in range(hkv):
            k, v = (torch.cat([prompt[j, h], mine[j, b, h, :own_keys]]).double() for j in (0, 1))
            score = x[:, h].reshape(n * G, hd) @ k.T * hd ** -0.5
            score = score.view(n, G, -1).masked_fill(~mask[:, None], -math.inf)
            p = torch.softmax(score, -1).view(n * G, -1)
            out[row:row + n, h] = (p @ v).view(n, G, hd)
        row += n
    return out.view(len(q), hq * hd)
