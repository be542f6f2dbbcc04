"""The operators on the K/V cache through the C ABI, against plain float64 forms.

Tolerances count roundings.  u = 2^-24 is half a step of fp32, U = 2^-8 of bf16;
a pair (hi, lo) of bf16 holds a value to U^2 = 2^-16.

append: a norm's sum of hd squares is off by at most hd u relative, its root,
quotient and the two products by a few more; the rotary factors are rounded to
fp32 and the two products added: (hd / 2 + 12) u of |x| + |y| for a rotated pair
(x, y) covers all.  Rows returned in bf16 add U of the value, cached keys and
values of bf16 models 2^-16.

attend: with S the largest sum |q_d k_d| / sqrt(hd), a score is off by at most
E = S (2^-15 + hd u) (queries and the dropped lo lo products 2^-16 each; fp32
caches: S hd u), so a weight by 2 E relative, the weights' own pairs and the
dropped lo lo by 2^-15 more, sums of n keys by n u and the exponent's argument
(log2 units, below 2^7) by 2^7 u each; every output is a mean of values, so its
error is at most that times the largest |v|.  The same roundings are independent
of each other, which the norm of the error over a whole output shows: it stays
below 2e-5 of the output's (an estimate of 5e-6: four roundings of 2^-18.6 rms).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
u, U = 2.0 ** -24, 2.0 ** -8


class Cache:
    """A cache, its model and their buffers."""

    def __init__(self, rv, dtype, hq, hkv, hd, batch, max_len, layers=1, max_block=64):
        import torch
        self.rv, self.dims, self.dtype, self.batch, self.max_len = rv, (hq, hkv, hd), dtype, batch, max_len
        cfg = rv.rv_config(layers, 256, hq, hkv, hd, 128, 16, rv.RV_BF16 if dtype == "bf16" else rv.RV_F32, 1e-5,
                           10000.0, 0.02)
        self.weights = torch.empty(rv.rv_model_bytes(cfg), dtype=torch.uint8, device="cuda")
        self.model = rv.rv_init_weights(cfg, 0, self.weights)
        self.buf = torch.empty(rv.rv_cache_bytes(self.model, batch, max_len, max_block, 1), dtype=torch.uint8,
                               device="cuda")
        torch.cuda.synchronize()
        self.h = rv.rv_cache_create(self.model, batch, max_len, max_block, 1, self.buf)

    def span(self, which, dtype):
        at, n = self.rv.rv_debug_cache_span(self.h, which)
        return self.buf[at:at + n].view(dtype)

    def read_all(self, layer=0):
        """K and V of every position, [batch][max_len][hkv][hd]."""
        import torch
        _, hkv, hd = self.dims
        k, v = (torch.empty((self.batch * self.max_len, hkv * hd), device="cuda") for _ in range(2))
        self.rv.rv_cache_read(self.h, layer, [0] * self.batch, [self.max_len] * self.batch, k, v)
        return [x.view(self.batch, self.max_len, hkv, hd).cpu().double().numpy() for x in (k, v)]

    def __del__(self):
        if getattr(self, "h", None):
            self.rv.rv_cache_free(self.h)
            self.rv.rv_model_free(self.model)


def rows_of(n, width, seed, io="f32", std=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = std * torch.randn((n, width), generator=g, device="cuda")
    return x.to(torch.bfloat16) if io == "bf16" else x


def f64(t):
    return t.double().cpu().numpy()


def pair(x):
    """What a bf16 cache holds of a float32 array's values."""
    import torch
    t = torch.from_numpy(np.asarray(x, dtype=np.float32))
    hi = t.to(torch.bfloat16).float()
    return (hi + (t - hi).to(torch.bfloat16).float()).double().numpy()


# ------------------------------------------------------------------- append, read

def ref_append(x, n, hd, pos, gain, rotate):
    """(rows, the scale |x| + |y| of each element's rotated pair)."""
    x = x.reshape(-1, n, hd)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5) * gain
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    size = np.concatenate([abs(a) + abs(b)] * 2, -1)
    if rotate:
        ang = pos[:, None, None] * 10000.0 ** (-2 * np.arange(hd // 2) / hd)
        x = np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)
    return x, size


APPEND = [  # type, rows' type, heads, positions, counts, gains of q and k, rotate
    ("bf16", "f32", (8, 2, 32), [0, 63, 31], [1, 1, 1], (True, True), True),
    ("bf16", "bf16", (8, 2, 64), [5, 0, 97], [7, 0, 33], (True, False), True),
    ("bf16", "f32", (4, 4, 128), [31, 64, 0], [34, 64, 100], (False, True), True),
    ("bf16", "f32", (5, 1, 128), [3], [129], (True, True), True),
    ("bf16", "bf16", (4, 2, 128), [17, 40], [15, 16], (False, False), False),
    ("bf16", "f32", (12, 3, 32), [100, 1], [2, 130], (True, True), True),
    ("f32", "f32", (4, 4, 64), [127], [21], (False, False), True),
    ("f32", "bf16", (8, 2, 128), [0, 33, 2, 60], [0, 40, 1, 5], (True, True), True),
    ("f32", "f32", (4, 1, 32), [1000, 7], [37, 64], (True, True), True),
    ("bf16", "f32", (4, 1, 64), [0] * 40, [1] * 40, (True, True), True),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{c[0]}-{c[1]}-{'x'.join(map(str, c[2]))}-{max(c[4])}")
@pytest.mark.parametrize("form", ["fused", "in-place"])
def test_append_and_read(rv, gpu, case, form):
    import torch
    dtype, io, (hq, hkv, hd), pos, n, (qn, kn), rotate = case
    B, M = len(pos), sum(n)
    c = Cache(rv, dtype, hq, hkv, hd, B, max(p + x for p, x in zip(pos, n)) + 3)
    # something at every position, so that what the call leaves alone shows
    old = rows_of(B * c.max_len, 2 * hkv * hd, 3)
    rv.rv_cache_append(c.h, 0, [0] * B, [c.max_len] * B, None, old[:, :hkv * hd], old[:, hkv * hd:], None, rotate=False)
    before = c.read_all()
    qkv = rows_of(M, (hq + 2 * hkv) * hd, 5, io)
    q, k, v = qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:]
    want_q, want_k, want_v = f64(q), f64(k), f64(v)
    gains = 1 + 0.2 * rows_of(2, hd, 6)
    out = q if form == "in-place" else torch.empty((M, hq * hd), dtype=q.dtype, device="cuda")
    rv.rv_cache_append(c.h, 0, pos, n, q, k, v, out, q_gain=gains[0] if qn else None, k_gain=gains[1] if kn else None,
                       rotate=rotate)
    at = np.concatenate([p + np.arange(x) for p, x in zip(pos, n)])
    seq = np.repeat(np.arange(B), n)
    g = f64(gains)
    ref, size = ref_append(want_q, hq, hd, at, g[0] if qn else None, rotate)
    tol = (hd / 2 + 12) * u * size + (U * abs(ref) if io == "bf16" else 0) + 1e-30
    assert (abs(f64(out).reshape(ref.shape) - ref) <= tol).all()
    ref_k, size_k = ref_append(want_k, hkv, hd, at, g[1] if kn else None, rotate)
    ref_v = want_v.reshape(-1, hkv, hd)
    after = c.read_all()
    held = 2.0 ** -16 if dtype == "bf16" else 0
    for got, was, ref, size in ((after[0], before[0], ref_k, size_k), (after[1], before[1], ref_v, 0 * ref_v)):
        assert (abs(got[seq, at] - ref) <= (hd / 2 + 12) * u * size + held * abs(ref) + 1e-30).all()
        got, was = got.copy(), was.copy()
        got[seq, at] = was[seq, at] = 0
        np.testing.assert_array_equal(got, was)
    # rows in their own type, and the inspection copy of one sequence
    ko, vo = (torch.empty((M, hkv * hd), dtype=q.dtype, device="cuda") for _ in range(2))
    rv.rv_cache_read(c.h, 0, pos, n, ko, vo)
    for got, ref in ((ko, after[0][seq, at]), (vo, after[1][seq, at])):
        want = torch.from_numpy(ref.reshape(M, -1)).float().to(q.dtype)
        assert torch.equal(got.cpu(), want)
    b = int(np.argmax(n))
    shape = (2, hkv, n[b], hd) if dtype == "bf16" else (hkv, n[b], hd)
    ek, ev = (torch.empty(shape, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
              for _ in range(2))
    rv.rv_debug_export_kv(c.h, 0, b, pos[b], n[b], ek, ev)
    for got, ref in ((ek, after[0]), (ev, after[1])):
        got = f64(got).sum(0) if dtype == "bf16" else f64(got)
        np.testing.assert_array_equal(got, ref[b, pos[b]:pos[b] + n[b]].transpose(1, 0, 2))


# ------------------------------------------------------------------- copy, fork

MOVES = {
    "swap": ([1, 0], [0, 1]), "ring": ([1, 2, 3, 4, 0], [0, 1, 2, 3, 4]), "fan": ([2] * 5, [0, 1, 3, 4, 5]),
    "ring-and-tails": ([1, 2, 0, 0, 3, 5], [0, 1, 2, 3, 4, 5]), "front": ([1, 3, 5], [0, 1, 2]),
    "chain": ([1, 2, 3, 4, 5], [0, 1, 2, 3, 4]), "one": ([4], [2]), "two-rings": ([1, 0, 3, 2], [0, 1, 2, 3]),
}


@pytest.mark.parametrize("name", MOVES)
@pytest.mark.parametrize("dtype,heads", [("bf16", (4, 1, 128)), ("bf16", (8, 2, 32)), ("f32", (4, 2, 64)),
                                         ("f32", (4, 1, 128))])
def test_copy_moves_everything_at_once(rv, gpu, name, dtype, heads):
    import torch
    hq, hkv, hd = heads
    B, max_len, layers = 6, 197, 3
    c = Cache(rv, dtype, hq, hkv, hd, B, max_len, layers)
    kv_len = 256
    bits = torch.int16 if dtype == "bf16" else torch.int32
    names = [rv.RV_SPAN_K, rv.RV_SPAN_V] + ([rv.RV_SPAN_K_LO, rv.RV_SPAN_V_LO] if dtype == "bf16" else [])
    planes = [c.span(w, bits).view(layers, B, hkv, kv_len // 64, 64 * hd) for w in names]
    ids = c.span(rv.RV_SPAN_IDS, torch.int32).view(B, max_len)
    for p in planes + [ids]:
        p.copy_(torch.randint(-30000, 30000, p.shape, device="cuda"))
    src, dst = MOVES[name]
    lens = [(1, 2, 64, 65, 66, 130, 197)[(i * 3 + len(name)) % 7] for i in range(len(src))]
    want, want_ids = [p.clone() for p in planes], ids.clone()
    for a, b, n in zip(src, dst, lens):
        for w, p in zip(want, planes):
            w[:, b, :, :(n - 1 + 63) // 64] = p[:, a, :, :(n - 1 + 63) // 64]
        want_ids[b, :n] = ids[a, :n]
    rv.rv_cache_copy(c.h, src, dst, lens)
    for w, p in zip(want, planes):
        assert torch.equal(w, p)
    assert torch.equal(want_ids, ids)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("f32", 32)])
def test_forks_read_what_they_continue(rv, gpu, dtype, hd):
    """Forks of forks, a copy of a fork, a fork made private, a new prefill of ids."""
    hkv, B, L = 2, 6, 300
    c = Cache(rv, dtype, 4, hkv, hd, B, L)

    def write(b, p, n, seed):
        x = rows_of(n, 2 * hkv * hd, seed)
        at, count = [0] * B, [0] * B
        at[b], count[b] = p, n
        rv.rv_cache_append(c.h, 0, at, count, None, x[:, :hkv * hd], x[:, hkv * hd:], None, rotate=False)

    for b in range(B):
        write(b, 0, L, b)
    k, v = c.read_all()

    def check(b, expect):  # expect: (sequence of the first state, first position, end)
        got = c.read_all()
        for ref, x in zip((k, v), got):
            for a, lo, hi in expect:
                np.testing.assert_array_equal(x[b, lo:hi], ref[a, lo:hi])

    rv.rv_cache_fork(c.h, 0, 200, [1, 2])       # 3 whole tiles shared, 192..198 copied
    check(1, [(0, 0, 199)])
    check(2, [(0, 0, 199)])
    rv.rv_cache_fork(c.h, 2, 130, [3])          # of a fork: its tiles lie with 0
    check(3, [(0, 0, 129)])
    rv.rv_cache_copy(c.h, [3, 1], [4, 5], [100, 199])  # copies of forks are their own
    check(4, [(0, 0, 99)])
    check(5, [(0, 0, 198)])
    for b, p in ((0, 10), (1, 191), (2, 0), (3, 127)):
        with pytest.raises(rv.RVError) as e:
            write(b, p, 1, 9)
        assert e.value.name == "RV_E_STATE"
    with pytest.raises(rv.RVError) as e:
        rv.rv_cache_copy(c.h, [4], [0], [10])
    assert e.value.name == "RV_E_STATE"
    write(4, 0, 99, 50)
    write(0, 199, 50, 51)
    check(1, [(0, 0, 199)])
    check(3, [(0, 0, 129)])
    rv.rv_cache_copy(c.h, [1], [1], [200])      # its own copy
    write(1, 0, 100, 52)
    check(2, [(0, 0, 199)])
    check(0, [(0, 0, 199)])
    # 2 and 3 re-forked together with their source's slot reused once they are gone
    rv.rv_cache_fork(c.h, 5, 150, [0, 2, 3])
    for b in (0, 2, 3):
        check(b, [(0, 0, 149)])


# ------------------------------------------------------------------- attend

def ref_attend(q, k, v, pos, n, G):
    """q [rows][hq][hd], k and v [B][L][hkv][hd] -> out, and the bounds' S and largest |v|."""
    out = np.zeros_like(q)
    hd, row, S = q.shape[-1], 0, 0.0
    for b in range(len(n)):
        for r in range(n[b]):
            p = pos[b] + r + 1
            for h in range(q.shape[1]):
                kk, vv = k[b, :p, h // G], v[b, :p, h // G]
                s = kk @ q[row, h] / np.sqrt(hd)
                S = max(S, (abs(kk) @ abs(q[row, h])).max() / np.sqrt(hd))
                w = np.exp(s - s.max())
                out[row, h] = (w / w.sum()) @ vv
            row += 1
    return out, S


ATTEND = [  # type, rows' type, heads, positions of the first rows, counts, forks (source, length, targets)
    # decode, nothing shared: one key, tile edges, more than one run
    ("bf16", "f32", (4, 1, 128), [0, 62, 63, 64, 65], [1] * 5, []),
    ("bf16", "bf16", (8, 2, 64), [0, 1, 127, 128, 700], [1, 2, 4, 3, 1], []),
    ("bf16", "f32", (16, 1, 32), [2500], [1], []),
    ("bf16", "f32", (8, 8, 128), [1100, 3], [1, 1], []),
    # decode over a shared prompt; padded sequences of the batch
    ("bf16", "f32", (4, 1, 128), [200, 260, 192, 300], [1] * 4, [(0, 193, [1, 2, 3])]),
    ("bf16", "bf16", (8, 1, 64), [400, 390, 0, 385, 500], [1, 1, 0, 1, 1], [(0, 386, [1, 2, 3, 4])]),
    ("bf16", "f32", (8, 2, 128), [1300] * 12, [1] * 12, [(3, 1250, [0, 1, 2] + list(range(4, 12)))]),
    ("bf16", "f32", (32, 8, 64), [130 + i for i in range(40)], [1] * 40, [(0, 130, list(range(1, 40)))]),
    # blocks: many queries, ragged counts, a member that the group leaves out
    ("bf16", "f32", (8, 2, 128), [300, 333, 257], [31, 31, 31], [(0, 258, [1, 2])]),
    ("bf16", "bf16", (8, 1, 32), [70, 640, 64, 100, 200], [40, 1, 17, 40, 33], [(1, 65, [0, 2, 3, 4])]),
    ("bf16", "f32", (6, 1, 64), [0, 65, 10], [150, 60, 1], []),
    ("bf16", "f32", (4, 4, 128), [129, 64, 128, 640], [10, 9, 3, 7], [(3, 129, [0, 1, 2])]),
    # rows before the end of what is shared: only the tiles below them count as shared
    ("bf16", "f32", (8, 2, 64), [100, 400, 390], [3, 3, 3], [(1, 391, [0, 2])]),
    # forks of forks: two groups, one inside the other's tiles
    ("bf16", "f32", (4, 1, 128), [520, 530, 540, 550, 90, 70], [2] * 6, [(0, 460, [1, 2, 3]), (1, 65, [4, 5])]),
    ("f32", "f32", (4, 4, 64), [0, 64, 63], [1, 1, 2], []),
    ("f32", "f32", (4, 1, 128), [200, 230, 193], [21, 21, 21], [(0, 193, [1, 2])]),
    ("f32", "bf16", (8, 2, 32), [1000, 990], [1, 5], [(0, 900, [1])]),
    ("f32", "f32", (8, 2, 128), [400] * 9, [1] * 9, [(8, 390, list(range(8)))]),
]


def filled(rv, case, layers=1):
    dtype, io, (hq, hkv, hd), pos, n, forks = case
    B = len(pos)
    c = Cache(rv, dtype, hq, hkv, hd, B, max(p + x for p, x in zip(pos, n)) + 5, layers, max_block=max(max(n), 8))
    x = rows_of(B * c.max_len, 2 * hkv * hd, 21)
    rv.rv_cache_append(c.h, layers - 1, [0] * B, [c.max_len] * B, None, x[:, :hkv * hd], x[:, hkv * hd:], None,
                       rotate=False)
    for src, length, dst in forks:
        rv.rv_cache_fork(c.h, src, length, dst)
    return c


def check_attend(rv, c, case, out, q, layer=0):
    dtype, io, (hq, hkv, hd), pos, n, _ = case
    k, v = c.read_all(layer)
    ref, S = ref_attend(f64(q).reshape(-1, hq, hd), k, v, pos, n, hq // hkv)
    got = f64(out).reshape(ref.shape)
    keys = max(p + x for p, x in zip(pos, n))
    rel = 2 * S * hd * u + keys * u + 2.0 ** 7 * u * 2
    if dtype == "bf16":
        rel += 2 * S * 2.0 ** -15 + 2.0 ** -15
    tol = rel * abs(v).max() + (U * abs(ref) if io == "bf16" else 0)
    assert np.isfinite(got).all()
    assert (abs(got - ref) <= tol).all(), (abs(got - ref) / tol).max()
    norm = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert norm < (2e-5 if io == "f32" else 4e-3), norm


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{c[0]}-{c[1]}-{'x'.join(map(str, c[2]))}-{c[3][0]}-{c[4][0]}"
                         f"-{len(c[3])}")
def test_attend(rv, gpu, case):
    import torch
    dtype, io, (hq, hkv, hd), pos, n, forks = case
    c = filled(rv, case)
    # rows as part of a wider tensor, and in the rows' place
    wide = rows_of(sum(n), (hq + 2 * hkv) * hd, 22, io)
    q = wide[:, :hq * hd]
    kept = wide.clone()
    out = torch.empty((sum(n), hq * hd), dtype=q.dtype, device="cuda")
    rv.rv_cache_attend(c.h, 0, pos, n, q, out)
    assert torch.equal(wide, kept)
    check_attend(rv, c, case, out, q)
    again = torch.empty_like(out)
    rv.rv_cache_attend(c.h, 0, pos, n, q, again)
    assert torch.equal(out, again)
    rv.rv_cache_attend(c.h, 0, pos, n, q, q)
    assert torch.equal(out, q)
    assert torch.equal(wide[:, hq * hd:], kept[:, hq * hd:])


@pytest.mark.parametrize("case", [ATTEND[1], ATTEND[4], ATTEND[8], ATTEND[9], ATTEND[15], ATTEND[16]],
                         ids=["few", "shared", "many", "ragged", "f32", "f32-few"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_masked_places_count_for_nothing(rv, gpu, case, bad):
    """Values that are not finite behind a row's position, in its block or in the cache, do not reach it;
    rows that see one get it."""
    import torch
    dtype, io, (hq, hkv, hd), pos, n, forks = case
    B, M = len(pos), sum(n)
    c = filled(rv, case)
    q = rows_of(M, hq * hd, 23, io)
    clean, out = torch.empty_like(q), torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, pos, n, q, clean)
    # everything behind the last row, and the last row's own key and value where the block has others
    at = [p + x - (1 if x > 1 else 0) for p, x in zip(pos, n)]
    count = [c.max_len - a for a in at]
    x = rows_of(sum(count), 2 * hkv * hd, 24)
    x[:] = bad
    rv.rv_cache_append(c.h, 0, at, count, None, x[:, :hkv * hd], x[:, hkv * hd:], None, rotate=False)
    rv.rv_cache_attend(c.h, 0, pos, n, q, out)
    row = 0
    for b in range(B):
        keep = n[b] - (1 if n[b] > 1 else 0)
        assert torch.equal(out[row:row + keep], clean[row:row + keep])
        if keep < n[b]:
            assert not torch.isfinite(out[row + keep]).any()
        row += n[b]


def test_attend_long_and_large(rv, gpu):
    """A long prompt in many runs, and as many rows as the workspace takes."""
    import torch
    case = ("bf16", "f32", (4, 1, 128), [9000] * 10, [1] * 10, [(0, 8990, list(range(1, 10)))])
    c = filled(rv, case)
    q = rows_of(10, 512, 25)
    out = torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, case[3], case[4], q, out)
    check_attend(rv, c, case, out, q)
    case = ("bf16", "bf16", (2, 2, 64), [64, 70], [1024, 1024], [(0, 65, [1])])
    c = filled(rv, case)
    q = rows_of(2048, 128, 26, "bf16")
    out = torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, case[3], case[4], q, out)
    check_attend(rv, c, case, out, q)


# ------------------------------------------------------------------- together

def test_a_layer_of_forked_sequences(rv, gpu):
    """append to a prompt, fork it, append to the forks, attend, reorder, attend: on a side stream,
    in the second of two layers."""
    import torch
    hq, hkv, hd, B, L = 8, 2, 64, 5, 150
    st = torch.cuda.Stream()
    c = Cache(rv, "bf16", hq, hkv, hd, B, 400, layers=2)
    gains = 1 + 0.2 * rows_of(2, hd, 1)
    prompt = rows_of(L, (hq + 2 * hkv) * hd, 2)
    step = rows_of(3 * B, (hq + 2 * hkv) * hd, 3)
    torch.cuda.synchronize()

    def split(x):
        return x[:, :hq * hd], x[:, hq * hd:(hq + hkv) * hd], x[:, (hq + hkv) * hd:]

    order = [2, 2, 0, 4, 1]
    with torch.cuda.stream(st):
        q0, q1, q2 = (torch.empty((n, hq * hd), device="cuda") for n in (L, 3 * B, B))
        q, k, v = split(prompt)
        rv.rv_cache_append(c.h, 1, [0] * B, [L] + [0] * (B - 1), q, k, v, q0, gains[0], gains[1])
        rv.rv_cache_fork(c.h, 0, L + 1, range(1, B))
        q, k, v = split(step)
        rv.rv_cache_append(c.h, 1, [L] * B, [3] * B, q, k, v, q1, gains[0], gains[1])
        out = torch.empty_like(q1)
        rv.rv_cache_attend(c.h, 1, [L] * B, [3] * B, q1, out)
        # the beams of the next step: copies of the forks, their own from now on
        k1, v1 = c.read_all(1)
        rv.rv_cache_copy(c.h, order, range(B), [L + 4] * B)
        k2, v2 = c.read_all(1)
        q2.copy_(rows_of(B, hq * hd, 4))
        out2 = torch.empty_like(q2)
        rv.rv_cache_attend(c.h, 1, [L + 2] * B, [1] * B, q2, out2)
        st.synchronize()
    # the whole in float64 from the inputs
    g = f64(gains)
    pk = ref_append(f64(prompt)[:, hq * hd:(hq + hkv) * hd], hkv, hd, np.arange(L), g[1], True)[0]
    at = np.tile(L + np.arange(3), B)
    sq = ref_append(f64(step)[:, :hq * hd], hq, hd, at, g[0], True)[0]
    sk = ref_append(f64(step)[:, hq * hd:(hq + hkv) * hd], hkv, hd, at, g[1], True)[0].reshape(B, 3, hkv, hd)
    pv = f64(prompt)[:, (hq + hkv) * hd:].reshape(L, hkv, hd)
    sv = f64(step)[:, (hq + hkv) * hd:].reshape(B, 3, hkv, hd)
    K = np.stack([np.concatenate([pk, sk[b]]) for b in range(B)])
    V = np.stack([np.concatenate([pv, sv[b]]) for b in range(B)])
    np.testing.assert_allclose(k1[:, :L + 3], K, atol=2.0 ** -16 * abs(K).max() + 60 * u * abs(K).max() * 2)
    ref, _ = ref_attend(sq, K, V, [L] * B, [3] * B, hq // hkv)
    assert np.linalg.norm(f64(out).reshape(ref.shape) - ref) < 2e-5 * np.linalg.norm(ref)
    np.testing.assert_array_equal(k2[:, :L + 3], k1[order][:, :L + 3])
    np.testing.assert_array_equal(v2[:, :L + 3], v1[order][:, :L + 3])
    ref, _ = ref_attend(f64(q2).reshape(B, hq, hd), K[order], V[order], [L + 2] * B, [1] * B, hq // hkv)
    assert np.linalg.norm(f64(out2).reshape(ref.shape) - ref) < 2e-5 * np.linalg.norm(ref)


def test_calls_in_a_captured_graph(rv, gpu):
    """A captured layer step, replayed over new rows with the program's own work between the replays."""
    import torch
    hq, hkv, hd, B = 8, 2, 128, 6
    prompt = rows_of(600, 2 * hkv * hd, 1)
    x = torch.zeros((B, (hq + 2 * hkv) * hd), device="cuda")
    q_out, out = (torch.empty((B, hq * hd), device="cuda") for _ in range(2))

    def forked():
        c = Cache(rv, "bf16", hq, hkv, hd, B, 700)
        rv.rv_cache_append(c.h, 0, [0] * B, [600] + [0] * (B - 1), None, prompt[:, :hkv * hd], prompt[:, hkv * hd:],
                           None)
        rv.rv_cache_fork(c.h, 0, 601, range(1, B))
        return c

    def step(c):
        rv.rv_cache_append(c.h, 0, [600] * B, [1] * B, x[:, :hq * hd], x[:, hq * hd:(hq + hkv) * hd],
                           x[:, (hq + hkv) * hd:], q_out)
        rv.rv_cache_attend(c.h, 0, [600] * B, [1] * B, q_out, out)

    c, eager = forked(), forked()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c)
        rv.rv_cache_copy(c.h, [2, 3], [3, 2], [602, 602])
    for i in range(4):
        x.copy_(rows_of(B, x.shape[1], 30 + i))
        graph.replay()
        got = out.clone()
        k, v = c.read_all()
        torch.cuda.synchronize()
        step(eager)
        assert torch.equal(out, got)
        ke, ve = eager.read_all()
        order = [0, 1, 3, 2, 4, 5]
        np.testing.assert_array_equal(k[order, :601], ke[:, :601])
        np.testing.assert_array_equal(v[order, :601], ve[:, :601])


def test_arguments_of_the_binding(rv, gpu):
    import torch
    c = Cache(rv, "bf16", 4, 2, 64, 3, 100)
    assert rv.rv_cache_dims(c.h) == (3, 4, 2, 64)
    k = rows_of(3, 128, 1)
    q = rows_of(3, 256, 1)
    rv.rv_cache_append(c.h, 0, [0] * 3, [1] * 3, q, k, k, q)
    for pos, n, a in (([0] * 2, [1] * 2, (q, k, k, q)), ([0] * 3, [1, 1], (q, k, k, q)),
                      ([0] * 3, [1, 1, 2], (q, k, k, q)), ([0] * 3, [1] * 3, (q, q, k, q)),
                      ([0] * 3, [1] * 3, (q, q, q, q)), ([0] * 3, [1] * 3, (k, k, k, k)),
                      ([0] * 3, [1] * 3, (q, k.double(), k, q)), ([0] * 3, [1] * 3, (q, k, k.bfloat16(), q)),
                      ([0] * 3, [1] * 3, (q, k.T.contiguous().T, k, q)), ([0] * 3, [1] * 3, (q, k.cpu(), k, q)),
                      ([0] * 3, [1] * 3, (q, k, k, q[:, :128])), ([0] * 3, [1] * 3, (q, k, k, None))):
        with pytest.raises((ValueError, rv.RVError)):
            rv.rv_cache_append(c.h, 0, pos, n, *a)
    for gain in (torch.ones(32, device="cuda"), torch.ones(64, device="cuda").double(),
                 torch.ones(128, device="cuda")[::2]):
        with pytest.raises(ValueError):
            rv.rv_cache_append(c.h, 0, [0] * 3, [1] * 3, q, k, k, q, q_gain=gain)
    with pytest.raises(rv.RVError):
        rv.rv_cache_attend(c.h, 0, [0] * 3, [1] * 3, k, k)
    with pytest.raises(ValueError):
        rv.rv_cache_attend(c.h, 0, [0] * 3, [1] * 3, q, q.bfloat16())
    with pytest.raises(rv.RVError):
        rv.rv_cache_read(c.h, 0, [0] * 3, [1] * 3, q, q.clone())
    with pytest.raises(ValueError):
        rv.rv_cache_copy(c.h, [0, 1], [2], [1])
    with pytest.raises(rv.RVError):
        rv.rv_cache_attend(c.h, 0, [0] * 3, [1] * 3, rows_of(3, 264, 1)[:, 2:258], q[:, :256].clone())
    none = torch.empty((0, 256), device="cuda")
    rv.rv_cache_attend(c.h, 0, [0] * 3, [0] * 3, none, none)


def test_attend_more_keys_than_the_last_level_cache(rv, gpu):
    """Decode steps over 300 MB of keys and values (nontemporal loads), ragged; float64 on the card."""
    import torch
    hq, hkv, hd, B = 16, 8, 128, 33
    lens = [1, 64, 1300] + [1000 + 7 * b for b in range(B - 3)]
    c = Cache(rv, "bf16", hq, hkv, hd, B, 1300)
    x = rows_of(sum(lens), 2 * hkv * hd, 41)
    rv.rv_cache_append(c.h, 0, [0] * B, lens, None, x[:, :hkv * hd], x[:, hkv * hd:], None, rotate=False)
    k, v = (torch.empty((sum(lens), hkv * hd), device="cuda") for _ in range(2))
    rv.rv_cache_read(c.h, 0, [0] * B, lens, k, v)
    q = rows_of(B, hq * hd, 42)
    out = torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, [n - 1 for n in lens], [1] * B, q, out)
    ref, at = torch.empty((B, hq, hd), dtype=torch.float64, device="cuda"), 0
    for b, n in enumerate(lens):
        kk, vv = (t[at:at + n].double().view(n, hkv, hd).transpose(0, 1) for t in (k, v))
        s = (kk @ q[b].double().view(hkv, hq // hkv, hd).transpose(1, 2).contiguous()) / hd ** 0.5
        ref[b] = (torch.softmax(s, 1).transpose(1, 2) @ vv).reshape(hq, hd)
        at += n
    assert float(torch.linalg.norm(out.view(B, hq, hd).double() - ref)) < 2e-5 * float(torch.linalg.norm(ref))


@pytest.mark.parametrize("counts", [[700, 0, 1, 1, 0, 3], [1] * 6, [0, 0, 0, 0, 0, 9]])
def test_attend_rows_of_few_sequences(rv, gpu, counts):
    """One sequence with many rows among others with few or none, over a prompt that all share."""
    import torch
    case = ("bf16", "f32", (4, 2, 64), [70 + 3 * b for b in range(6)], counts, [(0, 65, [1, 2, 3, 4, 5])])
    c = filled(rv, case)
    q = rows_of(sum(counts), 4 * 64, 43)
    out = torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, case[3], counts, q, out)
    check_attend(rv, c, case, out, q)


@pytest.mark.parametrize("dtype,hkv,B", [("bf16", 4, 80), ("f32", 16, 150)])
def test_attend_many_forks_of_unlike_lengths(rv, gpu, dtype, hkv, B):
    """More sequences than run at once: their workgroups start in the order of their keys."""
    import torch
    counts = [0 if b % 11 == 3 else 1 + b % 2 for b in range(B)]
    case = (dtype, "f32", (hkv, hkv, 32), [66 + b * 37 % 300 for b in range(B)], counts, [(0, 66, list(range(2, B, 2)))])
    c = filled(rv, case)
    q = rows_of(sum(counts), hkv * 32, 44)
    out = torch.empty_like(q)
    rv.rv_cache_attend(c.h, 0, case[3], counts, q, out)
    check_attend(rv, c, case, out, q)


def test_attend_in_place_with_two_strides(rv, gpu):
    import torch
    c = filled(rv, ("bf16", "f32", (4, 2, 64), [70, 3], [1, 2], []))
    wide = rows_of(3, 512, 45)
    flat = wide.view(-1)[:3 * 256].view(3, 256)
    with pytest.raises(rv.RVError, match="RV_E_ARG"):
        rv.rv_cache_attend(c.h, 0, [70, 3], [1, 2], wide[:, :256], flat)
    apart = torch.empty((3, 256), device="cuda")
    rv.rv_cache_attend(c.h, 0, [70, 3], [1, 2], wide[:, :256], apart)
    rv.rv_cache_attend(c.h, 0, [70, 3], [1, 2], wide[:, :256], wide[:, :256])
    assert torch.equal(wide[:, :256], apart)
