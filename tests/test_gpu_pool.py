"""The page pool on the GPU against the definitions in 64 bits: rows into pages and back, one new token over pages, packed
prompts; at the sizes, masks and contents where each can go wrong.

Tolerances.  Rows as they are: exact.  8 bits: a value is at most half a step off, s/2 with s = max|x| / 127, and a rounding of
x / s (2^-23 of 127 steps) and of s * c more.  Attention, as a whole (2-norm): bf16 out rounds once (at most 2^-9 of a value, rms
2^-9 / sqrt(3) and less) and may round the probabilities once more: together below 2^-8.  fp32: sums of at most 2^17 products, each
rounded to 2^-24, grow as their root: 2^-24 * 2^8.5 < 3e-5, products split in three parts (2^-21 each) below that.  By element
the contract of the attention of a block: 2e-2 or one step of bf16, and 1e-4 in fp32 for values of order one."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2604_16734_b200.binding import KVC_EINVAL, KVC_OK, KvcError
    from paper_2604_16734_b200.pool import Pool

BF16, F32 = torch.bfloat16, torch.float32
GUARD = 4096


class Guarded:
    """Device tensors between stretches of a known byte, which nobody may write."""

    def __init__(self):
        self.raw = []

    def empty(self, shape, dtype):
        size = math.prod(shape) * dtype.itemsize
        up = -(-size // 256) * 256
        raw = torch.full((GUARD + up + GUARD,), 0xA5, dtype=torch.uint8, device="cuda")
        self.raw.append((raw, size))
        return raw[GUARD:GUARD + size].view(dtype).view(shape)

    def check(self):
        for raw, size in self.raw:
            assert bool((raw[:GUARD] == 0xA5).all()) and bool((raw[GUARD + size:] == 0xA5).all()), "written outside a buffer"


def make_pool(guard, hq, hkv, d, dtype, n_pages, page, fmt, max_seqs=64, **kw):
    rows = n_pages * hkv * page
    nbytes = 2 * rows * d * dtype.itemsize if fmt == "plain" else 2 * rows * d + 2 * (-(-rows * 4 // 256) * 256)
    return Pool(hq, hkv, d, dtype, n_pages, page, fmt, max_seqs=max_seqs, blob=guard.empty((1, nbytes), torch.uint8), **kw)


def fill(pool, gen, bad=float("nan")):
    """Every place of the pool holds something that must not be used."""
    for x in pool.pages(0):
        if x.dtype == torch.int8:
            x.copy_(torch.randint(-128, 128, x.shape, generator=gen, device="cuda", dtype=torch.int16))
        else:
            x.fill_(bad)


def held(pool, k, v):
    """What the pool stands for after rows k, v were written, in 64 bits (by the formula of the codes)."""
    if pool.page_format == "plain":
        return k.double(), v.double()
    out = []
    for x in (k, v):
        x = x.float()
        s = x.abs().amax(-1, keepdim=True) * torch.full_like(x[..., :1], 1 / 127)
        s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
        inv = torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))
        out.append(s.double() * torch.round(x * inv).double())
    return out


def attend64(q, k, v, scale, causal=False):
    """q [m][Hq][d], k, v [n][Hkv][d] in 64 bits -> out, lse; a row without keys gives 0 and -inf."""
    m, hq, d = q.shape
    group = hq // k.shape[1]
    k, v = (x.double().repeat_interleave(group, 1) for x in (k, v))
    z = torch.einsum("mhd,nhd->hmn", q.double(), k) * scale
    if causal:
        z = z.masked_fill(torch.ones(m, k.shape[0], dtype=torch.bool, device=q.device).triu(1), -math.inf)
    if k.shape[0] == 0:
        return torch.zeros(m, hq, d, dtype=torch.float64, device=q.device), torch.full((m, hq), -math.inf, dtype=torch.float64, device=q.device)
    lse = torch.logsumexp(z, -1)
    return torch.einsum("hmn,nhd->mhd", torch.exp(z - lse[..., None]), v), lse.T


def close(got, want, dtype, what):
    g, w = got.double(), want.double()
    assert g.shape == w.shape and bool(torch.isfinite(g).all()), f"{what}: not finite"
    off = (g - w).abs()
    if dtype == BF16:
        step = (got.view(torch.int16).int() - want.to(BF16).view(torch.int16).int()).abs()
        assert bool(((off <= 2e-2) | (step <= 1)).all()), f"{what}: {off.max()}"
    else:
        assert off.max() <= 1e-4 * max(1.0, w.abs().max().item()), f"{what}: {off.max()}"
    if w.norm() > 0:
        assert (g - w).norm() / w.norm() <= (2.0 ** -8 if dtype == BF16 else 3e-5), f"{what}: {(g - w).norm() / w.norm()}"


def close_lse(got, want, dtype, what):
    assert got.shape == want.shape and bool(((got == -math.inf) == (want == -math.inf)).all()), what
    fin = want > -math.inf
    assert bool(((got.double() - want).abs()[fin] <= (2e-3 if dtype == BF16 else 1e-4) * (1 + 1e-2 * want.abs()[fin])).all()), what


# ---------------------------------------------------------------------------------------------------------------------- rows
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", ["plain", "int8"])
@pytest.mark.parametrize("hkv,d,page,n", [(1, 64, 16, 1), (3, 128, 32, 7), (8, 128, 64, 257), (32, 64, 256, 100), (4, 128, 128, 1000)])
@pytest.mark.parametrize("layout", ["tokens", "heads", "wide"])
def test_rows_into_pages_and_back(dtype, fmt, hkv, d, page, n, layout):
    gen = torch.Generator(device="cuda").manual_seed(n + hkv)
    guard = Guarded()
    n_pages = -(-n // page) + 2
    pool = make_pool(guard, hkv, hkv, d, dtype, n_pages, page, fmt)
    fill(pool, gen)
    before = pool.blob.clone()
    shape = {"tokens": (n, hkv, d), "heads": (hkv, n + 3, d), "wide": (n, 2 * hkv + 1, d)}[layout]
    k, v = (torch.randn(shape, generator=gen, device="cuda").mul_(torch.logspace(-3, 3, d, device="cuda")).to(dtype) for _ in range(2))
    if layout == "heads":
        k, v = k[:, 2:n + 2].transpose(0, 1), v[:, 2:n + 2].transpose(0, 1)
    if layout == "wide":
        k, v = k[:, 1:hkv + 1], v[:, 1:hkv + 1]
    slots = torch.randperm(n_pages * page, generator=gen, device="cuda")[:n]
    slots[n // 2] = -1 if n > 1 else slots[0]
    pool.write(0, k, v, slots)
    put = slots >= 0
    pages, rows = slots[put] // page, slots[put] % page
    want_k, want_v = held(pool, k[put], v[put])
    parts = pool.pages(0)
    for part, x, want in zip(parts, (k, v), (want_k, want_v)):
        if fmt == "plain":
            assert torch.equal(part[pages, :, rows], x[put])
        else:
            scale = parts[2 + (x is v)][pages, :, rows].double()
            got = part[pages, :, rows].double() * scale[..., None]
            assert torch.equal(got, want)                          # the same three operations
            x64 = x[put].double()
            top = x64.abs().amax(-1, keepdim=True)
            assert bool(((got - x64).abs() <= top / 127 * (0.5 + 2.0 ** -14)).all()) and bool(((scale - top.squeeze(-1) / 127).abs() <= scale * 2.0 ** -22).all())
    # nothing else was written
    out_k, out_v = pool.read(0, slots)
    assert torch.equal(out_k[put].double(), want_k.to(dtype).double()) and torch.equal(out_v[put].double(), want_v.to(dtype).double())
    assert not out_k[~put].any() and not out_v[~put].any()
    after = pool.blob.clone()
    for part, old in zip(parts, before_parts(pool, before)):
        part[pages, :, rows] = old[pages, :, rows]
    assert torch.equal(pool.blob, before) and not torch.equal(after, before)
    # back into rows of another layout
    wide = guard.empty((2, hkv, n + 1, d), dtype)
    wide.zero_()
    pool.blob.copy_(after)
    pool.read(0, slots, wide[0, :, :n].transpose(0, 1), wide[1, :, :n].transpose(0, 1))
    assert torch.equal(wide[0, :, :n].transpose(0, 1), out_k) and torch.equal(wide[1, :, :n].transpose(0, 1), out_v) and not wide[:, :, n].any()
    assert pool.status() == KVC_OK
    guard.check()


def before_parts(pool, blob):
    other = Pool.__new__(Pool)
    other.__dict__.update({k: v for k, v in pool.__dict__.items() if k not in ("_h", "_calls")})
    other.blob = blob
    return other.pages(0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_eight_bits_of_rows_at_the_edges(dtype, d):
    pool = Pool(2, 2, d, dtype, 2, 16, "int8")
    x = torch.randn(8, 2, d, device="cuda")
    x[0] = 0                                                       # nothing
    x[1] *= 1e-41 if dtype == F32 else 1e-39                       # subnormal: held as zeros
    x[2] = 2.0 ** 127                                              # the largest magnitudes
    x[2, :, ::2] = -torch.finfo(dtype).max
    x[3, 0, 5] = math.inf
    x[4, 1, 7] = math.nan
    x[5, 0] = 0
    x[5, 0, d - 1] = -3.0                                          # one value: exact
    x[6] *= 1e-30
    x[7] = torch.where(x[7] > 0, 127.0, 126.5)                     # a tie: to even
    x = x.to(dtype)
    slots = torch.arange(8, device="cuda") * 3
    pool.write(0, x, x.flip(0), slots)
    k, v = pool.read(0, slots)
    assert torch.equal(torch.nan_to_num(v.flip(0), nan=7e7), torch.nan_to_num(k, nan=7e7))
    assert not k[0].any() and not k[1].any()
    assert bool(k[3, 0].isnan().all()) and bool(k[4, 1].isnan().all()) and bool(torch.isfinite(k[3, 1]).all()) and bool(torch.isfinite(k[4, 0]).all())
    codes, _, scales, _ = pool.pages(0)
    for i in (2, 6):                                               # (what the page stands for; a row read back is rounded to its type)
        stands = codes[slots[i] // 16, :, slots[i] % 16].double() * scales[slots[i] // 16, :, slots[i] % 16].double()[..., None]
        assert bool(torch.isfinite(k[i]).all()) and torch.equal(k[i], stands.to(dtype))
        assert bool(((stands - x[i].double()).abs() <= x[i].double().abs().amax(-1, keepdim=True) / 127 * 0.51).all())
    assert k[5, 0, d - 1] == -3.0 and not k[5, 0, :d - 1].any()
    if dtype == F32:
        assert bool((k[7] == torch.where(x[7] > 126.9, 127.0, 126.0)).all())
    assert pool.status() == KVC_OK


def test_places_outside_the_pool_are_left_out_and_reported():
    guard = Guarded()
    pool = make_pool(guard, 4, 2, 64, BF16, 3, 16, "plain")
    pool.blob.zero_()
    x = torch.ones(5, 2, 64, device="cuda", dtype=BF16)
    pool.write(0, x, x, torch.tensor([0, 48, 2 ** 40, -7, 47], device="cuda"))
    with pytest.raises(KvcError) as e:
        pool._check(pool.status())
    assert e.value.code == KVC_EINVAL
    pool.workspace_init()
    k, v = pool.read(0, torch.tensor([0, 47, 1], device="cuda"))
    assert bool((k[:2] == 1).all()) and bool((v[:2] == 1).all()) and not k[2].any() and pool.status() == KVC_OK
    k, _ = pool.read(0, torch.tensor([0, 48, -1, 2 ** 62], device="cuda"))
    assert bool((k[0] == 1).all()) and not k[1:].any() and pool.status() == KVC_EINVAL
    # a page outside the pool, a length beyond the table, a negative length: the other sequences are right
    pool.workspace_init()
    q = torch.randn(4, 4, 64, device="cuda", dtype=BF16)
    for table, lens in (([[0, 3], [0, -1], [2, 1], [0, 1]], [17, 17, 17, 1]), ([[0, 1], [0, 1], [2, 1], [0, 1]], [33, -4, 17, 1])):
        out, lse = pool.decode(0, q, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        assert pool.status() == KVC_EINVAL
        pool.workspace_init()
        assert torch.isfinite(out[2:]).all() and bool((out[3] == 1).all())
        assert bool((out[2] == out[2, :, :1]).all()) and bool(((out[2] > 0) & (out[2] < 1)).all())   # (one of 17 rows is ones: slot 47)
    assert bool((lse[1] == -math.inf).all()) and not out[1].any()
    guard.check()


def test_calls_with_nothing_to_do():
    pool = Pool(4, 2, 64, BF16, 3, 16)
    none = torch.empty(0, 2, 64, device="cuda", dtype=BF16)
    pool.write(0, none, none, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert pool.read(0, torch.empty(0, dtype=torch.int64, device="cuda"))[0].shape == (0, 2, 64)
    out, lse = pool.decode(0, torch.empty(0, 4, 64, device="cuda", dtype=BF16), torch.empty(0, 1, dtype=torch.int32, device="cuda"),
                           torch.empty(0, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    for lens in ([], [0, 0]):
        out, _ = pool.prompt(torch.empty(0, 4, 64, device="cuda", dtype=BF16), none, none, pool.plan(lens))
        assert out.shape == (0, 4, 64)
    assert pool.launch_count() == 0 and pool.status() == KVC_OK


# ---------------------------------------------------------------------------------------------------------------------- decode
def decode_case(hq, hkv, d, dtype, fmt, page, lens, append, seed, gain=1.0, wide=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    guard = Guarded()
    b = len(lens)
    per = -(-(max(lens) + 1) // page) + 1
    n_pages = b * per + 1
    pool = make_pool(guard, hq, hkv, d, dtype, n_pages, page, fmt, max_seqs=b)
    fill(pool, gen)                                                # behind a sequence's end: NaN
    table = torch.randperm(n_pages, generator=gen, device="cuda")[:b * per].view(b, per).int()
    rows = []
    for i, n in enumerate(lens):
        k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda") for _ in range(2))
        k, v = (k * gain).to(dtype), v.to(dtype)
        pool.write(0, k, v, pool.slots(table[i], n))
        rows.append((k, v))
    # entries behind the page that a sequence reaches are not read
    for i, n in enumerate(lens):
        table[i, -(-(n + append) // page):] = -2 ** 31
    heads = hq + 2 * hkv if wide else hq
    packed = torch.randn(b, heads, d, generator=gen, device="cuda").to(dtype)
    q = packed[:, :hq]
    k_new = v_new = None
    if append:
        k_new, v_new = (packed[:, hq:hq + hkv], packed[:, hq + hkv:]) if wide else (torch.randn(b, hkv, d, generator=gen, device="cuda").to(dtype) for _ in range(2))
    out, lse = guard.empty((b, hq, d), dtype), guard.empty((b, hq), F32)
    before = pool.blob.clone()
    lens_t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pool.decode(0, q, table, lens_t, k_new, v_new, out, lse)
    assert pool.status() == KVC_OK
    guard.check()
    for i, n in enumerate(lens):
        k, v = rows[i]
        if append:
            k, v = torch.cat([k, k_new[i:i + 1]]), torch.cat([v, v_new[i:i + 1]])
        k64, v64 = held(pool, k, v)
        o, z = attend64(q[i:i + 1], k64, v64, 1 / math.sqrt(d))
        close(out[i:i + 1], o, dtype, f"sequence {i} of {n}")
        close_lse(lse[i:i + 1], z, dtype, f"sequence {i} of {n}")
    if append:                                                     # the rows are where they belong, and nothing else was touched
        slots = torch.stack([pool.slots(table[i], 1, n)[0] for i, n in enumerate(lens)])
        k64, v64 = held(pool, k_new, v_new)
        got = pool.read(0, slots)
        assert torch.equal(got[0].double(), k64.to(dtype).double()) and torch.equal(got[1].double(), v64.to(dtype).double())
        for part, old in zip(pool.pages(0), before_parts(pool, before)):
            part[slots // page, :, slots % page] = old[slots // page, :, slots % page]
    assert torch.equal(pool.blob, before)
    return pool, q, table, lens_t, out, lse


LENS = [1, 0, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 300]


@pytest.mark.parametrize("dtype,fmt", [(BF16, "plain"), (BF16, "int8"), (F32, "plain"), (F32, "int8")])
@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 64, 16), (8, 2, 128, 32), (28, 4, 128, 64), (3, 3, 64, 128), (32, 2, 128, 256), (9, 1, 128, 16), (17, 1, 64, 32),
                                           (128, 1, 128, 64)])
def test_decode_over_lengths_and_shapes(dtype, fmt, append, hq, hkv, d, page):
    decode_case(hq, hkv, d, dtype, fmt, page, LENS, append, hq + page)


@pytest.mark.parametrize("dtype,fmt", [(BF16, "plain"), (BF16, "int8"), (F32, "plain"), (F32, "int8")])
@pytest.mark.parametrize("lens", [[0], [1], [20011], [5000, 1, 0, 77], [1500] * 40, list(range(0, 700, 7))])
def test_decode_splits_and_joins(dtype, fmt, lens):
    pool, q, table, lens_t, out, lse = decode_case(8, 2, 128, dtype, fmt, 64, lens, True, 3, wide=True)
    # the same bits again, also behind other work in the same workspace
    first = pool.decode(0, q, table, lens_t)
    pool.decode(0, q[:1], table[:1], lens_t[:1])
    again = pool.decode(0, q, table, lens_t)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("dtype,fmt", [(BF16, "plain"), (BF16, "int8"), (F32, "plain"), (F32, "int8")])
@pytest.mark.parametrize("gain", [0.0, 1e-3, 20.0, 200.0])
def test_decode_of_flat_and_of_peaked_scores(dtype, fmt, gain):
    decode_case(7, 1, 64, dtype, fmt, 32, [900, 3, 64], True, 5, gain=gain)


@pytest.mark.parametrize("dtype,fmt", [(BF16, "plain"), (BF16, "int8"), (F32, "plain"), (F32, "int8")])
@pytest.mark.parametrize("size", [1e-20, 1e-4, 1e4, 1e20])
def test_decode_of_large_and_small_values(dtype, fmt, size):
    # values (and in 8 bits their scales) far from one: rows of very different size in one sequence
    pool = Pool(4, 2, 128, dtype, 40, 16, fmt)
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = 500
    k, v = (torch.randn(n, 2, 128, generator=gen, device="cuda") for _ in range(2))
    v *= size * torch.exp(torch.randn(n, 2, 1, generator=gen, device="cuda"))
    v[100:120] = 0
    k, v = k.to(dtype), v.to(dtype)
    table = torch.arange(40, dtype=torch.int32, device="cuda")[None]
    pool.write(0, k, v, pool.slots(table[0], n))
    q = torch.randn(1, 4, 128, generator=gen, device="cuda").to(dtype)
    out, lse = pool.decode(0, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    o, z = attend64(q, *held(pool, k, v), 128 ** -0.5)
    assert (out.double() - o).norm() / o.norm() <= (2.0 ** -8 if dtype == BF16 else 3e-5)
    close_lse(lse, z, dtype, "lse")


@pytest.mark.parametrize("fmt", ["plain", "int8"])
def test_decode_of_queries_far_from_one(fmt):
    # heads whose queries differ by many orders of magnitude, single channels far above the others; a query of zeros
    pool = Pool(4, 1, 64, BF16, 20, 16, fmt)
    gen = torch.Generator(device="cuda").manual_seed(11)
    k, v = (torch.randn(300, 1, 64, generator=gen, device="cuda").to(BF16) for _ in range(2))
    q = torch.randn(1, 4, 64, generator=gen, device="cuda")
    q[0, 0] *= 1e-30
    q[0, 1, 3] = 300.0
    q[0, 2] = 0
    q[0, 3] *= 1e10
    q = q.to(BF16)
    table = torch.arange(20, dtype=torch.int32, device="cuda")[None]
    pool.write(0, k, v, pool.slots(table[0], 300))
    out, lse = pool.decode(0, q, table, torch.tensor([300], dtype=torch.int32, device="cuda"))
    k64, v64 = held(pool, k, v)
    o, z = attend64(q, k64, v64, 0.125)
    close(out, o, BF16, "out")
    close_lse(lse, z, BF16, "lse")


def test_decode_replayed_as_lengths_grow_and_on_another_stream():
    hq, hkv, d, page, b = 8, 2, 128, 32, 5
    gen = torch.Generator(device="cuda").manual_seed(2)
    pool = Pool(hq, hkv, d, BF16, b * 4, page, "int8", n_layers=2, max_seqs=b)
    table = torch.arange(b * 4, dtype=torch.int32, device="cuda").view(b, 4)
    lens = torch.tensor([0, 1, 30, 31, 60], dtype=torch.int32, device="cuda")
    start = lens.tolist()
    rows = [[[], []] for _ in range(b)]
    for i, n in enumerate(start):
        k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").to(BF16) for _ in range(2))
        for layer in (0, 1):
            pool.write(layer, k, v, pool.slots(table[i], n))
        rows[i] = [k, v]
    q, k, v = (torch.zeros(b, h, d, device="cuda", dtype=BF16) for h in (hq, hkv, hkv))
    out, lse = torch.empty_like(q), torch.empty(b, hq, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pool.decode(0, q, table, lens, k, v, out, lse)             # (also written to row lens[i]; the next step writes there again)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in (0, 1):
            pool.decode(layer, q, table, lens, k, v, out, lse)
        lens += 1
    lens.copy_(torch.tensor(start, dtype=torch.int32))
    for step in range(40):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graph.replay()
        for i in range(b):
            rows[i] = [torch.cat([rows[i][0], k[i:i + 1]]), torch.cat([rows[i][1], v[i:i + 1]])]
            if step % 13 == 0 or step == 39:
                o, z = attend64(q[i:i + 1], *held(pool, *rows[i]), d ** -0.5)
                close(out[i:i + 1], o, BF16, f"step {step}, sequence {i}")
                close_lse(lse[i:i + 1], z, BF16, f"step {step}, sequence {i}")
    assert pool.status() == KVC_OK and lens.tolist() == [n + 40 for n in start]


def test_decode_of_a_page_far_into_a_large_pool():
    # offsets past 2^31 elements and bytes: the last pages of a pool of five billion codes
    hkv, d, page = 8, 128, 256
    n_pages = 20000
    pool = Pool(8, hkv, d, BF16, n_pages, page, "int8")
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn(300, hkv, d, generator=gen, device="cuda").to(BF16) for _ in range(2))
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    slots = pool.slots(table[0], 300)
    pool.write(0, k, v, slots)
    k64, v64 = held(pool, k, v)
    got = pool.read(0, slots)
    assert torch.equal(got[0].double(), k64.to(BF16).double()) and torch.equal(got[1].double(), v64.to(BF16).double())
    q = torch.randn(1, 8, d, generator=gen, device="cuda").to(BF16)
    out, lse = pool.decode(0, q, table, torch.tensor([300], dtype=torch.int32, device="cuda"))
    o, z = attend64(q, k64, v64, d ** -0.5)
    close(out, o, BF16, "out")
    assert pool.status() == KVC_OK


# ---------------------------------------------------------------------------------------------------------------------- prompts
def prompt_case(hq, hkv, d, dtype, lens, seed, wide=False, gain=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    guard = Guarded()
    n = sum(lens)
    pool = Pool(hq, hkv, d, dtype, 1)
    heads = hq + 2 * hkv
    packed = guard.empty((n, heads, d), dtype)
    packed.copy_(torch.randn(n, heads, d, generator=gen, device="cuda"))
    packed[:, hq:hq + hkv] *= gain
    q, k, v = packed.split([hq, hkv, hkv], 1)
    if not wide:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    out, lse = guard.empty((n, hq, d), dtype), guard.empty((n, hq), F32)
    keep = packed.clone()
    plan = pool.plan(lens)
    pool.prompt(q, k, v, plan, out, lse)
    assert pool.status() == KVC_OK and torch.equal(packed, keep)
    guard.check()
    first = 0
    for i, m in enumerate(lens):
        if m:
            part = slice(first, first + m)
            o, z = attend64(q[part], k[part], v[part], 1 / math.sqrt(d), causal=True)
            close(out[part], o, dtype, f"prompt {i} of {m}")
            close_lse(lse[part], z, dtype, f"prompt {i} of {m}")
        first += m
    return pool, plan, q, k, v, out, lse


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (8, 2, 128), (7, 1, 128), (3, 3, 64), (32, 2, 128), (5, 1, 64), (128, 1, 64), (28, 4, 128)])
@pytest.mark.parametrize("lens", [[1], [2, 0, 1, 31, 32, 33], [127, 128, 129, 1, 0, 255, 257], [700, 5, 64]])
def test_prompts_over_lengths_and_shapes(dtype, hq, hkv, d, lens):
    prompt_case(hq, hkv, d, dtype, lens, hq + len(lens), wide=hkv == 2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hkv,d,lens", [(8, 2, 128, [2500, 1, 1300]), (4, 1, 64, [3000]), (16, 4, 128, [1100, 900, 517, 1, 2047]), (8, 8, 128, [513] * 9), (6, 2, 64, [40] * 120),
                                           (32, 8, 128, [777, 640, 1025])])
def test_prompts_long_and_many(dtype, hq, hkv, d, lens):
    prompt_case(hq, hkv, d, dtype, lens, 1, wide=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gain", [0.0, 30.0])
def test_prompts_of_flat_and_of_peaked_scores(dtype, gain):
    prompt_case(8, 2, 128, dtype, [600, 77, 130], 2, gain=gain)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hkv,lens", [(4, 1, [100, 129, 40, 127, 300]), (32, 8, [700, 333, 1290, 650, 900]), (7, 7, [1, 1, 1, 200])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3e38])
def test_prompts_do_not_see_each_other(dtype, hq, hkv, lens, bad):
    # whatever a neighbour holds: the same bits
    pool, plan, q, k, v, out, lse = prompt_case(hq, hkv, 128, dtype, lens, 3)
    first = 0
    for i, m in enumerate(lens):
        if i % 2:
            for x in (q, k, v):
                x[first:first + m] = bad
        first += m
    again, lse2 = pool.prompt(q, k, v, plan)
    first = 0
    for i, m in enumerate(lens):
        if not i % 2:
            assert torch.equal(again[first:first + m], out[first:first + m]) and torch.equal(lse2[first:first + m], lse[first:first + m]), i
        first += m
    assert pool.status() == KVC_OK


# ---------------------------------------------------------------------------------------------------------------------- refusals
@pytest.mark.parametrize("dtype,fmt", [(BF16, "plain"), (BF16, "int8"), (F32, "plain"), (F32, "int8")])
def test_calls_that_follow_one_another_wait_for_one_another(dtype, fmt):
    """Each call reads what the call before it writes, and writes over what that one reads, with nothing in between: the bits are
    those of a run in which the host waits after every call."""
    gen = torch.Generator(device="cuda").manual_seed(17)
    heads, d, page, seqs, size = 4, 64, 32, 5, 700
    pool = Pool(heads, heads, d, dtype, 256, page, fmt, max_seqs=seqs)
    table = torch.randperm(256, generator=gen, device="cuda").int()[:seqs * 24].view(seqs, 24)
    slots = torch.cat([pool.slots(table[i], size) for i in range(seqs)])
    start = torch.randn(3, seqs * size, heads, d, generator=gen, device="cuda").to(dtype)
    plans = [pool.plan([size] * seqs), pool.plan([1] * seqs), pool.plan([seqs * size])]
    lens = torch.full((seqs,), size, dtype=torch.int32, device="cuda")

    def run(wait):
        x, y, z = start.clone()
        pool.blob.zero_()
        out, lse = torch.zeros_like(x), torch.zeros(seqs * size, heads, device="cuda")
        few, few_lse = torch.zeros(seqs, heads, d, device="cuda", dtype=dtype), torch.zeros(seqs, heads, device="cuda")
        torch.cuda.synchronize()
        for step in range(12):
            plan = plans[step % 3]
            n = plan.n_tokens
            calls = [lambda: pool.prompt(x[:n], y[:n], z[:n], plan, out[:n], lse[:n]),
                     lambda: pool.write(0, out, z, slots),
                     lambda: pool.read(0, slots, y, x),
                     lambda: pool.decode(0, y[:seqs], table, lens, x[:seqs], y[:seqs], few, few_lse),
                     lambda: pool.write(0, few, y[:seqs], slots[:seqs]),
                     lambda: pool.read(0, slots[:seqs], x[:seqs], z[:seqs]),
                     lambda: pool.decode(0, x[:seqs], table, lens, None, None, y[-seqs:], few_lse)]
            for call in calls:
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return [t.clone() for t in (x, y, z, out, lse, few, few_lse, pool.blob)]

    want = run(True)
    assert bool(torch.isfinite(want[0].float()).all()) and pool.status() == KVC_OK
    for _ in range(5):
        for a, b in zip(run(False), want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_refusals():
    pool = Pool(4, 2, 64, BF16, 3, 16, max_seqs=2)
    x, q = torch.zeros(2, 2, 64, device="cuda", dtype=BF16), torch.zeros(2, 4, 64, device="cuda", dtype=BF16)
    slots, table, lens = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    plan = pool.plan([2])
    for call in (lambda: pool.write(0, x.float(), x, slots), lambda: pool.write(0, x, x[:1], slots), lambda: pool.write(0, x, x, slots.int()),
                 lambda: pool.write(0, x, x, slots.cpu()), lambda: pool.write(0, x.cpu(), x, slots), lambda: pool.write(0, x, x.transpose(0, 1).contiguous().transpose(0, 1), slots),
                 lambda: pool.write(0, torch.zeros(2, 2, 128, device="cuda", dtype=BF16)[..., ::2], x, slots), lambda: pool.read(0, slots, x), lambda: pool.read(0, slots.int()),
                 lambda: pool.decode(0, x, table, lens), lambda: pool.decode(0, q, table.long(), lens), lambda: pool.decode(0, q, table[:1], lens),
                 lambda: pool.decode(0, q, table, lens.long()), lambda: pool.decode(0, q, table, lens, x), lambda: pool.decode(0, q, table, lens, x, x.half()),
                 lambda: pool.decode(0, q.transpose(0, 1).contiguous().transpose(0, 1), table, lens), lambda: pool.decode(0, q, table, lens, out=q.float()),
                 lambda: pool.decode(0, q, table, lens, lse=torch.zeros(2, 3, device="cuda")), lambda: pool.prompt(q, x, x[:1], plan),
                 lambda: pool.prompt(q[:1], x, x, plan), lambda: pool.prompt(q, x, x, plan, out=torch.zeros(2, 8, 64, device="cuda", dtype=BF16)[:, ::2]),
                 lambda: pool.plan([2 ** 31])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pool.plan([3, -1]), lambda: pool.decode(0, torch.zeros(3, 4, 64, device="cuda", dtype=BF16), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: pool.write(0, torch.zeros(2, 2, 65, device="cuda", dtype=BF16)[..., :64], torch.zeros(2, 2, 65, device="cuda", dtype=BF16)[..., :64], slots),
                 lambda: pool.write(0, torch.zeros(257, device="cuda", dtype=BF16)[1:].view(2, 2, 64), x, slots)):
        with pytest.raises(KvcError) as e:
            call()
        assert e.value.code == KVC_EINVAL
    for layer in (-1, 1):
        with pytest.raises(IndexError):
            pool.write(layer, x, x, slots)
    for bad in (dict(dtype=torch.float16), dict(page_format="fp8")):
        with pytest.raises(KeyError):
            Pool(**{**dict(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=BF16, n_pages=1), **bad})
    with pytest.raises(KvcError):
        Pool(4, 2, 96, BF16, 1)
    with pytest.raises(ValueError):
        Pool(4, 2, 64, BF16, 4, 16, blob=torch.zeros(1, 100, dtype=torch.uint8, device="cuda"))
    assert pool.launch_count() == 0 and pool.status() == KVC_OK
    keep, pool.blob = pool.blob, pool.blob[:, :-256]
    with pytest.raises(ValueError):
        pool.write(0, x, x, slots)
    pool.blob = keep
    pool.close()
    for call in (lambda: pool.write(0, x, x, slots), lambda: pool.read(0, slots), lambda: pool.decode(0, q, table, lens), lambda: pool.prompt(q, x, x, plan)):
        with pytest.raises(ValueError):
            call()
