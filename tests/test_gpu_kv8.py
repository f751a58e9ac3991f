"""The paged 8-bit cache on the GPU against the 64-bit oracle of kv8_common:
page resizing and slot maps, append, attention, and rounds of all three."""
import numpy as np
import pytest

from .kv8_common import PAGE, Cache, Pages, attention, attention_bound

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CAPACITY, BAD_PAGE, BAD_SLOT = 2, 4, 8


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(x, dt=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dt is None else t.to(dt)).cuda()


def i32(x):
    return dev(np.asarray(x, np.int32))


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, dtype):
    """x as the storage type holds it, in float64."""
    return torch.from_numpy(np.asarray(x)).to(DT[dtype]).double().numpy()


def upload(c):
    from paper_2609_06498_amd import KV8Cache
    return KV8Cache(dev(c.code["k"]), dev(c.code["v"].transpose(0, 1, 3, 2)), dev(c.scale["k"], torch.float32),
                    dev(c.scale["v"], torch.float32))


def random_cache(pages, heads, dh, rng):
    """Filled cache: every group's values of a size of its own."""
    c = Cache(pages, heads, dh)
    for n in "kv":
        size = np.exp(rng.normal(0, 1, (pages, heads, 4)))
        x = rng.normal(0, 1, (pages, heads, PAGE, dh)) * np.repeat(size, 16, 2)[..., None]
        scale = 2.0 ** np.ceil(np.log2(np.abs(x).reshape(pages, heads, 4, -1).max(-1) / 448))
        c.scale[n] = scale
        t = torch.from_numpy(x / np.repeat(scale, 16, 2)[..., None]).float().to(torch.float8_e4m3fn)
        c.code[n] = t.view(torch.uint8).numpy().copy()
    return c


def tables(kv_len, max_pages, pages, rng):
    ids = rng.permutation(pages)
    t, at = np.full((len(kv_len), max_pages), -1, np.int32), 0
    for s, n in enumerate(kv_len):
        need = -(-n // PAGE)
        t[s, :need] = ids[at:at + need]
        at += need
    return t


def junk_behind(c, t, kv_len, rng):
    """Any byte, NaN codes among them, behind every sequence's end."""
    for s, n in enumerate(kv_len):
        if n % PAGE:
            p = t[s, n // PAGE]
            for x in "kv":
                tail = c.code[x][p, :, n % PAGE:]
                tail[:] = rng.integers(0, 256, tail.shape)
                tail[..., ::7] = 127
            first = -(-(n % PAGE) // 16)                        # scales of groups that hold nothing
            for x in "kv":
                c.scale[x][p, :, first:] = [0.0, np.nan, np.inf, -1.0][s % 4]


def check(got, want, A, S, dtype, dh, keys):
    got = got.double().cpu().numpy()
    bound = attention_bound(want, A, S, dtype, dh, keys)
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), (err / bound).max()
    return (err / bound).max()


#        heads, kv heads, dh, kv lens, rows, max_len beyond the longest
CASES = [
    (4, 2, 64, [1], [1], 0),
    (8, 2, 128, [1, 2, 15, 16, 17], [1, 1, 1, 1, 1], 0),
    (8, 8, 128, [63, 64, 65], [1, 16, 5], 100),
    (12, 4, 64, [0, 300, 5], [0, 7, 5], 0),
    (16, 8, 128, [700, 0, 129, 257], [16, 0, 1, 16], 5000),
    (32, 8, 128, [130, 1000], [16, 16], 0),
    (64, 8, 128, [90, 16], [16, 16], 40000),
    (10, 2, 128, [600], [600], 0),                              # a prompt from its first token on
    (5, 5, 64, [333, 200], [130, 77], 0),
    (8, 2, 128, [40, 3], [16, 16], 0),                          # more rows than tokens: the first see nothing
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, dtype, causal):
    hq, hkv, dh, kv_len, n, beyond = CASES[case]
    rng = np.random.default_rng(100 + case)
    pages = sum(-(-x // PAGE) for x in kv_len) + 3
    max_pages = max(-(-max(kv_len) // PAGE), 1) + beyond // PAGE + 1
    c = random_cache(pages, hkv, dh, rng)
    t = tables(kv_len, max_pages, pages, rng)
    junk_behind(c, t, kv_len, rng)
    start = np.concatenate([[0], np.cumsum(n)])
    rows = int(start[-1]) + 2                                   # two rows behind the last sequence
    q = rounded(rng.normal(0, 1.2, (rows, hq, dh)), dtype)
    h = upload(c)
    out = torch.full((rows, hq, dh), 7.0, dtype=DT[dtype], device="cuda")
    h.attention(dev(q, DT[dtype]), i32(t), i32(kv_len), i32(start), max(n), max(kv_len) + beyond, causal=causal, out=out)
    want, A, S = attention(c, t, kv_len, start, q[:-2], causal, dh ** -0.5)
    check(out[:-2], want, A, S, dtype, dh, max(kv_len))
    assert (out[-2:] == 7).all(), "rows behind the last sequence"
    assert h.status() == 0


def test_attention_strides_scale_and_unused_row_sizes():
    """q and out as parts of wider rows, another softmax scale, max_rows and max_len above the real ones."""
    rng = np.random.default_rng(5)
    kv_len, n = [150, 70], [3, 2]
    c = random_cache(8, 2, 128, rng)
    t = tables(kv_len, 9, 8, rng)
    start = np.array([0, 3, 5])
    wide = rounded(rng.normal(0, 1, (5, 3, 8, 128)), "bf16")
    q = dev(wide, torch.bfloat16)
    out = torch.zeros(5, 2, 8, 128, dtype=torch.bfloat16, device="cuda")
    h = upload(c)
    h.attention(q[:, 1], i32(t), i32(kv_len), i32(start), 64, 9 * PAGE, scale=0.3, out=out[:, 1])
    want, A, S = attention(c, t, kv_len, start, wide[:, 1], True, 0.3)
    check(out[:, 1], want, A, S, "bf16", 128, 150)
    assert (out[:, 0] == 0).all() and h.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_nan_that_some_rows_see(dtype):
    """A NaN in the block's own keys or values reaches the rows that see it (a value: its channel only) and no other."""
    rng = np.random.default_rng(6)
    hq, hkv, dh, n, rows = 8, 2, 128, 75, 16
    for name, t_nan in (("v", n - 5), ("k", n - 9), ("v", 20)):
        c = random_cache(2, hkv, dh, rng)
        t = np.array([[1, 0]], np.int32)
        c.code[name][t[0, t_nan // PAGE], 1, t_nan % PAGE, 33] = 0xFF
        q = rounded(rng.normal(0, 1, (rows, hq, dh)), dtype)
        h = upload(c)
        out = h.attention(dev(q, DT[dtype]), i32(t), i32([n]), i32([0, rows]), rows, n).double().cpu().numpy()
        sees = np.arange(n - rows, n) >= t_nan
        nan = np.zeros(out.shape, bool)
        if name == "v":
            nan[sees, 4:, 33] = True
        else:
            nan[sees, 4:] = True
        assert (np.isnan(out) == nan).all(), name
        with np.errstate(invalid="ignore"):
            want, A, S = attention(c, t, [n], [0, rows], q, True, dh ** -0.5)
        bound = attention_bound(want, A, S, dtype, dh, n)
        assert (np.abs(out - want)[~nan] <= bound[~nan]).all()


@pytest.mark.parametrize("rows", [1, 16])
def test_attention_nan_keys_of_a_whole_head(rows):
    """Every key of a head NaN, over several splits: its rows are NaN, the other head's are not."""
    rng = np.random.default_rng(16)
    n = 500
    c = random_cache(8, 2, 64, rng)
    c.code["k"][:, 1] = 0x7F
    t = np.arange(8, dtype=np.int32)[None]
    q = rounded(rng.normal(0, 1, (rows, 8, 64)), "bf16")
    out = upload(c).attention(dev(q, torch.bfloat16), i32(t), i32([n]), i32([0, rows]), rows, n)
    assert out[:, 4:].isnan().all() and not out[:, :4].isnan().any()


def test_attention_large_and_small_magnitudes():
    """Scales from 2^-60 to 2^60 in one sequence, scores far apart: the softmax picks what 64 bits pick."""
    rng = np.random.default_rng(7)
    c = random_cache(3, 1, 64, rng)
    c.scale["v"][:] *= 2.0 ** rng.integers(-60, 60, c.scale["v"].shape)
    c.scale["k"][:] *= 2.0 ** rng.integers(-3, 3, c.scale["k"].shape)
    t = np.array([[2, 0, 1]], np.int32)
    for dtype in ("bf16", "f32"):
        q = rounded(rng.normal(0, 3, (4, 2, 64)), dtype)
        h = upload(c)
        out = h.attention(dev(q, DT[dtype]), i32(t), i32([190]), i32([0, 4]), 4, 190)
        want, A, S = attention(c, t, [190], [0, 4], q, True, 0.125)
        check(out, want, A, S, dtype, 64, 190)


def test_attention_bad_pages_and_lengths():
    """What only the device sees: status bits, and the other sequences' results as they are without it."""
    rng = np.random.default_rng(8)
    c = random_cache(9, 2, 128, rng)
    kv_len = [200, 130, 100, 64]
    t = tables(kv_len, 6, 10, rng) % 9
    q = rounded(rng.normal(0, 1, (8, 4, 128)), "bf16")
    start = np.array([0, 2, 4, 6, 8])
    h, args = upload(c), (i32(start), 2, 200)
    good = h.attention(dev(q, torch.bfloat16), i32(t), i32(kv_len), *args)
    assert h.status() == 0
    for bad in (9, -5, 1 << 30):
        t2 = t.copy()
        t2[1, 1] = bad
        out = h.attention(dev(q, torch.bfloat16), i32(t2), i32(kv_len), *args)
        want, A, S = attention(c, t2, kv_len, start, q, True, 128 ** -0.5)
        check(out, want, A, S, "bf16", 128, 200)
        assert torch.equal(out[:2], good[:2]) and torch.equal(out[4:], good[4:])
        assert h.status() == BAD_PAGE and h.status() == 0
    for lens in ([200, -3, 100, 64], [200, 201, 100, 64], [200, 2 ** 31 - 1, 100, 64]):
        out = h.attention(dev(q, torch.bfloat16), i32(t), i32(lens), *args)
        assert torch.equal(out[:2], good[:2]) and torch.equal(out[4:], good[4:])
        if lens[1] < 0:
            assert (out[2:4] == 0).all()
        assert h.status() & CAPACITY
    for starts in ([0, 2, 99, 6, 8], [0, 2, 1, 6, 8], [0, 2, -1, 6, 8]):
        out = torch.full((8, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda")
        h.attention(dev(q, torch.bfloat16), i32(t), i32(kv_len), i32(starts), 2, 200, out=out)
        own = 1 if starts[2] == 1 else 2                        # [.., 1, 6, ..] gives sequence 2 row 1 on
        assert torch.equal(out[:own], good[:own]) and torch.equal(out[6:], good[6:])
        assert h.status() == CAPACITY


def test_attention_row_does_not_depend_on_the_other_sequences():
    rng = np.random.default_rng(9)
    hq, hkv, dh = 32, 8, 128
    c = random_cache(60, hkv, dh, rng)
    lens = [900, 400, 70]
    t = tables(lens, 16, 60, rng)
    q = dev(rng.normal(0, 1, (48, hq, dh)), torch.bfloat16)
    h = upload(c)
    a = h.attention(q, i32(t), i32(lens), i32([0, 16, 32, 48]), 16, 1000)
    b = h.attention(q, i32(t), i32([900, 30, 1]), i32([0, 16, 30, 31]), 16, 1000)
    assert torch.equal(a[:16], b[:16])
    swap = h.attention(torch.cat([q[32:], q[16:32], q[:16]]), i32(t[::-1].copy()), i32(lens[::-1]), i32([0, 16, 32, 48]),
                       16, 1000)
    assert torch.equal(a[:16], swap[32:]) and torch.equal(a[32:], swap[:16])


# ---------------------------------------------------------------- append
def same_cache(h, c):
    k, v = h.k.cpu().numpy(), h.v.cpu().numpy().transpose(0, 1, 3, 2)
    np.testing.assert_array_equal(h.k_scale.cpu().numpy().astype(np.float64), c.scale["k"])
    np.testing.assert_array_equal(h.v_scale.cpu().numpy().astype(np.float64), c.scale["v"])
    nan = lambda x: np.where((x & 127) == 127, 127, x)          # NaN has no sign
    np.testing.assert_array_equal(nan(k), nan(c.code["k"]))
    np.testing.assert_array_equal(nan(v), nan(c.code["v"]))


def runs(spec):
    """Slots of [(first slot, count)]."""
    return np.concatenate([np.arange(a, a + n) for a, n in spec]).astype(np.int32)


SLOTS = {
    "one token": runs([(5, 1)]),
    "first of a page": runs([(64, 1)]),
    "last of a page": runs([(127, 1)]),
    "block over a page's end": np.concatenate([runs([(64 * 3 + 55, 9)]), runs([(64 * 1, 7)])]),
    "whole group": runs([(32, 16)]),
    "ragged batch": runs([(3, 8), (64 + 60, 4), (64 * 5, 4), (64 * 2 + 17, 1), (64 * 6, 64), (64 * 4 + 30, 33)]),
    "rows without a slot": np.array([-1, 40, 41, -1, -1, 200, -1], np.int32),
    "gaps in a group": np.array([18, 20, 25, 31], np.int32),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dh", [(2, 64), (3, 128)])
@pytest.mark.parametrize("name", sorted(SLOTS))
def test_append(name, heads, dh, dtype):
    rng = np.random.default_rng(len(name))
    slots = SLOTS[name]
    c = random_cache(7, heads, dh, rng)
    h = upload(c)
    k, v = (rounded(rng.normal(0, 1, (len(slots), heads, dh)) * np.exp(2 * rng.normal(0, 1, (len(slots), heads, 1))),
                    dtype) for _ in range(2))
    h.append(dev(k, DT[dtype]), dev(v, DT[dtype]), i32(slots))
    c.append(k, v, slots)
    same_cache(h, c)
    assert h.status() == 0


@pytest.mark.parametrize("rows", [2048, 2049, 5000])
def test_append_many_rows(rows):
    """The launch of one row per wave and the one of 32 agree with the oracle at their border, groups cut by it."""
    rng = np.random.default_rng(rows)
    pages = rows // PAGE + 3
    order = rng.permutation(pages)
    pos = np.arange(13, 13 + rows)
    slots = (order[pos // PAGE] * PAGE + pos % PAGE).astype(np.int32)
    c = random_cache(pages, 1, 64, rng)
    h = upload(c)
    k, v = (rounded(rng.normal(0, 1, (rows, 1, 64)), "bf16") for _ in range(2))
    h.append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), i32(slots))
    c.append(k, v, slots)
    same_cache(h, c)
    assert h.status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_values_at_the_ends(dtype):
    """Zeros, infinities, NaN, the smallest and the largest finite values, ties of the rounding."""
    heads, dh = 1, 64
    big = float(torch.finfo(DT[dtype]).max)
    fills = [0.0, np.inf, np.nan, 1e-38, 2.0 ** -130, big, -big, 448.0, 449.0, 464.0, 0.4375, 1.0625, 1.1875]
    slots = (np.arange(len(fills)) * 16 % (7 * PAGE)).astype(np.int32)
    k = np.ones((len(fills), heads, dh))
    for i, x in enumerate(fills):
        k[i, :, ::3] = x
        if x == 0:
            k[i] = 0
    k[3:5] = np.array(fills[3:5])[:, None, None]
    k = rounded(k, dtype)
    c = Cache(7, heads, dh)
    h = upload(c)
    h.append(dev(k, DT[dtype]), dev(k[::-1].copy(), DT[dtype]), i32(slots))
    c.append(k, k[::-1], slots)
    same_cache(h, c)


def test_append_token_by_token_is_append_at_once():
    """Power-of-two scales: a group filled one token at a time ends with the codes of one call, while kept values
    stay normal under the new scale (magnitudes within 2^8 of each other here, e4m3's normal range is 2^15)."""
    rng = np.random.default_rng(11)
    rows = rng.uniform(1, 2, (40, 2, 64)) * np.sign(rng.normal(0, 1, (40, 2, 64))) * 2.0 ** rng.integers(0, 7, (40, 1, 1))
    rows = rounded(rows, "bf16")
    slots = np.arange(20, 60).astype(np.int32)
    a, b = upload(Cache(1, 2, 64)), upload(Cache(1, 2, 64))
    x = dev(rows, torch.bfloat16)
    a.append(x, x, i32(slots))
    for i in range(40):
        b.append(x[i:i + 1], x[i:i + 1], i32(slots[i:i + 1]))
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n


def test_append_bad_slots_and_strides():
    """Bad slots are skipped.  (A group's rows stay consecutive, as the call asks: 70 and 90 are of two groups.)"""
    rng = np.random.default_rng(12)
    c = random_cache(4, 2, 128, rng)
    h = upload(c)
    wide = rounded(rng.normal(0, 1, (6, 4, 2, 128)), "bf16")
    x = dev(wide, torch.bfloat16)
    for slots in ([3, 4, 4 * PAGE, 70, -2, 90], [3, 4, 4, 70, 69, 72], [20, 1 << 30, 45, 46, -9, 100]):
        slots = np.array(slots, np.int32)
        h.append(x[:, 1], x[:, 2], i32(slots))
        fine = np.where((slots < -1) | (slots >= 4 * PAGE), -1, slots)
        c.append(wide[:, 1], wide[:, 2], fine)
        same_cache(h, c)
        assert h.status() == BAD_SLOT and h.status() == 0


# ---------------------------------------------------------------- pages
def pool_of(o, num_pages):
    from paper_2609_06498_amd import PagePool
    free = np.zeros(num_pages, np.int32)
    free[:len(o.free)] = o.free
    return PagePool(i32(o.table), i32(o.held), i32(free), i32([len(o.free)]))


def same_pool(p, o):
    np.testing.assert_array_equal(p.page_table.cpu().numpy(), o.table)
    assert p.n_held.cpu().tolist() == o.held
    assert int(p.n_free) == len(o.free)
    assert p.free_pages.cpu().tolist()[:len(o.free)] == o.free


@pytest.mark.parametrize("nseq,max_pages,num_pages,longest", [(1, 1, 1, 64), (3, 8, 30, 400), (70, 12, 300, 700),
                                                               (1024, 20, 5000, 1000), (8, 130, 900, 8000)])
def test_page_resize(nseq, max_pages, num_pages, longest):
    """Growing, shrinking, emptying and refilling rows, with more asked for than the pool and the rows hold."""
    rng = np.random.default_rng(nseq)
    o = Pages(np.full((nseq, max_pages), -1, np.int32), [0] * nseq, rng.permutation(num_pages))
    p = pool_of(o, num_pages)
    cap = 300000 if nseq == 1024 else 20000 if rng.random() < 0.5 else 4000
    refused = 0
    lens = np.zeros(nseq, int)
    for step in range(6):
        new = rng.integers(0, longest // 3 + 1, nseq) if step % 2 == 0 else rng.integers(0, 17, nseq)
        slot = torch.full((cap,), -77, dtype=torch.int32, device="cuda")
        start = torch.zeros(nseq + 1, dtype=torch.int32, device="cuda")
        p.resize(i32(lens), i32(new), slot, start)
        want, starts, ok = o.resize(lens.tolist(), new.tolist(), cap)
        same_pool(p, o)
        got = slot.cpu().numpy()
        np.testing.assert_array_equal(got[:len(want)], want)
        assert (got[len(want):] == -77).all()
        np.testing.assert_array_equal(start.cpu().numpy(), starts)
        assert p.status() == (0 if ok and sum(new) <= cap else CAPACITY)
        refused += not ok
        lens = np.minimum(lens + rng.integers(0, new + 1), np.array(o.held) * PAGE)   # what was committed
        lens[rng.random(nseq) < 0.2] = 0                                              # finished requests
        p.resize(i32(lens))
        assert o.resize(lens.tolist(), None)[2]
        same_pool(p, o)
        assert p.status() == 0
    print(f"refused in {refused} of 6 steps")


def test_page_resize_restores_the_stack_and_survives_bad_state():
    rng = np.random.default_rng(2)
    o = Pages(np.full((5, 9), -1, np.int32), [0] * 5, rng.permutation(40))
    p = pool_of(o, 40)
    lens = i32([100, 1, 0, 64, 65])
    p.resize(lens)
    before = p.free_pages.clone(), p.page_table.clone()
    p.resize(lens, i32([200, 64, 1, 0, 130]))
    p.resize(lens)
    assert torch.equal(p.free_pages, before[0]) and torch.equal(p.page_table, before[1]) and p.status() == 0
    for bad in ([-1, 0, 0, 0, 0], [0, 0, 0, 0, -(2 ** 31)]):      # negative lengths: the sequence keeps its row
        slot, start = i32(np.zeros(8)), i32(np.zeros(6))
        p.resize(i32(bad), i32([1, 1, 1, 1, 1]), slot, start)
        assert p.status() == CAPACITY
        s = slot.cpu().tolist()[:5]
        assert [x == -1 for x in s] == [b < 0 for b in bad]
    p.resize(i32([2 ** 31 - 1] * 5), i32([2 ** 31 - 1] * 5))
    assert p.status() == CAPACITY
    for n in (-4, 1000):                                        # a stack count no pool of 40 has
        p.n_free.fill_(n)
        p.resize(i32([10, 0, 0, 0, 0]))
        assert p.status() == CAPACITY and 0 <= int(p.n_free) <= 40


# ---------------------------------------------------------------- together
def serve(rounds, graph, stream):
    """Rounds of a small serving loop: reserve, append the block, attend, commit a part, trim."""
    from paper_2609_06498_amd import KV8Cache, PagePool
    rng = np.random.default_rng(21)
    nseq, B, hq, hkv, dh, max_pages = 4, 8, 8, 2, 128, 8
    kv = KV8Cache.alloc(20, hkv, dh)
    pool = PagePool.alloc(nseq, max_pages, 20)
    c, o = Cache(20, hkv, dh), Pages(np.full((nseq, max_pages), -1, np.int32), [0] * nseq, range(19, -1, -1))
    lens = i32(np.zeros(nseq))
    new, kv_len = i32(np.zeros(nseq)), i32(np.zeros(nseq))
    slot, start = i32(np.zeros(nseq * 64)), i32(np.zeros(nseq + 1))
    x = torch.zeros(2, nseq * B, hkv, dh, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(nseq * B, hq, dh, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    rows = nseq * B

    def step():
        pool.resize(lens, new, slot, start)
        kv.append(x[0], x[1], slot[:rows])
        kv.attention(q, pool.page_table, kv_len, start, B, max_pages * PAGE, out=out)

    g = None
    host = np.array([100, 0, 63, 17])
    with torch.cuda.stream(stream):
        # prompts
        prompt = rounded(rng.normal(0, 1, (2, int(host.sum()), hkv, dh)), "bf16")
        big = i32(np.zeros(int(host.sum())))
        pool.resize(lens, i32(host), big, start)
        slots, _, ok = o.resize([0] * nseq, host.tolist(), len(big))
        assert ok
        kv.append(dev(prompt[0], torch.bfloat16), dev(prompt[1], torch.bfloat16), big)
        c.append(prompt[0], prompt[1], slots)
        for r in range(rounds):
            kvn = rounded(rng.normal(0, 1, (2, rows, hkv, dh)), "bf16")
            qn = rounded(rng.normal(0, 1, (rows, hq, dh)), "bf16")
            x.copy_(torch.from_numpy(kvn))
            q.copy_(torch.from_numpy(qn))
            lens.copy_(i32(host))
            new.fill_(B)
            kv_len.copy_(i32(host + B))
            if graph and r == 1:
                g = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(g):
                    step()
                torch.cuda.synchronize()
            if g is not None:
                g.replay()
            else:
                step()
            slots, starts, ok = o.resize(host.tolist(), [B] * nseq, nseq * 64)
            assert ok
            c.append(kvn[0], kvn[1], slots)
            want, A, S = attention(c, o.table, (host + B).tolist(), starts, qn, True, dh ** -0.5)
            torch.cuda.current_stream().synchronize()
            check(out, want, A, S, "bf16", dh, int(host.max()) + B)
            same_cache(kv, c)
            same_pool(pool, o)
            host = host + rng.integers(1, B + 1, nseq)
            if r == 2:
                host[0] = 0                                     # a finished request's slot starts over
            pool.resize(i32(host))
            assert o.resize(host.tolist(), None)[2]
        assert pool.status() == 0 and kv.status() == 0


def test_rounds_together():
    serve(5, False, torch.cuda.current_stream())


def test_rounds_together_on_another_stream():
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    serve(3, False, s)


def test_rounds_captured_and_replayed():
    serve(6, True, torch.cuda.Stream())
