"""The paged 8-bit cache at the ends of its ranges: refusals of the Python layer,
captures, two caches at once, caches and row counts past 32-bit offsets."""
import numpy as np
import pytest

from .kv8_common import PAGE

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

CAPACITY = 2


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def randn(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def filled(pages, heads, dh, table, kv_len, seed):
    """A cache with random rows of the given lengths appended through the table."""
    from paper_2609_06498_amd import KV8Cache
    kv = KV8Cache.alloc(pages, heads, dh)
    slots = np.concatenate([table[s][np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE for s, n in enumerate(kv_len)])
    rows = len(slots)
    kv.append(randn(seed, rows, heads, dh), randn(seed + 1, rows, heads, dh), i32(slots))
    return kv


ARGS = dict(q=lambda: randn(1, 4, 8, 64), page_table=lambda: i32([[0, 1], [2, 3]]), kv_len=lambda: i32([70, 100]),
            row_start=lambda: i32([0, 2, 4]), max_rows=lambda: 2, max_len=lambda: 128)


@pytest.mark.parametrize("name,value", [
    ("q", lambda: randn(1, 4, 8, 64, dtype=torch.float16)), ("q", lambda: randn(1, 4, 8, 128)),
    ("q", lambda: randn(1, 4, 7, 64)), ("q", lambda: randn(1, 4, 512)), ("q", lambda: randn(1, 4, 8, 64).cpu()),
    ("q", lambda: randn(1, 4, 8, 128)[:, :, ::2]), ("q", lambda: randn(1, 4, 16, 64)[:, ::2]),
    ("q", lambda: randn(1, 4, 8 * 64 + 4)[:, 4:].view(4, 8, 64)),       # rows that are not 16-byte aligned
    ("q", lambda: randn(1, 8, 64).expand(4, 8, 64)), ("page_table", lambda: i32([[0, 1], [2, 3]]).long()),
    ("page_table", lambda: i32([[0, 1]])), ("page_table", lambda: i32([[0, 2], [1, 3]]).t()),
    ("page_table", lambda: i32([0, 1])), ("kv_len", lambda: i32([70, 100]).long()), ("kv_len", lambda: i32([70, 100]).cpu()),
    ("kv_len", lambda: i32([])), ("row_start", lambda: i32([0, 2])), ("row_start", lambda: i32([0, 2, 4]).float()),
    ("max_rows", lambda: -1), ("max_rows", lambda: 2 ** 20 + 1), ("max_len", lambda: -1), ("scale", lambda: 0.0),
    ("scale", lambda: float("nan")), ("scale", lambda: float("inf")), ("out", lambda: randn(1, 4, 8, 64).float()),
    ("out", lambda: randn(1, 3, 8, 64)), ("out", lambda: randn(1, 4, 8, 64).cpu()),
    ("out", lambda: randn(1, 1, 8, 64).expand(4, 8, 64)),
])
def test_attention_refusals(name, value):
    from paper_2609_06498_amd import DFlowError, KV8Cache
    kv = KV8Cache.alloc(4, 2, 64)
    args = {k: f() for k, f in ARGS.items()}
    out = torch.full((4, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    args["out"] = out
    args[name] = value()
    with pytest.raises(DFlowError):
        kv.attention(**args)
    torch.cuda.synchronize()
    assert (out == 7).all() and kv.status() == 0


@pytest.mark.parametrize("name,value", [
    ("k", lambda: randn(1, 5, 2, 64).half()), ("k", lambda: randn(1, 5, 2, 64).float()), ("k", lambda: randn(1, 4, 2, 64)),
    ("k", lambda: randn(1, 5, 4, 64)), ("k", lambda: randn(1, 5, 4, 64)[:, ::2]), ("v", lambda: randn(1, 5, 2, 64).cpu()),
    ("v", lambda: randn(1, 5, 2, 128)), ("slot", lambda: i32([0, 1, 2, 3])), ("slot", lambda: i32([0, 1, 2, 3, 4]).long()),
    ("slot", lambda: i32(range(10))[::2]), ("slot", lambda: i32([0, 1, 2, 3, 4]).cpu()),
])
def test_append_refusals(name, value):
    from paper_2609_06498_amd import DFlowError, KV8Cache
    kv = KV8Cache.alloc(4, 2, 64)
    args = dict(k=randn(1, 5, 2, 64), v=randn(2, 5, 2, 64), slot=i32([0, 1, 2, 3, 4]))
    args[name] = value()
    with pytest.raises(DFlowError):
        kv.append(**args)
    torch.cuda.synchronize()
    assert int(kv.k.sum()) == 0 and int(kv.v.sum()) == 0 and kv.status() == 0


@pytest.mark.parametrize("args", [
    lambda: (i32([1, 1, 1, 1]),), lambda: (i32([]),), lambda: (i32([1, 1]).long(),), lambda: (i32([1, 1]).cpu(),),
    lambda: (i32([1, 1]), i32([1])), lambda: (i32([1, 1, 1, 1])[::2],), lambda: (i32([1, 1]), i32([1, 1]), i32([0] * 4)),
    lambda: (i32([1, 1]), None, i32([0] * 4), i32([0] * 3)), lambda: (i32([1, 1]), i32([1, 1]), None, i32([0] * 3)),
    lambda: (i32([1, 1]), i32([1, 1]), i32([0] * 4), i32([0] * 2)),
    lambda: (i32([1, 1]), i32([1, 1]), i32([0] * 4).long(), i32([0] * 3)),
])
def test_page_resize_refusals(args):
    from paper_2609_06498_amd import DFlowError, PagePool
    pool = PagePool.alloc(3, 4, 8)
    with pytest.raises(DFlowError):
        pool.resize(*args())
    torch.cuda.synchronize()
    assert int(pool.n_free) == 8 and int(pool.n_held.sum()) == 0 and pool.status() == 0


def test_constructor_refusals():
    from paper_2609_06498_amd import DFlowError, KV8Cache, PagePool
    kv = KV8Cache.alloc(4, 2, 128)
    parts = [kv.k, kv.v, kv.k_scale, kv.v_scale]
    for i, bad in ((0, kv.k[:, :, :63]), (0, kv.k.to(torch.int8)), (1, kv.k), (1, kv.v.cpu()), (2, kv.k_scale.double()),
                   (3, kv.v_scale[:3]), (0, kv.k[0])):
        with pytest.raises(DFlowError):
            KV8Cache(*[bad if j == i else t for j, t in enumerate(parts)])
    p = PagePool.alloc(3, 4, 8)
    parts = [p.page_table, p.n_held, p.free_pages, p.n_free]
    for i, bad in ((0, p.page_table.long()), (1, p.n_held[:2]), (2, p.free_pages.cpu()), (3, p.n_free[:0])):
        with pytest.raises(DFlowError):
            PagePool(*[bad if j == i else t for j, t in enumerate(parts)])


def test_first_call_of_a_size_is_not_captured():
    """The workspace of a captured call has to be there, zeroed, before."""
    from paper_2609_06498_amd import DFlowError
    table = np.arange(64).reshape(1, 64)
    kv = filled(64, 2, 128, table, [4000], 3)
    q, lens, start = randn(5, 1, 8, 128), i32([4000]), i32([0, 1])
    pt = i32(table)
    call = lambda out: kv.attention(q, pt, lens, start, 1, 4096, out=out)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    with pytest.raises(DFlowError, match="captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            call(out)
    call(out)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        again = torch.zeros_like(q)
        call(again)
        assert torch.equal(again, want)
    assert kv.status() == 0


def test_two_caches_on_two_streams():
    """Caches with workspaces of their own run side by side."""
    table = np.arange(128).reshape(2, 64)
    calls = []
    for i in range(2):
        kv = filled(128, 2, 128, table, [4000, 3500], 30 + i)
        rows = (1, 16)[i]
        q, lens, start, pt = randn(40 + i, 2 * rows, 8, 128), i32([4000, 3500]), i32([0, rows, 2 * rows]), i32(table)
        want = kv.attention(q, pt, lens, start, rows, 4096).clone()
        outs = [torch.zeros_like(q) for _ in range(20)]
        calls.append((kv, q, pt, lens, start, rows, outs, want, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for n in range(20):
        for kv, q, pt, lens, start, rows, outs, want, stream in calls:
            with torch.cuda.stream(stream):
                kv.attention(q, pt, lens, start, rows, 4096, out=outs[n])
    torch.cuda.synchronize()
    for kv, _, _, _, _, _, outs, want, _ in calls:
        assert all(torch.equal(o, want) for o in outs) and kv.status() == 0


def test_sequences_that_share_pages():
    """A common prefix: page rows that name the same pages read them alike."""
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]])
    kv = filled(8, 2, 64, table, [200, 256], 11)
    shared = table.copy()
    shared[1, :3] = table[0, :3]
    q = randn(12, 2, 4, 64)
    q[1] = q[0]
    got = kv.attention(q, i32(shared), i32([190, 190]), i32([0, 1, 2]), 1, 256)
    assert torch.equal(got[0], got[1]) and bool(got.float().abs().sum() > 0)


@pytest.mark.parametrize("rows", [1, 16, 60])
def test_cache_past_32_bit_offsets(rows):
    """Pages whose bytes lie behind 4 GiB hold and give what the first pages do."""
    from paper_2609_06498_amd import KV8Cache
    heads, dh, pages = 8, 128, 70000                            # 64 KiB a page: 4.6 GB of keys, as many of values
    near = np.arange(20).reshape(2, 10)
    far = near + (pages - 20)
    assert far[0, 0] * heads * PAGE * dh > 2 ** 32
    lens = [600, 333]
    small, big = filled(20, heads, dh, near, lens, 50), None
    big = KV8Cache.alloc(pages, heads, dh)
    slots = np.concatenate([far[s][np.arange(n) // PAGE] * PAGE + np.arange(n) % PAGE for s, n in enumerate(lens)])
    big.append(randn(50, sum(lens), heads, dh), randn(51, sum(lens), heads, dh), i32(slots))
    for a, b in ((small.k, big.k), (small.v, big.v), (small.k_scale, big.k_scale), (small.v_scale, big.v_scale)):
        assert torch.equal(a, b[-20:])
        assert torch.equal(b[:20].float().unique(), b[20:40].float().unique())       # untouched
    q, start = randn(52, 2 * rows, 16, dh), i32([0, rows, 2 * rows])
    want = small.attention(q, i32(near), i32(lens), start, rows, 640)
    got = big.attention(q, i32(far), i32(lens), start, rows, 640)
    assert torch.equal(want, got) and small.status() == 0 and big.status() == 0


def test_append_of_millions_of_rows():
    """More row blocks than a launch's second dimension holds; the last rows are written."""
    from paper_2609_06498_amd import KV8Cache
    rows = 64 * 65536 + 37
    x = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device="cuda")
    slot = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    tail = randn(7, 30, 1, 64)
    x[-30:] = tail
    slot[-30:] = torch.arange(30, dtype=torch.int32, device="cuda")
    kv, few = KV8Cache.alloc(2, 1, 64), KV8Cache.alloc(2, 1, 64)
    kv.append(x, x, slot)
    few.append(tail, tail, slot[-30:])
    for a, b in ((kv.k, few.k), (kv.v, few.v), (kv.k_scale, few.k_scale), (kv.v_scale, few.v_scale)):
        assert torch.equal(a, b)
    assert int(kv.k.sum()) > 0 and kv.status() == 0


def test_slot_map_of_the_largest_capacity():
    """Room for 2^31 - 1 slots, of which a few are written."""
    from paper_2609_06498_amd import PagePool
    cap = 2 ** 31 - 1
    pool, slot = PagePool.alloc(3, 4, 8), torch.full((cap,), -77, dtype=torch.int32, device="cuda")
    start = torch.zeros(4, dtype=torch.int32, device="cuda")
    pool.resize(i32([0, 0, 0]), i32([70, 0, 3]), slot, start)
    assert start.tolist() == [0, 70, 70, 73] and pool.status() == 0
    assert slot[:74].tolist() == list(range(70)) + [128, 129, 130, -77]
    assert int(slot[73:].max()) == -77 and int(slot[73:].min()) == -77
    pool.resize(i32([0, 0, 0]), i32([2 ** 31 - 1, 0, 3]), slot, start)     # the first is refused, rows past the capacity cut
    assert pool.status() == CAPACITY
    assert start.tolist() == [0, cap, cap, cap] and int(slot[::4093].max()) == -1
