"""The 8-bit target cache and the page pool inside the round and the serving
engine.

Verification over the 8-bit cache is compared with the oracle's target forward
over the values that the device's cache holds (decoded by the oracle's own
table), so the comparison has the tolerance of the storage type and no rounding of
the cache in it; the cached rows themselves are compared with the oracle's keys and
values to within e4m3's rounding.  Engines over a page pool give the tokens of
engines whose slots own whole page-table rows.
"""
import numpy as np
import pytest

from tests.gpu_common import TOL, rel_rows
from tests.kv8_common import DECODE, PAGE
from workload import get_config
from workload.synth import make_weights

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cached(rt, s, n):
    """Values and scales per layer and side: [n, kv heads, dh] of slot s's first n tokens."""
    table = rt.page_table.cpu().numpy()
    pos = np.arange(n)
    page = table[s, pos // PAGE]
    k, v, ks, vs = (t.cpu().numpy() for t in rt.kv8)
    out = []
    for l in range(rt.dims.n_layers):
        grp = pos % PAGE // 16
        sk, sv = (x[l][page, :, grp].astype(np.float64)[..., None] for x in (ks, vs))
        out.append((DECODE[k[l][page, :, pos % PAGE]] * sk, DECODE[v[l][page, :, :, pos % PAGE]] * sv, sk, sv))
    return out


class OverCache:
    """The oracle's target whose layers attend over given keys and values instead of the rows' own."""

    def __new__(cls, dims, raw, mode, kv):
        from oracle import OracleModel

        class M(OracleModel):
            rows = {}

            def attention(self, q, k, v, visible):
                n, l = k.shape[0], self.layer
                self.rows[l] = (k, v)
                kk, vv = (x[:n].astype(self.mode.dt) for x in kv[l][:2])
                return super().attention(q, kk, vv, visible)

            def decoder_layer(self, prefix, *a):
                self.layer = int(prefix.split(".")[1])
                return super().decoder_layer(prefix, *a)
        return M(dims, raw, mode)


@pytest.mark.parametrize("name,max_rows,paged", [("tiny-f32", 24, False), ("small-f32", 64, True),
                                                 ("small-bf16", 128, False), ("small-bf16", 100, True)])
def test_verify_over_the_8_bit_cache(name, max_rows, paged):
    from oracle import Mode
    from paper_2609_06498_amd import Runtime
    wl = get_config(name)
    dm, B = wl.dims, wl.block
    w = make_weights(dm, wl.seed_w)
    rng = np.random.default_rng(31)
    lens = [70, 200, 33]
    mode = Mode("fp32" if dm.dtype == "f32" else "bf16")
    rt = Runtime(dm, B, 4, 300, w, wl.carry_window, max_rows=max_rows, kv_cache="fp8", num_pages=14 if paged else None)
    start = torch.tensor(lens + [0], dtype=torch.int32, device="cuda")
    if paged:
        rt.page_pool.resize(start, torch.tensor([2 * B] * 3 + [0], dtype=torch.int32, device="cuda"))
    prompts = [rng.integers(0, dm.vocab, n).astype(np.int32) for n in lens]
    first = torch.zeros(4, dtype=torch.int32, device="cuda")
    rt.prefill_batch(torch.from_numpy(np.concatenate(prompts)).cuda(), lens, first)
    pos = list(lens)
    toks = [list(p) for p in prompts]
    for step in range(3):                       # the second and third overwrite a rejected part of the block before
        blk = rng.integers(0, dm.vocab, (3, B)).astype(np.int32)
        lg = torch.zeros(3 * B, dm.vocab, dtype=torch.float32, device="cuda")
        rt.verify_block(3, torch.from_numpy(blk).cuda(), torch.tensor(pos, dtype=torch.int32, device="cuda"), None, lg)
        torch.cuda.synchronize()
        assert rt.status() == 0
        got = lg.cpu().numpy().reshape(3, B, -1)
        for s in range(3):
            kv = cached(rt, s, pos[s] + B)
            m = OverCache(dm, w, mode, kv)
            past = [(k[:pos[s]], v[:pos[s]]) for k, v, _, _ in kv]
            want = m.target_block(blk[s], pos[s], [a.astype(mode.dt) for a, _ in past],
                                  [b.astype(mode.dt) for _, b in past])[0]
            e = rel_rows(got[s], want).max()
            assert e <= TOL[dm.dtype], f"{name} step {step} sequence {s}: logits {e}"
            # the block's rows in the cache: e4m3's half step of normal values (2^-4) or of subnormal ones (2^-10 of the
            # scale), of a row that itself agrees to the storage type's tolerance
            for l, (k, v, sk, sv) in enumerate(kv):
                for x, y, sc in ((k, m.rows[l][0], sk), (v, m.rows[l][1], sv)):
                    x, y, sc = x[pos[s]:], y[pos[s]:].astype(np.float64), sc[pos[s]:]
                    tol = TOL[dm.dtype] * np.sqrt((y ** 2).mean(-1, keepdims=True)) * 4
                    assert (np.abs(x - y) <= 2.0 ** -4 * (np.abs(y) + tol) + 2.0 ** -10 * sc + tol).all(), (step, s, l)
            keep = int(rng.integers(1, B))
            toks[s] += blk[s][:keep].tolist()
            pos[s] += keep
    rt.close()


def test_prompt_results_do_not_depend_on_the_chunks():
    """Prompts in chunks of 64 and of 256 rows, alone and together: the same first tokens and caches, except values that a
    group's later scale makes subnormal (a chunk may end inside a group)."""
    from paper_2609_06498_amd import Runtime
    wl = get_config("small-bf16")
    w = make_weights(wl.dims, wl.seed_w)
    rng = np.random.default_rng(33)
    prompts = [rng.integers(0, wl.dims.vocab, n).astype(np.int32) for n in (250, 20, 131)]
    got = []
    for rows, together in ((64, True), (256, True), (128, False)):
        rt = Runtime(wl.dims, wl.block, 3, 300, w, max_rows=rows, kv_cache="fp8")
        first = torch.zeros(3, dtype=torch.int32, device="cuda")
        if together:
            rt.prefill_batch(torch.from_numpy(np.concatenate(prompts)).cuda(), [len(p) for p in prompts], first)
        else:
            for s, p in enumerate(prompts):
                rt.prefill(s, torch.from_numpy(p).cuda(), first[s:s + 1])
        torch.cuda.synchronize()
        assert rt.status() == 0
        got.append((first.cpu().numpy(), [cached(rt, s, len(p)) for s, p in enumerate(prompts)]))
        rt.close()
    for first, kv in got[1:]:
        np.testing.assert_array_equal(first, got[0][0])
        for s in range(3):
            for a, b in zip(kv[s], got[0][1][s]):
                for i in (0, 1):
                    # (layer 0's rows are the same, so its codes are; below, a subnormal's rounding travels on)
                    scale = np.maximum(a[2 + i], b[2 + i])
                    off = np.abs(a[i] - b[i])
                    assert (off <= 2.0 ** -3 * np.abs(b[i]) + 2.0 ** -9 * scale).mean() > 0.999
        for i in (0, 1):
            a, b = kv[0][0], got[0][1][0][0]
            assert (np.abs(a[i] - b[i]) <= 2.0 ** -9 * np.maximum(a[2 + i], b[2 + i])).all()


def _engine(name, slots, kv_cache, num_pages, temperature=None, carry=True):
    from paper_2609_06498_amd import Runtime
    from paper_2609_06498_amd.engine import Engine
    wl = get_config(name)
    w = make_weights(wl.dims, wl.seed_w)
    rng = np.random.default_rng([wl.seed_prompt, 78])
    rt = Runtime(wl.dims, wl.block, 3, 400, w, wl.carry_window, kv_cache=kv_cache, num_pages=num_pages)
    eng = Engine(rt, max_active=slots, carry_on=carry, temperature=temperature, sample_seed=9)
    rids = [eng.submit(rng.integers(0, wl.dims.vocab, int(rng.integers(5, 300))).astype(np.int32), n)
            for n in (1, 9, 40, 17, 30, 3)]
    outs = eng.run()
    torch.cuda.synchronize()
    assert rt.status() == 0
    if num_pages is not None:
        assert eng.pool.status() == 0 and int(eng.pool.n_free) == num_pages and eng.free_pages == num_pages
        assert eng.pool.n_held.sum() == 0 and sorted(eng.pool.free_pages.cpu().tolist()) == list(range(num_pages))
    rt.close()
    return [outs[r] for r in rids]


@pytest.mark.parametrize("kv_cache", ["model", "fp8"])
@pytest.mark.parametrize("name", ["tiny-f32", "small-bf16"])
def test_serving_from_a_page_pool(name, kv_cache):
    """The tokens of slots that own whole rows, from pools that hold three, two and one request at a time."""
    whole = _engine(name, 3, kv_cache, None)
    for pages in (21, 11, 7):
        assert _engine(name, 3, kv_cache, pages) == whole, pages
    assert _engine(name, 1, kv_cache, 7) == whole


def test_sampled_serving_from_a_page_pool():
    whole = _engine("small-bf16", 3, "fp8", None, temperature=0.8)
    assert _engine("small-bf16", 2, "fp8", 12, temperature=0.8) == whole


def test_requests_beyond_the_pool_are_refused():
    from paper_2609_06498_amd import Runtime
    from paper_2609_06498_amd.engine import Engine
    from paper_2609_06498_amd.runtime import DFlowError
    wl = get_config("tiny-f32")
    w = make_weights(wl.dims, wl.seed_w)
    rt = Runtime(wl.dims, wl.block, 2, 600, w, kv_cache="fp8", num_pages=3)
    eng = Engine(rt)
    with pytest.raises(DFlowError, match="pool"):
        eng.submit(np.zeros(200, np.int32), 10)
    # a prefill without pages: nothing is written, the status says so
    rt.prefill(0, torch.zeros(10, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert rt.status() == 4 and int(rt.kv8[0].sum()) == 0
    rt.close()
    for bad in (dict(kv_cache="int4"), dict(num_pages=0)):
        with pytest.raises(DFlowError):
            Runtime(wl.dims, wl.block, 2, 600, w, **bad)


def test_round_over_the_8_bit_cache_captured():
    """A greedy round recorded into a graph and replayed, with eager work between the replays, gives the eager rounds."""
    from paper_2609_06498_amd import Runtime
    from paper_2609_06498_amd.session import Session
    wl = get_config("small-bf16")
    w = make_weights(wl.dims, wl.seed_w)
    rng = np.random.default_rng(35)
    prompts = [rng.integers(0, wl.dims.vocab, n).astype(np.int32) for n in (100, 40)]
    runs = []
    for graph in (False, True):
        rt = Runtime(wl.dims, wl.block, 2, 500, w, wl.carry_window, kv_cache="fp8")
        s = Session(rt, 2)
        s.prefill(prompts)
        s.round()
        replay = s.capture_round() if graph else s.round
        out = []
        for _ in range(4):
            replay()
            torch.cuda.synchronize()
            out.append((s.committed.cpu().numpy().copy(), s.seq_len.cpu().numpy().copy()))
        assert rt.status() == 0
        runs.append(out)
        rt.close()
    for a, b in zip(*runs):
        np.testing.assert_array_equal(a[0], b[0])
        np.testing.assert_array_equal(a[1], b[1])


def test_an_engine_after_one_that_was_given_up():
    """A pool's pages belong to the engine that was built last."""
    from paper_2609_06498_amd import Runtime
    from paper_2609_06498_amd.engine import Engine
    wl = get_config("tiny-f32")
    w = make_weights(wl.dims, wl.seed_w)
    rng = np.random.default_rng(4)
    prompts = [rng.integers(0, wl.dims.vocab, n).astype(np.int32) for n in (150, 90, 120)]
    outs = []
    for given_up in (False, True):
        rt = Runtime(wl.dims, wl.block, 3, 400, w, kv_cache="fp8", num_pages=9)
        if given_up:
            eng = Engine(rt)
            for p in prompts[1:]:
                eng.submit(p, 30)
            eng._admit()
            torch.cuda.synchronize()
            assert int(rt.page_pool.n_free) < 9
        eng = Engine(rt)
        rids = [eng.submit(p, 12) for p in prompts]
        got = eng.run()
        torch.cuda.synchronize()
        assert rt.status() == 0 and eng.pool.status() == 0 and int(eng.pool.n_free) == 9
        outs.append([got[r] for r in rids])
        rt.close()
    assert outs[0] == outs[1]
