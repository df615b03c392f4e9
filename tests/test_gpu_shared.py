"""Attention of a batch over a shared prefix and own keys, in pages, against the float64 oracle, which gets each sequence's keys in a row."""
import numpy as np
import pytest
import torch

from oracle import flashblock_oracle as orc
from paper_2602_05305_amd import flashblock as fb
from paper_2602_05305_amd import workloads as wl

import cache_testlib as C
import fb_testlib as T

pytestmark = pytest.mark.gpu


class Case:
    """Keys of a batch in a pool whose every other value is NaN; the tensors of a call."""

    def __init__(self, dtype, B, Hq, Hkv, d, Bq, shared, lens, page, prefix=None, seed=5, scale=1.0):
        print(f"[case] shared {dtype} {B}x{Bq} {Hq}/{Hkv} d={d} shared={shared} lens={list(lens)} page={page} seed={seed}", flush=True)
        rng = np.random.default_rng(seed)
        self.dtype, self.shared, self.lens = dtype, shared, [int(n) for n in lens]
        prefix = max(self.lens) if prefix is None else prefix
        self.w = wl.Workload("shared", B, Hq, Hkv, d, prefix, Bq, 1, 1, dtype, 1.0)

        def normal(*shape):
            return wl.round_storage(rng.standard_normal(shape, dtype=np.float32) * np.float32(scale), dtype)
        self.seqs = [(normal(Hkv, n, d), normal(Hkv, n, d)) for n in [shared] + self.lens]
        need = [-(-n // page) for n in [shared] + self.lens]
        ids = rng.permutation(sum(need) + 2).astype(np.int32)
        pools = [np.full((len(ids), Hkv, page, d), np.nan, dtype=np.float32) for _ in range(2)]
        tables, at = [], 0
        for n, pages, kv in zip([shared] + self.lens, need, self.seqs):
            tables.append(ids[at:at + pages])
            at += pages
            for j in range(pages):
                lo, hi = j * page, min(n, (j + 1) * page)
                for pool, x in zip(pools, kv):
                    pool[tables[-1][j], :, :hi - lo] = x[:, lo:hi]
        table = np.full((B, max(1, -(-prefix // page))), -1, dtype=np.int32)
        for b, t in enumerate(tables[1:]):
            table[b, :len(t)] = t
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(T.DEV)
        self.k_pool, self.v_pool = (T.to_dev(x, dtype) for x in pools)
        self.table, self.prefix_lens, self.pages = dev(table), dev(np.asarray(self.lens, dtype=np.int32)), dev(tables[0])
        self.Q, self.Kb, self.Vb = normal(B, Hq, Bq, d), normal(B, Hkv, Bq, d), normal(B, Hkv, Bq, d)
        self.q, self.kb, self.vb = (T.to_dev(x, dtype) for x in (self.Q, self.Kb, self.Vb))
        self.shape = T.shape_of(self.w)
        self.kv = fb.make_paged_kv(self.k_pool, self.v_pool, self.table, self.prefix_lens)
        self.bytes = fb.fb_shared_workspace_bytes(self.shape, shared)
        self.buffers()

    def buffers(self):
        self.ext = T.Partial(self.w)
        self.out = torch.full_like(self.q, float("nan"))
        self.lse_out = torch.full(self.q.shape[:3], float("nan"), device=T.DEV)
        self.ws = torch.full((self.bytes + 512,), 0xA5, device=T.DEV, dtype=torch.uint8)     # (as floats -2.9e-16; nothing is to be read before it is written)

    def partial(self, stream=None):
        fb.fb_external_partial_shared(self.shape, self.q, self.kv, self.pages if self.shared else None, self.shared, self.ext.o, self.ext.m, self.ext.lse,
                                      self.ws[:self.bytes], stream)

    def refresh(self, lse=True, stream=None):
        fb.fb_refresh_step_shared(self.shape, self.q, self.kv, self.pages if self.shared else None, self.shared, self.kb, self.vb, self.ext.o, self.ext.m,
                                  self.ext.lse, self.out, self.lse_out if lse else None, self.ws[:self.bytes], stream)

    def want_partial(self):
        Ks, Vs = self.seqs[0]
        parts = []
        for b, (K, V) in enumerate(self.seqs[1:]):
            K, V = np.concatenate([Ks, K], axis=1)[None], np.concatenate([Vs, V], axis=1)[None]
            parts.append(orc.partial(self.Q[b:b + 1], K, V) if K.shape[2] else orc.empty_partial(1, self.w.n_q_heads, self.w.block_len, self.w.head_dim))
        return {k: np.concatenate([p[k] for p in parts], axis=0) for k in ("o", "m", "lse")}

    def check(self, want=None, step=True):
        torch.cuda.synchronize()
        want = self.want_partial() if want is None else want
        T.check_partial(self.ext.numpy(), want, self.dtype, "shared ext")
        if step:
            out, lse = orc.merge(want, orc.partial(self.Q, self.Kb, self.Vb))
            T.assert_close(self.out.double().cpu().numpy(), out, self.dtype, "shared out")
            T.assert_close(self.lse_out.double().cpu().numpy(), lse, self.dtype, "shared lse", lse=True)
        assert bool((self.ws[self.bytes:] == 0xA5).all()), "written behind the workspace"

    def run(self):
        want = self.want_partial()
        self.partial()
        self.check(want, step=False)
        self.buffers()
        self.refresh()
        self.check(want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,d,Bq,shared,lens,page", [
    (2, 1, 1, 64, 1, 1, [1, 0], 64),                               # the smallest: one row a sequence, one key
    (3, 4, 2, 64, 1, 63, [0, 64, 65], 64),
    (2, 4, 4, 128, 5, 64, [0, 0], 64),                             # own caches empty
    (3, 4, 2, 128, 4, 0, [70, 0, 3], 64),                          # nothing shared; a row with no key at all
    (2, 2, 1, 64, 3, 0, [0, 0], 64),                               # no key anywhere
    (4, 8, 2, 128, 8, 1000, [5, 300, 64, 129], 128),               # 128 rows a KV head
    (5, 8, 2, 128, 8, 1000, [5, 300, 64, 129, 0], 128),            # 160
    (7, 8, 8, 64, 9, 2113, [1, 2, 3, 64, 65, 127, 128], 64),       # 63 rows, odd everything
    (16, 4, 1, 128, 16, 1300, [17 * i for i in range(16)], 256),   # 1024 rows
    (33, 8, 2, 64, 8, 777, [3 * i for i in range(33)], 64),        # 1056 rows, the last workgroup short
    (6, 32, 1, 128, 11, 650, [0, 9, 90, 200, 31, 64], 64),         # 32 query heads to a KV head
    (9, 12, 12, 128, 40, 515, [4, 40, 400, 0, 1, 2, 3, 5, 6], 128),
    (2, 4, 2, 128, 70, 4097, [100, 33], 256),                      # a block beyond 64 rows
    (130, 2, 1, 64, 1, 200, [i % 70 for i in range(130)], 64),     # more sequences than are ranked inside the kernel
])
def test_shared_matches_oracle(dtype, B, Hq, Hkv, d, Bq, shared, lens, page):
    Case(dtype, B, Hq, Hkv, d, Bq, shared, lens, page).run()


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,Bq,shared,lens,page", [
    ("bf16", 8, 8, 1, 128, 32, 16384 + 17, [100 * i for i in range(8)], 256),       # long streams, many rows
    ("bf16", 8, 8, 1, 64, 32, 16384 + 17, [100 * i for i in range(8)], 64),
    ("bf16", 4, 4, 1, 128, 1, 40001, [0, 64, 1000, 7], 64),                         # 16 rows, 626 pages
    ("bf16", 64, 4, 1, 128, 1, 8192, [8 * i for i in range(64)], 256),              # 256 rows
    ("f32", 4, 4, 1, 64, 16, 5003, [0, 64, 1000, 7], 64),
])
def test_shared_long(dtype, B, Hq, Hkv, d, Bq, shared, lens, page):
    Case(dtype, B, Hq, Hkv, d, Bq, shared, lens, page, seed=6).run()


def test_no_own_pages_at_all():
    """prefix_len 0: table, lengths and max_pages are not looked at."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 3, 4, 2, 64, 6, 300, [0, 0, 0], 64, prefix=0)
        c.kv.block_table = c.kv.prefix_lens = None
        c.kv.max_pages = -1
        c.run()


def test_one_slab_is_a_pool_of_one_page():
    c = Case("bf16", 4, 8, 2, 128, 4, 2048, [0] * 4, 2048, prefix=0)
    c.run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_as_the_paged_step_over_all_pages(dtype):
    """The paged step whose tables list the shared pages first: the same keys, other sums."""
    c = Case(dtype, 5, 8, 2, 128, 8, 1024, [0, 10, 200, 128, 77], 128)
    c.refresh()
    table = torch.cat([c.pages[None].expand(5, -1), c.table], dim=1).contiguous()
    lens = c.prefix_lens + 1024
    shape = T.shape_of(c.w, prefix_len=1024 + c.w.prefix_len)
    kv = fb.make_paged_kv(c.k_pool, c.v_pool, table, lens)
    other, out, lse = T.Partial(c.w), torch.empty_like(c.q), torch.empty_like(c.lse_out)
    ws = T.workspace(shape, n_splits=fb.fb_paged_splits(shape))
    fb.fb_refresh_step_paged(shape, c.q, kv, c.kb, c.vb, other.o, other.m, other.lse, out, lse, ws)
    torch.cuda.synchronize()
    T.check_partial(c.ext.numpy(), other.numpy(), dtype, "against the paged step")
    T.assert_close(c.out.double().cpu().numpy(), out.double().cpu().numpy(), dtype, "out against the paged step")


def test_lengths_are_clamped_and_bad_pages_stay_in_the_pool():
    c = Case("bf16", 3, 4, 2, 64, 4, 200, [64, 100, 3], 64)
    c.prefix_lens.copy_(torch.tensor([64, 10 ** 6, 3], dtype=torch.int32))            # clamped to 100
    c.refresh()
    c.check()
    c = Case("bf16", 3, 4, 2, 64, 4, 256, [64, 128, 3], 64)
    c.prefix_lens[2] = -5
    c.k_pool.nan_to_num_(0.5)
    c.v_pool.nan_to_num_(0.5)
    c.pages[1], c.pages[2], c.table[1, 0] = -7, 10 ** 6, 1 << 30
    c.refresh()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(c.out.float()).all())


@pytest.mark.parametrize("dtype,B,Bq", [("bf16", 8, 16), ("bf16", 3, 2), ("f32", 5, 7)])
def test_the_same_bits_every_time_and_in_place(dtype, B, Bq):
    c = Case(dtype, B, 8, 2, 128, Bq, 3000, [37 * i for i in range(B)], 64)
    c.refresh()
    first = [t.clone() for t in (c.ext.o, c.ext.m, c.ext.lse, c.out, c.lse_out)]
    c.buffers()
    c.out = c.q                                                                       # out in the place of q
    c.refresh()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.ext.o, c.ext.m, c.ext.lse, c.out, c.lse_out)))


def test_graph_replays_and_streams():
    """Two captured steps with workspaces of their own, replayed on another stream, and an eager call between."""
    cases = [Case("bf16", 4, 8, 2, 128, 8, 1500, [10, 0, 300, 64], 64, seed=s) for s in (8, 9)]
    side = torch.cuda.Stream()
    for c in cases:
        c.refresh(stream=side)
    side.synchronize()
    want = [c.out.clone() for c in cases]
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.refresh()
        graphs.append(g)
    for _ in range(3):
        for c in cases:
            c.out.zero_()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c.out, x) for c, x in zip(cases, want))
        cases[0].refresh(lse=False)
        torch.cuda.synchronize()
        assert torch.equal(cases[0].out, want[0])
    cases[0].check()


def test_large_scores():
    """Scores over some 60 log2 units: references move in mid-stream and differ between the two key sets."""
    Case("bf16", 9, 8, 2, 128, 8, 2500, [61 * i for i in range(9)], 128, scale=2.0, seed=12).run()


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    dtype = ["bf16", "bf16", "f32"][seed % 3]
    Hkv, G, d = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 4, 7])), int(rng.choice([64, 128]))
    B, Bq = int(rng.choice([2, 3, 5, 17, 40])), int(rng.choice([1, 2, 4, 7, 16, 33]))
    while B * Bq * G * Hkv > 6000:
        B = max(2, B // 2)
        Bq = max(1, Bq // 2)
    page = int(rng.choice([64, 128, 192]))
    shared = int(rng.choice([0, 1, 64, 130, 700, 1777, 4000]))
    lens = rng.integers(0, int(rng.choice([1, 60, 500])) + 1, size=B)
    Case(dtype, B, Hkv * G, Hkv, d, Bq, shared, lens, page, seed=seed).run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_block_on_its_way_into_the_cache_and_the_next_one(dtype):
    """The operators as a program has them: two blocks of a batch behind a shared prompt.  The prompt goes into the pool through the append, each
    block's q, k, v come token-major, are rotated, attend to prompt, own cache and themselves, and are appended; the second block sees them."""
    rng = np.random.default_rng(31)
    B, Hq, Hkv, d, Bq, S, page, pairs = 3, 4, 2, 64, 8, 100, 64, 32
    counts = np.array([8, 5, 1], dtype=np.int32)                  # the blocks are padded
    normal = lambda *s: wl.round_storage(rng.standard_normal(s, dtype=np.float32), dtype)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(T.DEV)
    tdt = T.tdtype(dtype)
    inv = C.inv_freq(pairs)
    t_inv, capacity = dev(inv), 2 * Bq
    pages = -(-S // page)
    k_pool, v_pool = (torch.full((pages + B + 1, Hkv, page, d), float("nan"), device=T.DEV, dtype=tdt) for _ in range(2))
    order = rng.permutation(pages + B + 1).astype(np.int32)
    shared_pages, table = dev(order[:pages]), dev(order[pages:pages + B, None])
    # the prompt: one sequence, appended at length 0
    pk, pv = normal(1, Hkv, S, d), normal(1, Hkv, S, d)
    zero = torch.zeros(1, device=T.DEV, dtype=torch.int32)
    rot = fb.make_rotary(t_inv, [pairs])
    fb.fb_append_paged(fb.make_shape(1, Hq, Hkv, d, S, S, dtype), fb.make_paged_kv(k_pool, v_pool, shared_pages[None], zero), rot, T.to_dev(pk, dtype),
                       T.to_dev(pv, dtype))
    turned = lambda x, pos: wl.round_storage(C.rotate(x.astype(np.float64), C.angles(pos[..., None], inv, [pairs]), fb.FB_ROTARY_HALVES), dtype)
    past_k = [turned(pk, np.arange(S)[None])[0] for _ in range(B)]
    past_v = [pv[0] for _ in range(B)]
    lens, lens_next = torch.zeros(B, device=T.DEV, dtype=torch.int32), torch.empty(B, device=T.DEV, dtype=torch.int32)
    shape = fb.make_shape(B, Hq, Hkv, d, Bq, capacity, dtype)
    w = wl.Workload("chain", B, Hq, Hkv, d, capacity, Bq, 1, 1, dtype, 1.0)
    ws = torch.empty(fb.fb_shared_workspace_bytes(shape, S), device=T.DEV, dtype=torch.uint8)
    np_lens = np.zeros(B, dtype=np.int64)
    for _ in range(2):
        fused = normal(B, Bq, Hq + 2 * Hkv, d)
        heads = T.to_dev(fused, dtype).transpose(1, 2)
        q_in, k_in, v_in = heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]
        q, k, v = (torch.empty(B, h, Bq, d, device=T.DEV, dtype=tdt) for h in (Hq, Hkv, Hkv))
        at_own = fb.make_rotary(t_inv, [pairs], first=lens, offset=S)
        fb.fb_rotate_block(shape, at_own, q_in, k_in, v_in, q, k, v)
        ext, out = T.Partial(w), torch.empty_like(q)
        lse = torch.empty(B, Hq, Bq, device=T.DEV)
        fb.fb_refresh_step_shared(shape, q, fb.make_paged_kv(k_pool, v_pool, table, lens), shared_pages, S, k, v, ext.o, ext.m, ext.lse, out, lse, ws)
        fb.fb_append_paged(shape, fb.make_paged_kv(k_pool, v_pool, table, lens), None, k, v, dev(counts), lens_out=lens_next)
        lens.copy_(lens_next)
        pos = S + np_lens[:, None] + np.arange(Bq)
        x = np.moveaxis(fused, 2, 1)
        qr, kr, vr = turned(x[:, :Hq], pos), turned(x[:, Hq:Hq + Hkv], pos), x[:, Hq + Hkv:]
        # a rounding that falls the other way moves a value by a step of its storage: what the attention's tolerance is for
        part = [orc.partial(qr[b:b + 1], past_k[b][None], past_v[b][None]) for b in range(B)]
        part = {n: np.concatenate([p[n] for p in part]) for n in ("o", "m", "lse")}
        want, want_lse = orc.merge(part, orc.partial(qr, kr, vr))
        T.assert_close(out.double().cpu().numpy(), want, dtype, "chain out")
        np.testing.assert_allclose(lse.double().cpu().numpy(), want_lse, atol=1e-5 if dtype == "f32" else 1e-2)
        for b in range(B):
            past_k[b] = np.concatenate([past_k[b], kr[b, :, :counts[b]]], axis=1)
            past_v[b] = np.concatenate([past_v[b], vr[b, :, :counts[b]]], axis=1)
        np_lens += counts
        assert lens.tolist() == np_lens.tolist()
