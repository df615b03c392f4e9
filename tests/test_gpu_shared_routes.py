"""Shared prefix: every kind of workgroup that the plan picks, with the own keys in the second launch and as splits of the first, in one round of the
second launch's workgroups and in several (sequences by length); pools and views beyond 32-bit offsets."""
import numpy as np
import pytest
import torch

import cache_testlib as C
import fb_testlib as T
from paper_2602_05305_amd import flashblock as fb
from test_gpu_shared import Case

pytestmark = pytest.mark.gpu


# rows of the first launch's workgroups (256: of 8 wavefronts, or of 4); own keys: "finish", "order" (long ones, several rounds: sequences by length), "split", "none"
@pytest.mark.parametrize("B,Hq,Hkv,d,Bq,shared,own,page", [
    (108, 4, 4, 64, 1, 65, 1, 64),            # 32 rows, finish
    (50, 8, 4, 64, 1, 2087, 1, 192),
    (131, 2, 2, 64, 1, 5460, 70, 64),
    (133, 4, 4, 64, 1, 62, 30, 64),           # ... in two rounds
    (139, 4, 4, 128, 4, 70, 33, 128),
    (133, 4, 4, 64, 1, 62, 1100, 64),         # 32, order
    (139, 4, 4, 128, 4, 70, 600, 128),
    (22, 1, 1, 128, 1, 10, 140, 64),          # 32, split
    (33, 1, 1, 128, 4, 6777, 300, 64),        # 32, finish
    (138, 4, 4, 64, 16, 25, 65, 64),          # 64, finish
    (138, 4, 4, 64, 16, 25, 1050, 64),        # 64, order
    (35, 2, 2, 128, 1, 4144, 70, 64),         # 64, split
    (33, 8, 4, 128, 2, 1543, 33, 64),         # 128, finish
    (11, 8, 4, 64, 3, 6221, 1, 64),
    (132, 4, 4, 128, 1, 1590, 100, 64),
    (132, 4, 4, 128, 1, 1590, 520, 64),       # 128, order
    (65, 2, 1, 64, 32, 982, 1, 64),           # 128, split
    (9, 2, 2, 128, 11, 4199, 33, 64),
    (65, 16, 4, 64, 1, 8174, 1, 64),          # 256 of 8 wavefronts, finish
    (113, 32, 4, 128, 3, 2096, 1, 64),
    (43, 8, 2, 128, 32, 2073, 1, 64),
    (130, 8, 1, 64, 11, 970, 33, 64),
    (136, 2, 2, 128, 40, 1893, 70, 64),       # ... blocks that the second launch leaves to the internal pass
    (136, 2, 2, 128, 40, 1893, 530, 64),      # ... order
    (27, 1, 1, 128, 200, 4179, 1500, 64),     # ... split
    (4, 2, 2, 64, 200, 8095, 1500, 64),
    (130, 32, 4, 128, 3, 3239, 0, 64),        # 256 of 4, none
    (39, 8, 4, 64, 40, 2572, 1, 64),          # ... finish
    (134, 4, 4, 64, 8, 7741, 70, 128),
    (134, 4, 4, 64, 8, 7741, 1030, 128),      # ... order
    (97, 16, 4, 128, 8, 3113, 60, 64),        # ... finish
    (45, 8, 4, 128, 31, 3962, 1, 256),
    (103, 16, 2, 64, 8, 3588, 1, 64),
    (4, 4, 2, 64, 200, 7168, 70, 64),         # ... split
    (13, 4, 4, 128, 100, 7354, 3000, 64),
    (63, 2, 2, 128, 1, 75, 70, 64),           # one row to a workgroup of the second launch
    (2, 16, 4, 128, 8, 13937, 3, 128),
    (4, 8, 1, 128, 1, 4095, 99, 64),
    (121, 1, 1, 128, 3, 137, 70, 64),         # two, the last one of a sequence short
    (46, 2, 2, 64, 3, 53, 1, 64),
    (61, 4, 2, 128, 3, 14, 70, 64),           # four, short
    (45, 4, 4, 64, 3, 13, 1, 64),
    (5, 4, 1, 128, 32, 26862, 31, 64),        # four, many splits
    (125, 4, 2, 128, 3, 15, 1, 64),           # eight, short
    (49, 2, 1, 64, 11, 11, 1, 64),
    (126, 2, 2, 128, 11, 11, 1, 64),          # 16, short
    (139, 4, 1, 64, 3, 13, 1, 64),
])
def test_routes(B, Hq, Hkv, d, Bq, shared, own, page):
    rng = np.random.default_rng(B * 1000 + own)
    lens = rng.integers(0, own + 1, size=B)
    lens[-1] = own
    Case("bf16", B, Hq, Hkv, d, Bq, shared, lens, page, seed=B).run()


def test_infinite_and_nan_keys_of_other_slots_stay_out():
    """A last own and a last shared key of weight and value as they are; the slots behind them, and every other page, hold infinities."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 3, 4, 2, 128, 4, 77, [5, 0, 65], 64)
        for pool in (c.k_pool, c.v_pool):
            pool.nan_to_num_(float("inf"))
        c.run()


def test_an_infinite_value_of_one_sequence_stays_there():
    """An infinity among one sequence's own values: its rows are infinite, those of the others as without it, also behind short tiles."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 4, 4, 2, 64, 3, 100, [33, 70, 1, 20], 64)
        want = c.want_partial()
        page = int(c.table[1, 1])
        c.v_pool[page, :, 5, 7] = float("inf")                   # the last of 70 keys
        c.refresh()
        torch.cuda.synchronize()
        out = c.out.double().cpu().numpy()
        assert np.isposinf(out[1, ..., 7]).all() and np.isfinite(np.delete(out[1], 7, axis=-1)).all()
        keep = [0, 2, 3]
        T.check_partial({k: v[keep] for k, v in c.ext.numpy().items()}, {k: v[keep] for k, v in want.items()}, dtype, "others")


def test_pools_beyond_32_bit_offsets():
    """Pages at the end of pools of more than 2^31 elements: appended to, and attended to, as at the start."""
    B, Hq, Hkv, d, page, S, n = 3, 16, 8, 128, 256, 300, 9
    pages = (1 << 31) // (Hkv * page * d) + 8
    k_pool, v_pool = (torch.empty(pages, Hkv, page, d, device=T.DEV, dtype=torch.bfloat16) for _ in range(2))
    assert k_pool.numel() > 1 << 31
    g = torch.Generator(device=T.DEV)
    g.manual_seed(3)
    q, k, v = (torch.randn(B, h, n, d, generator=g, device=T.DEV, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    sk, sv = (torch.randn(1, Hkv, S, d, generator=g, device=T.DEV, dtype=torch.bfloat16) for _ in range(2))
    results = []
    for base in (0, pages - 5):
        ids = torch.tensor([4, 1, 0, 3, 2], dtype=torch.int32, device=T.DEV) + base
        shared, table = ids[:2].contiguous(), ids[2:, None].contiguous()
        zero, lens = torch.zeros(B, dtype=torch.int32, device=T.DEV), torch.empty(B, dtype=torch.int32, device=T.DEV)
        fb.fb_append_paged(fb.make_shape(1, Hq, Hkv, d, S, 2 * page, "bf16"), fb.make_paged_kv(k_pool, v_pool, shared[None], zero), None, sk, sv)
        shape = fb.make_shape(B, Hq, Hkv, d, n, page, "bf16")
        fb.fb_append_paged(shape, fb.make_paged_kv(k_pool, v_pool, table, zero), None, k, v, lens_out=lens)
        assert torch.equal(k_pool[ids[2].long(), :, :n], k[0]) and torch.equal(v_pool[ids[4].long(), :, :n], v[2])
        o, m, lse = torch.empty(B, Hq, n, d, device=T.DEV), torch.empty(B, Hq, n, device=T.DEV), torch.empty(B, Hq, n, device=T.DEV)
        out = torch.empty_like(q)
        ws = torch.empty(fb.fb_shared_workspace_bytes(shape, S), device=T.DEV, dtype=torch.uint8)
        fb.fb_refresh_step_shared(shape, q, fb.make_paged_kv(k_pool, v_pool, table, lens), shared, S, k, v, o, m, lse, out, None, ws)
        results.append((o, m, lse, out))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and bool(torch.isfinite(results[0][3].float()).all())


def test_views_beyond_32_bit_strides():
    """A batch stride of more than 2^31 elements, read and written."""
    B, H, n, d, far = 2, 2, 3, 64, (1 << 31) + 64
    buf = torch.empty(far + H * n * d, device=T.DEV, dtype=torch.bfloat16)
    wide = buf.as_strided((B, H, n, d), (far, d, H * d, 1))
    x = torch.randn(B, H, n, d, device=T.DEV).to(torch.bfloat16)
    inv = torch.from_numpy(C.inv_freq(32)).to(T.DEV)
    shape, rot = fb.make_shape(B, H, H, d, n, 0, "bf16"), fb.make_rotary(inv, [32], offset=5)
    want, got = torch.empty_like(x), torch.empty_like(x)
    fb.fb_rotate_block(shape, rot, x, None, None, want, None, None)
    fb.fb_rotate_block(shape, rot, x, None, None, wide, None, None)
    assert torch.equal(wide, want)
    wide.copy_(x)
    fb.fb_rotate_block(shape, rot, wide, None, None, got, None, None)
    assert torch.equal(got, want)


def test_two_calls_at_once():
    """Calls of their own workspaces on two streams, many in flight, against the same calls one by one."""
    cases = [Case("bf16", 6, 8, 2, 128, 4, 3000, [40 * i for i in range(6)], 64, seed=s) for s in (1, 2)]
    want = []
    for c in cases:
        c.refresh()
        torch.cuda.synchronize()
        want.append((c.out.clone(), c.ext.lse.clone()))
        c.out.zero_()
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for c, s in zip(cases, streams):
            c.refresh(stream=s)
    torch.cuda.synchronize()
    for c, (out, lse) in zip(cases, want):
        assert torch.equal(c.out, out) and torch.equal(c.ext.lse, lse)


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,Bq,shared", [
    ("bf16", 22, 1, 1, 128, 1, 10), ("bf16", 35, 2, 2, 128, 1, 4145), ("bf16", 132, 4, 4, 128, 1, 1591), ("bf16", 113, 32, 4, 128, 3, 2096), ("bf16", 130, 32, 4, 128, 3, 3239),
    ("bf16", 108, 4, 4, 64, 1, 65), ("bf16", 50, 8, 4, 64, 1, 2087), ("bf16", 131, 2, 2, 64, 1, 5460), ("bf16", 39, 8, 4, 64, 40, 2572),
    ("f32", 3, 4, 2, 64, 5, 1000), ("f32", 9, 8, 2, 128, 8, 130),
])
def test_an_infinite_value_of_the_last_shared_key(dtype, B, Hq, Hkv, d, Bq, shared):
    """In front of the masked rest of a tile, in every kind of workgroup: its column of its KV head is infinite, nothing else is."""
    c = Case(dtype, B, Hq, Hkv, d, Bq, shared, [0] * B, 64, prefix=1)
    page, at = int(c.pages[(shared - 1) // 64]), (shared - 1) % 64
    c.v_pool[page, 0, at, 7] = float("inf")
    c.refresh()
    torch.cuda.synchronize()
    out = c.out.double().cpu().numpy()
    first = Hq // Hkv
    assert np.isposinf(out[:, :first, :, 7]).all()
    out[:, :first, :, 7] = 0
    assert np.isfinite(out).all()


# fp32: rows of the workgroups of the shared keys and of the own ones (64 with a wavefront's parts of the columns, or without: head_dim 64); of one kind
# they are one launch; "order": sequences by length
@pytest.mark.parametrize("B,Hq,Hkv,d,Bq,shared,own,page", [
    (274, 1, 1, 64, 1, 70, 600, 64),          # 16 16 order
    (137, 2, 2, 128, 1, 70, 600, 192),
    (26, 8, 4, 64, 20, 70, 1, 64),            # 32 32
    (13, 16, 2, 128, 20, 70, 65, 64),
    (65, 2, 2, 64, 20, 130, 600, 64),         # 32 32 order
    (132, 1, 1, 128, 20, 300, 600, 128),
    (13, 32, 4, 64, 20, 70, 64, 64),          # 64 64
    (26, 16, 2, 64, 20, 300, 200, 64),        # 64 in parts, both
    (205, 2, 1, 128, 20, 70, 33, 64),
    (131, 2, 1, 64, 20, 700, 600, 64),        # ... order
    (133, 1, 1, 128, 40, 300, 600, 64),
    (9, 1, 1, 64, 40, 70, 900, 64),           # 16 and 64
    (13, 2, 1, 128, 20, 70, 600, 64),         # 16 and 64 in parts
    (174, 8, 4, 64, 1, 300, 600, 64),         # 32 and 16, order
    (171, 2, 2, 64, 4, 700, 600, 64),         # 64 and 16, order
    (129, 2, 2, 128, 4, 1500, 600, 64),       # 64 in parts and 16, order
    (87, 4, 4, 64, 1, 0, 600, 64),            # own keys alone, order
])
def test_routes_f32(B, Hq, Hkv, d, Bq, shared, own, page):
    rng = np.random.default_rng(B * 1000 + own)
    lens = rng.integers(0, own + 1, size=B)
    lens[-1] = own
    Case("f32", B, Hq, Hkv, d, Bq, shared, lens, page, seed=B).run()


@pytest.mark.parametrize("B,Hq,Hkv,d,Bq,shared", [(26, 8, 4, 64, 20, 70), (13, 16, 2, 128, 20, 70), (13, 32, 4, 64, 20, 70), (26, 16, 2, 64, 20, 300), (205, 2, 1, 128, 20, 70)])
def test_infinite_values_of_last_keys_f32(B, Hq, Hkv, d, Bq, shared):
    """The last shared key's in one column, one sequence's last own key's in another."""
    c = Case("f32", B, Hq, Hkv, d, Bq, shared, [3] * B, 64)
    c.v_pool[int(c.pages[(shared - 1) // 64]), 0, (shared - 1) % 64, 7] = float("inf")
    c.v_pool[int(c.table[1, 0]), 0, 2, 9] = float("inf")
    c.refresh()
    torch.cuda.synchronize()
    out = c.out.double().cpu().numpy()
    first = Hq // Hkv
    assert np.isposinf(out[:, :first, :, 7]).all() and np.isposinf(out[1, :first, :, 9]).all()
    out[:, :first, :, 7] = out[1, :first, :, 9] = 0
    assert np.isfinite(out).all()
