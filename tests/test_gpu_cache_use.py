"""Rotation, append and shared-prefix attention in the calls that a serving program makes: one sequence, outputs in place, shared heads as views of
stride 0, decoding captured into a graph while the caches grow."""
import numpy as np
import pytest
import torch

import cache_testlib as C
from paper_2602_05305_amd import flashblock as fb
from test_gpu_shared import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,Bq,shared,own", [
    (8, 2, 128, 1, 3000, 100), (8, 2, 64, 1, 64, 0), (4, 4, 64, 32, 1000, 333), (32, 8, 128, 40, 2100, 65), (1, 1, 64, 1, 0, 1), (4, 1, 128, 16, 0, 5000),
])
def test_one_sequence(dtype, Hq, Hkv, d, Bq, shared, own):
    Case(dtype, 1, Hq, Hkv, d, Bq, shared, [own], 64, seed=41).run()


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,Bq,shared,own", [
    ("bf16", 3, 8, 2, 128, 40, 1000, 100), ("bf16", 2, 4, 4, 64, 130, 700, 65), ("bf16", 40, 8, 2, 64, 8, 500, 300), ("f32", 3, 8, 2, 128, 40, 1000, 100),
    ("f32", 2, 4, 4, 64, 130, 700, 65), ("f32", 40, 8, 2, 64, 2, 500, 300), ("f32", 5, 4, 1, 128, 32, 300, 64), ("f32", 5, 4, 1, 64, 16, 0, 64),
    ("f32", 3, 4, 2, 64, 8, 0, 0),
])
def test_out_in_the_place_of_q(dtype, B, Hq, Hkv, d, Bq, shared, own):
    """(blocks of more than 32 keys have another kernel for it: not the same bits)"""
    c = Case(dtype, B, Hq, Hkv, d, Bq, shared, [own * i // max(1, B - 1) for i in range(B)], 64, seed=42)
    c.out = c.q
    c.refresh()
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_and_sequences_that_coincide(dtype):
    """One head's and one sequence's rows, expanded, give what copies of them give."""
    rng = np.random.default_rng(43)
    B, Hq, Hkv, d, n, page = 3, 6, 3, 64, 5, 64
    one = C.rows_tensor(rng, dtype, 1, 1, n, d, True)
    inv = torch.from_numpy(C.inv_freq(32)).to(C.DEV)
    first = torch.tensor([4, 0, 61], dtype=torch.int32, device=C.DEV)
    shape, rot = fb.make_shape(B, Hq, Hkv, d, n, 2 * page, dtype), fb.make_rotary(inv, [32], first=first)
    table = torch.arange(2 * B, dtype=torch.int32, device=C.DEV).view(B, 2)
    results = []
    for view in (lambda h: one.expand(B, h, n, d), lambda h: one.expand(B, h, n, d).contiguous()):
        q, k, v = view(Hq), view(Hkv), view(Hkv)
        outs = [torch.empty(B, h, n, d, device=C.DEV, dtype=C.TORCH[dtype]) for h in (Hq, Hkv, Hkv)]
        fb.fb_rotate_block(shape, rot, q, k, v, *outs)
        pools = [torch.zeros(2 * B, Hkv, page, d, device=C.DEV, dtype=C.TORCH[dtype]) for _ in range(2)]
        fb.fb_append_paged(shape, fb.make_paged_kv(*pools, table, first), rot, k, v)
        results.append(outs + pools)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert torch.equal(results[0][3][0, :, 4:4 + n], results[0][1][0]) and torch.equal(results[0][3][5, :, :2], results[0][1][2][:, 3:])


@pytest.mark.parametrize("dtype,B,Hq,Hkv,d,Bq,S,start,page,steps", [
    ("bf16", 5, 8, 2, 128, 1, 700, [0, 60, 63, 64, 126], 64, 5),
    ("bf16", 140, 4, 4, 128, 4, 70, [i % 60 for i in range(140)], 64, 3),
    ("bf16", 140, 4, 4, 128, 1, 70, [(37 * i) % 561 for i in range(140)], 64, 3),      # sequences by length
    ("bf16", 22, 1, 1, 128, 1, 10, [6 * i for i in range(22)], 64, 4),           # own keys as splits
    ("bf16", 3, 4, 2, 64, 40, 300, [0, 30, 100], 128, 3),
    ("bf16", 4, 4, 2, 64, 2, 0, [0, 5, 62, 200], 64, 3),                         # nothing shared
    ("f32", 137, 2, 2, 128, 1, 70, [4 * i for i in range(137)], 64, 3),          # ordered by a launch
    ("f32", 4, 8, 2, 64, 7, 500, [0, 5, 62, 200], 64, 4),
])
def test_captured_decoding_while_the_caches_grow(dtype, B, Hq, Hkv, d, Bq, S, start, page, steps):
    """Rotation, step and append in one graph: every replay, with eager work between them, against the same calls made one by one."""
    print(f"[case] decoding {dtype} {B}x{Bq} {Hq}/{Hkv} d={d} shared={S} page={page}", flush=True)
    g = torch.Generator(device=C.DEV)
    g.manual_seed(44)
    tdt = C.TORCH[dtype]
    capacity = max(start) + (steps + 1) * Bq
    per, ns = -(-capacity // page), -(-S // page)
    pool = [torch.randn(ns + B * per, Hkv, page, d, generator=g, device=C.DEV).to(tdt) for _ in range(2)]
    ids = torch.randperm(ns + B * per, generator=g, device=C.DEV).to(torch.int32)
    shared = ids[:ns].contiguous() if S else None
    table = ids[ns:].view(B, per).contiguous()
    inv = torch.from_numpy(C.inv_freq(d // 2)).to(C.DEV)
    fused = torch.randn(B, Bq, Hq + 2 * Hkv, d, generator=g, device=C.DEV).to(tdt)
    heads = fused.transpose(1, 2)
    shape = fb.make_shape(B, Hq, Hkv, d, Bq, capacity, dtype)

    class Side:
        def __init__(self):
            self.k_pool, self.v_pool = (x.clone() for x in pool)
            self.lens = torch.tensor(start, dtype=torch.int32, device=C.DEV)
            self.next = torch.empty_like(self.lens)
            self.q, self.k, self.v = (torch.empty(B, h, Bq, d, device=C.DEV, dtype=tdt) for h in (Hq, Hkv, Hkv))
            self.o, self.m, self.lse = torch.empty(B, Hq, Bq, d, device=C.DEV), torch.empty(B, Hq, Bq, device=C.DEV), torch.empty(B, Hq, Bq, device=C.DEV)
            self.out, self.lse_out = torch.empty_like(self.q), torch.empty_like(self.lse)
            self.ws = torch.empty(fb.fb_shared_workspace_bytes(shape, S), device=C.DEV, dtype=torch.uint8)
            self.rot = fb.make_rotary(inv, [d // 2], first=self.lens, offset=S)
            self.kv = fb.make_paged_kv(self.k_pool, self.v_pool, table, self.lens)

        def step(self):
            fb.fb_rotate_block(shape, self.rot, heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], self.q, self.k, self.v)
            fb.fb_refresh_step_shared(shape, self.q, self.kv, shared, S, self.k, self.v, self.o, self.m, self.lse, self.out, self.lse_out, self.ws)
            fb.fb_append_paged(shape, self.kv, None, self.k, self.v, None, None, None, self.next)
            self.lens.copy_(self.next)

        def all(self):
            return self.k_pool, self.v_pool, self.lens, self.out, self.lse_out, self.o, self.m, self.lse

    captured, eager = Side(), Side()
    captured.step()
    eager.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for i in range(steps):
        fused.mul_(0.9).add_(0.05)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured.all(), eager.all())), f"replay {i}"
    assert captured.lens.tolist() == [n + (steps + 1) * Bq for n in start]
    assert bool(torch.isfinite(captured.out.float()).all())
