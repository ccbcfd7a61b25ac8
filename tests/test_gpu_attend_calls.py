"""finch_attend in the ways it is called: eagerly and in a replayed graph, many problems of different length in one batch."""
import random

import pytest
import torch

import paper_2408_00167_amd as F
from tests.test_attend_plan_cpu import plan
from tests.test_gpu_attend import problem, verify

pytestmark = pytest.mark.gpu

# dtype, channels, heads, 8 bits; (n_que, c, m) of the problems: one workgroup a tile of rows, a few splits, many
CALLS = [
    ("bf16", 128, 4, 0, [(1, 1408, 100), (1, 3900, 100), (1, 20, 1), (1, 20000, 3)]),
    ("bf16", 128, 4, 64, [(1, 30000, 77), (1, 100, 1)]),
    ("bf16", 128, 4, 0, [(4, 20000, 4), (2, 5000, 2)]),
    ("bf16", 128, 4, 0, [(8, 20000, 8), (5, 3000, 5), (16, 9000, 16)]),
    ("bf16", 128, 1, 0, [(1, 40000, 1)]),
    ("bf16", 64, 8, 0, [(1, 9000, 9), (2, 20000, 9)]),
    ("bf16", 64, 8, 32, [(4, 20000, 9)]),
    ("bf16", 64, 2, 0, [(1, 20000, 9)]),
    ("bf16", 128, 4, 0, [(75, 9000, 75)]),
    ("f32", 64, 1, 0, [(1, 5000, 1), (256, 48, 256)]),
    ("f32", 64, 4, 0, [(17, 3000, 17), (3, 9000, 3)]),
    ("f32", 128, 4, 0, [(1, 5000, 1), (1, 20000, 5)]),
    ("f32", 128, 2, 0, [(17, 3000, 17), (3, 9000, 3)]),
]


@pytest.mark.parametrize("dtype,d,G,block,shapes", CALLS)
def test_a_replayed_call_has_the_eager_call_s_bits(dtype, d, G, block, shapes):
    """The last split to come joins the others in an eager call, a launch of its own in a captured one."""
    fin, gen = F.Finch(F.FINCH_BF16 if dtype == "bf16" else F.FINCH_F32, d, G), torch.Generator().manual_seed(21)
    if block:
        fin.set_scale_block(block)
    pbs = [problem(gen, dtype, d, G, *s, eight=block) for s in shapes]
    batch = F.AttentionBatch(pbs)
    fin.reserve_attend(batch)
    fin.attend(batch)
    torch.cuda.synchronize()
    eager = [(pb["full"].clone(), pb["lse_full"].clone()) for pb in pbs]
    for s, pb in zip(shapes, pbs):
        verify(pb, f"eager {dtype} d={d} G={G} {s}", block or 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        fin.attend(batch)
    for replay in range(3):
        for pb in pbs:
            pb["out"].fill_(9)
            pb["lse"].fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        for s, pb, (out, lse) in zip(shapes, pbs, eager):
            assert torch.equal(pb["full"], out) and torch.equal(pb["lse_full"], lse), f"{dtype} d={d} G={G} {s} replay {replay}"
        fin.attend(batch)
        torch.cuda.synchronize()
    fin.close()


def unlike(rng, n_long, heads):
    """Requests of all kinds, each with a few problems: more groups of like problems than a launch's table has room for."""
    shapes = []
    for i in range(80):
        n = rng.choice([0, 1, 1, 2, 4, 9, 20, rng.randint(1, 90)])
        shapes += [(n, rng.choice([0, 1, 40, rng.randint(0, 600)]), n + rng.choice([0, 0, 3]))] * rng.choice([1, heads])
    for at in (0, 30, 70):
        shapes.insert(at, (n_long, 9000 + at, n_long))
    return shapes


@pytest.mark.parametrize("dtype,d,G,block", [("bf16", 128, 4, 0), ("bf16", 64, 1, 0), ("bf16", 128, 4, 32), ("f32", 64, 2, 0)])
@pytest.mark.parametrize("n_long", [1, 12, 70])
def test_unlike_problems_in_one_batch(dtype, d, G, block, n_long):
    rng = random.Random(n_long)
    fin, gen = F.Finch(F.FINCH_BF16 if dtype == "bf16" else F.FINCH_F32, d, G), torch.Generator().manual_seed(22)
    fin.set_scale_block(block or 64)
    shapes = unlike(rng, n_long, 2)
    pbs = [problem(gen, dtype, d, G, *s, causal=i % 5 != 0, eight=block, lse=i % 3 != 0) for i, s in enumerate(shapes)]
    batch = F.AttentionBatch(pbs)
    fin.attend(batch)
    torch.cuda.synchronize()
    for s, pb in zip(shapes, pbs):
        verify(pb, f"{dtype} d={d} G={G} block={block} {s}", block or 64)
    eager = [pb["full"].clone() for pb in pbs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        fin.attend(batch)
    for _ in range(3):
        for pb in pbs:
            pb["out"].fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        for s, pb, out in zip(shapes, pbs, eager):
            assert torch.equal(pb["full"], out), s
    fin.close()


def test_more_tiles_of_rows_than_a_launch_has_workgroups():
    """Five problems of 2^24 rows (2^20 tiles each): two launches.  One query row for all, one key: every output is its value."""
    fin, gen, n = F.Finch(F.FINCH_F32, 64, 1), torch.Generator().manual_seed(23), 1 << 24
    pbs = []
    for i in range(5):
        q, k, v = (torch.randn(1, 64, generator=gen).cuda() for _ in range(3))
        pbs.append(dict(q=q[:, None].expand(n, 1, 64), k_cache=k, v_cache=v, out=torch.full((n, 1, 64), 7.0, device="cuda"), causal=False))
    fin.attend(F.AttentionBatch(pbs))
    torch.cuda.synchronize()
    for i, pb in enumerate(pbs):
        for part in pb["out"].view(16, -1, 64):
            assert bool((part == pb["v_cache"]).all()), i
    fin.close()


@pytest.mark.parametrize("dtype,d,G,n,kernel", [("bf16", 64, 4, 1, 0), ("bf16", 64, 4, 6, 1), ("f32", 64, 2, 1, 1)])
def test_ragged_requests_whose_last_splits_join(dtype, d, G, n, kernel):
    """Many runs, of one to a few splits each: the last split of each tile of rows joins the others."""
    rng = random.Random(5)
    lengths = [rng.randint(30, 2500) for _ in range(30)]
    shapes = [(n, c, n + 2) for c in lengths for _ in range(24)]
    how = plan([(*s, 1) for s in shapes], kernel, G, d, F.FINCH_BF16 if dtype == "bf16" else F.FINCH_F32)
    assert 1 < how["splits"] < 16 and how["workgroups"] > 512 and len({x[3] for x in how["pieces"]}) > 1
    fin, gen = F.Finch(F.FINCH_BF16 if dtype == "bf16" else F.FINCH_F32, d, G), torch.Generator().manual_seed(24)
    pbs = [problem(gen, dtype, d, G, *s) for s in shapes]
    batch = F.AttentionBatch(pbs)
    for again in range(2):  # (the counters are back at zero)
        for pb in pbs:
            pb["out"].fill_(9)
        fin.attend(batch)
        torch.cuda.synchronize()
        for i in range(again, len(pbs), 3):
            verify(pbs[i], f"{dtype} {shapes[i]}")
    fin.close()
