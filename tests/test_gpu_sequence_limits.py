"""The sequence path at the ends of what its calls allow: the most heads of keys over long histories, scratch asked for once and used for
smaller batches, scores without a finite one among them, kernels that run for seconds.  Inputs, oracle and error bounds are those of
test_gpu_sequence.py."""
import numpy as np
import pytest
import torch

from paper_2510_18239_b200 import binding
from test_gpu_sequence import check_history, check_tree, lime, off_of, paged, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,heads,dh,keys", [("f32", 640, 72, 100), ("f32", 1024, 128, 300), ("bf16", 593, 72, 950), ("bf16", 1024, 128, 1000)])
def test_the_most_heads_over_histories_of_many_tiles(dtype, heads, dh, keys):
    """So many heads of keys occupy the card by themselves: no row tile is cut, however long, and there is nothing to join."""
    gen = torch.Generator().manual_seed(heads)
    m = lime(dtype, heads, heads, dh)
    check_history(m, gen, dtype, heads, heads, dh, [2], [keys], 1 / np.sqrt(dh))
    check_tree(m, gen, dtype, heads, heads, dh, [3], [keys], 64, "drafts")
    check_tree(m, gen, dtype, heads, heads, dh, [1], [keys], 64, "none")


@pytest.mark.parametrize("dtype,Hq,Hkv,dh", [("f32", 8, 2, 64), ("f32", 1, 1, 8), ("f32", 32, 1, 32), ("f32", 16, 4, 128), ("bf16", 8, 2, 64), ("bf16", 1, 1, 8),
                                             ("bf16", 16, 4, 128), ("bf16", 32, 2, 32), ("bf16", 1024, 1024, 128)])
def test_scratch_serves_fewer_users_and_rows(dtype, Hq, Hkv, dh):
    """What is enough for B users with so many rows is enough for fewer users, and for fewer rows."""
    m = lime(dtype, Hq, Hkv, dh)
    steps = [0, 1, 2, 3, 5, 8, 13, 16, 31, 64, 100, 257, 1000, 4096, 30000, 250000, 1000000, 9000000]
    size = np.array([[binding.lime_sequence_workspace_bytes(m.ctx, b, r) for r in steps] for b in steps], np.int64)
    assert (size > 0).all() and (np.diff(size, axis=0) >= 0).all() and (np.diff(size, axis=1) >= 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_in_scratch_of_a_larger_batch(dtype):
    """Scratch of the size for 64 users with 64 rows, nothing behind it written, for all batches of at most as many users and rows."""
    gen = torch.Generator().manual_seed(61)
    Hq, Hkv, dh, page = 8, 2, 64, 16
    m = lime(dtype, Hq, Hkv, dh)
    seq = binding.lime_sequence(Hq, Hkv, dh)
    need = binding.lime_sequence_workspace_bytes(m.ctx, 64, 64)
    room = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    ws = room[:need]
    for B, rows in ((64, 64), (1, 64), (2, 64), (15, 64), (16, 64), (1, 1), (3, 50), (32, 33)):
        n = [rows // B + (b < rows % B) for b in range(B)]
        c = [40 + 4000 * b // B for b in range(B)]
        q, k, v = (rand(gen, rows, h, dh, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
        out = torch.empty_like(q)
        pk, pv = (rand(gen, rows + sum(c), Hkv, dh, dtype=dtype).cuda() for _ in range(2))
        off, kv_off = off_of(n), off_of([a + b for a, b in zip(n, c)])
        binding.lime_attend_history(m.ctx, seq, q, off, pk, pv, kv_off, out, ws)
        assert torch.equal(out, m.attend_history(q, pk, pv, off, kv_off=kv_off))
        ck, cv, table = (t.cuda() for t in paged(gen, c, page, Hkv, dh, dtype))
        ctx = torch.tensor(c, dtype=torch.int32).cuda()
        for new in ((None, None), (k, v)):
            binding.lime_attend_tree(m.ctx, seq, q, off, None, *new, ck, cv, table, ctx, None, out, ws)
            assert torch.equal(out, m.attend_tree(q, ck, cv, table, ctx, off, tree_k=new[0], tree_v=new[1]))
    assert (room[need:] == 0x5a).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scratch_of_a_million_users_serves_fewer_rows(dtype):
    """9 rows a user are tiled otherwise than 8, whose list of work items is the longer one.  A key a user: its value is the result."""
    m = lime(dtype, 1, 1, 8)
    B = 1000000
    ws = torch.empty(binding.lime_sequence_workspace_bytes(m.ctx, B, 9 * B), dtype=torch.uint8, device="cuda")
    cache = torch.arange(16 * 8, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32).view(1, 16, 1, 8)
    table, ctx = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    for each in (8, 9):
        q = torch.ones(each * B, 1, 8, dtype=cache.dtype, device="cuda")
        out, off = torch.zeros_like(q), (torch.arange(B + 1, device="cuda") * each).to(torch.int32)
        binding.lime_attend_tree(m.ctx, binding.lime_sequence(1, 1, 8), q, off, None, None, None, cache, cache, table, ctx, None, out, ws)
        assert (out == cache[0, 0]).all()


def test_scratch_of_absurd_batches():
    """More row tiles than the lists can count: no size."""
    m = lime("bf16", 8, 1, 8)
    assert binding.lime_sequence_workspace_bytes(m.ctx, 2 ** 31 - 1, 0x7fff0000) == 0
    assert binding.lime_sequence_workspace_bytes(m.ctx, 2 ** 31 - 1, 1) > 0
