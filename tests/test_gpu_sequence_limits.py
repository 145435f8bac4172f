"""The sequence path at the ends of what its calls allow: the most heads of keys over long histories, scratch asked for once and used for
smaller batches, scores without a finite one among them, kernels that run for seconds.  Inputs, oracle and error bounds are those of
test_gpu_sequence.py."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from paper_2510_18239_b200 import binding
from test_gpu_sequence import check_history, check_tree, close, f64, lime, off_of, paged, rand

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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,dh", [(8, 2, 64), (4, 4, 32), (16, 4, 128)])
def test_scratch_goes_by_the_rows(dtype, Hq, Hkv, dh):
    """Partial results are kept for the rows that there are, not for whole tiles: one event takes a few MB, as every call has its own."""
    m = lime(dtype, Hq, Hkv, dh)
    assert binding.lime_sequence_workspace_bytes(m.ctx, 1, 1) < 4 << 20


def infinite_scores(q, at, k, bad):
    """Feature 0 decides the sign of a score against the key rows `at`, whose feature 0 is `bad`: the one for even query heads, the other for odd."""
    q[:, 0::2, 0], q[:, 1::2, 0] = 1.0, -1.0
    k[at, :, 0] = bad


def check_infinite(got, q, k, v, sees, at, bad, scale, dh, dtype):
    """A row and head that sees a key with score +inf, or none with a finite one, has NaN (inf - inf); a score of -inf is a probability of 0."""
    Hq = q.shape[1]
    hot = np.zeros(k.shape[0], bool)
    hot[at] = True
    cold = k.copy()
    cold[hot] = 0.0
    ref, mag, size = so.attend(q, cold, v, sees & ~hot, scale)
    for h in range(Hq):
        positive = (bad > 0) == (h % 2 == 0)
        nan = (sees & hot).any(1) if positive else sees.any(1) & ~(sees & ~hot).any(1)
        assert torch.isnan(got[:, h][torch.from_numpy(nan).to(got.device)]).all()
        rest = np.flatnonzero(~nan)
        close(got[rest.tolist(), h:h + 1], ref[rest, h:h + 1], mag[rest, h:h + 1], size[rest, h:h + 1], dh, k.shape[0], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf")])
@pytest.mark.parametrize("Hq,Hkv,dh", [(2, 1, 64), (4, 4, 32), (2, 2, 128)])
def test_infinite_scores(dtype, bad, Hq, Hkv, dh):
    gen = torch.Generator().manual_seed(67)
    m, scale = lime(dtype, Hq, Hkv, dh), 1 / np.sqrt(dh)
    # causal: user 0 begins with such a key and has another further on, user 1 has one in the middle; user 2 has more queries than keys
    nq, nk, at = [150, 140, 9], [150, 140, 4], [[0, 90], [70], [0]]
    q, k, v = rand(gen, sum(nq), Hq, dh, dtype=dtype), rand(gen, sum(nk), Hkv, dh, dtype=dtype), rand(gen, sum(nk), Hkv, dh, dtype=dtype)
    infinite_scores(q, [j + a for j, i in zip((0, 150, 290), at) for a in i], k, bad)
    got = m.attend_history(q.cuda(), k.cuda(), v.cuda(), off_of(nq), kv_off=off_of(nk))
    i = j = 0
    for a, b, hot in zip(nq, nk, at):
        check_infinite(got[i:i + a], f64(q[i:i + a]), f64(k[j:j + b]), f64(v[j:j + b]), so.causal(a, b), hot, bad, scale, dh, dtype)
        i, j = i + a, j + b
    # over the cache: nothing but such keys, in one tile and in pieces that are joined; one among many; one alone; no keys
    c = [1, 100, 5000, 3000, 0, 5000]
    hot = [range(1), range(100), range(5000), [2999], [], [0, 777, 4999]]
    for n, form in (([1] * 6, "none"), ([3] * 6, "roots"), ([20] * 6, "none")):
        ck, cv, table = paged(gen, c, 64, Hkv, dh, dtype)
        q, tk, tv = (rand(gen, sum(n), h, dh, dtype=dtype) for h in (Hq, Hkv, Hkv))
        flat = ck.view(-1, Hkv, dh)
        infinite_scores(q, [int(table[b, j // 64]) * 64 + j % 64 for b in range(6) for j in hot[b]], flat, bad)
        new = {} if form == "none" else dict(tree_k=tk.cuda(), tree_v=tv.cuda())
        got = m.attend_tree(q.cuda(), ck.cuda(), cv.cuda(), table.cuda(), torch.tensor(c, dtype=torch.int32).cuda(), off_of(n), **new)
        i = 0
        for b, (a, cb) in enumerate(zip(n, c)):
            kk, vv = so.cached_rows(f64(ck), table[b].tolist(), cb), so.cached_rows(f64(cv), table[b].tolist(), cb)
            sees = np.ones((a, cb), bool)
            if form == "roots":
                kk, vv, sees = np.concatenate((kk, f64(tk[i:i + a]))), np.concatenate((vv, f64(tv[i:i + a]))), np.concatenate((sees, np.eye(a, dtype=bool)), 1)
            check_infinite(got[i:i + a], f64(q[i:i + a]), kk, vv, sees, list(hot[b]), bad, scale, dh, dtype)
            i += a


@pytest.mark.parametrize("Hq,Hkv,dh", [(2, 1, 32), (2, 1, 64), (1, 1, 128)])
def test_values_that_are_not_finite_in_a_long_chain(Hq, Hkv, dh):
    """Causal rows as a chain of drafts, with a NaN and an infinity among the first values: what every later row adds of them takes a walk up
    its chain, not one for every tile of it, which would keep the warps that wait for its result longer than they may."""
    n, m = 100000, lime("bf16", Hq, Hkv, dh)
    gen = torch.Generator(device="cuda").manual_seed(73)
    q, k, v = (torch.randn(n, h, dh, generator=gen, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    page = torch.zeros(1, 16, Hkv, dh, dtype=torch.bfloat16, device="cuda")
    args = (page, page, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), off_of([n]))
    chain = torch.arange(-1, n - 1, dtype=torch.int32, device="cuda")
    clean = m.attend_tree(q, *args, parent=chain, tree_k=k, tree_v=v)
    v[300, :, 1], v[70, :, 5] = float("nan"), float("inf")
    got = m.attend_tree(q, *args, parent=chain, tree_k=k, tree_v=v)
    assert binding.lime_device_status(m.ctx) == 0
    assert torch.isnan(got[300:, :, 1]).all() and torch.equal(got[:300, :, 1], clean[:300, :, 1])
    assert (got[70:, :, 5] == float("inf")).all() and torch.equal(got[:70, :, 5], clean[:70, :, 5])
    rest = [c for c in range(dh) if c not in (1, 5)]
    assert torch.equal(got[:, :, rest], clean[:, :, rest])


def test_a_call_of_seconds_whose_first_ragged_tile_comes_last():
    """The first user's history fills its key tiles, which leaves nothing to mend in them for longer than a wait may take; the second's,
    whose few rows come last, ends inside one."""
    Hq, dh, page, n, c = 16, 128, 128, [180000, 4000], [1 << 21, 100]
    m = lime("bf16", Hq, 1, dh)
    gen = torch.Generator(device="cuda").manual_seed(71)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    pages = c[0] // page + 1
    ck, cv, q = normal(pages, page, 1, dh), normal(pages, page, 1, dh), normal(sum(n), Hq, dh)
    cv[-1, c[1]:] = float("nan")
    table = torch.full((2, pages - 1), -1, dtype=torch.int32)
    table[0], table[1, 0] = torch.arange(pages - 1), pages - 1
    out = torch.empty_like(q)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    args = (ck, cv, table.cuda(), torch.tensor(c, dtype=torch.int32).cuda(), off_of(n))
    begin.record()
    m.attend_tree(q, *args, out=out)
    end.record()
    torch.cuda.synchronize()
    assert binding.lime_device_status(m.ctx) == 0
    assert begin.elapsed_time(end) > 2200                        # or the case no longer outlasts a wait
    assert torch.isfinite(out).all()
    # rows of both ends: |out - ref| is bounded as in test_gpu_sequence.py; A = sum p |v| from the same sum
    for b, first in ((0, 0), (1, n[0])):
        rows = [first, first + n[b] // 2, first + n[b] - 1]
        kk, vv = (x.view(-1, dh)[:c[0]] if b == 0 else x[-1, :c[1], 0] for x in (ck, cv))
        for r in rows:
            s = q[r].double() @ kk.double().T / np.sqrt(dh)
            p = torch.softmax(s, -1)
            size = (q[r].double().abs() @ kk.double().abs().T).amax(-1) / np.sqrt(dh)
            close(out[r:r + 1], (p @ vv.double()).cpu().numpy()[None], (p @ vv.double().abs()).cpu().numpy()[None], size.cpu().numpy()[None], dh, c[b], "bf16")
