"""The sequence path on the GPU against its fp64 statement (oracle/sequence_oracle.py).

Error bounds.  u = 2^-24 bounds an fp32 rounding relative to the value, b = 2^-8 a bf16 one.
Norm and rotation: the sum of squares of up to 128 terms through at most 16 additions, its square root's reciprocal, two products, the
cosine and sine of an angle that is off by at most 2 u pi, two more products: together less than 32 u (|y_a| + |y_b|); then one rounding
to the storage type, b |y| for bf16.
Attention: a score is a sum of d products, off by at most d u S with S = scale sum |q| |k|, and 2 u S more from the scale; so is the
reference maximum, so a probability is off by the factor exp(2 (d + 4) u S), and by 2^-21 from the exponential and the rescalings of the
running sums (at most one in a tile, 2^-24 each).  Numerator and denominator each have that error, and n u from adding n terms one after
the other.  With A = sum p |v|, the result is off by at most (2 expm1(2 (d + 4) u S) + 2^-20 + 2 n u) A.  bf16: each probability is
rounded once for the value product, b A more, and the result once, b |o| more."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from paper_2510_18239_b200 import binding

pytestmark = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def lime(dtype, Hq, Hkv, dh, **kw):
    m = binding.Lime(d=64, H=2, ell=8, n_layers=1, dtype=binding.LIME_F32 if dtype == "f32" else binding.LIME_BF16)
    m.set_sequence(Hq, Hkv, dh, **kw)
    return m


def rand(gen, *shape, dtype):
    return torch.randn(shape, generator=gen, dtype=torch.float32).to(TYPES[dtype])


def f64(t):
    return t.detach().cpu().double().numpy()


def off_of(lens):
    return torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32).cuda()


def close_rotated(got, x, gamma, pos, rot, inter, base, eps, dtype):
    ref = so.norm_rotate(x, gamma, pos, rot, inter, base, eps)
    y = np.abs(so.norm_rotate(x, gamma, pos, 0, inter, base, eps))
    size = y.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        size[..., a] = size[..., b] = y[..., a] + y[..., b]
    tol = 32 * U * size + (BF * np.abs(ref) if dtype == "bf16" else 0.0)
    err = np.abs(f64(got) - ref)
    assert (err <= tol).all(), f"{(err - tol).max()} over the bound"


def attend_bound(mag, size, ref, d, n, dtype):
    tol = (2 * np.expm1(2 * (d + 4) * U * size[..., None]) + 2.0 ** -20 + 2 * n * U) * mag
    return tol + (BF * (mag * 1.001 + np.abs(ref)) if dtype == "bf16" else 0.0)


def close(got, ref, mag, size, d, n, dtype):
    err, tol = np.abs(f64(got) - ref), attend_bound(mag, size, ref, d, n, dtype)
    assert np.isfinite(f64(got)).all()
    assert (err <= tol).all(), f"{(err - tol).max()} over the bound, at {np.argwhere(err > tol)[:5].tolist()}"


# ----------------------------------------------------------------------------- norm and rotation
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,dh,rot,inter", [(1, 1, 8, 8, False), (4, 2, 16, 16, True), (3, 1, 24, 10, False), (4, 4, 32, 32, False),
                                                 (8, 2, 40, 40, True), (8, 2, 40, 36, False), (6, 2, 64, 64, False), (5, 5, 96, 48, False),
                                                 (16, 4, 128, 128, False), (2, 2, 128, 2, True), (7, 1, 128, 0, False)])
def test_norm_rotate(dtype, Hq, Hkv, dh, rot, inter):
    gen = torch.Generator().manual_seed(dh * 7 + rot)
    m = lime(dtype, Hq, Hkv, dh, rot_dim=rot, rot_interleaved=inter, rot_base=5000.0)
    for rows in (1, 3, 37, 130):
        q, k = rand(gen, rows, Hq, dh, dtype=dtype), rand(gen, rows, Hkv, dh, dtype=dtype)
        gq, gk = rand(gen, dh, dtype=dtype), rand(gen, dh, dtype=dtype)
        pos = torch.randint(-50, 5000, (rows,), generator=gen, dtype=torch.int32)
        oq, ok = m.norm_rotate(q.cuda(), k.cuda(), pos.cuda(), gamma_q=gq.cuda(), gamma_k=gk.cuda())
        close_rotated(oq, f64(q), f64(gq), pos.numpy(), rot, inter, 5000.0, 1e-6, dtype)
        close_rotated(ok, f64(k), f64(gk), pos.numpy(), rot, inter, 5000.0, 1e-6, dtype)
        oq, ok = m.norm_rotate(q.cuda(), k.cuda(), pos.cuda())                     # no gains
        close_rotated(oq, f64(q), None, pos.numpy(), rot, inter, 5000.0, 1e-6, dtype)
        close_rotated(ok, f64(k), None, pos.numpy(), rot, inter, 5000.0, 1e-6, dtype)


def test_rotation_far_out_and_at_the_ends():
    """Positions up to the ends of int32, the largest base, and base 1 (every pair turns alike): the angle keeps its bits."""
    gen = torch.Generator().manual_seed(3)
    pos = torch.tensor([0, 1, -1, 1 << 20, (1 << 24) + 1, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32)
    q, k = rand(gen, 8, 2, 64, dtype="f32"), rand(gen, 8, 1, 64, dtype="f32")
    for base in (1.0, 10000.0, 1e6, 1e30):
        m = lime("f32", 2, 1, 64, rot_dim=64, rot_base=base)
        oq, ok = m.norm_rotate(q.cuda(), k.cuda(), pos.cuda())
        # the reference's angle, a product in fp64, is off by up to 2^31 * 2^-53 radians: under 4 u
        close_rotated(oq, f64(q), None, pos.numpy(), 64, False, base, 1e-6, "f32")
        close_rotated(ok, f64(k), None, pos.numpy(), 64, False, base, 1e-6, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_rotate_into_a_cache(dtype):
    """Parts of one wider row in, keys and values to their slots; unnamed rows stay, -1 is silent, other bad slots are reported."""
    gen = torch.Generator().manual_seed(5)
    Hq, Hkv, dh, rows = 4, 2, 64, 45
    m = lime(dtype, Hq, Hkv, dh, rot_dim=32)
    qkv = rand(gen, rows, Hq + 2 * Hkv, dh, dtype=dtype).cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    pos = torch.arange(rows, dtype=torch.int32)
    for bad in (False, True):
        ck, cv = rand(gen, 5, 16, Hkv, dh, dtype=dtype).cuda(), rand(gen, 5, 16, Hkv, dh, dtype=dtype).cuda()
        before_k, before_v = ck.clone(), cv.clone()
        slots = torch.randperm(80, generator=gen)[:rows].to(torch.int32)
        slots[7] = slots[20] = -1
        if bad:
            slots[30], slots[11] = 80, -2
        flag = torch.full((1,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        oq, ok = m.norm_rotate(q, k, pos.cuda(), v=v, cache_k=ck, cache_v=cv, slots=slots.cuda(), dev_flag=flag, keep_k=True)
        assert int(flag) == (11 if bad else 2 ** 31 - 1)
        close_rotated(ok, f64(k), None, pos.numpy(), 32, False, 10000.0, 1e-6, dtype)
        want_k, want_v = before_k.view(80, Hkv, dh), before_v.view(80, Hkv, dh)
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < 80:
                want_k[s], want_v[s] = ok[t], v[t]
        assert torch.equal(ck.view(80, Hkv, dh), want_k) and torch.equal(cv.view(80, Hkv, dh), want_v)
        assert m.norm_rotate(q, k, pos.cuda(), v=v, cache_k=ck, cache_v=cv, slots=slots.cuda())[1] is None
    # keys alone to a cache, and outputs over their inputs
    m.norm_rotate(q, k, pos.cuda(), cache_k=ck, slots=slots.cuda())
    q_in, k_in = f64(q), f64(k)
    m.norm_rotate(q, k, pos.cuda(), q_out=q, k_out=k)
    close_rotated(q, q_in, None, pos.numpy(), 32, False, 10000.0, 1e-6, dtype)
    close_rotated(k, k_in, None, pos.numpy(), 32, False, 10000.0, 1e-6, dtype)


def test_norm_rotate_of_zero_infinite_and_tiny_rows():
    m = lime("f32", 1, 1, 16)
    q = torch.zeros(4, 1, 16).cuda()
    q[1] = 1e-30
    q[2, 0, 3] = float("inf")
    q[3, 0, 5] = float("nan")
    k = torch.ones(4, 1, 16).cuda()
    oq, ok = m.norm_rotate(q, k, None)
    assert (oq[0] == 0).all() and torch.allclose(oq[1], torch.full((1, 16), 1e-27, device="cuda"), rtol=1e-5)
    assert torch.isnan(oq[2, 0, 3]) and (oq[2, 0, :3] == 0).all() and torch.isnan(oq[3]).all()
    assert torch.isfinite(ok).all()
    e = m.norm_rotate(q[:0], k[:0], None)
    assert e[0].shape == (0, 1, 16) and e[1].shape == (0, 1, 16)


# ----------------------------------------------------------------------------- causal attention over packed histories
def check_history(m, gen, dtype, Hq, Hkv, dh, nq, nk, scale, kv_off=True, tail=0, std=1.0):
    rows, keys = sum(nq), sum(nk)
    q = rand(gen, rows + tail, Hq, dh, dtype=dtype) * std
    k, v = rand(gen, keys + tail, Hkv, dh, dtype=dtype) * std, rand(gen, keys + tail, Hkv, dh, dtype=dtype)
    out = torch.full((rows + tail, Hq, dh), 7.0, dtype=TYPES[dtype], device="cuda")
    m.attend_history(q.cuda(), k.cuda(), v.cuda(), off_of(nq), kv_off=off_of(nk) if kv_off else None, out=out)
    assert (out[rows:] == 7).all()                                                   # rows behind the last history
    i = j = 0
    for a, b in zip(nq, nk):
        ref, mag, size = so.attend(f64(q[i:i + a]), f64(k[j:j + b]), f64(v[j:j + b]), so.causal(a, b), scale)
        close(out[i:i + a], ref, mag, size, dh, b, dtype)
        i, j = i + a, j + b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,dh", [(1, 1, 8), (2, 2, 32), (4, 1, 16), (3, 1, 40), (8, 2, 64), (6, 6, 72), (4, 2, 128), (14, 2, 96), (20, 1, 32), (64, 1, 64)])
def test_history(dtype, Hq, Hkv, dh):
    gen = torch.Generator().manual_seed(Hq * 1000 + dh)
    m = lime(dtype, Hq, Hkv, dh)
    scale = 1 / np.sqrt(dh)
    for lens in ([1], [2, 0, 1, 0, 0, 17], [64, 63, 65], [127, 1, 129, 128], [0, 0], [200, 5]):
        check_history(m, gen, dtype, Hq, Hkv, dh, lens, lens, scale, kv_off=len(lens) % 2 == 0, tail=3 if len(lens) % 2 == 0 else 0)
    # new rows behind older ones; more queries than keys (the first see nothing); no keys at all
    check_history(m, gen, dtype, Hq, Hkv, dh, [1, 3, 16, 5], [1, 300, 130, 5], scale)
    check_history(m, gen, dtype, Hq, Hkv, dh, [5, 3, 140], [2, 0, 70], scale, tail=2)
    check_history(m, gen, dtype, Hq, Hkv, dh, [4], [0], scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_histories_are_cut_into_parts(dtype):
    """One query row, and a few, over thousands of keys: several work items per row tile, joined; scores of some spread."""
    gen = torch.Generator().manual_seed(11)
    m = lime(dtype, 4, 2, 64, attn_scale=0.3)
    check_history(m, gen, dtype, 4, 2, 64, [1], [9000], 0.3)
    check_history(m, gen, dtype, 4, 2, 64, [3, 40, 1, 0, 2], [5000, 2500, 1, 17, 12000], 0.3, std=1.5)
    check_history(m, gen, dtype, 4, 2, 64, [1500], [1500], 0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("rise", [0.02, -0.02, 0.5, -0.5])
def test_scores_that_grow_and_fall(dtype, dh, rise):
    """Scores that rise or fall along the keys by far more than the range a probability has: the reference moves again and again, or what
    comes later vanishes.  And a constant offset of all scores, far from zero, changes nothing."""
    gen = torch.Generator().manual_seed(43)
    m = lime(dtype, 2, 1, dh, attn_scale=1.0)
    n = 700
    q, k, v = rand(gen, n, 2, dh, dtype=dtype), rand(gen, n, 1, dh, dtype=dtype) * 0.25, rand(gen, n, 1, dh, dtype=dtype)
    q[:, :, 0], k[:, 0, 0] = 1.0, (torch.arange(n) * rise).to(TYPES[dtype])
    q[:, :, 1], k[:, 0, 1] = 1.0, -300.0
    out = m.attend_history(q.cuda(), k.cuda(), v.cuda(), off_of([n]))
    ref, mag, size = so.attend(f64(q), f64(k), f64(v), so.causal(n, n), 1.0)
    close(out, ref, mag, size, dh, n, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_history_with_strides(dtype):
    gen = torch.Generator().manual_seed(13)
    Hq, Hkv, dh, lens = 4, 2, 32, [70, 1, 33]
    m = lime(dtype, Hq, Hkv, dh)
    qkv = rand(gen, sum(lens), Hq + 2 * Hkv, dh, dtype=dtype).cuda()
    wide = torch.full((sum(lens), Hq + 3, dh), 5.0, dtype=TYPES[dtype], device="cuda")
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    got = m.attend_history(q, k, v, off_of(lens), out=wide[:, 1:1 + Hq])
    want = m.attend_history(q.contiguous(), k.contiguous(), v.contiguous(), off_of(lens))
    assert torch.equal(got, want) and (wide[:, 0] == 5).all() and (wide[:, 1 + Hq:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_has_no_influence(dtype, bad):
    """A key or value row with infinities or NaN: rows before it, other users and rows past the end are as without it; rows that see it
    get what the formula gives."""
    gen = torch.Generator().manual_seed(17)
    for Hq, Hkv, dh in ((2, 1, 64), (4, 4, 32), (2, 2, 128)):
        m = lime(dtype, Hq, Hkv, dh)
        lens, at = [150, 140, 3], 90
        n = sum(lens)
        q, k, v = (rand(gen, n + 5, h, dh, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
        clean = m.attend_history(q, k, v, off_of(lens))
        k2, v2 = k.clone(), v.clone()
        k2[n:] = bad
        v2[n:] = bad                                                                  # behind the last history
        v2[at, :, 1] = bad
        got = m.attend_history(q, k2, v2, off_of(lens))
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[150:n], clean[150:n])
        seen = got[at:150].float()
        assert (torch.isnan(seen[:, :, 1]) if bad != bad else seen[:, :, 1] == bad).all()
        keep = [c for c in range(dh) if c != 1]
        assert torch.equal(got[at:150][:, :, keep], clean[at:150][:, :, keep])
        k2[at] = bad                                                                  # the score is then not finite either
        got = m.attend_history(q, k2, v2, off_of(lens))
        assert torch.equal(got[:at], clean[:at]) and torch.equal(got[150:n], clean[150:n])
        assert torch.isnan(got[149]).all() or bad == -float("inf") or bad == float("inf")


# ----------------------------------------------------------------------------- trees over a paged cache
def paged(gen, lens, page, Hkv, dh, dtype, spare=2):
    need = [-(-n // page) for n in lens]
    pool = sum(need) + spare
    order = torch.randperm(pool, generator=gen)
    table = torch.full((len(lens), max(1, max(need))), -5, dtype=torch.int32)
    first = 0
    for b, n in enumerate(need):
        table[b, :n] = order[first:first + n]
        first += n
    return rand(gen, pool, page, Hkv, dh, dtype=dtype), rand(gen, pool, page, Hkv, dh, dtype=dtype), table


def check_tree(m, gen, dtype, Hq, Hkv, dh, n, c, page, form, tail=0, parent=None):
    scale, rows = 1 / np.sqrt(dh), sum(n)
    ck, cv, table = paged(gen, c, page, Hkv, dh, dtype)
    q, tk, tv = (rand(gen, rows + tail, h, dh, dtype=dtype) for h in (Hq, Hkv, Hkv))
    if form == "drafts" and parent is None:
        parent = torch.cat([(torch.rand(a, generator=gen) * (torch.arange(a) + 1)).long() - 1 for a in n] + [torch.zeros(tail, dtype=torch.long)]).to(torch.int32)
    out = torch.full((rows + tail, Hq, dh), 7.0, dtype=TYPES[dtype], device="cuda")
    new = dict(tree_k=tk.cuda(), tree_v=tv.cuda()) if form != "none" else {}
    flag = torch.full((1,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    m.attend_tree(q.cuda(), ck.cuda(), cv.cuda(), table.cuda(), torch.tensor(c, dtype=torch.int32).cuda(), off_of(n),
                  parent=parent.cuda() if form == "drafts" else None, out=out, dev_flag=flag, **new)
    assert int(flag) == 2 ** 31 - 1 and (out[rows:] == 7).all()
    i = 0
    for b, (a, cb) in enumerate(zip(n, c)):
        k, v = so.cached_rows(f64(ck), table[b].tolist(), cb), so.cached_rows(f64(cv), table[b].tolist(), cb)
        sees = np.ones((a, cb), bool)
        if form != "none":
            k, v = np.concatenate((k, f64(tk[i:i + a]))), np.concatenate((v, f64(tv[i:i + a])))
            sees = np.concatenate((sees, so.ancestors(parent[i:i + a].tolist()) if form == "drafts" else np.eye(a, dtype=bool)), 1)
        ref, mag, size = so.attend(f64(q[i:i + a]), k, v, sees, scale)
        close(out[i:i + a], ref, mag, size, dh, cb + a, dtype)
        i += a


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["none", "roots", "drafts"])
@pytest.mark.parametrize("Hq,Hkv,dh,page", [(1, 1, 8, 16), (4, 4, 32, 32), (8, 2, 64, 16), (3, 1, 40, 64), (4, 2, 128, 128), (10, 2, 96, 256), (40, 2, 64, 64)])
def test_tree(dtype, form, Hq, Hkv, dh, page):
    gen = torch.Generator().manual_seed(Hq * 100 + dh + len(form))
    m = lime(dtype, Hq, Hkv, dh)
    check_tree(m, gen, dtype, Hq, Hkv, dh, [1], [0], page, form)
    check_tree(m, gen, dtype, Hq, Hkv, dh, [1, 1, 1, 1], [1, page, page + 1, 300], page, form, tail=2)
    check_tree(m, gen, dtype, Hq, Hkv, dh, [5, 0, 63, 1, 64], [129, 40, 0, 1, 128], page, form, tail=1)
    check_tree(m, gen, dtype, Hq, Hkv, dh, [150, 3], [70, 257], page, form)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_over_long_caches_is_cut_into_parts(dtype):
    gen = torch.Generator().manual_seed(19)
    m = lime(dtype, 4, 2, 64)
    check_tree(m, gen, dtype, 4, 2, 64, [1], [9001], 64, "none")
    check_tree(m, gen, dtype, 4, 2, 64, [1, 20, 1], [10, 7000, 4097], 32, "drafts")
    check_tree(m, gen, dtype, 4, 2, 64, [2, 3], [11000, 0], 128, "roots")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chains_and_bad_parents(dtype):
    """A chain (every row the child of the one before) is causal attention; entries that are no earlier row make roots."""
    gen = torch.Generator().manual_seed(23)
    m = lime(dtype, 4, 2, 32)
    n = [70, 140]
    chain = torch.cat([torch.arange(a) - 1 for a in n]).to(torch.int32)
    check_tree(m, gen, dtype, 4, 2, 32, n, [100, 33], 16, "drafts", parent=chain)
    wild = chain.clone()
    wild[5], wild[6], wild[80], wild[100], wild[140] = 5, 1 << 30, -7, -2 ** 31, 69
    check_tree(m, gen, dtype, 4, 2, 32, n, [100, 33], 16, "drafts", parent=wild)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_that_are_not_there_and_lengths_past_the_table(dtype):
    """Such a page reads as rows of zeros and its place in the table is reported; lengths are cut to the table; pages may be shared."""
    gen = torch.Generator().manual_seed(29)
    Hq, Hkv, dh, page = 4, 2, 64, 16
    m = lime(dtype, Hq, Hkv, dh)
    ck, cv = (rand(gen, 6, page, Hkv, dh, dtype=dtype) for _ in range(2))
    table = torch.tensor([[0, 1, 2, 3], [3, 6, -1, 5], [5, 5, 0, 9]], dtype=torch.int32)
    ctx = torch.tensor([1000, 50, 20], dtype=torch.int32)                 # the last user's bad page is past its length
    q = rand(gen, 3, Hq, dh, dtype=dtype)
    flag = torch.full((1,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    out = m.attend_tree(q.cuda(), ck.cuda(), cv.cuda(), table.cuda(), ctx.cuda(), off_of([1, 1, 1]), dev_flag=flag)
    assert int(flag) == 5
    for b, n in enumerate((64, 50, 20)):
        k, v = so.cached_rows(f64(ck), table[b].tolist(), n), so.cached_rows(f64(cv), table[b].tolist(), n)
        ref, mag, size = so.attend(f64(q[b:b + 1]), k, v, np.ones((1, n), bool), 1 / 8)
        close(out[b:b + 1], ref, mag, size, dh, n, dtype)
    neg = m.attend_tree(q.cuda(), ck.cuda(), cv.cuda(), table.cuda(), torch.tensor([-3, -2 ** 31, 0], dtype=torch.int32).cuda(), off_of([1, 1, 1]))
    assert (neg == 0).all()
    none = m.attend_tree(q.cuda(), ck[:0].cuda(), cv[:0].cuda(), table.cuda(), ctx.cuda(), off_of([1, 1, 1]), dev_flag=flag)
    assert (none == 0).all() and int(flag) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_unwritten_cache_rows_have_no_influence(dtype, bad):
    """What lies behind a user's length in its last page, in other pages, and in draft rows of other branches."""
    gen = torch.Generator().manual_seed(31)
    for Hq, Hkv, dh, page in ((4, 2, 64, 32), (2, 2, 128, 16), (4, 4, 32, 128)):
        m = lime(dtype, Hq, Hkv, dh)
        ck, cv, table = paged(gen, [37, 128], page, Hkv, dh, dtype)
        n, ctx = [6, 3], torch.tensor([37, 128], dtype=torch.int32).cuda()
        q, tk, tv = (rand(gen, 9, h, dh, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
        parent = torch.tensor([-1, 0, 0, 1, 2, 4, -1, 0, -1], dtype=torch.int32).cuda()
        args = dict(parent=parent, tree_k=tk, tree_v=tv)
        clean = m.attend_tree(q, ck.cuda(), cv.cuda(), table.cuda(), ctx, off_of(n), **args)
        used = torch.zeros(ck.shape[:2], dtype=torch.bool)
        for b, c in enumerate((37, 128)):
            for j in range(c):
                used[table[b, j // page], j % page] = True
        ck[~used], cv[~used] = bad, bad
        assert torch.equal(m.attend_tree(q, ck.cuda(), cv.cuda(), table.cuda(), ctx, off_of(n), **args), clean)
        tk[1], tv[1] = bad, bad                                                # seen by rows 1 and 3 only
        got = m.attend_tree(q, ck.cuda(), cv.cuda(), table.cuda(), ctx, off_of(n), **args)
        others = [0, 2, 4, 5, 6, 7, 8]
        assert torch.equal(got[others], clean[others]) and not torch.isfinite(got[[1, 3]]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_users_and_offsets_past_the_rows(dtype):
    """More users than the work lists keep near (2048), most of them empty; offsets past the rows given are cut to them."""
    gen = torch.Generator().manual_seed(47)
    m = lime(dtype, 2, 1, 32)
    lens = [0] * 5000
    for b, n in ((0, 3), (17, 200), (2047, 1), (2048, 70), (4999, 64)):
        lens[b] = n
    check_history(m, gen, dtype, 2, 1, 32, lens, lens, 1 / np.sqrt(32), kv_off=False, tail=5)
    q, k, v = (rand(gen, 40, h, 32, dtype=dtype) for h in (2, 1, 1))
    off = torch.tensor([0, 30, 90, 1 << 30], dtype=torch.int32).cuda()
    out = torch.full((40, 2, 32), 7.0, dtype=TYPES[dtype], device="cuda")
    m.attend_history(q.cuda(), k.cuda(), v.cuda(), off, out=out)
    for lo, hi in ((0, 30), (30, 40)):
        ref, mag, size = so.attend(f64(q[lo:hi]), f64(k[lo:hi]), f64(v[lo:hi]), so.causal(hi - lo, hi - lo), 1 / np.sqrt(32))
        close(out[lo:hi], ref, mag, size, 32, hi - lo, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(dtype):
    """Rows 2^20 elements apart, the last ones more than 2^31 elements in; a cache of more than 2^31 elements, used at its end."""
    gen = torch.Generator().manual_seed(37)
    Hq, Hkv, dh, rows, n = 4, 2, 64, 2200, 130
    m = lime(dtype, Hq, Hkv, dh, rot_dim=64)
    wide = torch.empty(rows, 1 << 20, dtype=TYPES[dtype], device="cuda")
    part = lambda at, h: wide[:, at:at + h * dh].unflatten(1, (h, dh))
    q, k, v, out = part(0, Hq), part(512, Hkv), part(1024, Hkv), part(4096, Hq)
    qkv = [rand(gen, rows, h, dh, dtype=dtype) for h in (Hq, Hkv, Hkv)]
    for to, x in zip((q, k, v), qkv):
        to.copy_(x)
    off = torch.tensor([0, rows - n, rows], dtype=torch.int32).cuda()
    out.fill_(7)
    m.attend_history(q, k, v, off, out=out)
    ref, mag, size = so.attend(*(f64(x[-n:]) for x in qkv), so.causal(n, n), 1 / 8)
    close(out[-n:], ref, mag, size, dh, n, dtype)
    # into the last pages of a cache, and from there; the rest of the last but one is whatever the memory held
    page, n_pages = 128, 131200
    ck = torch.empty(n_pages, page, Hkv, dh, dtype=TYPES[dtype], device="cuda")
    cv = torch.empty_like(ck)
    slots = torch.full((rows,), -1, dtype=torch.int32)
    slots[-n:-2] = (n_pages - 1) * page + torch.arange(page, dtype=torch.int32)
    slots[-2:] = (n_pages - 2) * page + torch.arange(2, dtype=torch.int32)
    pos = torch.arange(rows, dtype=torch.int32)
    m.norm_rotate(q, k, pos.cuda(), v=v, q_out=q, k_out=k, cache_k=ck, cache_v=cv, slots=slots.cuda())
    close_rotated(q[-n:], f64(qkv[0][-n:]), None, pos[-n:].numpy(), 64, False, 10000.0, 1e-6, dtype)
    assert torch.equal(ck[-1], k[-n:-2]) and torch.equal(cv[-2, :2], v[-2:])
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32).cuda()
    got = m.attend_tree(q[-3:], ck, cv, table, torch.tensor([n], dtype=torch.int32).cuda(), off_of([3]))
    ref, mag, size = so.attend(f64(q[-3:]), f64(k[-n:]), f64(v[-n:]), np.ones((3, n), bool), 1 / 8)
    close(got, ref, mag, size, dh, n, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,dh", [(1024, 1024, 8), (1024, 16, 128), (1024, 512, 64), (64, 1, 8)])
def test_the_most_heads(dtype, Hq, Hkv, dh):
    gen = torch.Generator().manual_seed(Hkv)
    m = lime(dtype, Hq, Hkv, dh, rot_dim=dh)
    check_history(m, gen, dtype, Hq, Hkv, dh, [3, 0, 1], [3, 5, 70], 1 / np.sqrt(dh), tail=1)
    check_tree(m, gen, dtype, Hq, Hkv, dh, [1, 3], [20, 0], 16, "drafts")
    q, k, gamma = rand(gen, 5, Hq, dh, dtype=dtype), rand(gen, 5, Hkv, dh, dtype=dtype), rand(gen, dh, dtype=dtype)
    pos = torch.tensor([0, 1, 7, 100, 5000], dtype=torch.int32)
    oq, ok = m.norm_rotate(q.cuda(), k.cuda(), pos.cuda(), gamma_q=gamma.cuda(), gamma_k=gamma.cuda())
    close_rotated(oq, f64(q), f64(gamma), pos.numpy(), dh, False, 10000.0, 1e-6, dtype)
    close_rotated(ok, f64(k), f64(gamma), pos.numpy(), dh, False, 10000.0, 1e-6, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_the_largest_pages_and_long_trees(dtype, dh):
    gen = torch.Generator().manual_seed(dh)
    m = lime(dtype, 2, 1, dh)
    check_tree(m, gen, dtype, 2, 1, dh, [2, 1], [5000, 4096], 4096, "drafts")
    check_tree(m, gen, dtype, 2, 1, dh, [700, 9], [65, 1], 32, "roots")
    check_tree(m, gen, dtype, 2, 1, dh, [900], [33], 16, "drafts", parent=torch.arange(900, dtype=torch.int32) - 1)


@pytest.mark.parametrize("dtype,Hq,Hkv,dh", [("f32", 8, 2, 64), ("bf16", 4, 4, 32), ("bf16", 8, 2, 64), ("bf16", 16, 4, 128)])
@pytest.mark.parametrize("form", ["history", "none", "roots", "drafts"])
def test_many_calls_in_a_row_give_the_same(dtype, Hq, Hkv, dh, form):
    """Calls overlap at their ends; their warps wait for one another in orders that differ from call to call.  Every result is the first
    one's, and no bounded wait runs out."""
    gen = torch.Generator().manual_seed(dh)
    m = lime(dtype, Hq, Hkv, dh)
    B, page = 48, 64
    n, c = [4] * B, [16 + 3000 * b // B for b in range(B)]
    q, k, v = (rand(gen, 4 * B, h, dh, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
    if form == "history":
        keys = [a // 8 + 4 for a in c]
        k, v = (rand(gen, sum(keys), Hkv, dh, dtype=dtype).cuda() for _ in range(2))
        off, kv_off = off_of(n), off_of(keys)
        call = lambda out: m.attend_history(q, k, v, off, kv_off=kv_off, out=out)
    else:
        ck, cv, table = paged(gen, c, page, Hkv, dh, dtype)
        ck, cv, table, ctx = ck.cuda(), cv.cuda(), table.cuda(), torch.tensor(c, dtype=torch.int32).cuda()
        rows = B if form == "none" else 4 * B
        off = off_of([rows // B] * B)
        new = {} if form == "none" else dict(tree_k=k, tree_v=v)
        if form == "drafts":
            new["parent"] = torch.tensor([-1, 0, 0, 1] * B, dtype=torch.int32).cuda()
        q = q[:rows]
        call = lambda out: m.attend_tree(q, ck, cv, table, ctx, off, out=out, **new)
    first = call(torch.empty_like(q))
    outs = [torch.empty_like(q) for _ in range(25)]
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(40):
        for o in outs:
            call(o)
        for o in outs:
            differ += (o != first).sum()
    assert int(differ) == 0
    binding.lime_device_status(m.ctx)


@pytest.mark.parametrize("dtype,Hq,Hkv,dh", [("f32", 16, 1, 64), ("bf16", 16, 1, 32), ("bf16", 16, 1, 64), ("bf16", 12, 1, 72), ("bf16", 48, 3, 128), ("bf16", 2, 2, 128)])
def test_runs_of_users_and_rows_that_see_nothing(dtype, Hq, Hkv, dh):
    """Users without keys, many in a row, between users with one (whose value is the result as it is); queries ahead of the first key.
    Again and again, as the warps that have nothing to do for them may be far ahead of the others."""
    gen = torch.Generator().manual_seed(dh + Hq)
    m = lime(dtype, Hq, Hkv, dh)
    B = 400
    has = [int(torch.randint(0, 5, (1,), generator=gen)) == 0 and b > 3 for b in range(B)]
    n = [1 + b % 9 for b in range(B)]
    ck, cv, table = paged(gen, [int(h) for h in has], 16, Hkv, dh, dtype)
    q = rand(gen, sum(n), Hq, dh, dtype=dtype).cuda()
    args = (ck.cuda(), cv.cuda(), table.cuda(), torch.tensor(has, dtype=torch.int32).cuda(), off_of(n))
    want = torch.zeros(B, Hkv, dh, dtype=TYPES[dtype])
    for b in range(B):
        if has[b]:
            want[b] = cv[table[b, 0], 0]
    want = want.repeat_interleave(torch.tensor(n), 0).repeat_interleave(Hq // Hkv, 1).cuda()
    out = torch.empty_like(q)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        differ += (m.attend_tree(q, *args, out=out) != want).sum()
    # 20 queries a user, the last of which see keys: 0 .. 3 of them
    nk = [b % 4 if b % 3 else 0 for b in range(B)]
    q = rand(gen, 20 * B, Hq, dh, dtype=dtype).cuda()
    k, v = (rand(gen, sum(nk), Hkv, dh, dtype=dtype).cuda() for _ in range(2))
    off, kv_off = off_of([20] * B), off_of(nk)
    first, out = m.attend_history(q, k, v, off, kv_off=kv_off), torch.empty_like(q)
    seen = first.view(B, 20, Hq, dh)
    j = 0
    for b, a in enumerate(nk):
        assert (seen[b, :20 - a] == 0).all()
        if a:                                                            # the first query that sees a key has that value
            assert torch.equal(seen[b, 20 - a], v[j].repeat_interleave(Hq // Hkv, 0))
        j += a
    for _ in range(300):
        differ += (m.attend_history(q, k, v, off, kv_off=kv_off, out=out) != first).sum()
    assert int(differ) == 0
    binding.lime_device_status(m.ctx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_graph_serves_other_lengths_than_it_was_captured_with(dtype):
    """Lengths, tables and trees are device data: a replay reads what stands there then."""
    gen = torch.Generator().manual_seed(53)
    Hq, Hkv, dh, page = 4, 2, 64, 16
    m = lime(dtype, Hq, Hkv, dh)
    ck, cv, table = paged(gen, [640, 640], page, Hkv, dh, dtype)
    q, tk, tv = (rand(gen, 12, h, dh, dtype=dtype) for h in (Hq, Hkv, Hkv))
    d = [t.cuda() for t in (q, ck, cv, table, tk, tv)]
    ctx, off = torch.tensor([1, 1], dtype=torch.int32).cuda(), off_of([1, 1])
    parent = torch.full((12,), -1, dtype=torch.int32, device="cuda")
    run = lambda: m.attend_tree(d[0], d[1], d[2], d[3], ctx, off, parent=parent, tree_k=d[4], tree_v=d[5])
    run()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for n, c, par in (([3, 9], [640, 5], [-1, 0, 1] + [-1, 0, 0, 1, 1, 2, 5, -1, 7]), ([0, 12], [0, 600], [-1] + list(range(11))), ([12, 0], [77, 640], [-1] * 12)):
        off.copy_(off_of(n))
        ctx.copy_(torch.tensor(c, dtype=torch.int32))
        parent.copy_(torch.tensor(par, dtype=torch.int32))
        g.replay()
        i = 0
        for b, (a, cb) in enumerate(zip(n, c)):
            kk = np.concatenate((so.cached_rows(f64(ck), table[b].tolist(), cb), f64(tk[i:i + a])))
            vv = np.concatenate((so.cached_rows(f64(cv), table[b].tolist(), cb), f64(tv[i:i + a])))
            sees = np.concatenate((np.ones((a, cb), bool), so.ancestors(par[i:i + a])), 1)
            ref, mag, size = so.attend(f64(q[i:i + a]), kk, vv, sees, 1 / 8)
            close(out[i:i + a], ref, mag, size, dh, cb + a, dtype)
            i += a


# ----------------------------------------------------------------------------- the operators together
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_history_grows_event_by_event(dtype):
    """Prompt through norm_rotate into the cache and through attend_history; then single events and a list of candidates over the cache
    give what whole histories with these rows at their end give."""
    gen = torch.Generator().manual_seed(37)
    Hq, Hkv, dh, page = 8, 2, 64, 16
    m = lime(dtype, Hq, Hkv, dh, rot_dim=dh)
    lens = [40, 1, 129]
    B, extra = len(lens), 3
    full = [n + extra for n in lens]
    raw = [rand(gen, n, Hq + 2 * Hkv, dh, dtype=dtype) for n in full]
    pages = [-(-n // page) for n in full]
    table = torch.full((B, max(pages)), -1, dtype=torch.int32)
    order = torch.randperm(sum(pages), generator=gen).to(torch.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    ck = torch.full((sum(pages), page, Hkv, dh), float("nan"), dtype=TYPES[dtype], device="cuda")
    cv = ck.clone()

    def slots(b, first, n):
        j = torch.arange(first, first + n)
        return table[b, j // page] * page + (j % page).to(torch.int32)

    def enter(rows, first):
        n = [r.shape[0] for r in rows]
        x = torch.cat(rows).cuda()
        pos = torch.cat([torch.arange(f, f + a) for f, a in zip(first, n)]).to(torch.int32).cuda()
        at = torch.cat([slots(b, f, a) for b, (f, a) in enumerate(zip(first, n))]).to(torch.int32).cuda()
        q, k = m.norm_rotate(x[:, :Hq], x[:, Hq:Hq + Hkv], pos, v=x[:, Hq + Hkv:], cache_k=ck, cache_v=cv, slots=at, keep_k=True)
        return q, k, x[:, Hq + Hkv:]

    # what whole histories give, every row of them
    cat = torch.cat(raw).cuda()
    pos = torch.cat([torch.arange(n) for n in full]).to(torch.int32).cuda()
    q, k = m.norm_rotate(cat[:, :Hq], cat[:, Hq:Hq + Hkv], pos)
    off = off_of(full)
    whole = m.attend_history(q, k, cat[:, Hq + Hkv:], off)
    at = np.concatenate(([0], np.cumsum(full)))
    tol = dict(atol=2e-5, rtol=2e-5) if dtype == "f32" else dict(atol=4 * BF * 4, rtol=2 * BF)     # both sides' bounds, |v| up to 4
    # the prompt
    q, k, v = enter([r[:n] for r, n in zip(raw, lens)], [0] * B)
    out = m.attend_history(q, k, v, off_of(lens))
    i = 0
    for b, n in enumerate(lens):
        assert torch.allclose(out[i:i + n].float(), whole[at[b]:at[b] + n].float(), **tol)
        i += n
    # event by event
    for e in range(extra):
        q, _, _ = enter([r[n + e:n + e + 1] for r, n in zip(raw, lens)], [n + e for n in lens])
        ctx = torch.tensor([n + e + 1 for n in lens], dtype=torch.int32).cuda()
        out = m.attend_tree(q, ck, cv, table.cuda(), ctx, off_of([1] * B))
        for b, n in enumerate(lens):
            assert torch.allclose(out[b].float(), whole[at[b] + n + e].float(), **tol)
    # the last three events as a chain of drafts behind the prompt, and the first of them as one of two candidates
    x = torch.cat([r[n:] for r, n in zip(raw, lens)]).cuda()
    pos = torch.cat([torch.arange(n, n + extra) for n in lens]).to(torch.int32).cuda()
    q, k = m.norm_rotate(x[:, :Hq], x[:, Hq:Hq + Hkv], pos)
    ctx = torch.tensor(lens, dtype=torch.int32).cuda()
    out = m.attend_tree(q, ck, cv, table.cuda(), ctx, off_of([extra] * B), parent=torch.tensor([-1, 0, 1] * B, dtype=torch.int32).cuda(), tree_k=k, tree_v=x[:, Hq + Hkv:])
    for b, n in enumerate(lens):
        assert torch.allclose(out[3 * b:3 * b + 3].float(), whole[at[b] + n:at[b] + n + 3].float(), **tol)
    out = m.attend_tree(q, ck, cv, table.cuda(), ctx, off_of([extra] * B), tree_k=k, tree_v=x[:, Hq + Hkv:])
    for b, n in enumerate(lens):
        assert torch.allclose(out[3 * b].float(), whole[at[b] + n].float(), **tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graphs_streams_and_both_ways_of_marshalling(dtype):
    gen = torch.Generator().manual_seed(41)
    Hq, Hkv, dh = 4, 2, 64
    m = lime(dtype, Hq, Hkv, dh, rot_dim=dh)
    lens = [300, 5, 0, 1200]
    q, k, v = (rand(gen, sum(lens), h, dh, dtype=dtype).cuda() for h in (Hq, Hkv, Hkv))
    pos = torch.arange(sum(lens), dtype=torch.int32).cuda()
    ck, cv, table = paged(gen, [5000, 3, 0, 700], 32, Hkv, dh, dtype)
    ck, cv, table, ctx = ck.cuda(), cv.cuda(), table.cuda(), torch.tensor([5000, 3, 0, 700], dtype=torch.int32).cuda()
    off, off1 = off_of(lens), off_of([1] * 4)

    def calls():
        a = m.norm_rotate(q, k, pos)
        return a[0], a[1], m.attend_history(a[0], a[1], v, off), m.attend_tree(q[:4], ck, cv, table, ctx, off1, tree_k=k[:4], tree_v=v[:4])

    want = [t.clone() for t in calls()]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(calls(), want))                 # bit for bit, every time
    native, m._native = m._native, binding._PlainCalls
    assert all(torch.equal(a, b) for a, b in zip(calls(), want))
    m._native = native
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = calls()
        graphs.append((g, r))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (g, r), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, r in graphs for a, b in zip(r, want))
    results = []
    for s in streams * 2:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            results.append(calls())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in results for a, b in zip(r, want))
    assert binding.lime_device_status(m.ctx) == 0


def test_refusals():
    m = binding.Lime(d=64, H=2, ell=8, n_layers=1, dtype=binding.LIME_BF16)
    q, k = torch.zeros(4, 4, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 2, 32, dtype=torch.bfloat16, device="cuda")
    off, pos = off_of([4]), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.LimeError) as e:
        m.attend_history(q, k, k, off)
    assert e.value.status == 5
    lib = binding.load_library()
    import ctypes
    seq = binding.lime_sequence
    for bad, status in ((seq(0, 1, 32), 1), (seq(4, 0, 32), 1), (seq(4, 3, 32), 1), (seq(4, 2, 0), 1), (seq(4, 2, 32, -1.0), 1), (seq(4, 2, 32, float("nan")), 1),
                        (seq(4, 2, 32, 0, -1.0), 1), (seq(4, 2, 32, 0, 0, 34), 1), (seq(4, 2, 32, 0, 0, 3), 1), (seq(4, 2, 32, 0, 0, 4, 2), 1),
                        (seq(4, 2, 32, 0, 0, 4, 0, 0.5), 1), (seq(4, 2, 32, 0, 0, 4, 0, 1e31), 1), (seq(4, 2, 32, 0, 0, 4, 0, float("nan")), 1), (seq(4, 2, 36), 2), (seq(4, 2, 136), 2),
                        (seq(65, 1, 32), 2), (seq(2048, 64, 8), 2)):
        assert lib.lime_set_sequence(m.ctx, ctypes.byref(bad)) == status
    assert lib.lime_set_sequence(m.ctx, None) == 1 and lib.lime_sequence_workspace_bytes(m.ctx, 1, 1) == 0
    for native in (binding._native(), binding._PlainCalls):
        m._native = native
        m.set_sequence(4, 2, 32, rot_dim=32)
        cache = torch.zeros(2, 16, 2, 32, dtype=torch.bfloat16, device="cuda")
        table, ctx = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        for call in (lambda: m.attend_history(q.float(), k, k, off), lambda: m.attend_history(q, k.float(), k, off), lambda: m.attend_history(q.cpu(), k, k, off),
                     lambda: m.attend_history(q, k, k[:3], off), lambda: m.attend_history(k, k, k, off), lambda: m.attend_history(q, k, k, off.long()),
                     lambda: m.attend_history(q.transpose(1, 2).contiguous().transpose(1, 2), k, k, off), lambda: m.attend_history(q, k, k, off, kv_off=off[:1]),
                     lambda: m.attend_history(q, k, k, off, out=q[:3]), lambda: m.norm_rotate(q, k, pos[:3]), lambda: m.norm_rotate(q, k, pos.float()),
                     lambda: m.norm_rotate(q, k, pos, gamma_q=torch.ones(32, device="cuda")), lambda: m.norm_rotate(q, k, pos, cache_k=cache[0], slots=pos),
                     lambda: m.norm_rotate(q, k, pos, v=k, cache_k=cache, cache_v=cache[:1], slots=pos),
                     lambda: m.attend_tree(q, cache, cache[:1], table, ctx, off), lambda: m.attend_tree(q, cache, cache, table[0], ctx, off),
                     lambda: m.attend_tree(q, cache, cache, table, ctx[:0], off), lambda: m.attend_tree(q, cache, cache, table, ctx, off, tree_k=k, tree_v=k, parent=pos[:2])):
            with pytest.raises(ValueError):
                call()
        with pytest.raises(TypeError):
            m.attend_history(q, k, [1], off)
        wide = torch.zeros(4, 4 * 32 + 4, dtype=torch.bfloat16, device="cuda")
        odd = wide[:, :128].view(4, 4, 32) if False else torch.as_strided(wide, (4, 4, 32), (132, 32, 1))
        shifted = torch.as_strided(torch.zeros(600, dtype=torch.bfloat16, device="cuda"), (4, 4, 32), (128, 32, 1), 4)
        over = torch.as_strided(torch.zeros(600, dtype=torch.bfloat16, device="cuda"), (4, 4, 32), (64, 32, 1))
        for call in (lambda: m.attend_history(odd, k, k, off), lambda: m.attend_history(shifted, k, k, off), lambda: m.attend_history(over, k, k, off),
                     lambda: m.attend_history(q, k[:3], k[:3], off), lambda: m.norm_rotate(q, k, None), lambda: m.norm_rotate(q, k, pos, cache_k=cache),
                     lambda: m.norm_rotate(q, k, pos, v=k), lambda: m.norm_rotate(q, k, pos, slots=pos), lambda: m.norm_rotate(odd, k, pos),
                     lambda: m.norm_rotate(q, k, pos, cache_v=cache, v=k), lambda: m.attend_tree(q, cache, cache, table, ctx, off, tree_k=k),
                     lambda: m.attend_tree(q, cache, cache, table, ctx, off, parent=pos), lambda: m.attend_tree(q, cache[:, :8].contiguous(), cache[:, :8].contiguous(), table, ctx, off),
                     lambda: m.attend_tree(q, cache.view(1, 32, 2, 32)[:, :24].contiguous(), cache.view(1, 32, 2, 32)[:, :24].contiguous(), table, ctx, off)):
            with pytest.raises(binding.LimeError) as e:
                call()
            assert e.value.status == 1
        assert m.attend_history(q[:0], k[:0], k[:0], off_of([0])).shape == (0, 4, 32)
        assert m.attend_tree(q[:0], cache, cache, table[:0], ctx[:0], off[:1]).shape == (0, 4, 32)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(binding.LimeError) as e:
        binding.lime_attend_history(m.ctx, binding.lime_sequence(4, 2, 32), q, off, k, k, None, torch.empty_like(q), small)
    assert e.value.status == 3
