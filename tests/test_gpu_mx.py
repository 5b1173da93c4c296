"""The 4-bit cache on the GPU against its definition in 64 bits on the host: bytes written and values read back equal, attention within
the bound that mx_reference.tolerance derives.  Caches start out full of 0xFF (every scale a NaN), so that whatever is read beyond a
sequence's end shows."""
import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2601_23180_amd import MXCache, mx_append, mx_attend, mx_read

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def random_rows(rng, shape, dtype, wild=False):
    """Normal numbers, some features several times as large; `wild`: also zeros, ties, huge and tiny blocks."""
    x = rng.standard_normal(shape) * (1 + 4 * (rng.random(shape[-1]) < 0.06))
    if wild:
        flat = x.reshape(-1, 32)
        pick = rng.integers(0, 8, len(flat))
        flat[pick == 0] = 0.0
        flat[pick == 1] *= 2.0 ** rng.integers(-140, 120, (pick == 1).sum())[:, None]
        flat[pick == 2] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, 6.9], flat[pick == 2].shape)
        flat[pick == 3, 0] = 7.0
        flat[pick == 4, 31] = -3.3e38
    return torch.from_numpy(x).float().to(DT[dtype])


def make_cache(batch, kv, d, capacity, paged, rng):
    if not paged:
        c = MXCache.empty(batch, kv, d, capacity)
        table = None
    else:
        pages = -(-capacity // R.PAGE)
        table = rng.permutation(batch * pages + 2)[: batch * pages].reshape(batch, pages).astype(np.int32)
        c = MXCache.empty(batch, kv, d, 0, torch.from_numpy(table).cuda(), batch * pages + 2)
    for t in c.tensors[:4]:
        t.fill_(0xFF)
    ref = R.Bytes(c.tensors[0].shape[0], kv, c.tensors[0].shape[2], d, 0xFF)
    return c, ref, table


def assert_bytes(cache, ref):
    torch.cuda.synchronize()
    for t, want in zip(cache.tensors[:4], ref.arrays):
        np.testing.assert_array_equal(t.cpu().numpy(), want)


@pytest.mark.parametrize("d,kv,dtype,paged,start,count", [
    (128, 2, "bf16", False, [0], [1]), (128, 8, "f32", False, [5, 8, 63], [1, 0, 2]), (64, 3, "bf16", False, [7, 0], [9, 64]),
    (64, 1, "f32", True, [250, 511], [13, 1]), (128, 2, "bf16", True, [0, 255, 3], [300, 2, 257]), (128, 1, "f32", False, [3], [130]),
])
def test_append_writes_its_bytes_and_no_others(d, kv, dtype, paged, start, count):
    rng = np.random.default_rng(d + kv + sum(start))
    n = max(count) + 2                                                   # a padded batch
    c, ref, table = make_cache(len(start), kv, d, 576, paged, rng)
    k, v = (random_rows(rng, (len(start), n, kv, d), dtype, wild=True) for _ in range(2))
    mx_append(c, k.cuda(), v.cuda(), start, count)
    for b, (s, m) in enumerate(zip(start, count)):
        for i in range(m):
            ref.write(*R.place(table, b, s + i), k[b, i].double().numpy(), v[b, i].double().numpy())
    assert_bytes(c, ref)
    lo = [max(0, s - 3) for s in start]
    for out in ("bf16", "f32"):
        rk, rv = mx_read(c, lo, n + 5, DT[out])
        for x, y in ((k, rk), (v, rv)):
            for b, (s, m) in enumerate(zip(start, count)):
                got = y[b].double().cpu().numpy()
                np.testing.assert_array_equal(got[s - lo[b]:s - lo[b] + m], R.rounded(x[b, :m].double().numpy()))
                assert np.isnan(got[:s - lo[b]]).all() and np.isnan(got[s - lo[b] + m:]).all()


def test_blocks_with_an_infinity_or_a_nan_read_back_as_nan():
    x = torch.ones(1, 4, 1, 64)
    x[0, 0, 0, 3], x[0, 1, 0, 40], x[0, 2, 0, 63] = float("nan"), float("inf"), float("-inf")
    c = MXCache.empty(1, 1, 64, 64)
    mx_append(c, x.cuda(), x.cuda(), [0])
    for t in mx_read(c, [0], 4, torch.float32):
        bad = torch.isnan(t[0, :, 0]).cpu()
        want = torch.zeros(4, 64, dtype=torch.bool)
        want[0, :32] = want[1, 32:] = want[2, 32:] = True
        assert torch.equal(bad, want) and (t[0, :, 0].cpu()[~want] == 1).all()


def test_rows_by_other_strides_and_one_side_alone():
    """Keys and values inside a fused row, sequences interleaved; only keys, or only values, read back, into such rows."""
    rng = np.random.default_rng(3)
    fused = random_rows(rng, (5, 2, 3 * 2, 64), "bf16").cuda()           # [row][sequence][q, k, v heads]
    k, v = fused[:, :, 2:4].transpose(0, 1), fused[:, :, 4:].transpose(0, 1)
    c = MXCache.empty(2, 2, 64, 64)
    mx_append(c, k, v, [1, 30])
    for out in mx_read(c, [1, 30], 5), :
        for x, y in ((k, out[0]), (v, out[1])):
            np.testing.assert_array_equal(y.double().cpu().numpy(), R.rounded(x.double().cpu().numpy()))
    import ctypes as C
    from paper_2601_23180_amd import binding as B
    to = torch.full((5, 2, 6, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    row, seq = to.stride(0), to.stride(1)
    one = B.MXRows(to[:, :, 2:4].data_ptr(), row, seq)
    ints = lambda *v: (C.c_int32 * len(v))(*v)  # noqa: E731
    B.check(B.lib().trispec_mx_read(c.ref, C.byref(one), None, B.TRISPEC_BF16, ints(1, 30), ints(5, 3), None))
    torch.cuda.synchronize()
    want = torch.full_like(to, 9.0)
    want[:, 0, 2:4] = torch.from_numpy(R.rounded(k[0].double().cpu().numpy())).to("cuda", torch.bfloat16)
    want[:3, 1, 2:4] = torch.from_numpy(R.rounded(k[1, :3].double().cpu().numpy())).to("cuda", torch.bfloat16)
    assert torch.equal(to, want)


def test_a_cache_beyond_32_bits():
    """Offsets that pass 2^32 bytes: the last sequence of a cache of 8 x 2^24 slots of 64 features."""
    cap = 1 << 24
    c = MXCache.empty(8, 1, 64, cap)
    rng = np.random.default_rng(1)
    x = random_rows(rng, (8, 40, 1, 64), "bf16").cuda()
    start = [0, 5, 0, 0, 0, 0, 3, cap - 40]
    mx_append(c, x, x, start)
    k, v = mx_read(c, start, 40)
    want = torch.from_numpy(R.rounded(x.double().cpu().numpy())).to("cuda", torch.bfloat16)
    assert torch.equal(k, want) and torch.equal(v, want)
    q = random_rows(rng, (8, 1, 1, 64), "f32").cuda()
    own = random_rows(rng, (8, 1, 1, 64), "f32").cuda()
    out = mx_attend(c, [0] * 7 + [40], q, own, own).double().cpu().numpy()
    # no context: its own value.  The one weight p stands in the sum and under it, so p (1 but for the score's rounding) cancels; what is left
    # is the rounding of at most 6 products' sum (three parts of p, three of v), of the merge's scaling on both sides and of its division: 10 of 2^-24
    want = own[:7].double().cpu().numpy()
    assert (np.abs(out[:7] - want) <= 10 * 2.0 ** -24 * np.abs(want)).all()


def test_a_range_that_takes_more_than_one_launch():
    """2^23 workgroups and some, over two pages that a table repeats."""
    from paper_2601_23180_amd import binding as B
    n, heads, row = (1 << 18) + 40, 1024, 1024 * 64
    table = (torch.arange(1025, dtype=torch.int32) % 2)[None].cuda()
    c = MXCache.empty(1, heads, 64, 0, table, 2)
    rows = random_rows(np.random.default_rng(5), (1, 512, heads, 64), "bf16").cuda()
    mx_append(c, rows, rows, [0])
    want = mx_read(c, [0], 512)[0][0]
    out = torch.empty((n, heads, 64), dtype=torch.bfloat16, device="cuda")
    out[-512:] = -1
    B.check(B.lib().trispec_mx_read(c.ref, B._pack_rows(out.data_ptr(), row, n * row), None, B.TRISPEC_BF16, c.ints([0]), c.ints([n]),
                                    torch.cuda.current_stream().cuda_stream))
    for first in (0, 512 * 300 + 7, (1 << 18) - 30, n - 100):
        for i in range(first, first + 100, 9):
            if i < n:
                assert torch.equal(out[i], want[i % 512]), i
    del out
    torch.cuda.empty_cache()


def tree(rng, m, kind):
    if kind == "chain":
        return np.arange(-1, m - 1, dtype=np.int32)
    p = np.full(m, -1, np.int32)
    for i in range(1, m):
        p[i] = rng.integers(0, i) if kind == "bush" else max(0, i - 1 - rng.integers(0, 4))
    return p


def attend_case(d, heads, kv, nodes, ctx, dtype, paged, kind, append, own=True, seed=0, fused=True):
    rng = np.random.default_rng([seed, d, heads, nodes, len(ctx)])
    batch = len(ctx)
    cap = max(64, -(-(max(ctx) + nodes) // 64) * 64)
    c, ref, table = make_cache(batch, kv, d, cap, paged, rng)
    n = max(ctx)
    k_ctx, v_ctx = (random_rows(rng, (batch, max(n, 1), kv, d), "f32") for _ in range(2))
    mx_append(c, k_ctx.cuda(), v_ctx.cuda(), [0] * batch, list(ctx))
    x = random_rows(rng, (batch, nodes, heads + 2 * kv, d), dtype).cuda()
    q, k, v = x[:, :, :heads], x[:, :, heads:heads + kv], x[:, :, heads + kv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    parents = np.stack([tree(rng, nodes, kind) for _ in range(batch)])
    given = None if kind == "chain" else parents
    before = [t.clone() for t in c.tensors[:4]]
    out = mx_attend(c, ctx, q, k if own else None, v if own else None, parents=given, append=append)
    assert out.dtype == DT[dtype] and out.shape == (batch, nodes, heads, d)
    got = out.double().cpu().numpy()
    worst = 0.0
    for b in range(batch):
        kb, vb = (R.rounded(t[b, :ctx[b]].double().numpy()) for t in (k_ctx, v_ctx))
        mine = [t[b].double().cpu().numpy() for t in (q, k, v)]
        want, mass, spread = R.attend(mine[0], kb, vb, mine[1] if own else None, mine[2] if own else None, parents[b])
        tol = R.tolerance(want, mass, spread, ctx[b] + nodes, d, dtype == "bf16")
        off = np.abs(got[b] - want)
        assert (off <= tol).all(), (b, float((off / tol).max()), np.argwhere(off > tol)[:3])
        worst = max(worst, float((off / tol).max()))
    if append:      # as if by mx_append, byte for byte
        other = MXCache(*before, c.tensors[4])
        mx_append(other, k.contiguous(), v.contiguous(), ctx)
        before = other.tensors[:4]
    for t, w in zip(c.tensors[:4], before):
        assert torch.equal(t, w)
    return worst


LENGTHS = [[0], [1], [7, 0], [31, 32, 33], [127], [129, 128], [255, 256, 257], [1000, 3], [513]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ctx", LENGTHS, ids=str)
def test_attend_single_token_over_every_kind_of_end(ctx, dtype):
    for d, heads, kv, paged in ((128, 8, 2, False), (64, 3, 3, True), (128, 8, 1, True)):
        attend_case(d, heads, kv, 1, ctx, dtype, paged, "chain", append=paged)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,heads,kv,nodes,ctx,paged,kind", [
    (128, 2, 2, 16, [300], False, "tree"),            # 16 rows: one block
    (128, 4, 1, 5, [77, 260], True, "bush"),          # 20 rows: two
    (64, 8, 2, 8, [515], False, "chain"),             # 32
    (128, 4, 2, 17, [200, 0, 40], True, "tree"),      # 34: two wavefronts side by side
    (64, 4, 2, 31, [640], True, "tree"),              # 62
    (128, 8, 2, 17, [1025], False, "tree"),           # 68: four
    (128, 8, 4, 60, [300], True, "bush"),             # 120
    (64, 8, 2, 33, [700, 129], False, "tree"),        # 132: 64 rows each
    (128, 8, 2, 60, [999], False, "tree"),            # 240
    (128, 4, 1, 128, [129, 64], True, "chain"),       # 512: two row groups
    (64, 8, 1, 64, [0, 300], False, "bush"),          # 512
    (128, 1, 1, 128, [65], True, "tree"),
])
def test_attend_trees_of_every_form(d, heads, kv, nodes, ctx, paged, kind, dtype):
    attend_case(d, heads, kv, nodes, ctx, dtype, paged, kind, append=nodes % 2 == 0, fused=nodes % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_a_long_context_in_many_splits(dtype):
    attend_case(128, 4, 1, 1, [20000], dtype, False, "chain", append=True)
    attend_case(64, 2, 2, 9, [9000, 4097], dtype, True, "tree", append=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_the_cache_alone_and_rows_without_a_key(dtype):
    attend_case(128, 4, 2, 3, [100, 0, 32], dtype, False, "chain", append=False, own=False)
    attend_case(64, 2, 1, 40, [0], dtype, True, "chain", append=False, own=False)
    attend_case(128, 8, 2, 60, [0, 70], dtype, False, "chain", append=False, own=False)


def test_scores_that_keep_growing_and_scores_far_apart():
    """Every run of keys has a new maximum; scores spread over thousands: weights of exactly 1 and 0."""
    for nodes in (1, 40):
        c = MXCache.empty(1, 1, 128, 1024)
        rng = np.random.default_rng(nodes)
        k = torch.from_numpy(rng.standard_normal((1, 900, 1, 128)) * np.linspace(0.01, 6, 900)[:, None, None]).float().cuda()
        v = random_rows(rng, (1, 900, 1, 128), "f32").cuda()
        mx_append(c, k, v, [0])
        q = 3 * random_rows(rng, (1, nodes, 2, 128), "f32").cuda()
        own = random_rows(rng, (1, nodes, 1, 128), "f32").cuda()
        out = mx_attend(c, [900], q, own, own).double().cpu().numpy()[0]
        kb, vb = R.rounded(k[0].double().cpu().numpy()), R.rounded(v[0].double().cpu().numpy())
        o = own[0].double().cpu().numpy()
        want, mass, spread = R.attend(q[0].double().cpu().numpy(), kb, vb, o, o, tree(rng, nodes, "chain"))
        assert (np.abs(out - want) <= R.tolerance(want, mass, spread, 900 + nodes, 128, False)).all()


@pytest.mark.parametrize("d,heads,kv,nodes,ctx", [(128, 4, 2, 1, 100), (64, 4, 1, 9, 700), (128, 4, 2, 9, 2500), (128, 8, 2, 60, 3000), (64, 2, 2, 40, 0)])
def test_fp32_rows_lose_nothing_to_the_matrix_instructions_type(d, heads, kv, nodes, ctx):
    """fp32 operands go in three parts of 8 bits, 24 in all, so a score is the fp32 sum of 3 d exact products: off by (3 d + 8) 2^-24 of
    sum |q| |k| / sqrt(d), the scale, the maximum and the parts' cut at the end among the 8.  A weight is off by that twice (numerator, and sum of weights), by
    its own cut and exponential, 4 of 2^-24, twice as well, and by the sums' (3 n + 64) 2^-24; a factor of 2 for second-order terms."""
    rng = np.random.default_rng([nodes, ctx])
    c = MXCache.empty(1, kv, d, 4096)
    k_ctx, v_ctx = (random_rows(rng, (1, max(ctx, 1), kv, d), "f32") for _ in range(2))
    mx_append(c, k_ctx.cuda(), v_ctx.cuda(), [0], [ctx])
    x = random_rows(rng, (1, nodes, heads + 2 * kv, d), "f32")
    q, k, v = x[:, :, :heads], x[:, :, heads:heads + kv], x[:, :, heads + kv:]
    y = x.cuda()
    out = mx_attend(c, [ctx], y[:, :, :heads], y[:, :, heads:heads + kv], y[:, :, heads + kv:])[0].double().cpu().numpy()
    kb, vb = (R.rounded(t[0, :ctx].double().numpy()) for t in (k_ctx, v_ctx))
    want, mass, spread = R.attend(q[0].double().numpy(), kb, vb, k[0].double().numpy(), v[0].double().numpy(), tree(rng, nodes, "chain"))
    weight = 2 * (3 * d + 8) * 2.0 ** -24 * spread + (2 * 4 + 3 * (ctx + nodes) + 64) * 2.0 ** -24
    assert (np.abs(out - want) <= 2 * weight * mass + 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,heads,kv,nodes,ctx,paged,kind", [
    (128, 4, 2, 1, [1600], False, "chain"),             # 16 rows a workgroup, one sequence
    (64, 4, 4, 3, [2687, 0, 5, 2688], True, "chain"),   # an empty sequence and a short one among the long
    (128, 6, 2, 8, [2000, 2049], True, "bush"),         # 32
    (64, 16, 2, 33, [3000], False, "tree"),             # 64, and two partials of nodes
    (128, 4, 1, 60, [2433, 77], True, "tree"),
    (128, 1, 1, 128, [4001], False, "chain"),           # four
    (64, 8, 8, 2, [3100] * 8, False, "bush"),           # splits for every CU twice, fewer than there are keys for
])
def test_attend_beyond_what_one_workgroup_takes(d, heads, kv, nodes, ctx, paged, kind, dtype):
    attend_case(d, heads, kv, nodes, ctx, dtype, paged, kind, append=nodes % 2 == 0, fused=nodes % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [1, 9])
def test_attend_on_both_sides_of_the_longest_context_of_one_workgroup(nodes, dtype):
    for ctx in (600, 640, 1100, 1200, 1500, 1600):
        attend_case(64, 4, 2, nodes, [ctx], dtype, False, "tree", append=True, seed=ctx)


@pytest.mark.parametrize("nodes,heads", [(1, 1), (9, 4), (40, 4)])
def test_nan_in_a_long_context_reaches_the_rows_that_see_it_and_no_others(nodes, heads):
    rng = np.random.default_rng(nodes)
    c = MXCache.empty(2, 2, 64, 4096)
    k, v = (random_rows(rng, (2, 4000, 2, 64), "f32") for _ in range(2))
    v[0, 2500, 1, 40] = float("nan")
    k[1, 3999, 0, 3] = float("inf")
    mx_append(c, k.cuda(), v.cuda(), [0, 0])
    q = random_rows(rng, (2, nodes, 2 * heads, 64), "f32").cuda()
    own_k, own_v = (random_rows(rng, (2, nodes, 2, 64), "f32") for _ in range(2))
    parents = np.zeros((2, nodes), np.int32)
    parents[:, 0] = -1
    if nodes > 2:
        own_v[0, 1, 0, 7], own_v[0, 2, 0, 8] = float("inf"), float("nan")
    for length, seen in ((4000, True), (2500, False)):
        out = torch.isnan(mx_attend(c, [length, length], q, own_k.cuda(), own_v.cuda(), parents=parents)).cpu().unflatten(2, (2, heads))
        want = torch.zeros(2, nodes, 2, heads, 64, dtype=torch.bool)
        want[0, :, 1, :, 32:] = seen
        want[1, :, 0] = seen
        if nodes > 2:
            want[0, 2, 0, :, 8] = True
        assert torch.equal(out, want)


@pytest.mark.parametrize("nodes,heads", [(1, 1), (9, 1), (9, 4), (40, 4)])
def test_nan_reaches_the_rows_that_see_it_and_no_others(nodes, heads):
    rng = np.random.default_rng(nodes)
    c = MXCache.empty(2, 2, 64, 128)
    k, v = (random_rows(rng, (2, 100, 2, 64), "f32") for _ in range(2))
    v[0, 50, 1, 40] = float("nan")                    # a value of sequence 0, head 1: features 32 .. 63 of all its rows
    k[1, 99, 0, 3] = float("inf")                     # a key of sequence 1, head 0: everything of its rows
    mx_append(c, k.cuda(), v.cuda(), [0, 0])
    q = random_rows(rng, (2, nodes, 2 * heads, 64), "f32").cuda()
    own_k, own_v = (random_rows(rng, (2, nodes, 2, 64), "f32") for _ in range(2))
    parents = np.zeros((2, nodes), np.int32)          # every node below the root: two levels
    parents[:, 0] = -1
    if nodes > 2:
        own_v[0, 1, 0, 7], own_v[0, 2, 0, 8] = float("inf"), float("nan")   # nodes 1 and 2 of sequence 0, head 0, see it; the others do not
    out = torch.isnan(mx_attend(c, [100, 100], q, own_k.cuda(), own_v.cuda(), parents=parents)).cpu().unflatten(2, (2, heads))
    want = torch.zeros(2, nodes, 2, heads, 64, dtype=torch.bool)
    want[0, :, 1, :, 32:] = True
    want[1, :, 0] = True
    if nodes > 2:
        want[0, 2, 0, :, 8] = True
    assert torch.equal(out, want)
    # one slot less: the key at the end of sequence 1 is no token any more
    out = torch.isnan(mx_attend(c, [50, 99], q, own_k.cuda(), own_v.cuda(), parents=parents)).cpu().unflatten(2, (2, heads))
    want[:] = False
    if nodes > 2:
        want[0, 2, 0, :, 8] = True
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ctx,first,count", [(1, 0, 1), (40, 0, 40), (300, 32, 32), (300, 0, 300), (3000, 0, 3000), (3000, 1024, 600)])
@pytest.mark.parametrize("nodes", [1, 9])
def test_keys_that_are_all_nan_reach_every_row(nodes, ctx, first, count, dtype):
    """Runs, and whole contexts, without a score that is a number."""
    rng = np.random.default_rng(ctx)
    c = MXCache.empty(1, 2, 64, 4096)
    k, v = (random_rows(rng, (1, ctx, 2, 64), "f32") for _ in range(2))
    k[0, first:first + count, 0] = float("nan")
    mx_append(c, k.cuda(), v.cuda(), [0])
    q, own = random_rows(rng, (1, nodes, 4, 64), dtype).cuda(), random_rows(rng, (1, nodes, 2, 64), dtype).cuda()
    for mine in (own, None):
        out = torch.isnan(mx_attend(c, [ctx], q, mine, mine)).cpu()
        assert out[:, :, :2].all() and not out[:, :, 2:].any()


def test_page_ids_outside_the_pool_are_clamped():
    table = torch.tensor([[-5, 1000]], dtype=torch.int32, device="cuda")
    c = MXCache.empty(1, 1, 64, 0, table, 3)
    x = torch.full((1, 512, 1, 64), 2.0, device="cuda")
    mx_append(c, x, x, [0])
    assert all((t == 2).all() for t in mx_read(c, [0], 512))
    assert torch.equal(c.tensors[0][0], c.tensors[0][2]) and not c.tensors[0][1].any()
    out = mx_attend(c, [512], x[:, :1], x[:, :1], x[:, :1])
    assert (out == 2).all()


def test_captured_calls_replay_on_another_stream_with_workspaces_of_their_own():
    rng = np.random.default_rng(8)
    c = MXCache.empty(1, 2, 128, 1024)
    k, v = (random_rows(rng, (1, 700, 2, 128), "bf16").cuda() for _ in range(2))
    mx_append(c, k, v, [0])
    xs = [random_rows(rng, (1, 3, 12, 128), "bf16").cuda() for _ in range(2)]
    split = lambda x: (x[:, :, :8], x[:, :, 8:10], x[:, :, 10:])  # noqa: E731
    ws = [torch.empty(c.workspace_bytes(3, 8), dtype=torch.uint8, device="cuda") for _ in range(2)]
    eager = [mx_attend(c, [700], *split(x)) for x in xs]
    torch.cuda.synchronize()
    graphs, outs, side = [], [], torch.cuda.Stream()
    for x, w in zip(xs, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = mx_attend(c, [700], *split(x), append=True, workspace=w, stream=side)
            outs.append((out, *mx_read(c, [700], 3, stream=side)))
        graphs.append(g)
    for turn in range(4):
        for g, x, o, e in zip(graphs, xs, outs, eager):
            with torch.cuda.stream(side):
                g.replay()
            side.synchronize()
            _, kk, vv = split(x)
            assert torch.equal(o[0], e)
            np.testing.assert_array_equal(o[1].double().cpu().numpy(), R.rounded(kk.double().cpu().numpy()))
            np.testing.assert_array_equal(o[2].double().cpu().numpy(), R.rounded(vv.double().cpu().numpy()))
            assert torch.equal(mx_attend(c, [700], *split(x)), e)          # eager work in between
        xs[0].mul_(1.0)


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(4)
    for nodes, ctx in ((1, 5000), (60, 3000)):
        c = MXCache.empty(1, 2, 128, 8192)
        k, v = (random_rows(rng, (1, ctx, 2, 128), "bf16").cuda() for _ in range(2))
        mx_append(c, k, v, [0])
        x = random_rows(rng, (1, nodes, 12, 128), "f32").cuda()
        first = mx_attend(c, [ctx], x[:, :, :8], x[:, :, 8:10], x[:, :, 10:])
        for _ in range(3):
            assert torch.equal(mx_attend(c, [ctx], x[:, :, :8], x[:, :, 8:10], x[:, :, 10:]), first)


def test_the_binding_refuses_what_does_not_fit():
    c = MXCache.empty(2, 2, 64, 64)
    x = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (x[:1], x[..., :32], x.cpu(), x[:, :, :1], x.half(), x.transpose(1, 3)):
        with pytest.raises(ValueError):
            mx_append(c, bad, x, [0, 0])
    with pytest.raises(ValueError):
        mx_append(c, x, x, [0, 0], [4, 0])          # more rows than there are
    with pytest.raises(ValueError):
        mx_append(c, x, x, [0])
    with pytest.raises(ValueError):
        mx_append(c, x, x[:, :2], [0, 0])
    with pytest.raises(ValueError):
        mx_attend(c, [0, 0], x, x, None)
    with pytest.raises(ValueError):
        mx_attend(c, [0, 0], x, x, x, parents=np.zeros((2, 2), np.int32))
    with pytest.raises(ValueError):
        mx_attend(c, [0, 0], x, x.float(), x.float())
    with pytest.raises(ValueError):
        mx_read(c, [0, 0], 1, torch.float16)
    with pytest.raises(ValueError):
        MXCache(c.tensors[0], c.tensors[1], c.tensors[2], c.tensors[3][:, :, :4])
    k, v = mx_read(c, [3, 4], 0)
    assert k.shape == v.shape == (2, 0, 2, 64)
