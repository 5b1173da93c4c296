"""The verification pass, the commit and the two-level rounds over a cache held in 4 bits, as a program uses them together."""
import numpy as np
import pytest
import torch

import mx_reference as R
from gpu_helpers import Case, compare_decisions, device_model
from helpers import prefill
from oracle import CRIT_MARGIN
from paper_2601_23180_amd import MXKVCache, TernaryDecoder, Verifier, fill_kv_layer
from paper_2601_23180_amd.binding import LAUNCH_PER_LAYER
from workloads import SHAPES, gen_context_tokens, gen_draft_tokens, gen_tree, tree_depths

pytestmark = pytest.mark.gpu


def problem(shape, seed, ctx, nodes, batch=1):
    parents = np.stack([gen_tree(nodes, 5, 3, seed + b) for b in range(batch)])
    ks, vs = [], []
    for b in range(batch):
        K, V = prefill(shape, seed, gen_context_tokens(shape.vocab, ctx - 7 * b, seed + b))
        ks.append(R.rounded(K)), vs.append(R.rounded(V))           # what such a cache holds of it
    tokens = np.stack([gen_draft_tokens(parents[b], shape.vocab, seed + b) for b in range(batch)])
    positions = np.stack([ctx - 7 * b + tree_depths(parents[b]) for b in range(batch)])
    return Case(shape, seed, ks, vs, tokens, parents, positions)


def run(case, paged, launch_mode=0):
    model = device_model(case.shape, case.seed)
    cap = (max(case.ctx_len) + case.n_nodes + 63) // 64 * 64
    kv = MXKVCache(model, case.batch, cap, paged=paged)
    for l in range(case.shape.n_layers):
        k = np.zeros((case.batch, case.shape.n_kv_heads, max(case.ctx_len), case.shape.head_dim))
        v = k.copy()
        for b in range(case.batch):
            k[b, :, :case.ctx_len[b]], v[b, :, :case.ctx_len[b]] = case.k_ctx[b][l], case.v_ctx[b][l]
        fill_kv_layer(kv, l, k, v)
    kv.set_len(case.ctx_len)
    ver = Verifier(model, case.batch, case.n_nodes, debug_logits=True)
    ver.launch_mode = launch_mode
    out = ver.verify(kv, torch.from_numpy(case.tokens).cuda(), case.parents, torch.from_numpy(case.positions).cuda(), 0.5, CRIT_MARGIN)
    torch.cuda.synchronize()
    got = {k: t.cpu().numpy() for k, t in out.items()}
    got["logits"] = ver.logits.cpu().numpy()
    return got, kv, model


@pytest.mark.parametrize("key,nodes,batch,paged,mode", [
    ("tiny_bf16", 24, 1, False, 0), ("tiny_bf16", 24, 1, True, LAUNCH_PER_LAYER), ("tiny_bf16", 9, 3, True, 0), ("tiny_bf16", 70, 1, False, 0)])
def test_pass_against_the_oracle(key, nodes, batch, paged, mode):
    """The context as the cache reads back, the nodes unrounded: the bars of the bf16 cache's parity tests."""
    case = problem(SHAPES[key], 5, 96, nodes, batch)
    got, kv, model = run(case, paged, mode)
    want = case.run_oracle()
    for b in range(batch):
        ref = want[b]["logits"]
        assert np.abs(got["logits"][b] - ref).max() <= 2e-2 * np.abs(ref).max()
        assert np.abs(got["logits"][b] - ref).max() <= 2e-3                          # and what they reach there
        np.testing.assert_array_equal(got["status"], [0])
    compare_decisions(case, got, want, 0.5, CRIT_MARGIN)
    # the nodes' rows went into the cache: within half a step of the oracle's (2 scales between the largest values, a scale is at most the
    # block's largest / 3.5; 2^-7: the oracle's are rounded to bf16, and what the rounding of its operands does), and but for values
    # next to a border the very same (bf16 moves a value by up to 2^-8 of it, a step is a sixth of it and more: 1 in 20 at most)
    for b in range(batch):
        n = case.ctx_len[b]
        for mine, theirs in ((kv.k, want[b]["k_new"]), (kv.v.transpose(-1, -2), want[b]["v_new"])):
            mine = mine[:, b, :, n:n + nodes].double().cpu().numpy()
            blocks = theirs.reshape(*theirs.shape[:-1], -1, 32)
            step = np.repeat(np.abs(blocks).max(-1) / 3.5, 32, -1)
            assert (np.abs(mine - theirs) <= step * (1 + 2.0 ** -7) + 2.0 ** -7 * np.abs(theirs)).all()
            same = mine == R.rounded(theirs)
            assert same.mean() > 0.95, same.mean()


@pytest.mark.parametrize("paged", [False, True])
def test_commit_moves_the_path_and_nothing_else(paged):
    case = problem(SHAPES["tiny_bf16"], 11, 90, 40, 2)
    got, kv, model = run(case, paged)
    before = [(kv.k.clone(), kv.v.clone())]
    paths = [[0, 3, 17, 39], []]
    kv.commit(paths)
    k, v = kv.k, kv.v
    want_k, want_v = before[0]
    want_k, want_v = want_k.clone(), want_v.clone()
    n = case.ctx_len[0]
    for i, node in enumerate(paths[0]):
        want_k[:, 0, :, n + i] = before[0][0][:, 0, :, n + node]
        want_v[:, 0, :, :, n + i] = before[0][1][:, 0, :, :, n + node]
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    kv.sync_len()
    assert kv.ctx_len == [n + 4, case.ctx_len[1]]


def test_a_pass_after_a_commit_reads_what_was_committed():
    """Two passes with a commit between them, against the oracle with the committed rows as the cache reads them back."""
    shape = SHAPES["tiny_bf16"]
    case = problem(shape, 21, 64, 12)
    got, kv, model = run(case, True)
    path = [0]
    while (case.parents[0] == path[-1]).any():
        path.append(int(np.flatnonzero(case.parents[0] == path[-1])[0]))
    kv.commit([path])
    n = kv.ctx_len[0]
    K, V = kv.k[:, 0, :, :n].double().cpu().numpy(), kv.v[:, 0, :, :, :n].transpose(-1, -2).double().cpu().numpy()
    np.testing.assert_array_equal(K[:, :, :64], case.k_ctx[0])
    parents = gen_tree(9, 4, 2, 3)
    again = Case(shape, 21, [K], [V], gen_draft_tokens(parents, shape.vocab, 3), parents, n + tree_depths(parents))
    ver = Verifier(model, 1, 9, debug_logits=True)
    ver.verify(kv, torch.from_numpy(again.tokens).cuda(), again.parents, torch.from_numpy(again.positions).cuda(), 0.5)
    ref = again.run_oracle()[0]["logits"]
    assert np.abs(ver.logits[0].cpu().numpy() - ref).max() <= 2e-3


def rounds(model, prompt, lam, drafts, n, paged):
    """A sequence of n tokens by rounds with `drafts` taken from a given sequence, right except for every third."""
    dec = TernaryDecoder(model, model, 256, max_nodes=16, paged=paged, mx=True)
    dec.start(prompt)
    while len(dec.seq) < n:
        at = len(dec.seq)
        chain = [int(t) ^ (1 if i == at % 3 + 1 else 0) for i, t in enumerate(drafts[at:at + 3])]
        dec.round(list(range(-1, len(chain))), [0] + chain, lam)
    return dec


@pytest.mark.parametrize("paged", [False, True])
def test_rounds_over_4_bit_caches(paged):
    """One model as proxy and target: rounds that the proxy ends and rounds that the target ends run the same passes, so their tokens and
    their caches are the same byte for byte; and rounds without drafts are passes of one token with a commit after each."""
    shape = SHAPES["tiny_bf16"]
    model = device_model(shape, 3)
    prompt = [int(t) for t in gen_context_tokens(shape.vocab, 20, 3)]
    plain = rounds(model, prompt, 0.0, [], 40, paged)
    kv, ver = MXKVCache(model, 1, 256, paged=paged), Verifier(model, 1, 1)
    for t in (0, 1):
        kv.pools[t].copy_(plain.kv_p.pools[t]), kv.pools[t + 2].copy_(plain.kv_p.pools[t + 2])
    kv.set_len([len(prompt) - 1])
    seq = prompt[:]
    while len(seq) < len(plain.seq):
        i32 = dict(dtype=torch.int32, device="cuda")
        out = ver.verify(kv, torch.tensor([[seq[-1]]], **i32), np.array([[-1]]), torch.tensor([[len(seq) - 1]], **i32), 0.0)
        seq.append(int(out["token"][0]))
        kv.commit([[0]])
    assert seq == [int(t) for t in plain.seq]
    for a, b in zip(kv.pools, plain.kv_p.pools):
        assert torch.equal(a, b)
    proxy, both = (rounds(model, prompt, lam, seq, 40, paged) for lam in (0.0, 1.5))
    assert list(proxy.seq) == list(both.seq) and both.target_passes > 0 and proxy.target_passes == 0
    n = proxy.kv_p.ctx_len[0]
    assert both.kv_t.ctx_len[0] == both.kv_p.ctx_len[0] == n
    for mine in (both.kv_p, both.kv_t):
        assert torch.equal(mine.k[:, :, :, :n], proxy.kv_p.k[:, :, :, :n]) and torch.equal(mine.v[..., :n], proxy.kv_p.v[..., :n])
