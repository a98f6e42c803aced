"""The operators between two steps as a program runs them, step after step
(GPU): a decode loop that evicts tokens, and a beam search whose beams share
pages, each against the oracle from the tokens' own keys and values."""

import types

import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import assert_parity
from oracle import upkeep
from paper_2509_02121_amd import halo
from test_gpu_step import _rope_reference
from test_step import rope_frequencies
from upkeep_helpers import BF16, F32, cuda, params, to_numpy, values

pytestmark = pytest.mark.gpu
PAGE, H, HQ, D = 16, 2, 8, 64
U = 2.0 ** -24


class Cache:
    """Pools of bf16 keys and values, NaN at first, and a free list of their pages."""

    def __init__(self, rows, width, pages, seed):
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator().manual_seed(seed)
        self.params = params(HQ, H, D, BF16, pages)
        self.k = torch.full((pages, H, PAGE * D), float("nan"), dtype=BF16, device="cuda")
        self.v = torch.full((pages, H, PAGE * D), float("nan"), dtype=BF16, device="cuda")
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        self.free = cuda(self.rng.permutation(pages))
        self.free_next = cuda([0])
        self.flag = cuda([0])
        self.scale = float(np.float32(D ** -0.5))

    def random(self, *shape):
        return torch.randn(shape, generator=self.gen).to(BF16)

    def append(self, seq_len, seq_new, k=None, v=None, table=None):
        """New tokens for the rows of a table, their pages from the free list; returns the StepTables."""
        table = self.table if table is None else table
        n = len(seq_len)
        total = int(seq_new.sum())
        steps = halo.StepTables(n, max(total, 1), n * table.shape[1])
        halo.kv_step_tables(steps, seq_len, seq_new, table, self.free, self.free_next, self.flag)
        if k is not None:
            halo.kv_page_scatter_kv(self.k, self.v, self.params, steps.page_ids, steps.seq_page_indptr, steps.seq_start,
                                    steps.seq_count, steps.in_token_offset, k, v, self.flag)
        self.free_next = steps.free_next.clone()
        return steps

    def lists(self, table, lengths):
        return [table[i, :upkeep.pages_of(int(n))].tolist() for i, n in enumerate(lengths)]

    def attend(self, q, lists, lengths):
        """Attention of a row each over page lists: (o, lse)."""
        forest = dict(seg_len=np.asarray(lengths), seg_page_indptr=np.cumsum([0] + [len(x) for x in lists]),
                      seg_page_ids=np.concatenate(lists), req_seg_indptr=np.arange(len(lists) + 1),
                      req_seg_ids=np.arange(len(lists)))
        return halo.PrefixAttention(self.params, forest).run(q, self.k, self.v)

    def check_attention(self, o, lse, q, keys, vals, label):
        n = len(keys)
        want = oracle.decode(q.double().cpu().numpy(), dict(enumerate(keys)), dict(enumerate(vals)),
                             [[i] for i in range(n)], self.scale)
        assert_parity(types.SimpleNamespace(dtype=BF16), o.double().cpu().numpy(), lse.double().cpu().numpy(), *want,
                      np.arange(n), label)

    def tokens(self, lists, lengths):
        """Keys and values [tokens, H, D] that the pools hold for each list."""
        host = [values(to_numpy(x), z, D, False) for z, x in enumerate((self.k, self.v))]
        return [[x[p].reshape(-1, H, D)[:n] for p, n in zip(lists, lengths)] for x in host]

    def pages_are_whole(self, lists):
        """Every page is in the free list's rest or in a list, and in one of the two."""
        used = {int(p) for x in lists for p in x}
        rest = self.free[int(self.free_next):].tolist()
        assert len(rest) == len(set(rest)) and not used & set(rest) and len(used) + len(rest) == len(self.free)
        assert int(self.flag) == 0


def test_decode_loop_that_evicts(gpu_lib):
    """Prompts, then steps of one token a sequence: tables, scatter, attention, weights, and every step the choice,
    the move and the pages given back, all without a look from the host but for the checks."""
    prompts = [70, 12, 48, 33, 1]
    n, budget, trigger, sinks, recent, decay = len(prompts), 40, 44, 2, 8, 0.9
    c = Cache(n, 6, 64, 21)
    keys, vals = [[x.double().numpy() for x in (c.random(p, H, D) for p in prompts)] for _ in range(2)]
    lengths = cuda([0] * n)
    steps = c.append(lengths, cuda(prompts), *[torch.from_numpy(np.concatenate(x)).to(BF16).cuda() for x in (keys, vals)])
    lengths = steps.seq_end.clone()
    width = c.table.shape[1] * PAGE
    weights = torch.zeros((n, H, width), device="cuda")
    kept = torch.full((n, H, budget), -1, dtype=torch.int32, device="cuda")
    new_len = cuda([0] * n)
    evicted = 0
    for step in range(14):
        new = [c.random(n, H, D) for _ in range(2)]
        start = lengths
        steps = c.append(lengths, cuda([1] * n), *[x.cuda() for x in new])
        lengths = steps.seq_end.clone()
        for x, y in zip((keys, vals), new):
            for i in range(n):
                x[i] = np.concatenate([x[i], y[i:i + 1].double().numpy()])
        host = lengths.tolist()
        assert host == [len(x) for x in keys]
        q = c.random(n, HQ, D).cuda()
        o, lse = c.attend(q, c.lists(c.table, host), host)
        c.check_attention(o, lse, q, keys, vals, f"step {step}")
        before = weights.double().cpu().numpy()
        halo.kv_page_weights(weights, c.k, c.params, steps.page_ids, steps.seq_page_indptr, start, lengths, q, lse,
                             decay=decay, error_flag=c.flag)
        after = weights.double().cpu().numpy()
        for i in range(n):
            want, products, sizes = upkeep.weights(keys[i], q[i:i + 1].double().cpu().numpy(),
                                                   lse[i:i + 1].double().cpu().numpy(), [host[i]], c.scale, before[i],
                                                   int(start[i]), float(np.float32(decay)))
            # (two sums of D products and the scale; score and lse in fp32; the exponential; the sums of HQ / H rows)
            bound = 2 * (D + 2) * U * products + 4 * U * sizes + (2.0 ** -21 + (HQ // H + 4) * U) * want
            assert (np.abs(after[i, :, :host[i]] - want) <= bound).all(), f"step {step}, sequence {i}"
        halo.kv_evict_select(weights, lengths, kept, new_len, trigger, sinks, recent, error_flag=c.flag)
        halo.kv_page_keep_kv(c.k, c.v, c.params, steps.page_ids, steps.seq_page_indptr, lengths, new_len, kept,
                             error_flag=c.flag)
        free, free_next = torch.empty_like(c.free), torch.empty_like(c.free_next)
        halo.kv_release_pages(c.table, lengths, new_len, c.free, c.free_next, free, free_next, c.flag)
        c.free, c.free_next, lengths = free, free_next, new_len.clone()
        for i in range(n):
            for h in range(H):
                stay = upkeep.evict(after[i, h], host[i], budget, trigger, sinks, recent)
                if stay is None:
                    continue
                assert kept[i, h].tolist() == stay and torch.equal(weights[i, h, :budget].double().cpu(),
                                                                   torch.from_numpy(after[i, h, stay]))
                for x in (keys, vals):
                    x[i][:budget, h] = x[i][stay, h]
            if host[i] > trigger:
                evicted += 1
                keys[i], vals[i] = keys[i][:budget], vals[i][:budget]
        now = lengths.tolist()
        assert now == [len(x) for x in keys]
        lists = c.lists(c.table, now)
        c.pages_are_whole(lists)
        for x, y in zip(c.tokens(lists, now), (keys, vals)):
            assert all(np.array_equal(a, b) for a, b in zip(x, y))
    assert evicted > n


def test_decode_loop_that_evicts_with_rotary_positions(gpu_lib):
    """Kept keys stay turned by the positions that they came with, so a new token's position is its place in the cache,
    which the step tables give, and the tokens that its sequence has lost; counted on the GPU."""
    prompts = [70, 12, 48, 33, 1]
    n, budget, trigger, sinks, recent = len(prompts), 40, 44, 2, 8
    c = Cache(n, 6, 64, 24)
    rope, (w, _) = halo.Rope(D), rope_frequencies(D, 10000.0, "none", 1.0, 8192, 32, 1)
    keys, vals = [[np.zeros((0, H, D))] * n for _ in range(2)]
    lengths, lost = cuda([0] * n), cuda([0] * n)
    weights = torch.zeros((n, H, c.table.shape[1] * PAGE), device="cuda")
    kept = torch.full((n, H, budget), -1, dtype=torch.int32, device="cuda")
    new_len = cuda([0] * n)
    came = [0] * n                    # tokens that each sequence has had
    apart = 0
    for step in range(14):
        counts = [1] * n if step else prompts
        q, k, v = (c.random(sum(counts), heads, D).cuda() for heads in (HQ, H, H))
        start = lengths
        steps = c.append(lengths, cuda(counts))
        lengths = steps.seq_end.clone()
        positions = steps.positions[:sum(counts)] + torch.repeat_interleave(lost, cuda(counts), output_size=sum(counts))
        true = torch.tensor([t for i in range(n) for t in range(came[i], came[i] + counts[i])], dtype=torch.int32)
        assert torch.equal(positions.cpu(), true)
        apart += int((steps.positions[:sum(counts)].cpu() != true).sum())
        wanted = [_rope_reference(x, true, w, 1.0, False) for x in (q, k)]
        halo.rope_qk(q, k, positions, rope)
        for x, (want, tol) in zip((q, k), wanted):
            assert ((x.double().cpu() - want).abs() <= tol).all()
        halo.kv_page_scatter_kv(c.k, c.v, c.params, steps.page_ids, steps.seq_page_indptr, steps.seq_start,
                                steps.seq_count, steps.in_token_offset, k, v, c.flag)
        first = np.cumsum([0] + counts)
        for x, y in zip((keys, vals), (k, v)):
            for i in range(n):
                x[i] = np.concatenate([x[i], y[first[i]:first[i + 1]].double().cpu().numpy()])
        came = [a + b for a, b in zip(came, counts)]
        host = lengths.tolist()
        q = q[first[1:] - 1].contiguous()             # each sequence's last query
        o, lse = c.attend(q, c.lists(c.table, host), host)
        c.check_attention(o, lse, q, keys, vals, f"step {step}")
        halo.kv_page_weights(weights, c.k, c.params, steps.page_ids, steps.seq_page_indptr, start, lengths, q, lse,
                             decay=0.9, error_flag=c.flag)
        before = weights.double().cpu().numpy()
        halo.kv_evict_select(weights, lengths, kept, new_len, trigger, sinks, recent, error_flag=c.flag)
        halo.kv_page_keep_kv(c.k, c.v, c.params, steps.page_ids, steps.seq_page_indptr, lengths, new_len, kept,
                             error_flag=c.flag)
        free, free_next = torch.empty_like(c.free), torch.empty_like(c.free_next)
        halo.kv_release_pages(c.table, lengths, new_len, c.free, c.free_next, free, free_next, c.flag)
        lost += lengths - new_len
        c.free, c.free_next, lengths = free, free_next, new_len.clone()
        for i in range(n):
            for h in range(H):
                stay = upkeep.evict(before[i, h], host[i], budget, trigger, sinks, recent)
                if stay is not None:
                    for x in (keys, vals):
                        x[i][:budget, h] = x[i][stay, h]
            if host[i] > trigger:
                keys[i], vals[i] = keys[i][:budget], vals[i][:budget]
        c.pages_are_whole(c.lists(c.table, lengths.tolist()))
    assert apart > n and [a - b for a, b in zip(came, lengths.tolist())] == lost.tolist()


def test_beam_search_that_shares_pages(gpu_lib):
    """Requests of several beams: the first step from one beam, then selection, the tables of the children, copies of
    the pages that they split, and once the tokens of every beam cut down into pages of its own."""
    items, beams, vocab, width = 3, 4, 301, 8
    rows, end = items * beams, 7
    prompts = [40, 16, 5]
    c = Cache(rows, width, 120, 22)
    tok = [torch.randn((vocab, H, D), generator=c.gen).to(BF16) for _ in range(2)]
    history = [[] for _ in range(rows)]     # each row's tokens as pairs of (token, K and V [H, D])

    def entry(t):
        x = [y[t] + c.random(H, D) for y in tok]
        return [y.to(BF16) for y in x]

    for i, p in enumerate(prompts):
        history[i * beams] = [entry(t) for t in c.rng.integers(0, vocab, p)]
    counts = [len(h) for h in history]
    flat = [e for h in history for e in h]
    steps = c.append(cuda([0] * rows), cuda(counts), *[torch.stack([e[z] for e in flat]).cuda() for z in range(2)])
    lengths = steps.seq_end.clone()
    scores = cuda([[0.0] + [-np.inf] * (beams - 1)] * items, F32).view(-1)
    ended = cuda([0] * rows)
    select = halo.BeamSelect(items, beams, vocab)
    tables = [halo.BeamTables(items, beams, width, len(c.free)) for _ in range(2)]
    shared = split = 0
    for step in range(24):
        # logits that make beams cross over often
        logits = (torch.randn((rows, vocab), generator=c.gen) * 2).to(BF16).cuda()
        halo.beam_select(select, logits, scores, ended, end)
        got = [x.cpu().numpy() for x in (select.scores, select.tokens, select.parents)]
        for i in range(items):
            at = slice(i * beams, (i + 1) * beams)
            s, t, p = upkeep.select(logits[at].double().cpu().numpy(), scores[at].double().cpu().numpy(),
                                    ended[at].cpu().numpy(), end, beams)
            # (the sums of `vocab` exponentials, and score, logit and their sum in fp32)
            assert np.allclose(got[0][i], s, rtol=0, atol=(vocab + 8) * U * (1 + np.abs(s).max()))
            assert got[1][i].tolist() == t and got[2][i].tolist() == p
        scores = select.scores.view(-1).clone()
        out = tables[step % 2]
        old = c.table.cpu().numpy(), lengths.tolist(), c.free.tolist(), int(c.free_next)
        halo.kv_beam_tables(out, select.parents, lengths, c.table, c.free, c.free_next, c.flag)
        want = upkeep.beam_tables(items, beams, got[2], old[1], old[0], old[2], old[3])
        assert out.copy_src.tolist() == want[4] and out.copy_dst.tolist() == want[5]
        assert out.seq_len.tolist() == want[1] and int(out.free_next) == want[3]
        assert out.free_pages[want[3]:].tolist() == want[2][want[3]:]
        for pool in (c.k, c.v):
            halo.kv_page_copy(pool, c.params, out.copy_src, out.copy_dst)
        c.table, lengths = out.block_table, out.seq_len
        c.free, c.free_next = out.free_pages, out.free_next
        history = [list(history[i * beams + p]) for i in range(items) for p in got[2][i]]
        split += int((out.copy_src >= 0).sum())
        # a beam that was ended keeps its tokens, the others have one more
        was = ended.view(items, beams)
        stopped = torch.gather(was, 1, select.parents.long()).view(-1)
        ended = (stopped.bool() | (select.tokens.view(-1) == end)).int()
        new = (1 - stopped).tolist()
        fresh = [entry(int(t)) for t in select.tokens.view(-1).tolist()]
        for r in range(rows):
            if new[r]:
                history[r].append(fresh[r])
        flat = [f for f, m in zip(fresh, new) if m]
        steps = c.append(lengths, cuda(new), *[torch.stack([e[z] for e in flat]).cuda() for z in range(2)])
        lengths = steps.seq_end.clone()
        host = lengths.tolist()
        assert host == [len(h) for h in history]
        lists = c.lists(c.table, host)
        c.pages_are_whole(lists)
        shared += sum(len(x) for x in lists) - len({p for x in lists for p in x})
        keys, vals = [[torch.stack([e[z] for e in h]).double().numpy() for h in history] for z in range(2)]
        for x, y in zip(c.tokens(lists, host), (keys, vals)):
            assert all(np.array_equal(a, b) for a, b in zip(x, y)), f"step {step}"
        q = c.random(rows, HQ, D).cuda()
        o, lse = c.attend(q, lists, host)
        c.check_attention(o, lse, q, keys, vals, f"step {step}")
        if step != 15:
            continue
        # every beam's tokens cut down: chosen by this step's weights, moved to pages of its own, the shared ones back
        budget = 24
        weights = torch.zeros((rows, H, width * PAGE), device="cuda")
        halo.kv_page_weights(None, c.k, c.params, steps.page_ids, steps.seq_page_indptr, None, lengths, q, lse, decay=0.0,
                             weights_out=weights, error_flag=c.flag)
        kept = torch.zeros((rows, H, budget), dtype=torch.int32, device="cuda")
        new_len = cuda([0] * rows)
        halo.kv_evict_select(weights, lengths, kept, new_len, sinks=1, recent=4, error_flag=c.flag)
        table = torch.full_like(c.table, -1)
        own = c.append(cuda([0] * rows), new_len, table=table)
        halo.kv_page_keep_kv(c.k, c.v, c.params, steps.page_ids, steps.seq_page_indptr, lengths, new_len, kept,
                             own.page_ids, own.seq_page_indptr, c.flag)
        gone = halo.BeamTables(items, beams, width, len(c.free))
        halo.kv_beam_tables(gone, cuda([[-1] * beams] * items), lengths, c.table, c.free, c.free_next, c.flag)
        c.table, c.free, c.free_next, lengths = table, gone.free_pages, gone.free_next, new_len
        host = new_len.tolist()
        c.pages_are_whole(c.lists(c.table, host))
        for r in range(rows):
            if len(history[r]) > budget:
                which = kept[r].tolist()
                history[r] = [[torch.stack([history[r][which[h][j]][z][h] for h in range(H)]) for z in range(2)]
                              for j in range(budget)]
        assert host == [len(h) for h in history] and max(host) == budget
    assert shared > 100 and split > 20
