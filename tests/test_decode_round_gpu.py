"""Decoding rounds as a serving program runs them: a small one-layer model whose blocks enter
the paged cache, attend to it, are verified against the output layer and committed."""
import numpy as np
import pytest
import torch

import paper_2608_03447_amd as asd
from oracle import decode

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
N, HQ, HKV, D, DM, V, PAGE, WIDTH = 3, 4, 2, 64, 256, 500, 8, 12


class Model:
    def __init__(self, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def make(*shape):
            return (torch.randn(shape, generator=gen) * shape[-1] ** -0.5).to(torch.bfloat16).to(DEV)

        self.embed, self.head = make(V, DM) * 16, make(V, DM) * 4
        self.qkv, self.out = make((HQ + 2 * HKV) * D, DM), make(DM, HQ * D)
        self.q_norm = torch.ones(D, dtype=torch.bfloat16, device=DEV)
        self.freq = (1e4 ** (-torch.arange(0, D, 2) / D)).float().to(DEV)

    def hidden(self, tokens, cache, cached, lens, mask=None, positions=None):
        """Final hidden states of the blocks' rows; their keys and values enter the cache."""
        x = self.embed[tokens.long()]
        q, k, v = (t.unflatten(1, (-1, D)) for t in
                   (x @ self.qkv.T).split([HQ * D, HKV * D, HKV * D], 1))
        q = asd.asd_rope_append(q, k, v, *cache, cached, lens, self.freq, q_norm=self.q_norm,
                                k_norm=self.q_norm, positions=positions)
        o = asd.asd_block_attention(q, *cache, cached, lens, mask=mask)
        return x + o.flatten(1) @ self.out.T


def new_cache(gen):
    pages = N * WIDTH
    table = torch.randperm(pages, generator=gen).to(torch.int32).reshape(N, WIDTH).to(DEV)
    k = torch.full((pages, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    return k, k.clone(), table


def test_rounds_with_drafts_commit_what_single_tokens_would():
    """Budget 0: the committed tokens are the greedy ones, however the drafts cut the sequence
    into blocks, and stale entries of rejected drafts are overwritten."""
    model, gen = Model(), torch.Generator().manual_seed(1)
    rng = np.random.default_rng(2)
    tokens = torch.zeros((N, 64), dtype=torch.int32, device=DEV)
    tokens[:, 0] = torch.tensor([5, 77, 400])
    seq_len = torch.ones(N, dtype=torch.int64, device=DEV)
    cache = new_cache(gen)
    budget = torch.zeros((N, 2), device=DEV)
    logits_of = {}
    for turn in range(8):
        lens = [int(x) for x in rng.integers(0, 5, N)]
        rows = []
        for i, k in enumerate(lens):
            last = int(tokens[i, int(seq_len[i]) - 1])
            rows += [last] + [int(x) for x in rng.integers(0, V, k)]
        # some drafts that are right: what a drafter that knows the model proposes
        block = torch.tensor(rows, dtype=torch.int32, device=DEV)
        k_lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        for _ in range(2):
            h = model.hidden(block, cache, seq_len - 1, k_lens)
            greedy = (h.float() @ model.head.float().T).argmax(1)
            at = 0
            for k in lens:
                if k:
                    block[at + 1] = greedy[at]
                at += k + 1
        # the verifier's drafts: row p holds draft p + 1
        draft = torch.zeros_like(block)
        at = 0
        for k in lens:
            draft[at:at + k] = block[at + 1:at + 1 + k]
            at += k + 1
        amax = torch.empty(len(rows), dtype=torch.int32, device=DEV)
        acc, nxt = asd.asd_lmhead_verify(h.contiguous(), model.head, draft, k_lens, 1.0, 1, budget,
                                         out_argmax=amax)
        before = seq_len.clone()
        asd.asd_commit(draft, k_lens, acc, nxt, tokens, seq_len)
        torch.cuda.synchronize()
        assert (seq_len > before).all()
        for i, k in enumerate(lens):
            assert int(acc[i]) >= (1 if k else 0)
    # the whole sequences again, in one block each: every committed token is the greedy one
    lens = [int(s) - 2 for s in seq_len]
    block = torch.cat([tokens[i, :int(s) - 1] for i, s in enumerate(seq_len)])
    again = new_cache(gen)
    h = model.hidden(block, again, torch.zeros_like(seq_len),
                     torch.tensor(lens, dtype=torch.int32, device=DEV))
    z = (h.float() @ model.head.float().T)
    at = 0
    for i, s in enumerate(seq_len.tolist()):
        for p in range(s - 1):
            # the greedy token, or one whose logit is within bfloat16's rounding of the hidden state
            chosen = z[at + p, int(tokens[i, p + 1])]
            assert z[at + p].max() - chosen <= 2.0 ** -5 * z[at + p].abs().max()
        at += s - 1


def test_a_tree_scores_each_branch_like_its_own_chain():
    model, gen = Model(3), torch.Generator().manual_seed(4)
    cached = torch.zeros(N, dtype=torch.int64, device=DEV)
    prompt = torch.randint(V, (N * 20,), generator=gen).to(torch.int32).to(DEV)
    cache = new_cache(gen)
    model.hidden(prompt, cache, cached, torch.full((N,), 19, dtype=torch.int32, device=DEV))
    cached += 20
    # 0 -> 1 -> 3, 0 -> 2 -> 4 in every request
    nodes = torch.randint(V, (N, 5), generator=gen).to(torch.int32).to(DEV)
    seen = torch.tensor([[1], [3], [5], [11], [21]], dtype=torch.int64, device=DEV).repeat(N, 1)
    depth = torch.tensor([0, 1, 1, 2, 2], device=DEV)
    tree = model.hidden(nodes.flatten(), cache, cached, torch.full((N,), 4, dtype=torch.int32,
                                                                   device=DEV), seen,
                        (cached[:, None] + depth).flatten().contiguous()).reshape(N, 5, DM)
    for path in ([0, 1, 3], [0, 2, 4]):
        chain = model.hidden(nodes[:, path].flatten().contiguous(), cache, cached,
                             torch.full((N,), 2, dtype=torch.int32, device=DEV)).reshape(N, 3, DM)
        # both round the same numbers, in another order of summation: bfloat16 steps of the sums
        assert ((tree[:, path] - chain).float().abs().max() <=
                2.0 ** -6 * chain.float().abs().max())


def test_sampled_proposals_and_rounds_in_a_graph():
    """A drafter's loop under capture: append, attend, sample, the token goes back in."""
    model, gen = Model(5), torch.Generator().manual_seed(6)
    cache = new_cache(gen)
    token = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    cached = torch.zeros(N, dtype=torch.int64, device=DEV)
    zero = torch.zeros(N, dtype=torch.int32, device=DEV)
    u = torch.zeros(N, device=DEV)
    ks = torch.full((N,), 40, dtype=torch.int32, device=DEV)
    logits = torch.empty((N, V), device=DEV)
    out = torch.empty_like(token)

    def step():
        h = model.hidden(token, cache, cached, zero)
        logits.copy_((h @ model.head.T).float())
        asd.asd_sample(logits, u, top_k=ks, out_token=out)
        token.copy_(out)
        cached.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    token.copy_(torch.tensor([1, 2, 3]))
    cached.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for turn in range(6):
        before = (token.clone(), cached.clone())
        u.copy_(torch.rand(N, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        got, z = token.clone(), logits.cpu().numpy()
        for r in range(N):
            assert int(got[r]) == decode.sample_row(z[r], float(u[r]), k=40)[0]
        # the same step, eager, from the same state
        token.copy_(before[0])
        cached.copy_(before[1])
        step()
        torch.cuda.synchronize()
        assert torch.equal(token, got) and torch.equal(cached, before[1] + 1)
