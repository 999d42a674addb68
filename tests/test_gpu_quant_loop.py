"""Decoding iterations over a target cache in 8 bits, as a program makes them: the prompt is written, every layer attends the draft
tree to the cache, logits become the wanted tokens, the accepted rows are committed, chunks are ranked for the draft model.  Each step
against 64 bits from what the step before left; the cache itself is compared exactly."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
import quant_util as qu
from parity_util import check_selection

pytestmark = pytest.mark.gpu


class _Target:
    """Seeded rows in place of a model: queries, keys and values of any tree, logits from the attention's output."""

    def __init__(self, layers, hq, hkv, d, vocab, seed):
        self.rng = np.random.default_rng(seed)
        self.layers, self.hq, self.hkv, self.d, self.vocab = layers, hq, hkv, d, vocab
        self.head = torch.from_numpy(self.rng.standard_normal((hq * d, vocab)).astype(np.float32)).cuda()

    def rows(self, *shape):
        return torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32)).bfloat16()

    def logits(self, out):
        return (out.reshape(out.shape[0], -1).float() @ self.head * 4).bfloat16()


@pytest.mark.parametrize("layers,hq,hkv,d,block,chunk,prompt,iterations", [(2, 8, 2, 128, 32, 32, 201, 4), (1, 6, 3, 64, 64, 96, 310, 3), (2, 4, 1, 128, 128, 64, 130, 4)])
def test_iterations(layers, hq, hkv, d, block, chunk, prompt, iterations):
    import paper_2505_20776_amd as sx
    model = _Target(layers, hq, hkv, d, 5000, prompt)
    t, cap = 24, prompt + 24 * iterations
    nb = -(-cap // block)
    codes = [torch.zeros((layers, hkv, cap, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((layers, hkv, nb), device="cuda") for _ in range(2)]
    ref = [qu.Cache(layers, hkv, cap, d, block) for _ in range(2)]
    first = [model.rows(layers, hkv, prompt, d) for _ in range(2)]
    sx.quant_kv_write(first[0].cuda(), first[1].cuda(), *codes, *scales, layers, hkv, d, prompt, 0, cap, block)
    for r, x in zip(ref, first):
        r.write(x.double().numpy(), 0)
    n = prompt
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    draft, path, n_accept, next_token = (torch.zeros(m, dtype=torch.int32, device="cuda") for m in (t, t, 1, 1))
    lse = torch.empty((hq, t), device="cuda")
    top = torch.empty((t, 1), dtype=torch.int32, device="cuda")
    row_lse, entropy, child = torch.empty(t, device="cuda"), torch.empty(t, device="cuda"), torch.empty((t, 1), device="cuda")
    ws_lp = torch.empty(sx.token_logprobs_bytes(t, model.vocab, 1), dtype=torch.uint8, device="cuda")
    for it in range(iterations):
        parent = np.array([-1] + [i - 1 if i % 3 else max(0, i - 4) for i in range(1, t)], dtype=np.int32)
        q = model.rows(layers, t, hq, d)
        tree = [model.rows(layers, hkv, t, d) for _ in range(2)]
        q_dev, tree_dev, parent_dev = q.cuda(), [x.cuda() for x in tree], torch.from_numpy(parent).cuda()
        common = dict(dtype=sx.SPECEXT_BF16, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, prefix_len=n, n_tree=t, kp_stride_h=cap * d, flags=block)
        desc, scored = sx.make_desc(**common), sx.make_desc(chunk_size=chunk, want_scores=True, **common)
        ws = torch.empty(max(sx.workspace_bytes(desc), sx.workspace_bytes(scored)), dtype=torch.uint8, device="cuda")
        out = torch.empty((layers, t, hq, d), dtype=torch.bfloat16, device="cuda")
        for y in range(layers):
            sx.verify_attn_quant(scored if y == layers - 1 else desc, q_dev[y], codes[0][y], codes[1][y], scales[0][y], scales[1][y],
                                 tree_dev[0][y], tree_dev[1][y], parent_dev, out[y], lse, ws, scale_stride_h=nb)
        logits = model.logits(out[-1])
        # the draft model is good at some nodes: their tokens are the target's, known from the same logits
        wanted = logits.float().argmax(dim=1).cpu().numpy()
        tokens = np.arange(t, dtype=np.int32) + 1
        for i in range(1, t):
            if i % 5 != 4:
                tokens[i] = wanted[parent[i]]
        draft.copy_(torch.from_numpy(tokens))
        sx.token_logprobs(logits, t, model.vocab, ws_lp, tokens=draft, n_given=1, logprob=child, k=1, top_id=top, lse=row_lse, entropy=entropy)
        sx.accept_greedy(parent_dev, draft, top, ints([int(tokens[0])]), t, path, n_accept, next_token)
        sx.commit_tree_quant(*tree_dev, *codes, *scales, path, n_accept, t, t, layers, hkv, d, n, cap, block)
        n_chunks = -(-n // chunk)
        scores, idx, n_idx = torch.empty(n_chunks, device="cuda"), ints([0] * 4), ints([0])
        sx.chunk_scores_select(scored, ws, 0, 4, idx, n_idx, scores=scores, path=path, n_accept=n_accept)
        torch.cuda.synchronize()

        # ---- the same in 64 bits
        lp = torch.log_softmax(logits.double().cpu(), dim=1)
        ids = torch.sort(logits.float().cpu(), dim=1, descending=True, stable=True).indices[:, 0]
        assert torch.equal(top[:, 0].cpu().long(), ids)
        assert (child[:, 0].cpu().double() - lp.gather(1, draft.cpu().long()[:, None])[:, 0]).abs().max() <= 2.0 ** -17
        assert ((row_lse.cpu().double() - torch.logsumexp(logits.double().cpu(), 1)).abs() <= 2.0 ** -17 + 2.0 ** -23 * row_lse.cpu().abs()).all()
        want_path, want_next = orc.accept_greedy(parent, tokens, ids.numpy(), int(tokens[0]))
        assert path.cpu().numpy()[:int(n_accept)].tolist() == want_path and int(next_token) == want_next and len(want_path) >= 2
        for y in range(layers):
            k, v = (torch.from_numpy(r.values[y, :, :n]) for r in ref)
            o, ref_lse, mag, spread, sc = qu.attention(q[y].double(), k, v, tree[0][y].double(), tree[1][y].double(), parent, 1 / math.sqrt(d), chunk)
            tol = (2.0 ** -10 + n * 2.0 ** -24 + 2.0 ** -15 * spread.T)[:, :, None] * mag[:, :, None] + 2.0 ** -8 * o.abs()
            assert ((out[y].cpu().double() - o).abs() <= tol).all()
        last = want_path[-1]
        assert (scores.cpu().double() - sc[last]).abs().max() <= 1e-4 * sc[last].max()
        check_selection(idx.cpu().numpy()[:int(n_idx)], sc[last].numpy(), 4, "chunks")
        for r, x, c, s in zip(ref, tree, codes, scales):
            r.append(x.double().numpy(), n, want_path)
            now = n + len(want_path)
            blocks = -(-now // block)
            assert torch.equal(s.cpu().double()[:, :, :blocks], torch.from_numpy(r.scale[:, :, :blocks]))
            got = c.cpu().view(torch.float8_e4m3fn).double()[:, :, :now] * s.cpu().double().repeat_interleave(block, 2)[:, :, :now, None]
            assert torch.equal(got, torch.from_numpy(r.values[:, :, :now]))
        n += len(want_path)


def test_a_step_in_one_graph():
    """Attention, logits, acceptance, commit and ranking captured once; every replay gives the eager results, with eager work between.
    (A commit at the same place writes the same bytes again.)"""
    import paper_2505_20776_amd as sx
    model = _Target(1, 8, 2, 128, 40000, 5)
    n, t, block, cap, d = 500, 20, 32, 600, 128
    codes = [torch.zeros((1, 2, cap, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros((1, 2, -(-cap // block)), device="cuda") for _ in range(2)]
    rows = [model.rows(1, 2, n, d).cuda() for _ in range(2)]
    sx.quant_kv_write(*rows, *codes, *scales, 1, 2, d, n, 0, cap, block)
    q, kt, vt = model.rows(t, 8, d).cuda(), model.rows(1, 2, t, d).cuda() * 3, model.rows(1, 2, t, d).cuda() * 3
    parent = torch.arange(-1, t - 1, dtype=torch.int32, device="cuda")
    desc = sx.make_desc(dtype=sx.SPECEXT_BF16, n_q_heads=8, n_kv_heads=2, head_dim=d, prefix_len=n, n_tree=t, kp_stride_h=cap * d, flags=block,
                        chunk_size=32, want_scores=True)
    ws = torch.empty(sx.workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    ws_lp = torch.empty(sx.token_logprobs_bytes(t, 40000, 1), dtype=torch.uint8, device="cuda")
    logits = torch.randn((t, 40000), device="cuda").bfloat16()
    out, lse = torch.empty((t, 8, d), dtype=torch.bfloat16, device="cuda"), torch.empty((8, t), device="cuda")
    draft = torch.cat([torch.zeros(1, device="cuda"), logits.float().argmax(1)[:-1].float()]).int()
    draft[12] = 39999
    top, path, scores = torch.zeros((t, 1), dtype=torch.int32, device="cuda"), torch.zeros(t, dtype=torch.int32, device="cuda"), torch.zeros(16, device="cuda")
    one = lambda: torch.zeros(1, dtype=torch.int32, device="cuda")  # noqa: E731
    n_accept, next_token, idx, n_idx, first = one(), one(), torch.zeros(4, dtype=torch.int32, device="cuda"), one(), one()

    def step():
        sx.verify_attn_quant(desc, q, *codes, *scales, kt, vt, parent, out, lse, ws, scale_stride_h=scales[0].shape[2])
        sx.token_logprobs(logits, t, 40000, ws_lp, k=1, top_id=top)
        sx.accept_greedy(parent, draft, top, first, t, path, n_accept, next_token)
        sx.commit_tree_quant(kt, vt, *codes, *scales, path, n_accept, t, t, 1, 2, d, n, cap, block)
        sx.chunk_scores_select(desc, ws, 0, 4, idx, n_idx, scores=scores, path=path, n_accept=n_accept)

    results = (out, lse, top, path, n_accept, next_token, idx, scores, *codes, *scales)
    step()
    # (the commit may move the codes of the block that it enters under a larger scale; the next attention reads those)
    step()
    torch.cuda.synchronize()
    assert int(n_accept) == 12
    eager = [x.clone() for x in results]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        for x in results[:8]:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, eager))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, eager))
