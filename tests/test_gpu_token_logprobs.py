"""Log probabilities, entropy and top tokens of logits against 64 bits.

Tolerances.  x - m is exact to 2^-24 |x - m|, so a term e^(x - m) to 2^-23 |x - m| + 2^-22; the terms that matter have |x - m| < 20,
and their sum's own roundings are below 2^-20.  lse, and with it a log probability, is m (exact) plus the log of such a sum: 2^-18, and
its rounding to fp32, 2^-24 of it.  The entropy is a mean of |x - m| under the same weights: 2^-17 (1 + its size)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _reference(x, tokens, k):
    """x [rows, vocab] float64 CPU."""
    top = x.amax(dim=1)
    empty = torch.isneginf(top)
    shifted = x - torch.where(empty, torch.zeros_like(top), top)[:, None]       # rows of -1e38: their logarithms are lost beside x
    log_z = torch.logsumexp(shifted, dim=1)
    lse = top + torch.where(empty, torch.zeros_like(top), log_z)
    lp = shifted - torch.where(empty, torch.zeros_like(top), log_z)[:, None]
    p = torch.exp(lp)
    entropy = -(torch.where(p > 0, p * lp, torch.zeros_like(p))).sum(dim=1)
    entropy[empty] = 0
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
    given = None
    if tokens is not None:
        ok = (tokens >= 0) & (tokens < x.shape[1])
        given = torch.where(ok, lp.gather(1, tokens.clamp(0, x.shape[1] - 1).long()), torch.full((1,), -math.inf, dtype=torch.float64))
    return lse, entropy, ids, lp.gather(1, ids), given


def _close(a, b, tol):
    same = (a == b) | (torch.isnan(a) & torch.isnan(b))
    return bool((same | ((a - b).abs() <= tol)).all())


def _run(logits, vocab, k=0, tokens=None, scale=0.0, stream=None, row_stride=None):
    import paper_2505_20776_amd as sx
    from paper_2505_20776_amd import harness as hx
    rows = logits.shape[0]
    made = {"ws": hx.guarded((sx.token_logprobs_bytes(rows, vocab, k),), torch.uint8), "lse": hx.guarded((rows,), torch.float32),
            "entropy": hx.guarded((rows,), torch.float32), "id": hx.guarded((rows, k), torch.int32), "lp": hx.guarded((rows, k), torch.float32),
            "given": hx.guarded((rows, tokens.shape[1] if tokens is not None else 0), torch.float32)}
    t = {n: v[0] for n, v in made.items()}
    sx.token_logprobs(logits, rows, vocab, t["ws"], dtype=sx.SPECEXT_BF16 if logits.dtype == torch.bfloat16 else sx.SPECEXT_F32,
                      row_stride=logits.stride(0) if row_stride is None else row_stride, logit_scale=scale,
                      tokens=None if tokens is None else tokens.cuda(), n_given=0 if tokens is None else tokens.shape[1], logprob=t["given"],
                      k=k, top_id=t["id"], top_logprob=t["lp"], lse=t["lse"], entropy=t["entropy"], stream=stream)
    torch.cuda.synchronize()
    for name, (_, base) in made.items():
        assert hx.guards_intact(base), name
    return {n: v.cpu() for n, v in t.items()}


def _check(x, k=0, tokens=None, scale=0.0, logits=None, **kw):
    """x [rows, vocab] as the kernel reads it, on the CPU; logits: the device tensor, if laid out otherwise."""
    got = _run(x.cuda() if logits is None else logits, x.shape[1], k, tokens, scale, **kw)
    ref = x.float()
    if scale:
        ref = ref * torch.tensor(scale, dtype=torch.float32)
    lse, entropy, ids, lp, given = _reference(ref.double(), tokens, k)
    tol = 2.0 ** -18 + 2.0 ** -23 * lse.abs().nan_to_num(0, 0, 0)
    assert _close(got["lse"].double(), lse, tol)
    assert _close(got["entropy"].double(), entropy, 2.0 ** -17 * (1 + entropy))
    assert torch.equal(got["id"].long(), ids)
    far = lambda v: tol[:, None] + 2.0 ** -23 * v.abs().nan_to_num(0, 0, 0)  # noqa: E731
    assert _close(got["lp"].double(), lp, far(lp))
    if tokens is not None:
        assert _close(got["given"].double(), given, far(given))


def _logits(seed, rows, vocab, dtype, sharp=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, vocab)) * sharp
    x[np.arange(rows), rng.integers(0, vocab, rows)] += 10
    return torch.from_numpy(x.astype(np.float32)).to(dtype), rng


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,k,given", [
    (1, 1, 1, 1), (3, 2, 2, 1), (2, 7, 7, 3), (5, 8, 1, 0), (1, 63, 63, 2), (4, 64, 64, 1), (2, 500, 32, 2), (3, 4089, 64, 1), (2, 4096, 5, 1),
    (2, 4097, 1, 1), (1, 8191, 16, 1), (60, 32000, 1, 4), (1, 32761, 4, 1), (2, 32762, 4, 1), (3, 32768, 4, 1), (2, 50257, 10, 2), (4, 65537, 2, 1),
    (7, 128256, 8, 1), (1, 262147, 64, 1), (1, 1 << 20, 3, 1)])
def test_sizes(dtype, rows, vocab, k, given):
    print(f"[case] {dtype} rows={rows} vocab={vocab} k={k}", flush=True)
    x, rng = _logits(rows + vocab, rows, vocab, dtype)
    tokens = torch.from_numpy(rng.integers(0, vocab, (rows, given)).astype(np.int32)) if given else None
    _check(x, k, tokens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,stride_more", [(0, 1), (1, 0), (3, 5), (7, 8), (2, 3)])
def test_rows_at_any_address(dtype, offset, stride_more):
    """Rows that begin anywhere between two multiples of 16 bytes, NaN between them."""
    rows, vocab = 9, 5001
    x, rng = _logits(offset, rows, vocab, dtype)
    ld = vocab + stride_more
    flat = torch.full((offset + rows * ld + 64,), math.nan, dtype=dtype, device="cuda")
    view = flat[offset:offset + rows * ld].view(rows, ld)[:, :vocab]
    view.copy_(x)
    tokens = torch.from_numpy(rng.integers(-2, vocab + 2, (rows, 3)).astype(np.int32))
    tokens[0] = torch.tensor([0, vocab - 1, vocab])
    _check(x, 6, tokens, logits=view)


@pytest.mark.parametrize("scale", [0.5, 1.0, 3.0, 1e-6])
def test_temperature(scale):
    x, rng = _logits(3, 6, 33000, torch.float32)
    _check(x, 5, torch.from_numpy(rng.integers(0, 33000, (6, 2)).astype(np.int32)), scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [300, 32768, 70001])
def test_banned_and_equal(dtype, vocab):
    """Rows with few tokens left, with none, all equal, of two values, with the lowest finite value, both zeros."""
    inf = math.inf
    x = torch.full((9, vocab), -inf)
    x[1, vocab // 2] = 3.0
    x[2, [5, vocab - 1, 17]] = torch.tensor([1.0, 1.0, -2.0])
    x[3] = 0.25
    x[4] = torch.finfo(dtype).min
    x[5] = torch.finfo(dtype).min
    x[5, 7] = 0.0
    x[6] = torch.where(torch.arange(vocab) % 3 == 0, 2.0, 1.0)
    x[7] = torch.where(torch.arange(vocab) % 2 == 0, -0.0, 0.0)
    x[8, ::100] = torch.arange(0, len(x[8, ::100])).float() * 0.5 % 7
    tokens = torch.tensor([[0, vocab // 2, 17]] * 9, dtype=torch.int32)
    for k in (1, 2, 40, 64):
        _check(x.to(dtype), k, tokens)


@pytest.mark.parametrize("vocab", [4096, 32768, 128256])
def test_crowded_list(vocab):
    """The largest values in the places of few lanes, thousands of them: the list of candidates overflows and its threshold is raised."""
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.standard_normal((2, vocab)).astype(np.float32))
    crowd = torch.arange(vocab) % 4096 < 8 * 70          # lanes 0 .. 69 of every slice of fp32 and bf16 vectors
    x[:, crowd] += 50
    x[1, crowd] = 60.0
    for dtype in (torch.float32, torch.bfloat16):
        for k in (1, 20, 64):
            _check(x.to(dtype), k)
    low = torch.arange(vocab, dtype=torch.float32).flip(0)[None] * 1e-3          # sorted by frequency
    _check(low, 64)


def test_infinities_and_nan():
    x, _ = _logits(5, 4, 1000, torch.float32)
    x[0, 10] = math.inf
    x[1, 20] = math.nan
    x[2, 30], x[2, 31] = math.inf, math.nan
    got = _run(x.cuda(), 1000, 2, torch.tensor([[1]] * 4, dtype=torch.int32))
    assert torch.isnan(got["lse"][:3]).all() and torch.isnan(got["entropy"][:3]).all() and torch.isnan(got["given"][:3]).all()
    assert got["id"][0, 0] == 10 and got["id"][1, 0] == 20 and got["id"][2].tolist() == [31, 30]
    assert torch.isfinite(got["lse"][3])


def test_nothing_asked():
    import paper_2505_20776_amd as sx
    x, _ = _logits(6, 2, 40000, torch.bfloat16)
    ws = torch.empty(sx.token_logprobs_bytes(2, 40000, 0), dtype=torch.uint8, device="cuda")
    lse = torch.zeros(2, device="cuda")
    sx.token_logprobs(x.cuda(), 2, 40000, ws, lse=lse)
    torch.cuda.synchronize()
    assert torch.allclose(lse.cpu().double(), torch.logsumexp(x.double(), dim=1), atol=1e-4)
    sx.token_logprobs(x.cuda(), 0, 40000, ws)
    sx.token_logprobs(x.cuda(), 2, 40000, ws)
    torch.cuda.synchronize()


def test_captured_and_replayed_on_a_side_stream():
    import paper_2505_20776_amd as sx
    x, _ = _logits(7, 60, 128256, torch.bfloat16)
    dev, k = x.cuda(), 3
    ws = torch.empty(sx.token_logprobs_bytes(60, 128256, k), dtype=torch.uint8, device="cuda")
    ids = torch.zeros((60, k), dtype=torch.int32, device="cuda")
    lse = torch.zeros(60, device="cuda")
    call = lambda: sx.token_logprobs(dev, 60, 128256, ws, k=k, top_id=ids, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    eager = ids.clone(), lse.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        ids.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, eager[0]) and torch.equal(lse, eager[1])
        call()
        torch.cuda.synchronize()
        assert torch.equal(ids, eager[0])


@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 1280), (torch.bfloat16, 12 * 4096 + 1280), (torch.float32, 700), (torch.bfloat16, 65), (torch.float32, 2048 * 9 + 300)])
@pytest.mark.parametrize("k", [4, 8, 9])
def test_slices_that_fill_few_waves(dtype, vocab, k):
    """The last slice of a row has values for fewer waves than answers are wanted."""
    x, _ = _logits(vocab + k, 5, vocab, dtype)
    _check(x, k)
