"""The 8-bit cache: rows written, appended and read back against the definition in 64 bits.  Every value is compared exactly: codes
and scales are determined by the input."""
import numpy as np
import pytest
import torch

from quant_util import Cache

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _rows(rng, shape, dtype, size=1.0):
    x = rng.standard_normal(shape) * size * np.exp(rng.standard_normal(shape[:-1] + (1,)))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


class _Pair:
    """K and V on the device, guarded, beside their definition."""

    def __init__(self, layers, heads, capacity, d, block):
        from paper_2505_20776_amd import harness as hx
        self.shape = (layers, heads, capacity, d)
        self.block = block
        self.ref = [Cache(layers, heads, capacity, d, block) for _ in range(2)]
        nb = -(-capacity // block)
        made = [hx.guarded((layers, heads, capacity, d), torch.uint8) for _ in range(2)]
        made += [hx.guarded((layers, heads, nb), torch.float32) for _ in range(2)]
        self.codes, self.scales = [made[0][0], made[1][0]], [made[2][0], made[3][0]]
        self.bases = [b for _, b in made]

    def check(self, upto, dtype=F32):
        """Every row in front of `upto`, read back through the library and straight from the codes; nothing outside written."""
        import paper_2505_20776_amd as sx
        from paper_2505_20776_amd import harness as hx
        y, h, cap, d = self.shape
        back = [hx.guarded((y, h, upto, d), dtype) for _ in range(2)]
        sx.quant_kv_read(*self.codes, *self.scales, back[0][0], back[1][0], y, h, d, upto, 0, cap, self.block,
                         dtype=sx.SPECEXT_BF16 if dtype == BF16 else sx.SPECEXT_F32)
        torch.cuda.synchronize()
        assert all(hx.guards_intact(b) for b in self.bases) and all(hx.guards_intact(b) for _, b in back)
        blocks = -(-upto // self.block)
        for i in range(2):
            want = torch.from_numpy(self.ref[i].values[:, :, :upto])
            scale = self.scales[i].cpu().double()[:, :, :blocks]
            assert torch.equal(scale, torch.from_numpy(self.ref[i].scale[:, :, :blocks]))
            codes = self.codes[i].cpu().view(torch.float8_e4m3fn).float().double()[:, :, :upto]
            assert torch.equal(torch.nan_to_num(codes * scale.repeat_interleave(self.block, 2)[:, :, :upto, None], nan=2.0 ** 100),
                               torch.nan_to_num(want, nan=2.0 ** 100))
            assert torch.equal(torch.nan_to_num(back[i][0].cpu().double(), nan=2.0 ** 100), torch.nan_to_num(want, nan=2.0 ** 100).to(dtype).double())


@pytest.mark.parametrize("d,block,dtype,layers,heads,pieces", [
    (128, 32, BF16, 2, 3, [(0, 1)]),                        # one token
    (128, 32, BF16, 1, 2, [(0, 31), (31, 1), (32, 33)]),    # a block filled by its last token, then one and a token more
    (128, 64, BF16, 2, 2, [(0, 100), (100, 5), (105, 150)]),
    (128, 128, BF16, 1, 2, [(0, 300), (300, 1)]),
    (64, 32, F32, 2, 5, [(0, 37), (37, 91)]),
    (64, 64, F32, 1, 3, [(0, 64), (64, 64)]),
    (64, 128, BF16, 1, 2, [(0, 129), (129, 127)]),
    (128, 128, F32, 1, 1, [(0, 127), (127, 2)]),
])
def test_written_in_pieces(d, block, dtype, layers, heads, pieces):
    import paper_2505_20776_amd as sx
    rng = np.random.default_rng(d + block + layers)
    cap = pieces[-1][0] + pieces[-1][1] + 7
    c = _Pair(layers, heads, cap, d, block)
    for i, (start, n) in enumerate(pieces):
        rows = [_rows(rng, (layers, heads, n, d), dtype, 3.0 ** i) for _ in range(2)]        # later ones larger: scales grow
        sx.quant_kv_write(rows[0].cuda(), rows[1].cuda(), *c.codes, *c.scales, layers, heads, d, n, start, cap, block,
                          dtype=sx.SPECEXT_BF16 if dtype == BF16 else sx.SPECEXT_F32)
        for ref, x in zip(c.ref, rows):
            ref.write(x.double().numpy(), start)
    c.check(pieces[-1][0] + pieces[-1][1])
    c.check(pieces[-1][0] + pieces[-1][1], BF16)


@pytest.mark.parametrize("block", [32, 64, 128])
def test_special_values(block):
    """Zeros, infinities, NaN, the borders of the scale and of the codes' range."""
    import paper_2505_20776_amd as sx
    d, n = 64, 3 * block
    x = np.zeros((1, 4, n, d), dtype=np.float32)
    x[0, 0, 0, :8] = [448.0, 449.0, -448.0, 0.0, -0.0, 1e-3, 2.0 ** -9, 2.0 ** -10]      # 449 > 448: scale 2
    x[0, 0, block, :4] = [1.75, -1.75, 2.0 ** -13, 1.0]         # exactly 448 x 2^-8
    x[0, 1, :, :] = np.float32(2.0 ** -120)                     # below the smallest scale's range
    x[0, 1, block:2 * block, 0] = np.float32(1e38)
    x[0, 2, 3, :5] = [np.inf, -np.inf, np.nan, 100.0, -3.0]
    x[0, 2, block + 1, 0] = np.inf                              # nothing finite but zeros beside it
    x[0, 3, 0, :4] = [17.0, 18.0, 19.0, 448.0]                  # ties to even at scale 1
    c = _Pair(1, 4, n, d, block)
    rows = torch.from_numpy(x)
    sx.quant_kv_write(rows.cuda(), (-rows).cuda(), *c.codes, *c.scales, 1, 4, d, n, 0, n, block, dtype=sx.SPECEXT_F32)
    c.ref[0].write(x.astype(np.float64), 0)
    c.ref[1].write(-x.astype(np.float64), 0)
    c.check(n)


@pytest.mark.parametrize("layers,heads,T,d,block,prefix,accept,dtype", [
    (2, 3, 60, 128, 32, 93, 5, BF16),         # over a block's end
    (1, 2, 128, 128, 64, 60, 128, BF16),      # three blocks
    (3, 1, 9, 64, 128, 127, 1, F32),
    (1, 4, 7, 64, 32, 32, 7, BF16),           # a fresh block
    (2, 2, 16, 128, 32, 0, 16, F32),          # an empty cache
    (1, 2, 20, 128, 64, 70, 0, BF16),         # nothing accepted: nothing written
])
def test_commit(layers, heads, T, d, block, prefix, accept, dtype):
    import paper_2505_20776_amd as sx
    rng = np.random.default_rng(T + prefix)
    code = sx.SPECEXT_BF16 if dtype == BF16 else sx.SPECEXT_F32
    cap = prefix + T + 3
    c = _Pair(layers, heads, cap, d, block)
    if prefix:
        old = [_rows(rng, (layers, heads, prefix, d), dtype, 0.3) for _ in range(2)]
        sx.quant_kv_write(old[0].cuda(), old[1].cuda(), *c.codes, *c.scales, layers, heads, d, prefix, 0, cap, block, dtype=code)
        for ref, x in zip(c.ref, old):
            ref.write(x.double().numpy(), 0)
    tree = [_rows(rng, (layers, heads, T, d), dtype) for _ in range(2)]
    path = np.full(T, -1, np.int32)
    path[:accept] = rng.permutation(T)[:accept]
    before = [x.clone() for x in c.codes]
    # the count may say more than the bound allows
    count = torch.tensor([accept if accept < T else T + 9], dtype=torch.int32, device="cuda")
    sx.commit_tree_quant(tree[0].cuda(), tree[1].cuda(), *c.codes, *c.scales, torch.from_numpy(path).cuda(), count, T, T, layers, heads, d,
                         prefix, cap, block, dtype=code)
    for ref, x in zip(c.ref, tree):
        ref.append(x.double().numpy(), prefix, [int(r) for r in path[:accept]])
    if prefix + accept:
        c.check(prefix + accept)
    for was, now in zip(before, c.codes):       # rows behind the last one
        assert torch.equal(was[:, :, prefix + accept:], now[:, :, prefix + accept:])


def test_commit_entries_that_are_no_nodes():
    """Their rows keep their bytes; the others are written, and the scale follows those."""
    import paper_2505_20776_amd as sx
    rng = np.random.default_rng(3)
    y, h, T, d, block, prefix, cap = 2, 2, 10, 128, 32, 30, 64
    c = _Pair(y, h, cap, d, block)
    old = _rows(rng, (y, h, cap, d), BF16)
    sx.quant_kv_write(old.cuda(), old.cuda(), *c.codes, *c.scales, y, h, d, cap, 0, cap, block)
    before = [x.clone() for x in c.codes]
    for ref in c.ref:
        ref.write(old.double().numpy(), 0)
    tree = _rows(rng, (y, h, T, d), BF16, 4.0)
    path = [3, -1, 7, 99, 0]
    sx.commit_tree_quant(tree.cuda(), tree.cuda(), *c.codes, *c.scales, torch.tensor(path, dtype=torch.int32, device="cuda"),
                         torch.tensor([5], dtype=torch.int32, device="cuda"), 5, T, y, h, d, prefix, cap, block)
    torch.cuda.synchronize()
    for i in range(2):
        c.ref[i].append(tree.double().numpy(), prefix, path)
        assert torch.equal(before[i][:, :, [31, 33]], c.codes[i][:, :, [31, 33]])
        want, scale = torch.from_numpy(c.ref[i].values), c.scales[i].cpu().double()
        assert torch.equal(scale, torch.from_numpy(c.ref[i].scale))
        got = c.codes[i].cpu().view(torch.float8_e4m3fn).double() * scale.repeat_interleave(block, 2)[:, :, :cap, None]
        rows = list(range(prefix)) + [30, 32, 34]
        assert torch.equal(got[:, :, rows], want[:, :, rows])


def test_strides_and_another_stream():
    """Token-major cache and sources, K and V side by side, scales with a gap; on a side stream."""
    import paper_2505_20776_amd as sx
    rng = np.random.default_rng(9)
    y, h, n, d, block, cap = 2, 3, 75, 64, 32, 96
    src = _rows(rng, (y, n, h, 2, d), BF16)
    dev = src.cuda()
    cache = torch.full((y, cap, h, 2, d), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, y, h, 8), 7.0, dtype=torch.float32, device="cuda")
    strides = dict(cache_stride_layer=cap * h * 2 * d, cache_stride_h=2 * d, cache_stride_l=h * 2 * d, scale_stride_layer=h * 8, scale_stride_h=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    back = torch.zeros((y, n, h, 2, d), dtype=torch.bfloat16, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    sx.quant_kv_write(dev, dev[:, :, :, 1:], cache, cache[:, :, :, 1:], scales[0], scales[1], y, h, d, n, 0, cap, block,
                      src_stride_layer=n * h * 2 * d, src_stride_h=2 * d, src_stride_t=h * 2 * d, stream=s, **strides)
    sx.quant_kv_read(cache, cache[:, :, :, 1:], scales[0], scales[1], back, back[:, :, :, 1:], y, h, d, n, 0, cap, block,
                     dst_stride_layer=n * h * 2 * d, dst_stride_h=2 * d, dst_stride_t=h * 2 * d, stream=s, **strides)
    s.synchronize()
    for i in range(2):
        ref = Cache(y, h, cap, d, block)
        ref.write(src[:, :, :, i].permute(0, 2, 1, 3).double().numpy(), 0)
        assert torch.equal(back[:, :, :, i].permute(0, 2, 1, 3).cpu().double(), torch.from_numpy(ref.values[:, :, :n]))
        assert torch.equal(scales[i, :, :, :3].cpu().double(), torch.from_numpy(ref.scale))
    assert (scales[:, :, :, 3:] == 7.0).all() and (cache[:, n:] == 0xA5).all()


def test_read_with_scales_that_are_no_powers_of_two():
    """value = code x scale, rounded once: at most half a step of bf16 (2^-8 relative) from the product, here exactly its rounding."""
    import paper_2505_20776_amd as sx
    rng = np.random.default_rng(4)
    y, h, n, d, block = 1, 2, 70, 128, 32
    codes = torch.from_numpy(rng.integers(0, 127, (y, h, n, d), dtype=np.uint8)).cuda()
    scale = torch.from_numpy(rng.uniform(1e-3, 3.0, (y, h, 3)).astype(np.float32)).cuda()
    for dtype, code in ((BF16, sx.SPECEXT_BF16), (F32, sx.SPECEXT_F32)):
        back = torch.empty((y, h, 41, d), dtype=dtype, device="cuda")
        sx.quant_kv_read(codes, codes, scale, scale, back, back.clone(), y, h, d, 41, 29, n, block, dtype=code)
        want = codes.cpu().view(torch.float8_e4m3fn).float() * scale.cpu().repeat_interleave(block, 2)[:, :, :n, None]
        assert torch.equal(back.cpu(), want[:, :, 29:].to(dtype))


def test_nothing_to_do():
    import paper_2505_20776_amd as sx
    c = _Pair(1, 1, 8, 64, 32)
    x = torch.ones((1, 1, 8, 64), dtype=BF16, device="cuda")
    before = [t.clone() for t in c.codes + c.scales]
    sx.quant_kv_write(x, x, *c.codes, *c.scales, 1, 1, 64, 0, 8, 8, 32)
    sx.quant_kv_read(*c.codes, *c.scales, x, x, 1, 1, 64, 0, 3, 8, 32)
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, c.codes + c.scales)) and (x == 1).all()


def test_count_of_nothing_changes_nothing():
    """In the middle of a block too, whatever its scale is."""
    import paper_2505_20776_amd as sx
    for scale in (2.0 ** -120, 0.3, 1.0):
        c = _Pair(2, 2, 64, 64, 32)
        for t in c.codes:
            t.view(torch.uint8).copy_(torch.randint(0, 0x7F, t.shape, dtype=torch.uint8))
        for t in c.scales:
            t.fill_(scale)
        before = [t.clone() for t in c.codes + c.scales]
        x = torch.ones((2, 2, 8, 64), dtype=BF16, device="cuda")
        for n in (0, -3):
            sx.commit_tree_quant(x, x, *c.codes, *c.scales, torch.arange(8, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"),
                                 8, 8, 2, 2, 64, 37, 64, 32)
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, c.codes + c.scales))
