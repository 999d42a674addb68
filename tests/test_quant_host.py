"""Refusals of the 8-bit cache and logits functions: reported before anything is launched, so nothing here needs a GPU."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK = 4096


@pytest.fixture(scope="module")
def sx():
    import paper_2505_20776_amd as sx
    if not os.path.exists(os.path.join(ROOT, "paper_2505_20776_amd", "libspecext.so")):
        from paper_2505_20776_amd.build import build_library
        build_library(verbose=False)
    sx.load_library()
    return sx


def _desc(sx, **kw):
    base = dict(dtype=sx.SPECEXT_BF16, n_q_heads=32, n_kv_heads=8, head_dim=128, prefix_len=4096, n_tree=60, chunk_size=32,
                want_scores=True, num_splits=8, flags=sx.SPECEXT_FLAG_QUANT_BLOCK_32)
    base.update(kw)
    return sx.make_desc(**base)


def _attend(sx, desc, args=None, ws=OK, nbytes=1 << 40, stride=0):
    return sx.verify_attn_quant(desc, *(args or [OK] * 10), ws, workspace_nbytes=nbytes, scale_stride_h=stride, stream=0, check=False)


@pytest.mark.parametrize("field,value,status", [
    ("flags", 32 | 64, -1), ("flags", 32 | 64 | 128, -1), ("flags", 64 | 16, -1), ("flags", 256 | 32, -1), ("reserved", 1, -1),
    ("flags", 32 | 1, -2), ("dtype", 0, -2), ("chunk_size", 48, -2), ("chunk_size", 16, -2), ("kp_stride_l", 136, -2), ("kp_stride_h", 1000 * 8, 0),
    ("kp_stride_h", 8, -2), ("kp_stride_l", 64, -1), ("head_dim", 96, -2), ("n_tree", 129, -2), ("prefix_len", -1, -1),
])
def test_descriptor(sx, field, value, status):
    d = _desc(sx)
    if field == "dtype":
        d.out_dtype = value
    setattr(d, field, value)
    if status == 0:
        assert sx.workspace_bytes(d) > 0 and sx.num_splits(d) == 8
        return
    assert sx.workspace_bytes(d) == 0 and sx.num_splits(d) == status
    assert _attend(sx, d) == status


def test_the_two_kinds_of_prefix_do_not_mix(sx):
    quant, plain = _desc(sx), _desc(sx, flags=0)
    assert _attend(sx, plain) == -1
    nbytes = 1 << 40
    assert sx.verify_attn(quant, *[OK] * 8, OK, workspace_nbytes=nbytes, stream=0, check=False) == -1
    none = _desc(sx, want_scores=False)
    assert sx.verify_attn_static(none, *[OK] * 8, stream=0, check=False) == -1
    assert sx.materialized_bytes(quant) == 0 and sx.materialized_ld(quant) == -1


def test_attention_pointers(sx):
    d = _desc(sx)
    for i in list(range(9)):                             # lse may be null
        a = [OK] * 10
        a[i] = None
        assert _attend(sx, d, a) == -1, i
    assert _attend(sx, d, ws=None) == -1
    for i, off in [(1, 8), (2, 8), (3, 2), (4, 2), (5, 8), (0, 8), (8, 8), (9, 2), (7, 2)]:
        a = [OK] * 10
        a[i] += off
        assert _attend(sx, d, a) == -2, i
    assert _attend(sx, d, ws=OK + 64) == -2
    assert _attend(sx, d, nbytes=sx.workspace_bytes(d) - 1) == -3
    assert _attend(sx, d, stride=-1) == -1
    with pytest.raises(sx.SpecextError):
        sx.verify_attn_quant(d, *[OK] * 10, OK, workspace_nbytes=0, stream=0)
    # without a prefix its pointers may be null; the workspace is looked at next
    empty = _desc(sx, prefix_len=0, want_scores=False, num_splits=0)
    a = [OK] * 10
    a[1] = a[2] = a[3] = a[4] = None
    assert _attend(sx, empty, a, nbytes=0) == -3


CACHE = dict(n_layers=32, n_kv_heads=8, head_dim=128, cache_capacity=1024, scale_block=32, stream=0, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(n_layers=0), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=0), -1), (dict(n_tokens=-1), -1), (dict(start=-1), -1),
    (dict(start=1020), -1), (dict(cache_capacity=9), -1), (dict(head_dim=96), -2), (dict(scale_block=16), -2), (dict(scale_block=0), -2),
    (dict(scale_block=48), -2), (dict(scale_block=256), -2), (dict(dtype=2), -2), (dict(n_layers=9000), -2), (dict(rows_stride_t=100), -2),
    (dict(rows_stride_t=64), -2), (dict(rows_stride_h=-128), -1), (dict(cache_stride_l=136), -2), (dict(cache_stride_l=64), -2),
    (dict(cache_stride_h=8), -2), (dict(scale_stride_h=-1), -1), (dict(cache_capacity=(1 << 30) + 1), -2),
])
def test_write_and_read(sx, change, status):
    kw = dict(CACHE, n_tokens=10, start=0)
    for f, rows in ((sx.quant_kv_write, "src"), (sx.quant_kv_read, "dst")):
        more = {k.replace("rows", rows): v for k, v in change.items()}
        assert f(*[OK] * 6, **{**kw, **more}) == status
        for i in range(6):
            a = [OK] * 6
            a[i] = None
            assert f(*a, **kw) == -1
            a[i] = OK + (2 if (i in (4, 5) if rows == "src" else i in (2, 3)) else 8)
            assert f(*a, **kw) == -2


def test_commit(sx):
    kw = dict(CACHE, max_accept=8, n_tree=60, prefix_len=1000)
    f = sx.commit_tree_quant
    for change, status in [(dict(max_accept=-1), -1), (dict(n_tree=0), -1), (dict(n_tree=129), -2), (dict(max_accept=129, prefix_len=0), -2),
                           (dict(prefix_len=1017), -1), (dict(prefix_len=-1), -1), (dict(scale_block=33), -2), (dict(dtype=7), -2),
                           (dict(tree_stride_t=64), -2), (dict(head_dim=32), -2)]:
        assert f(*[OK] * 8, **{**kw, **change}) == status, change
    for i in range(8):
        a = [OK] * 8
        a[i] = None
        assert f(*a, **kw) == -1
        a[i] = OK + (2 if i >= 4 else 8)
        assert f(*a, **kw) == -2


def test_logits(sx):
    assert sx.token_logprobs_bytes(60, 128256, 4) >= 60 * 4 * (16 + 32)
    for bad in ((-1, 100, 1), (5, 0, 0), (5, 10, 11), (5, 100, -1), (5, 100, 65), (5, (1 << 20) + 1, 1), ((1 << 24) + 1, 10, 1)):
        assert sx.token_logprobs_bytes(*bad) == 0
    nbytes = sx.token_logprobs_bytes(60, 128256, 4)
    good = dict(tokens=OK, n_given=3, logprob=OK, k=4, top_id=OK, top_logprob=OK, lse=OK, entropy=OK, workspace_nbytes=nbytes, stream=0, check=False)

    def call(logits=OK, rows=60, vocab=128256, ws=OK, **kw):
        return sx.token_logprobs(logits, rows, vocab, ws, **{**good, **kw})
    for kw, status in [(dict(logits=None), -1), (dict(ws=None), -1), (dict(rows=-1), -1), (dict(vocab=0), -1), (dict(k=-1), -1),
                       (dict(vocab=3), -1), (dict(n_given=-1), -1), (dict(tokens=None), -1), (dict(logprob=None), -1), (dict(top_id=None), -1),
                       (dict(row_stride=128255), -1), (dict(row_stride=-5), -1), (dict(logit_scale=-1.0), -1), (dict(logit_scale=float("inf")), -1),
                       (dict(logit_scale=float("nan")), -1), (dict(k=65), -2), (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), -2), (dict(dtype=3), -2),
                       (dict(logits=OK + 1), -2), (dict(logits=OK + 2, dtype=0), -2), (dict(ws=OK + 128), -2), (dict(lse=OK + 2), -2),
                       (dict(entropy=OK + 1), -2), (dict(top_id=OK + 2), -2), (dict(tokens=OK + 2), -2), (dict(workspace_nbytes=nbytes - 1), -3)]:
        assert call(**kw) == status, kw


@pytest.mark.parametrize("d,hq,hkv,T,L,splits", [
    (128, 32, 8, 1, 2048, 16), (128, 32, 8, 1, 4096, 32), (128, 32, 8, 16, 4096, 32), (128, 32, 8, 30, 4096, 32), (128, 32, 8, 60, 4096, 16),
    (128, 8, 2, 60, 4096, 32), (128, 32, 8, 60, 512, 8), (128, 32, 8, 60, 513, 5), (128, 32, 8, 8, 512, 4), (64, 12, 12, 60, 4096, 16),
    (128, 32, 8, 128, 32731, 16), (128, 32, 32, 60, 8155, 8), (128, 32, 8, 1, 1, 1)])
def test_automatic_splits(sx, d, hq, hkv, T, L, splits):
    """256 compute units: 128 keys up to 32 splits for at most 128 rows per KV head or few KV heads, else 16; 64 keys up to 512."""
    for block in (32, 64, 128):
        for chunk in (0, 32):
            kw = dict(dtype=sx.SPECEXT_BF16, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, prefix_len=L, n_tree=T, flags=block, chunk_size=chunk,
                      want_scores=chunk > 0)
            assert sx.num_splits(sx.make_desc(**kw)) == splits
            assert sx.num_splits(sx.make_desc(num_splits=splits, **kw)) == splits


@pytest.mark.parametrize("d,hq,hkv,T", [(128, 32, 8, 1), (128, 32, 8, 16), (128, 32, 8, 30), (128, 32, 8, 60), (128, 8, 2, 128), (64, 12, 12, 60), (64, 32, 8, 60)])
def test_the_reported_split_count_holds_at_every_length(sx, d, hq, hkv, T):
    for L in [*range(1, 1200, 7), *range(1200, 8300, 97), 16384, 50000, 131035]:
        for chunk in (0, 32, 96, 1024):
            kw = dict(dtype=sx.SPECEXT_BF16, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, prefix_len=L, n_tree=T, chunk_size=chunk, want_scores=chunk > 0,
                      flags=64)
            auto = sx.make_desc(**kw)
            asked = sx.make_desc(num_splits=sx.num_splits(auto), **kw)
            assert sx.num_splits(asked) == sx.num_splits(auto) and sx.workspace_bytes(asked) == sx.workspace_bytes(auto), (L, chunk)


def test_nothing_to_do_needs_no_rows(sx):
    """Empty tensors have no address."""
    for f in (sx.quant_kv_write, sx.quant_kv_read):
        a = [OK] * 6
        for i in ((0, 1) if f is sx.quant_kv_write else (4, 5)):
            a[i] = None
        assert f(*a, **CACHE, n_tokens=0, start=1024) == 0
        assert f(*a, **CACHE, n_tokens=1, start=0) == -1
    assert sx.commit_tree_quant(None, None, *[OK] * 6, **CACHE, max_accept=0, n_tree=4, prefix_len=8) == 0
    kw = dict(n_given=2, k=3, workspace_nbytes=sx.token_logprobs_bytes(0, 50, 3), stream=0, check=False)
    assert sx.token_logprobs(None, 0, 50, OK, **kw) == 0
    assert sx.token_logprobs(None, 0, 50, None, **kw) == -1
    assert sx.token_logprobs(None, 1, 50, OK, **kw) == -1


def test_sizes_beyond_one_launch(sx):
    """Threads along x stay below 2^32."""
    kw = dict(CACHE, n_layers=1, n_kv_heads=1, n_tokens=1 << 28, start=0)
    for f in (sx.quant_kv_write, sx.quant_kv_read):
        assert f(*[OK] * 6, **{**kw, "cache_capacity": (1 << 28) + 1}) == -2
        assert f(*[OK] * 4, None, OK, **{**kw, "cache_capacity": 1 << 28}) == -1          # (the sizes themselves are allowed)
    for rows, vocab, allowed in ((8388607, 10, True), (8388608, 10, False), (131071, 1 << 20, False), (129055, 1 << 20, True), (8388607, 16379, True),
                                 (8388607, 16380, False), (4194303, 16380, True)):
        assert (sx.token_logprobs_bytes(rows, vocab, 1) > 0) == allowed, (rows, vocab)
        if not allowed:
            assert sx.token_logprobs(OK, rows, vocab, OK, workspace_nbytes=1 << 50, stream=0, check=False) == -2


@pytest.mark.parametrize("scale,status", [(2.0 ** -101, -2), (2.0 ** 101, -2), (1e-45, -2), (2.0 ** -100, -3), (2.0 ** 100, -3), (0.0, -3)])
def test_range_of_the_logit_scale(sx, scale, status):
    assert sx.token_logprobs(OK, 1, 50, OK, logit_scale=scale, workspace_nbytes=0, stream=0, check=False) == status
