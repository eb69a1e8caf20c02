"""Rotation and 8-bit cache without a GPU: the oracle against hand-worked and brute-force values, and the refusals of the
entry points, which come before anything touches the device."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import kv8 as O
from paper_2404_12457_amd import binding as B

A = 0x10000  # a fake, aligned, non-NULL address: validation never dereferences device pointers
FAR = 0x40000000


@pytest.fixture(scope="module", autouse=True)
def lib():
    return B.load()


# ---- the oracle -----------------------------------------------------------------------------
def test_e4m3_values_and_rounding_by_hand():
    assert O.VALUES[0x7E] == 448 and O.VALUES[0x01] == 2.0**-9 and O.VALUES[0x08] == 2.0**-6 and O.VALUES[0xB8] == -1.0
    assert math.isnan(O.VALUES[0x7F]) and math.isnan(O.VALUES[0xFF])
    x = np.array([448, 432, 431.9, 433, 1.0625, 1.1875, 2.0**-10, 1.01 * 2.0**-10, -0.0, np.inf, np.nan, -17.0])
    want = [0x7E, 0x7E, 0x7D, 0x7E, 0x38, 0x3A, 0x00, 0x01, 0x80, 0x7F, 0x7F, 0xD8]  # 432, 1.0625 and 2^-10 are ties, -17 too
    assert O.encode(x).tolist() == want
    codes = np.array([c for c in range(256) if c & 0x7F != 0x7F], np.uint8)
    assert np.array_equal(O.encode(O.VALUES[codes]), codes)


def test_e4m3_rounding_against_torch():
    torch = pytest.importorskip("torch")
    x = np.random.Generator(np.random.PCG64(5)).standard_normal(20000).astype(np.float32) * 40
    assert np.array_equal(O.encode(x.astype(np.float64)), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("amax,want", [(0.0, 1), (448.0, 127), (448.0001, 128), (224.0, 126), (1.0, 119), (1.75, 119), (1.7500001, 120),
                                       (3.3e38, 247), (2.0**-133, 1)])
def test_scale_is_the_smallest_that_holds_the_largest_value(amax, want):
    assert O.scale_byte(amax) == want


@pytest.mark.parametrize("d", [64, 128])
def test_tile_orders_are_permutations_with_the_documented_neighbours(d):
    k, v = O.byte_of(d, True), O.byte_of(d, False)
    assert np.array_equal(np.sort(k.ravel()), np.arange(16 * d)) and np.array_equal(np.sort(v.ravel()), np.arange(16 * d))
    assert (k[0, :16] == np.arange(16)).all() and (k[:, 0] == 16 * np.arange(16)).all()
    assert (v[:4, 0] == np.arange(4)).all() and (v[0, :64:16] == 4 * np.arange(4)).all() and (v[0, :16] == 16 * np.arange(16)).all()


def test_a_raised_scale_leaves_normal_numbers_alone():
    g = np.random.Generator(np.random.PCG64(6))
    x = g.standard_normal((9, 1, 64))
    plane = np.zeros((1, O.block_bytes(1, 64)), np.uint8)
    O.write_tokens(plane, [0], 0, x, True)
    before = O.read_tokens(plane, [0], 9, 1, 64, True)
    O.write_tokens(plane, [0], 9, 30 * x[:1], True)
    after = O.read_tokens(plane, [0], 10, 1, 64, True)
    e = int(plane[0, 16 * 64]) - 127
    normal = np.abs(before) >= 2.0 ** (e - 6)
    assert np.array_equal(before[normal], after[:9][normal]) and np.abs(after[:9] - before).max() <= 2.0 ** (e - 10)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_relative_angles(interleaved):
    g = np.random.Generator(np.random.PCG64(7))
    cs = O.angles(50, 32)
    x, y = g.standard_normal((2, 1, 1, 64))
    dot = lambda p, q: float((O.rotate(x, p, cs, interleaved) * O.rotate(y, q, cs, interleaved)).sum())  # noqa: E731
    assert abs(dot(40, 37) - dot(5, 2)) < 1e-5 and abs(dot(0, 0) - float((x * y).sum())) < 1e-12
    assert np.array_equal(O.rotate(x, 9, cs, interleaved)[..., 32:], x[..., 32:])


def test_a_row_of_q_as_two_e4m3_numbers_is_off_by_the_documented_bound():
    """hi = nearest to q 2^-e, lo = nearest to 16 times the rest.  Elements far below the row's largest lose bits: their own error is
    not bounded by 2^-12 of them, only by 2^-21 of the largest."""
    g = np.random.Generator(np.random.PCG64(8))
    m = (128 + g.integers(0, 128, (500, 64))) / 128 * g.choice([-1, 1], (500, 64))  # the 8 significant bits of a bf16 number
    q = np.ldexp(m, g.integers(-30, 1, (500, 64)))
    worst = 0.0
    for row in q:
        top = np.abs(row).max()
        e = O.scale_byte(top) - 127
        f = np.ldexp(row, -e)
        hi = O.VALUES[O.encode(f)]
        off = np.abs(hi + O.VALUES[O.encode((f - hi) * 16)] / 16 - f) * 2.0**e
        assert (off <= 2.0**-21 * top).all() and (off[np.abs(row) > 2.0**-13 * top] == 0).all()
        worst = max(worst, float((off / np.abs(row)).max()))
    assert worst > 2.0**-12


# ---- the refusals ---------------------------------------------------------------------------
def _pool(dtype=B.RAGC_DTYPE_BF16, **kw):
    args = dict(k=A, v=A, num_blocks=64, kv_heads=2, head_dim=128, dtype=dtype)
    args.update(kw)
    return B.make_pool(**args)


def _pool8(**kw):
    return _pool(B.RAGC_DTYPE_E4M3, **kw)


def _batch(p=(10,), n=(5,), stride=4, table=None, dev=A, start=None):
    hp, hn = np.asarray(p, np.int32), np.asarray(n, np.int32)
    hs = np.concatenate([[0], np.cumsum(np.maximum(hn, 0))]).astype(np.int32) if start is None else np.asarray(start, np.int32)
    b = B.make_batch(len(p), stride, dev, dev, dev, dev, hp, hn, hs, table)
    b.keep = (hp, hn, hs, table)
    return b


def _rope(**kw):
    args = dict(cos_sin=A, positions=64, rot_dim=128)
    args.update(kw)
    return B.make_rope(**args)


def _code(f, *a):
    with pytest.raises(B.RagcError) as e:
        f(*a)
    return e.value.code


def _rope_code(pool=None, batch=None, rope=None, q=A, k=A, v=A, qo=A, ko=None, hq=8):
    return _code(B.ragc_kv_append_rope, pool or _pool(), batch or _batch(), rope or _rope(), q, k, v, qo, ko, hq)


def _append8_code(pool=None, batch=None, rope="", q=A, k=A, v=A, qo=A, hq=8):
    return _code(B.ragc_kv8_append, pool or _pool8(), batch or _batch(), _rope() if rope == "" else rope, q, k, v, qo, hq)


@pytest.mark.parametrize("code", [_rope_code, _append8_code])
def test_appends_with_a_rotation_refuse(code):
    r = _rope()
    r.reserved = 1
    assert code(rope=r) == B.RAGC_ERR_SHAPE
    r = _rope()
    r.interleaved = 2
    assert code(rope=r) == B.RAGC_ERR_SHAPE
    assert code(rope=_rope(cos_sin=None)) == B.RAGC_ERR_NULL
    assert code(rope=_rope(cos_sin=A + 4)) == B.RAGC_ERR_ALIGN
    for rot in (0, -16, 8, 24, 144):
        assert code(rope=_rope(rot_dim=rot)) == B.RAGC_ERR_SHAPE
    assert code(rope=_rope(positions=0)) == B.RAGC_ERR_SHAPE
    assert code(rope=_rope(positions=14)) == B.RAGC_ERR_RANGE  # the last new token is at position 14
    assert "position 14" in B.ragc_last_error()
    assert code(hq=7) == B.RAGC_ERR_SHAPE and code(hq=-2) == B.RAGC_ERR_SHAPE
    assert code(hq=0) == B.RAGC_ERR_NULL and code(q=None) == B.RAGC_ERR_NULL and code(qo=None) == B.RAGC_ERR_NULL
    assert code(k=None) == B.RAGC_ERR_NULL and code(v=None) == B.RAGC_ERR_NULL
    for name in ("q", "k", "v", "qo"):
        assert code(**{name: A + 8}) == B.RAGC_ERR_ALIGN
    assert code(qo=A + 256) == B.RAGC_ERR_SHAPE and "overlaps" in B.ragc_last_error()
    assert code(batch=_batch(dev=None)) == B.RAGC_ERR_NULL
    assert code(batch=_batch(p=(60,), n=(10,))) == B.RAGC_ERR_RANGE
    assert code(batch=_batch(p=(-1,))) == B.RAGC_ERR_RANGE
    assert code(batch=_batch(p=(1, 1), n=(5, 2), start=(0, 6, 8))) == B.RAGC_ERR_RANGE
    assert code(batch=_batch(p=(20,), n=(5,), table=np.array([[1, 64, 0, 0]], np.int32))) == B.RAGC_ERR_RANGE


def test_rope_append_refuses_what_is_its_own():
    assert _rope_code(pool=_pool8()) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_kv_append_rope, _pool(), _batch(), None, A, A, A, A, None, 8) == B.RAGC_ERR_NULL
    assert _rope_code(ko=A + 64) == B.RAGC_ERR_SHAPE
    assert _rope_code(ko=FAR + 8) == B.RAGC_ERR_ALIGN


def test_appends_refuse_outputs_that_overlap_what_others_read():
    """Five rows from number 7 on: q and q_out have 8 heads, the rest 2.  Arrays a megabyte apart, one of them moved."""
    b, mb, row = _batch(p=(10,), n=(5,), start=(7, 12)), 1 << 20, 128 * 2
    at = dict(q=A, k=A + mb, v=A + 2 * mb, qo=A + 3 * mb, ko=A + 4 * mb)
    rows = {n: (at[n] + 7 * h * row, at[n] + 12 * h * row) for n, h in dict(q=8, k=2, v=2, qo=8, ko=2).items()}
    heads = dict(qo=8, ko=2)
    for out, other in (("qo", "k"), ("qo", "v"), ("qo", "ko"), ("ko", "q"), ("ko", "v"), ("ko", "qo")):
        first, end = rows[other]
        for start in (first - 5 * heads[out] * row + 16, first, end - 16):  # of the rows that the call writes
            assert _rope_code(batch=b, **{**at, out: start - 7 * heads[out] * row}) == B.RAGC_ERR_SHAPE, (out, other, start)
            assert "overlaps" in B.ragc_last_error()
        if other not in ("ko", "qo"):
            assert "_new" in B.ragc_last_error() or other == "q"
    for start in (A + 5 * mb, A + 5 * mb + 64 * 128 * 4 - 16):
        rope = _rope(cos_sin=A + 5 * mb)
        assert _rope_code(batch=b, rope=rope, **{**at, "ko": start - 7 * 2 * row}) == B.RAGC_ERR_SHAPE and "cos_sin" in B.ragc_last_error()
        assert _append8_code(batch=b, rope=rope, q=A, k=A + mb, v=A + 2 * mb, qo=start - 7 * 8 * row) == B.RAGC_ERR_SHAPE
    assert _append8_code(q=A, k=A + mb, v=A + 2 * mb, qo=A + mb) == B.RAGC_ERR_SHAPE and "k_new" in B.ragc_last_error()  # rows from number 0 on


def test_kv8_append_refuses_what_is_its_own():
    for dtype in (B.RAGC_DTYPE_F32, B.RAGC_DTYPE_BF16, 3):
        assert _append8_code(pool=_pool(dtype)) == B.RAGC_ERR_SHAPE
    assert _append8_code(rope=None) == B.RAGC_ERR_SHAPE  # q without a rotation
    assert _append8_code(rope=None, q=None, qo=None, hq=8) == B.RAGC_ERR_SHAPE
    assert _append8_code(pool=_pool8(block_stride_elems=2 * 16 * 128 + 8)) == B.RAGC_ERR_SHAPE  # no room for the scales
    assert _append8_code(pool=_pool8(block_stride_elems=2 * 16 * 128 + 24)) == B.RAGC_ERR_ALIGN
    assert _append8_code(pool=_pool8(k=A + 8)) == B.RAGC_ERR_ALIGN


def test_other_calls_refuse_an_8_bit_pool():
    b = _batch()
    assert _code(B.ragc_prefill_attn, _pool8(), b, A, A, A, A, 8, 0.1) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_prefill_attn_static, _pool8(), b, A, A, A, A, 8, 0.1) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_prefill_attn_workspace, _pool8(), b, 8) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_kv_append, _pool8(), b, A, A) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_kv_gather, _pool8(), b, 0, 4, A, A) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_debug_get_attn_plan, _pool8(), b, 8) == B.RAGC_ERR_SHAPE


def test_empty_batches_are_nothing():
    none = _batch(p=(10,), n=(0,))
    assert B.ragc_kv_append_rope(_pool(), none, _rope(), None, None, None, None, None, 0) == 0
    assert B.ragc_kv8_append(_pool8(), none, None, None, None, None, None, 0) == 0


def test_swap_of_8_bit_pools_counts_the_scales():
    need = B.kv8_block_bytes(2, 128)
    assert need == 2 * 16 * 128 + 16 and B.kv8_block_bytes(17, 64) == 17 * 16 * 64 + 32
    ids = np.zeros(1, np.int32)
    assert _code(B.ragc_kv_swap, _pool8(), A, A, need - 16, 4, ids, ids, B.RAGC_SWAP_TO_HOST) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_kv_swap, _pool8(), A, A, need + 8, 4, ids, ids, B.RAGC_SWAP_TO_HOST) == B.RAGC_ERR_ALIGN
    assert B.ragc_kv_swap(_pool8(), A, A, need, 4, np.zeros(0, np.int32), np.zeros(0, np.int32), B.RAGC_SWAP_TO_HOST) == 0


def test_bytes_per_token_of_8_bit_pools_count_the_scales():
    for layers, heads, d in ((32, 8, 128), (1, 1, 64), (80, 17, 128), (7, 32, 64)):
        assert 16 * B.ragc_kv_bytes_per_token(layers, heads, d, B.RAGC_DTYPE_E4M3) == 2 * layers * B.kv8_block_bytes(heads, d)
    assert B.ragc_kv_bytes_per_token(0, 8, 128, B.RAGC_DTYPE_E4M3) == 0


def _attn_code(pool=None, batch=None, q=A, o=A, hq=8, scale=0.1, flags=0, ws=None, n=0):
    return _code(B.ragc_kv8_attn, pool or _pool8(), batch or _batch(), q, o, hq, scale, flags, ws, n)


def test_kv8_attention_refuses():
    for dtype in (B.RAGC_DTYPE_F32, B.RAGC_DTYPE_BF16, 5):
        assert _attn_code(pool=_pool(dtype)) == B.RAGC_ERR_SHAPE
        assert _code(B.ragc_kv8_attn_workspace, _pool(dtype), _batch(), 8) == B.RAGC_ERR_SHAPE
    assert _attn_code(hq=3) == B.RAGC_ERR_SHAPE and _attn_code(hq=0) == B.RAGC_ERR_SHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _attn_code(scale=scale) == B.RAGC_ERR_SHAPE
    assert _attn_code(flags=B.RAGC_ATTN_APPEND_FUSED) == B.RAGC_ERR_SHAPE and _attn_code(flags=0x80) == B.RAGC_ERR_SHAPE
    assert _code(B.ragc_kv8_attn_workspace, _pool8(), _batch(), 8, B.RAGC_ATTN_APPEND_FUSED) == B.RAGC_ERR_SHAPE
    assert _attn_code(q=None) == B.RAGC_ERR_NULL and _attn_code(o=None) == B.RAGC_ERR_NULL
    assert _attn_code(q=A + 8) == B.RAGC_ERR_ALIGN and _attn_code(o=A + 2) == B.RAGC_ERR_ALIGN
    assert _attn_code(batch=_batch(dev=None)) == B.RAGC_ERR_NULL
    assert _attn_code(batch=_batch(p=(60,), n=(10,))) == B.RAGC_ERR_RANGE
    assert _attn_code(batch=_batch(p=(20,), n=(5,), table=np.array([[1, 64, 0, 0]], np.int32))) == B.RAGC_ERR_RANGE
    assert B.ragc_kv8_attn(_pool8(), _batch(n=(0,)), None, None, 8, 0.1) == 0


def test_kv8_attention_workspace():
    long = _batch(p=(100000,), n=(1,), stride=6251)
    need = B.ragc_kv8_attn_workspace(_pool8(num_blocks=7000), long, 8)
    assert need > 0 and need % (2 * 16 * (128 + 2) * 4) == 0
    assert B.ragc_kv8_attn_workspace(_pool8(num_blocks=7000), long, 8, B.RAGC_ATTN_NO_SPLIT) == 0
    assert B.ragc_kv8_attn_workspace(_pool8(), _batch(), 8) == 0 and B.ragc_kv8_attn_workspace(_pool8(), _batch(n=(0,)), 8) == 0
    p = _pool8(num_blocks=7000)
    assert _attn_code(pool=p, batch=long) == B.RAGC_ERR_WORKSPACE
    assert _attn_code(pool=p, batch=long, ws=A, n=need - 1) == B.RAGC_ERR_WORKSPACE
    assert _attn_code(pool=p, batch=long, ws=A + 16, n=need) == B.RAGC_ERR_ALIGN


def test_kv8_plan_hook():
    long = _batch(p=(100000,), n=(1,), stride=6251)
    p = _pool8(num_blocks=7000)
    try:
        for bad in ((7, 8, 0), (16, 5, 0), (16, 8, 24), (16, 8, -16), (128, 4, 1 << 20)):
            assert _code(B.ragc_debug_set_kv8_plan, *bad) == B.RAGC_ERR_SHAPE
        B.ragc_debug_set_kv8_plan(32, 4, 64)
        assert B.ragc_debug_get_kv8_plan(p, long, 8) == (32, 4, 64)
        assert B.ragc_kv8_attn_workspace(p, long, 8) == 98 * 2 * 32 * (128 + 2) * 4  # 6251 blocks in copies of 64, two heads
        assert B.ragc_debug_get_kv8_plan(p, long, 8, B.RAGC_ATTN_NO_SPLIT) == (32, 4, 0)
        assert B.ragc_debug_get_kv8_plan(p, _batch(n=(0,)), 8) == (0, 0, 0)
    finally:
        B.ragc_debug_set_kv8_plan(0)


def _plan(p, n, hq, hkv, d=128, flags=0):
    stride = max(-(-(a + b) // 16) for a, b in zip(p, n))
    return B.ragc_debug_get_kv8_plan(_pool8(num_blocks=1 << 20, kv_heads=hkv, head_dim=d), _batch(p=p, n=n, stride=stride), hq, flags)


def test_kv8_plans_of_known_batches():
    """256 compute units (no GPU here): measured on both sides of the lines."""
    assert _plan((1000,) * 64, (1,) * 64, 64, 8)[::2] == (16, 0)      # a full batch of decode steps is not split
    assert _plan((200,) * 64, (1,) * 64, 32, 32) == (16, 4, 0)        # many short workgroups: two per CU
    rows, _, chunk = _plan((100003,), (1,), 64, 8)                    # one long step is
    assert rows == 16 and 128 <= chunk <= 512
    assert _plan((1024,), (100,), 32, 32) [::2] == (32, 0)
    assert _plan((4096,) * 4, (128,) * 4, 64, 8) == (128, 8, 0)       # an item per CU
    assert _plan((2000,) * 40, (300,) * 40, 32, 8) == (128, 4, 0)     # many: two workgroups per CU
    assert _plan((50000,), (64,), 32, 8)[0] == 128 and _plan((50000,), (64,), 32, 8)[2] > 0
    assert _plan((50000,), (64,), 32, 8, flags=B.RAGC_ATTN_NO_SPLIT)[2] == 0


def test_kv8_plans_of_few_long_prompts():
    """Copies of equal length that the compute units hold at once: one more of them per row tile would be a second round."""
    rows, waves, chunk = _plan((8000,), (300,), 32, 8)
    copies = -(-(8300 // 16 + 1) // chunk)
    assert (rows, waves) == (128, 8) and 10 * 8 * copies <= 256 < 10 * 8 * (copies + 1)
    assert _plan((8000, 8000), (200, 200), 32, 8)[2] > 0 and _plan((16000,), (100,), 64, 8)[2] > 0
    assert _plan((8000,) * 40, (200,) * 40, 32, 8)[2] == 0  # a full batch is whole


def _outcome(f, *args, **kwargs):
    try:
        return f(*args, **kwargs)
    except B.RagcError as e:
        return e.code, str(e)
    except Exception as e:
        return type(e)


_ROWS = [(A,) * 4, (None, A, A, None), (A, None, A, A), (A + 8, A, A, A)]


@pytest.mark.parametrize("call", range(2, 5))
def test_new_calls_marshalled_in_c_behave_as_through_ctypes(call):
    """Refused or empty calls only: nothing reaches the device."""
    import inspect

    slow = B._ctypes_calls[call]
    fast = getattr(B, slow.__name__)
    assert type(fast).__name__ == "builtin_function_or_method" and inspect.signature(fast).parameters.keys() == inspect.signature(slow).parameters.keys()
    pool, batch, none = (_pool() if call == 2 else _pool8(k=A + 8)), _batch(p=(60,), n=(10,)), _batch(n=(0,))
    for b in (batch, none, None, 7):
        for rope in (_rope(), None, 3):
            for q, k, v, o in _ROWS:
                for hq in (8, 7, "8", 2**40):
                    args = {2: (pool, b, rope, q, k, v, o, None, hq), 3: (pool, b, rope, q, k, v, o, hq), 4: (pool, b, q, o, hq, 0.1)}[call]
                    for extra in ((), (0,), (None,)) if call != 4 else ((), (0,), (1 << 33,), (0, None, 0, 0)):
                        assert _outcome(fast, *args, *extra) == _outcome(slow, *args, *extra), (args, extra)
    assert _outcome(fast) is TypeError and _outcome(fast, *args, nothing=1) is TypeError
    keys = list(inspect.signature(slow).parameters)
    assert _outcome(fast, **dict(zip(keys, args))) == _outcome(slow, **dict(zip(keys, args)))


def test_rows_that_whole_numbers_do_not_hold_are_refused():
    big = _batch(p=(0,), n=(1 << 24,), stride=1 << 20)
    assert _attn_code(pool=_pool8(num_blocks=1 << 21), batch=big, hq=8) == B.RAGC_ERR_RANGE
    assert _code(B.ragc_kv8_attn_workspace, _pool8(num_blocks=1 << 21), big, 8) == B.RAGC_ERR_RANGE
    wide = _batch(p=(0,), n=(2000,), stride=200)
    assert _attn_code(pool=_pool8(kv_heads=1), batch=wide, hq=2048) == B.RAGC_ERR_RANGE


@pytest.mark.parametrize("call", ["ragc_batch_validate(pool, batch, 1)", "ragc_kv8_attn(pool, batch, A, A, 8, 0.1, B.RAGC_ATTN_VALIDATE)",
                                  "ragc_prefill_attn(pool16, batch, A, A, A, A, 8, 0.1, B.RAGC_ATTN_VALIDATE)"])
def test_host_memory_that_is_not_there_is_an_error(call):
    """A block table of 2^49 bytes to be read back.  In a process of its own, which an exception through the C entry would end."""
    code = f"""
import numpy as np
from paper_2404_12457_amd import binding as B
A, n = {A}, 65535
pool, pool16 = (B.make_pool(A, A, 64, 2, 128, t) for t in (B.RAGC_DTYPE_E4M3, B.RAGC_DTYPE_BF16))
lens = [np.ones(n, np.int32), np.ones(n, np.int32), np.arange(n + 1, dtype=np.int32)]
batch = B.make_batch(n, 2**31 - 1, A, A, A, A, *lens, None)
try:
    B.{call}
except B.RagcError as e:
    print(e.code, B.ragc_last_error())
"""
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert got.returncode == 0 and got.stdout == f"{B.RAGC_ERR_HIP} out of host memory\n", got


def test_an_output_may_stand_right_behind_its_input():
    """Rows 5.. of a packed array: what lies before them is not the call's.  Refused only for the alignment that comes later."""
    b = _batch(p=(10,), n=(5,), start=(5, 10))
    size = 5 * 8 * 128 * 2
    assert _rope_code(batch=b, qo=A + size - 16) == B.RAGC_ERR_SHAPE
    assert _rope_code(batch=b, qo=A + size, ko=A + 16) == B.RAGC_ERR_SHAPE and "k_out" in B.ragc_last_error()
