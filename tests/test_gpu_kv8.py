"""GPU parity of the append with position rotation and of the 8-bit cache against the oracle in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv8 as O
from paper_2404_12457_amd import binding as B

from kv8_util import Case

pytestmark = pytest.mark.gpu

ODD = [(0, 1), (5, 1), (15, 1), (15, 2), (16, 16), (3, 40), (0, 0), (31, 0), (100, 133), (47, 17), (16, 1), (0, 64)]
STEPS = [(int(p), 1) for p in np.random.Generator(np.random.PCG64(1)).integers(0, 400, 70)]  # more requests than a wave has lanes
HALF_STEP = {"bf16": 2.0**-8, "f32": 2.0**-24}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _rope(c, rot_dim, interleaved):
    cs = O.angles(int((c.h_prefix + c.h_new).max()), rot_dim)
    dev = torch.from_numpy(cs).cuda()
    return cs, dev, B.make_rope(dev, len(cs), rot_dim, interleaved)


def _near(got, want, sides, dtype):
    """One rounding to the type, and in fp32 one of a product and one of the sum."""
    off = np.abs(got - want) - (HALF_STEP[dtype] * np.abs(want) * 1.001 + 2.0**-23 * sides + 1e-38)
    worst = float(off.max())
    assert worst <= 0


def _sides(x, cs, interleaved, c):
    """|a cos| + |b sin| for the first of each turned pair, |a sin| + |b cos| for the second, |x| elsewhere.  The first is
    |a| |cos| - |b| (-|sin|), the first element of |x| turned by (|cos|, -|sin|); the second that of |x| turned by (|cos|, |sin|).
    What these two turns give for the other element of the pair is a difference of the same sides, no larger than they are."""
    half = cs.shape[1] // 2
    minus = np.abs(cs) * np.concatenate([np.ones(half), -np.ones(half)]).astype(np.float32)
    return np.maximum(c.rotated(np.abs(x), minus, interleaved), c.rotated(np.abs(x), np.abs(cs), interleaved))


@pytest.mark.parametrize("lens", [ODD, STEPS, [(7, 1)], [(0, 515)]], ids=["odd", "steps", "one", "prompt"])
@pytest.mark.parametrize("dtype,hq,hkv,d,rot,inter", [("bf16", 8, 2, 128, 128, False), ("bf16", 6, 3, 64, 16, False), ("bf16", 5, 5, 128, 64, True),
                                                     ("f32", 4, 2, 64, 32, True), ("f32", 3, 1, 128, 128, False), ("f32", 7, 7, 64, 48, False)])
def test_append_rope(lens, dtype, hq, hkv, d, rot, inter):
    c = Case(lens, hq, hkv, d, dtype, seed=hq, pad=hkv % 2, first_row=3)
    cs, keep, rope = _rope(c, rot, inter)
    q, k, v = (c.host(t) for t in (c.q, c.k_new, c.v_new))
    before = [c.host(p) for p in c.planes]
    q_out, k_out = torch.full_like(c.q, 7.0), torch.full_like(c.k_new, 7.0)
    B.ragc_kv_append_rope(c.pool, c.batch, rope, c.q, c.k_new, c.v_new, q_out, k_out, hq, _stream())
    torch.cuda.synchronize()
    tol = [_sides(x, cs, inter, c)[3:] for x in (q, k)]
    qr, kr = c.rotated(q, cs, inter), c.rotated(k, cs, inter)
    _near(c.host(q_out)[3:], qr[3:], tol[0], dtype)
    _near(c.host(k_out)[3:], kr[3:], tol[1], dtype)
    assert torch.all(q_out[:3] == 7) and torch.all(k_out[:3] == 7)  # rows before the first are not the call's
    # the pool has the very rows of k_out and v_new, and nothing else has changed
    want = [b.copy() for b in before]
    for plane, rows in zip(want, (c.host(k_out), v)):
        tiles = plane[:, :hkv * 16 * d].reshape(-1, hkv, 16, d)
        for r, p, n, at in c.spans():
            pos = np.arange(p, p + n)
            tiles[c.h_table[r, pos // 16], :, pos % 16] = rows[at]
        plane[:, :hkv * 16 * d] = tiles.reshape(len(plane), -1)
    for got, w in zip(c.planes, want):
        assert np.array_equal(c.host(got), w)
    # in place, and the same bits
    q2, k2 = c.q.clone(), c.k_new.clone()
    B.ragc_kv_append_rope(c.pool, c.batch, rope, q2, k2, c.v_new, q2, k2, hq, _stream())
    assert torch.equal(q2[3:], q_out[3:]) and torch.equal(k2[3:], k_out[3:])
    # without Q and without the copy of K
    B.ragc_kv_append_rope(c.pool, c.batch, rope, None, c.k_new, c.v_new, None, None, 0, _stream())
    for got, w in zip(c.planes, want):
        assert np.array_equal(c.host(got), w)


@pytest.mark.parametrize("lens", [ODD, STEPS, [(7, 1)], [(0, 515)]], ids=["odd", "steps", "one", "prompt"])
@pytest.mark.parametrize("hq,hkv,d,rot,inter", [(8, 2, 128, 128, False), (6, 3, 64, 16, False), (5, 5, 128, 64, True), (9, 9, 64, 48, False), (0, 17, 64, 0, False)])
def test_kv8_append_gives_the_bytes_of_the_definition(lens, hq, hkv, d, rot, inter):
    c = Case(lens, max(hq, 1), hkv, d, seed=hkv, pad=hkv % 2, first_row=5)
    k, v, q = (c.host(t) for t in (c.k_new, c.v_new, c.q))
    q_out = torch.full_like(c.q, 7.0)
    cs, keep, rope = _rope(c, rot, inter) if rot else (None, None, None)
    want = c.appended8(c.rotated(k, cs, inter) if rot else k, v)
    B.ragc_kv8_append(c.pool, c.batch, rope, c.q if hq else None, c.k_new, c.v_new, q_out if hq else None, hq, _stream())
    torch.cuda.synchronize()
    for got, w in zip(c.planes, want):
        assert np.array_equal(got.cpu().numpy(), w)
    if hq:
        _near(c.host(q_out)[5:], c.rotated(q, cs, inter)[5:], _sides(q, cs, inter, c)[5:], "bf16")
    assert torch.all(q_out[:5 if hq else None] == 7)
    # a second time: the tokens are there, the scales hold them, nothing changes
    B.ragc_kv8_append(c.pool, c.batch, rope, None, c.k_new, c.v_new, None, 0, _stream())
    for got, w in zip(c.planes, want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_kv8_append_token_by_token_raises_scales_as_the_definition_says():
    """40 single tokens, each larger than the last by a random factor, so that blocks are rounded anew again and again."""
    c = Case([(0, 40), (9, 40)], 2, 2, 64, seed=3)
    grow = torch.from_numpy(np.exp2(np.cumsum(c.rng.uniform(0, 1.5, 40)) - 20).astype(np.float32)).cuda()
    for t in (c.k_new, c.v_new):
        t.mul_(torch.cat([grow, grow])[:, None, None].to(t.dtype))
    start = c.h_prefix.copy()
    for i in range(40):
        hp, hn, hs = (start + i).astype(np.int32), np.ones(2, np.int32), np.arange(3, dtype=np.int32)
        rows = torch.tensor([i, 40 + i], device="cuda")
        k, v = c.k_new[rows].contiguous(), c.v_new[rows].contiguous()
        want = []
        for plane, is_k, x in zip(c.planes, (True, False), (k, v)):
            b = plane.cpu().numpy().copy()
            for r in range(2):
                O.write_tokens(b, c.h_table[r], int(hp[r]), c.host(x)[r:r + 1], is_k)
            want.append(b)
        dev = [torch.from_numpy(a).cuda() for a in (hp, hn, hs)]
        batch = B.make_batch(2, c.h_table.shape[1], *dev, c.dev[3], hp, hn, hs, c.h_table)
        B.ragc_kv8_append(c.pool, batch, None, None, k, v, None, 0, _stream())
        for got, w in zip(c.planes, want):
            assert np.array_equal(got.cpu().numpy(), w), i


def test_kv8_append_of_zeros_tiny_huge_and_what_is_not_finite():
    c = Case([(0, 48), (6, 20)], 1, 2, 128, seed=4)
    k = c.k_new.float()
    k[0:16] = 0
    k[16:32] *= 2.0**-130          # below the smallest scale: subnormal codes and zeros
    k[32:48] *= 2.0**125
    k[50, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0])
    k[55] = float("nan")           # a whole token
    c.k_new.copy_(k)
    c.v_new.copy_(k.flip(-1))
    want = c.appended8(c.host(c.k_new), c.host(c.v_new))
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    for got, w in zip(c.planes, want):
        assert np.array_equal(got.cpu().numpy(), w)


def test_appends_follow_the_device_arrays_when_a_graph_is_replayed():
    """A decode step captured once: prefix_len moves on between the replays, new_len stays.  Every request has blocks of its
    own for the tokens of all steps, as the calls require."""
    c = Case([(p, 1) for p in (0, 14, 15, 100)], 8, 2, 128, seed=5, room=4)
    t = Case([(p, 1) for p in (0, 14, 15, 100)], 8, 2, 128, "bf16", seed=5, room=4)
    cs = O.angles(200, 128)
    dev = torch.from_numpy(cs).cuda()
    rope = B.make_rope(dev, 200, 128)
    q_out = torch.empty_like(c.q)
    tq, tk = torch.empty_like(t.q), torch.empty_like(t.k_new)

    def calls(s):
        B.ragc_kv8_append(c.pool, c.batch, rope, c.q, c.k_new, c.v_new, q_out, 8, s)
        B.ragc_kv_append_rope(t.pool, t.batch, rope, t.q, t.k_new, t.v_new, tq, tk, 8, s)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(side.cuda_stream)
    first = c.h_prefix.copy()
    for step in range(4):
        for x in (c, t):
            x.h_prefix[:] = first + step
            x.dev[0].copy_(torch.from_numpy(x.h_prefix))
            for rows in (x.q, x.k_new, x.v_new):
                rows.normal_()
        want = c.appended8(c.rotated(c.host(c.k_new), cs, False), c.host(c.v_new))
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(c.planes, want):
            assert np.array_equal(got.cpu().numpy(), w)
        qr = c.rotated(c.host(c.q), cs, False)
        _near(c.host(q_out), qr, _sides(c.host(c.q), cs, False, c), "bf16")
        eager_q, eager_k = torch.empty_like(tq), torch.empty_like(tk)
        pools = [p.clone() for p in t.planes]
        B.ragc_kv_append_rope(t.pool, t.batch, rope, t.q, t.k_new, t.v_new, eager_q, eager_k, 8, _stream())
        assert torch.equal(eager_q, tq) and torch.equal(eager_k, tk)
        for a, b in zip(pools, t.planes):
            assert torch.equal(a, b)


def test_swap_moves_8_bit_blocks_with_their_scales():
    c = Case([(64, 1)], 4, 3, 64, seed=6)
    need = O.block_bytes(3, 64)
    host = [torch.zeros(6, need, dtype=torch.uint8).pin_memory() for _ in range(2)]
    before = [p.clone() for p in c.planes]
    ids, slots = np.array([4, 1, 2], np.int32), np.array([0, 5, 3], np.int32)
    for flags in (B.RAGC_SWAP_KERNEL, B.RAGC_SWAP_MEMCPY):
        for x in host:
            x.zero_()
        B.ragc_kv_swap(c.pool, *host, need, 6, ids, slots, B.RAGC_SWAP_TO_HOST, flags, _stream())
        torch.cuda.synchronize()
        for h, b in zip(host, before):
            assert torch.equal(h[slots.tolist()], b[ids.tolist(), :need].cpu()) and not h[[1, 2, 4]].any()
        for p in c.planes:
            p[ids.tolist()] = 0
        B.ragc_kv_swap(c.pool, *host, need, 6, ids, slots, B.RAGC_SWAP_TO_DEVICE, flags, _stream())
        torch.cuda.synchronize()
        for p, b in zip(c.planes, before):
            assert torch.equal(p, b)


def test_append_rope_then_prefill_attention_is_attention_over_rotated_rows():
    """The run of the two as a server uses them: turned in place, stored, then attended to."""
    from oracle import attention as OA

    c = Case([(40, 21), (0, 33), (130, 1)], 8, 2, 128, "bf16", seed=8)
    cs, keep, rope = _rope(c, 128, False)
    B.ragc_kv_append_rope(c.pool, c.batch, rope, c.q, c.k_new, c.v_new, c.q, c.k_new, 8, _stream())
    out = torch.empty_like(c.q)
    B.ragc_prefill_attn(c.pool, c.batch, c.q, c.k_new, c.v_new, out, 8, 128**-0.5, 0, None, 0, _stream())
    torch.cuda.synchronize()
    tiles = [c.host(p)[:, :2 * 16 * 128].reshape(-1, 2, 16, 128) for p in c.planes]
    for r, p, n, rows in c.spans():
        pos = np.arange(p + n)
        k, v = (x[c.h_table[r, pos // 16], :, pos % 16] for x in tiles)
        want = OA.prefill_attn(c.host(c.q)[rows], k, v, p, 128**-0.5)
        assert np.max(np.abs(c.host(out)[rows] - want)) <= 2e-2


# ---- attention ------------------------------------------------------------------------------
# Against exact arithmetic on the same bytes.  Probabilities are rounded to bf16 (2^-9 relative each on average over many, 2^-8 at most)
# and so is the output: |error| <= 2^-8 |out| + 2^-8 sum_j p_j |v_j|, plus the scores' own error in the exponent.  With e4m3 K and bf16 Q
# as two e4m3 numbers the matrix unit keeps 16 bits below the largest product of a group of 16: at most 16 * 2^-16 of sum |q k| per
# score, times scale, and twice that (numerator and denominator) of sum_j p_j |v_j|.
def _attention(c, q, scale):
    """(exact output, bound of the error), [rows, q_heads, head_dim]."""
    want, tol = np.zeros((c.rows, c.hq, c.d)), np.zeros((c.rows, c.hq, c.d))
    planes = [p.cpu().numpy() for p in c.planes]
    for r, p, n, rows in c.spans():
        k, v = (O.read_tokens(x, c.h_table[r], p + n, c.hkv, c.d, is_k) for x, is_k in zip(planes, (True, False)))
        hidden = np.arange(p + n)[None] > p + np.arange(n)[:, None]
        for h in range(c.hq):
            g = h // (c.hq // c.hkv)
            x = q[rows, h]
            s = np.where(hidden, -np.inf, scale * (x @ k[:, g].T))
            e = np.exp(s - s.max(-1, keepdims=True))
            w = e / e.sum(-1, keepdims=True)
            vv = np.where(np.isnan(v[:, g]), 0.0, v[:, g])
            seen_nan = (~hidden).astype(float) @ np.isnan(v[:, g])
            want[rows, h] = np.where(seen_nan > 0, np.nan, w @ vv)
            off = scale * 2.0**-12 * np.where(hidden, 0.0, np.abs(x) @ np.abs(k[:, g]).T).max(-1, keepdims=True)
            tol[rows, h] = 2.0**-8 * np.abs(want[rows, h]) + (2.0**-8 + 2 * off) * (w @ np.abs(vv)) + 1e-30
    return want, tol


def _run(c, scale, flags=0, q=None, out=None):
    need = B.ragc_kv8_attn_workspace(c.pool, c.batch, c.hq, flags)
    ws = torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda")  # NaN everywhere: nothing may be read before it is written
    out = torch.full_like(c.q, 7.0) if out is None else out
    B.ragc_kv8_attn(c.pool, c.batch, c.q if q is None else q, out, c.hq, scale, flags, ws, need, _stream())
    torch.cuda.synchronize()
    return out


def _check(c, scale, flags=0):
    want, tol = _attention(c, c.host(c.q), scale)
    out = _run(c, scale, flags)
    got = c.host(out)[c.first:]
    want, tol = want[c.first:], tol[c.first:]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    worst = float(np.nanmax(np.abs(got - want) / tol)) if not np.isnan(want).all() else 0.0
    assert worst <= 1
    assert torch.all(out[:c.first] == 7)
    again = _run(c, scale, flags)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))  # the order of sums is fixed
    return out


ATTN = {
    "steps": [(int(p), 1) for p in np.random.Generator(np.random.PCG64(2)).integers(0, 600, 70)],
    "one": [(0, 1)],
    "short": [(15, 1), (16, 1), (31, 1), (32, 1), (33, 1), (0, 2), (14, 3), (0, 0), (255, 1)],
    "few": [(40, 4), (513, 3), (0, 7), (1000, 5)],
    "questions": [(100, 33), (0, 40), (47, 17), (260, 1), (15, 64)],
    "prompts": [(0, 300), (301, 129), (64, 64), (1000, 200), (3, 1)],
    "crowd": [(int(p), 17 + int(p) % 23) for p in np.random.Generator(np.random.PCG64(3)).integers(0, 300, 40)],
    "long_step": [(9000, 1), (300, 1)],
    "long_question": [(5000, 19)],
}
HEADS = [(8, 2, 128), (4, 4, 64), (7, 1, 128), (28, 4, 64), (16, 1, 128), (20, 1, 64), (3, 3, 128), (64, 8, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("lens", list(ATTN))
def test_kv8_attention(lens, hq, hkv, d):
    c = Case(ATTN[lens], hq, hkv, d, seed=hq, pad=hkv % 3, first_row=hkv % 2)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    _check(c, d**-0.5)


@pytest.mark.parametrize("lens", ["long_step", "long_question", "few"])
def test_kv8_attention_without_a_split(lens):
    c = Case(ATTN[lens], 8, 2, 128, seed=9)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    assert B.ragc_kv8_attn_workspace(c.pool, c.batch, 8, B.RAGC_ATTN_NO_SPLIT) == 0
    _check(c, 128**-0.5, B.RAGC_ATTN_NO_SPLIT)


@pytest.mark.parametrize("lens", ["steps", "few", "questions", "prompts", "long_step", "long_question"])
@pytest.mark.parametrize("d", [64, 128])
def test_kv8_attention_with_a_sharp_softmax(lens, d):
    """Scores of some tens: the running reference is raised often."""
    c = Case(ATTN[lens], 8, 2, d, seed=10)
    c.fill_prefixes()
    c.q.mul_(6.0)
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    _check(c, d**-0.5)


@pytest.mark.parametrize("lens", ["short", "few", "questions", "prompts", "long_step"])
@pytest.mark.parametrize("d", [64, 128])
def test_kv8_attention_nan_goes_to_the_rows_that_see_it(lens, d):
    """NaN in V of every request's fourth token from the end and in K of another's; slots behind the last token are NaN too."""
    c = Case(ATTN[lens], 8, 2, d, seed=11)
    c.fill_prefixes()
    for r, (p, n) in enumerate(zip(c.h_prefix, c.h_new)):
        at = int(c.h_start[r]) + int(n) - 4
        if n >= 4:
            c.v_new[at, 0, 5] = float("nan")
            c.v_new[at + 2, 1] = float("nan")
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    planes = [p.cpu().numpy() for p in c.planes]
    for plane, is_k in zip(planes, (True, False)):
        order = O.byte_of(d, is_k)
        for r, (p, n) in enumerate(zip(c.h_prefix, c.h_new)):
            end = int(p) + int(n)
            if end % 16:
                for h in range(2):
                    plane[c.h_table[r, end // 16], h * 16 * d + order[end % 16:]] = 0x7F
    for plane, host in zip(c.planes, planes):
        plane.copy_(torch.from_numpy(host))
    _check(c, d**-0.5)


def test_kv8_attention_nan_in_k_reaches_the_rows_that_see_the_key():
    c = Case([(20, 50)], 4, 2, 128, seed=12)
    c.fill_prefixes()
    c.k_new[30, 1] = float("nan")
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    out = c.host(_run(c, 128**-0.5))
    assert not np.isnan(out[:30]).any() and np.isnan(out[30:, 2:]).all() and not np.isnan(out[30:, :2]).any()


@pytest.mark.parametrize("lens", ["few", "prompts"])
def test_kv8_attention_scales_of_all_sizes(lens):
    """Blocks of very different magnitude next to each other; q is small where K is large."""
    c = Case(ATTN[lens], 4, 2, 64, seed=13)
    sat = 2 * 16 * 64
    for plane in c.planes:
        plane[:, :sat] &= 0xF7  # no NaN codes
    c.planes[0][:, sat:sat + 2] = torch.from_numpy(c.rng.integers(95, 160, (c.blocks, 2)).astype(np.uint8)).cuda()
    c.planes[1][:, sat:sat + 2] = torch.from_numpy(c.rng.integers(60, 200, (c.blocks, 2)).astype(np.uint8)).cuda()
    c.q.mul_(2.0**-38)
    _check(c, 0.125)


def test_kv8_append_then_attention_equals_one_prefill():
    """The run of the two as a server uses them: a prompt at once, or its first part, then the rest token by token.  The scales of partly
    filled blocks may come about differently, so the second way is compared with the oracle on its own bytes and with the first loosely."""
    whole = Case([(0, 45)], 8, 2, 128, seed=14, room=16)
    cs, keep, rope = _rope(whole, 128, False)
    q0 = whole.q.clone()
    q = torch.empty_like(q0)
    B.ragc_kv8_append(whole.pool, whole.batch, rope, q0, whole.k_new, whole.v_new, q, 8, _stream())
    whole.q.copy_(q)
    once = _check(whole, 128**-0.5)
    parts = Case([(0, 45)], 8, 2, 128, seed=14, room=16)
    got = []
    for lo, hi in [(0, 30)] + [(i, i + 1) for i in range(30, 45)]:
        hp, hn, hs = (np.asarray(x, np.int32) for x in ([lo], [hi - lo], [0, hi - lo]))
        dev = [torch.from_numpy(a).cuda() for a in (hp, hn, hs)]
        batch = B.make_batch(1, parts.h_table.shape[1], *dev, parts.dev[3], hp, hn, hs, parts.h_table)
        qq, out = torch.empty_like(q0[lo:hi]), torch.empty_like(q0[lo:hi])
        B.ragc_kv8_append(parts.pool, batch, rope, q0[lo:hi], parts.k_new[lo:hi], parts.v_new[lo:hi], qq, 8, _stream())
        assert torch.equal(qq, q[lo:hi])
        B.ragc_kv8_attn(parts.pool, batch, qq, out, 8, 128**-0.5, 0, None, 0, _stream())
        got.append(out)
    got = torch.cat(got).double()
    assert float((got - once.double()).norm() / once.double().norm()) < 2e-2


def test_kv8_attention_on_streams_and_in_a_graph():
    """Two batches on two streams with workspaces of their own, and a captured call replayed over changed bytes and tables."""
    cases = [Case([(3000, 1), (70, 1)], 8, 2, 128, seed=15), Case([(2500, 2), (9, 1)], 8, 2, 64, seed=16)]
    streams, outs, spaces = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for c in cases:
        c.fill_prefixes()
        B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
        spaces.append(torch.empty(max(1, B.ragc_kv8_attn_workspace(c.pool, c.batch, c.hq)), dtype=torch.uint8, device="cuda"))
        outs.append(torch.empty_like(c.q))
    want = [_run(c, 0.1) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s, o, w in zip(cases, streams, outs, spaces):
            B.ragc_kv8_attn(c.pool, c.batch, c.q, o, c.hq, 0.1, 0, w, w.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
    c, space = cases[0], spaces[0]
    side, graph, out = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.empty_like(c.q)
    with torch.cuda.graph(graph, stream=side):
        B.ragc_kv8_attn(c.pool, c.batch, c.q, out, c.hq, 0.1, 0, space, space.numel(), side.cuda_stream)
    for _ in range(3):
        c.q.normal_()
        c.dev[3][0, :50] = c.dev[3][0, :50].flip(0)  # other blocks, as far as the replay is concerned
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _run(c, 0.1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,waves,chunk", [(r, w, c) for r in (16, 32, 128) for w in (4, 8) for c in (0, 16, 48)])
def test_kv8_attention_in_every_layout(rows, waves, chunk, d):
    """Every kernel on lengths that end inside its tiles, split and whole: copies without a key for some rows, and more of them than keys."""
    c = Case([(700, 37), (15, 1), (0, 130), (1030, 3), (255, 16), (2100, 1)], 8, 2, d, seed=17, pad=1, first_row=1)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        _check(c, d**-0.5)
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("rows,waves", [(r, w) for r in (16, 32, 128) for w in (4, 8)])
def test_kv8_attention_nan_in_every_layout(rows, waves):
    c = Case([(700, 37), (20, 130)], 8, 2, 128, seed=18)
    c.fill_prefixes()
    for at in (3, 20, 36, 37 + 64, 37 + 128):
        c.v_new[at, 0, 7 * at % 128] = float("nan")
        c.v_new[at, 1, 127] = float("inf")
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    try:
        for chunk in (0, 16):
            B.ragc_debug_set_kv8_plan(rows, waves, chunk)
            _check(c, 128**-0.5)
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("chunk", [0, 16])
def test_kv8_attention_of_more_requests_than_an_argument_list_holds(chunk):
    g = np.random.Generator(np.random.PCG64(19))
    c = Case([(int(p), int(n)) for p, n in zip(g.integers(0, 700, 200), g.integers(0, 4, 200))], 4, 2, 64, seed=20)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    try:
        if chunk:
            B.ragc_debug_set_kv8_plan(16, 8, chunk)
        _check(c, 0.125)
    finally:
        B.ragc_debug_set_kv8_plan(0)


def test_kv8_calls_without_host_arrays_and_with_validation():
    c = Case([(33, 7), (0, 18)], 8, 2, 128, seed=21)
    c.fill_prefixes()
    bare = B.make_batch(2, c.h_table.shape[1], *c.dev, None, None, None, None)  # lengths are read back
    want = c.appended8(c.host(c.k_new), c.host(c.v_new))
    B.ragc_kv8_append(c.pool, bare, None, None, c.k_new, c.v_new, None, 0, _stream())
    for got, w in zip(c.planes, want):
        assert np.array_equal(got.cpu().numpy(), w)
    out = torch.empty_like(c.q)
    B.ragc_kv8_attn(c.pool, bare, c.q, out, 8, 0.1, B.RAGC_ATTN_VALIDATE, None, 0, _stream())
    torch.cuda.synchronize()
    assert torch.equal(out, _run(c, 0.1))
    B.ragc_batch_validate(c.pool, c.batch, True)
    c.dev[3][1, 0] = c.blocks  # the device's table names a block that does not exist: found before anything is launched
    with pytest.raises(B.RagcError) as e:
        B.ragc_kv8_attn(c.pool, c.batch, c.q, out, 8, 0.1, B.RAGC_ATTN_VALIDATE, None, 0, _stream())
    assert e.value.code == B.RAGC_ERR_RANGE
    with pytest.raises(B.RagcError):
        B.ragc_batch_validate(c.pool, c.batch, True)


def test_kv8_calls_leave_other_blocks_and_rows_alone():
    """A batch in the middle of packed arrays and of a pool: nothing outside it changes."""
    c = Case([(20, 9), (64, 33)], 8, 2, 128, seed=22, pad=2, first_row=4, spare=20)
    c.fill_prefixes()
    before = [p.clone() for p in c.planes]
    cs, keep, rope = _rope(c, 128, False)
    q = c.q.clone()
    B.ragc_kv8_append(c.pool, c.batch, rope, c.q, c.k_new, c.v_new, c.q, 8, _stream())  # Q in place
    out = torch.full((c.rows + 6, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    _run(c, 0.1, out=out)
    assert torch.all(out[:4] == 7) and torch.all(out[c.rows:] == 7) and torch.equal(c.q[:4], q[:4])
    used = set()
    for r, p, n, _ in c.spans():
        used |= set(c.h_table[r, p // 16:-(-(p + n) // 16)].tolist())
    others = [b for b in range(c.blocks) if b not in used]
    for a, b in zip(before, c.planes):
        assert torch.equal(a[others], b[others]) and torch.equal(a[:, -32:], b[:, -32:])


def test_kv8_attention_in_two_graphs_replayed_in_turn():
    """Two captured calls with workspaces of their own and eager work between their replays."""
    cases, graphs, outs, spaces = [Case([(2000 + 300 * i, 1), (40, 70)], 8, 2, 128, seed=23 + i) for i in range(2)], [], [], []
    for c in cases:
        c.fill_prefixes()
        B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
        B.ragc_debug_set_kv8_plan(32, 8, 32)
        need = B.ragc_kv8_attn_workspace(c.pool, c.batch, 8)
        assert need > 0
        spaces.append(torch.empty(need, dtype=torch.uint8, device="cuda"))
        outs.append(torch.empty_like(c.q))
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.ragc_kv8_attn(c.pool, c.batch, c.q, outs[-1], 8, 0.1, 0, spaces[-1], need, side.cuda_stream)
        graphs.append(graph)
    try:
        for turn in range(3):
            for c, graph, out in zip(cases, graphs, outs):
                c.q.normal_()
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, _run(c, 0.1))
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("dtype", ["e4m3", "bf16"])
def test_blocks_behind_the_first_four_gib_of_a_plane(dtype):
    """The same blocks 128 MiB apart: offsets that 32 bits do not hold, in every call and kernel."""
    c = Case([(200, 17), (300, 1), (61, 40)], 8, 2, 128, dtype, seed=29)
    if dtype == "e4m3":
        c.fill_prefixes()
    size, stride = c.planes[0].element_size(), (1 << 27) // c.planes[0].element_size()
    assert int(c.h_table.max()) * (1 << 27) > 1 << 32
    far = [torch.empty(c.blocks * stride, dtype=p.dtype, device="cuda").view(c.blocks, stride) for p in c.planes]
    for f, p in zip(far, c.planes):
        f[:, :c.stride] = p
    pool = B.make_pool(*far, c.blocks, 2, 128, c.pool.dtype, stride)
    cs, keep, rope = _rope(c, 128, False)
    q_out = [torch.empty_like(c.q) for _ in range(2)]
    for p, q in zip((c.pool, pool), q_out):
        if dtype == "e4m3":
            B.ragc_kv8_append(p, c.batch, rope, c.q, c.k_new, c.v_new, q, 8, _stream())
        else:
            B.ragc_kv_append_rope(p, c.batch, rope, c.q, c.k_new, c.v_new, q, None, 8, _stream())
    torch.cuda.synchronize()
    bits = torch.uint8 if size == 1 else torch.int16
    assert torch.equal(q_out[0].view(torch.int16), q_out[1].view(torch.int16))
    for f, p in zip(far, c.planes):
        assert torch.equal(f[:, :c.stride].contiguous().view(bits), p.contiguous().view(bits))
    if dtype == "bf16":
        return
    try:
        for plan in [(16, 8, 0), (16, 4, 16), (32, 4, 0), (128, 4, 0), (128, 8, 16)]:
            B.ragc_debug_set_kv8_plan(*plan)
            need = B.ragc_kv8_attn_workspace(c.pool, c.batch, 8)
            ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
            outs = [torch.empty_like(c.q) for _ in range(2)]
            for p, o in zip((c.pool, pool), outs):
                B.ragc_kv8_attn(p, c.batch, q_out[0], o, 8, 0.1, 0, ws, need, _stream())
            torch.cuda.synchronize()
            assert not torch.isnan(outs[0]).any() and torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("rows,waves,chunk", [(16, 4, 0), (16, 8, 16), (32, 4, 16), (128, 4, 0), (128, 8, 0), (128, 8, 16)])
@pytest.mark.filterwarnings("ignore:invalid value")
def test_kv8_attention_rows_of_q_that_are_not_finite_stay_alone(rows, waves, chunk):
    c = Case([(300, 40), (17, 1), (0, 3)], 8, 2, 64, seed=31)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    c.q[3, 1, 5] = float("nan")
    c.q[20, 7, 60] = float("inf")
    c.q[40, 0, 0] = -float("inf")
    c.q[42, 2, :] = 0.0
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        _check(c, 0.125)
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("steps", [3, 7, 16, 17, 19, 23])
def test_kv8_attention_key_loops_that_end_anywhere_in_a_window(steps, split, d):
    """128 rows, two wave groups, a tile of 64 keys each per step: loops that end where block ids or scales of steps 16 on would be
    asked for (3, 7, 19, 23) and around the change of windows, with and without a last tile for the second group; whole and as the last copy."""
    chunk = 16 * -(-steps // 2) if split else 0  # blocks: at least as many steps as the last copy has
    keys = [16 * chunk + 128 * steps, 16 * chunk + 128 * steps - 64 - 9]
    c = Case([(k - n, n) for k, n in zip(keys, (40, 33))], 8, 2, d, seed=steps)
    c.fill_prefixes()
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    try:
        B.ragc_debug_set_kv8_plan(128, 8, chunk)
        assert B.ragc_debug_get_kv8_plan(c.pool, c.batch, 8) == (128, 8, chunk)
        _check(c, d**-0.5)
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("rows,waves,chunk", [(r, w, c) for r in (16, 32, 128) for w in (4, 8) for c in (0, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_kv8_attention_numbers_that_bf16_does_not_hold_count_only_where_they_are_seen(rows, waves, chunk, d):
    """V of 2^128 and above: the largest bf16 numbers round up to it, and scale bytes above 246 reach further.  A row that sees one
    has an infinity or NaN in its column; nothing comes to any other row or column."""
    c = Case([(300, 37), (20, 130), (47, 2)], 8, 2, d, seed=33)
    c.fill_prefixes()
    big = float(torch.finfo(torch.bfloat16).max)
    for at in (3, 20, 36, 37 + 64, 37 + 128):
        c.v_new[at, 0, 7 * at % d] = big if at % 2 else -big
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    # the last block of the last request, head 1: of its two new tokens the first has one number just below 2^128, the second others above
    sat, order, tile = 2 * 16 * d, O.byte_of(d, False), c.planes[1][c.h_table[2, 2]]
    tile[16 * d:2 * 16 * d] = 0
    tile[sat + 1] = 254                                   # 2^127
    tile[16 * d + int(order[15, 4])] = 0x3F               # 1.875
    last = c.planes[1][c.h_table[2, 3]]
    last[16 * d:2 * 16 * d] = 0
    last[sat + 1] = 251                                   # 2^124
    for e, code in ((9, 0x58), (d - 1, 0xFE), (17, 0x57)):  # 16, -448, 15
        last[16 * d + int(O.byte_of(d, False)[0, e])] = code
    c.q[-2:, 4:] = 0  # weights of 1 before the division: 1.875 * 2^127 times a larger one would overflow fp32
    want, tol = _attention(c, c.host(c.q), d**-0.5)
    planes, inf = c.planes[1].cpu().numpy(), np.zeros_like(want, bool)
    for r, p, n, at in c.spans():
        v = O.read_tokens(planes, c.h_table[r], p + n, 2, d, False)
        for i in range(n):
            inf[at.start + i] = np.repeat((np.abs(v[:p + i + 1]) >= 2.0**128).any(0), 4, axis=0)
    assert inf[-1, 4:, [9, d - 1]].all() and not inf[-2, 4:].any() and not inf[-1, 4:, 17].any()
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        got = c.host(_run(c, d**-0.5))
    finally:
        B.ragc_debug_set_kv8_plan(0)
    assert np.array_equal(np.isfinite(got), ~inf)
    assert float((np.abs(got - want) / tol)[~inf].max()) <= 1


@pytest.mark.parametrize("rows,waves,chunk", [(16, 8, 0), (32, 4, 0), (128, 4, 0), (128, 8, 0), (128, 8, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_kv8_attention_of_small_numbers_beside_a_large_one(rows, waves, chunk, d):
    """q is 2^15 where K is 0, and between 1 and 1.6 where K is 0 or 4: what decides is 2^-15 of the row's largest number, of which
    the second of two e4m3 numbers keeps steps of 2^-7 of 1.  One key in 100 is of the second kind, V 1 there and -1 elsewhere, so that the weights
    are of one size and the output follows the score by up to half.
    A score is off by at most off = scale (2^-12 sum |q K| + 2^-21 max|q| sum |K|) = 2^-12 * 6.4 + 2^-21 * 2^15 * 4 = 0.064, a weight by a factor of
    e^off, and so are their sums: (e^(2 off) - 1) sum p |v|, with 2^-8 of it for the weights' rounding and 2^-8 of the output for its own."""
    c = Case([(0, 230), (0, 60)], 8, 2, d, seed=35)
    kind = torch.cat([torch.arange(n, device="cuda") % 100 == 0 for n in (230, 60)])
    c.k_new.zero_()
    c.k_new[kind, :, 5] = 4.0
    c.v_new.copy_(torch.where(kind, 1.0, -1.0)[:, None, None].expand_as(c.v_new))
    c.q.copy_(torch.from_numpy(c.rng.uniform(1, 1.6, c.q.shape).astype(np.float32)))
    c.q[:, :, 0] = 2.0**15
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    q = c.host(c.q)
    want, _ = _attention(c, q, 1.0)
    off = 2.0**-12 * 4 * np.abs(q[..., 5:6]) + 2.0**-21 * 2.0**15 * 4
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        got = c.host(_run(c, 1.0))
    finally:
        B.ragc_debug_set_kv8_plan(0)
    assert (np.abs(got - want) <= 2.0**-8 * np.abs(want) + 2.0**-8 + np.expm1(2 * off)).all()
    if rows < 128:  # the products of these are exact: fp32 roundings of an exponent of 9.2 (two) and of exp2 in the weights, twice
        assert (np.abs(got - want) <= 2.0**-8 * np.abs(want) + 2.0**-8 + 4e-6).all()


@pytest.mark.parametrize("rows,waves", [(r, w) for r in (16, 32, 128) for w in (4, 8)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.filterwarnings("ignore:invalid value")
def test_kv8_attention_nan_in_k_in_every_layout(rows, waves, d):
    """A key of one head that is NaN: in the frontier, in an early tile, and a run of 256 of them, so that a copy of 16 blocks and the
    waves in it see nothing else (a sum that is NaN beside a maximum that was never raised)."""
    c = Case([(700, 37), (20, 130), (0, 600)], 8, 2, d, seed=36)
    c.fill_prefixes()
    for at in (30, 37 + 5, 37 + 100):
        c.k_new[at, 0, 7 * at % d] = float("nan")
    c.k_new[167 + 256:167 + 512, 1] = float("nan")
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    want, tol = _attention(c, c.host(c.q), d**-0.5)
    try:
        for chunk in (0, 16):
            B.ragc_debug_set_kv8_plan(rows, waves, chunk)
            got = c.host(_run(c, d**-0.5))
            assert np.array_equal(np.isnan(got), np.isnan(want))
            assert float(np.nanmax(np.abs(got - want) / tol)) <= 1
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("rows,waves,chunk", [(0, 8, 0), (16, 8, 16), (32, 4, 0), (128, 4, 0), (128, 8, 16)])
def test_kv8_attention_of_requests_that_read_the_same_blocks(rows, waves, chunk):
    """Five questions about one document, one of them about its first 20 blocks: its blocks are in every table."""
    lens = [(480, 1), (480, 40), (480, 3), (320, 17), (480, 16)]
    c = Case(lens, 8, 2, 128, seed=37)
    for r, (p, _) in enumerate(lens[1:], 1):
        c.h_table[r, :p // 16] = c.h_table[0, :p // 16]
    c.dev[3].copy_(torch.from_numpy(c.h_table))
    c.fill_prefixes()
    B.ragc_batch_validate(c.pool, c.batch, True)
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        _check(c, 128**-0.5)
    finally:
        B.ragc_debug_set_kv8_plan(0)


@pytest.mark.parametrize("rows,waves,chunk", [(r, w, c) for r in (16, 32, 128) for w in (4, 8) for c in (0, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_kv8_attention_keys_that_bf16_does_not_hold_count_only_where_they_are_seen(rows, waves, chunk, d):
    """K of 2^128 in one head: rows that come before it, and the other head, are as if it were not there."""
    c = Case([(300, 37), (20, 130)], 8, 2, d, seed=38)
    c.fill_prefixes()
    first = {0: 20, 1: 37 + 64}
    for at in (*first.values(), 30, 37 + 128):
        c.k_new[at, 0, 7 * at % d] = float(torch.finfo(torch.bfloat16).max)
    B.ragc_kv8_append(c.pool, c.batch, None, None, c.k_new, c.v_new, None, 0, _stream())
    free = np.ones((c.rows, c.hq), bool)
    for r, _, n, at in c.spans():
        free[first[r]:at.stop, :4] = False
    want, tol = _attention(c, c.host(c.q), d**-0.5)
    try:
        B.ragc_debug_set_kv8_plan(rows, waves, chunk)
        got = c.host(_run(c, d**-0.5))
    finally:
        B.ragc_debug_set_kv8_plan(0)
    assert float((np.abs(got - want) / tol)[free].max()) <= 1
