"""Performance cases of the cache operators with position rotation and of the 8-bit cache, in plain torch and through the
public entry points (`ragc_kv_append_rope`, `ragc_kv8_append`, `ragc_kv8_attn` of the ctypes binding).

A case is a dict of plain values:

    op                    "append" (rotated K and V into a pool of `dtype`, Q rotated by the same call),
                          "append8" (the same into an 8-bit pool) or "attn8" (attention over an 8-bit pool)
    dtype                 "bf16" or "f32" (append): the type of the tensors
    q_heads, kv_heads, head_dim
    rot_dim, interleaved  how many elements of a head turn, and whether neighbours or halves are the pairs   (append, append8)
    requests              requests of the batch
    cached_min/_max       cached tokens per request, drawn from the range
    new_min/_max          new tokens per request, drawn from the range
    lengths               seed of those draws: the lengths belong to the case, not to the inputs

An 8-bit pool holds e4m3 numbers and one power-of-two scale 2^(s-127), s a byte, per block of 16 tokens, plane and head:
s is the smallest with which the largest finite |x| of the block's rows is at most 448.  Rows join a partly filled block at
the larger of its scale and theirs, and what it held is rounded anew to a larger one.  Numbers that are not finite become NaN.
One block of a plane: [kv_heads] tiles of 16 * head_dim bytes, [kv_heads] scale bytes, padding to 16.  A K tile is
[head_dim / 16][token][16], a V tile [head_dim / 64][token / 4][16][4][token % 4] with element 64 * first + 16 * fourth + third.

K and V are of unit variance with queries of standard deviation 2 (a moderately sharp softmax); blocks sit at random places of
the pool, as after hours of evictions.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
POOL_SLACK = 1.25  # pool blocks per block in use
MAX_POOL_BYTES = 1 << 30
ROPE_BASE = 10000.0


def _append(op, dtype, heads, head_dim, requests, cached, new, lengths, rot_dim=None, interleaved=False):
    return dict(op=op, dtype=dtype, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, requests=requests,
                cached_min=cached[0], cached_max=cached[1], new_min=new[0], new_max=new[1], lengths=lengths,
                rot_dim=rot_dim or head_dim, interleaved=interleaved)


def _attn(heads, head_dim, requests, cached, new, lengths):
    return dict(op="attn8", dtype="bf16", q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, requests=requests,
                cached_min=cached[0], cached_max=cached[1], new_min=new[0], new_max=new[1], lengths=lengths)


def listed():
    return [
        # A decode step of a full batch: one token each, 70B-shaped layer.
        dict(_append("append", "bf16", (64, 8), 128, 64, (512, 2048), (1, 1), 1), name="rope_steps"),
        # Freshly computed documents and questions of a loaded server.
        dict(_append("append", "bf16", (32, 8), 128, 16, (256, 4096), (64, 768), 2), name="rope_prompts"),
        # fp32 model with half of each head turned, neighbours as pairs; short and odd lengths.
        dict(_append("append", "f32", (12, 4), 64, 5, (0, 300), (3, 217), 3, 32, True), name="rope_f32_odd"),
        # One token of one request: what a step of a lone user pays.
        dict(_append("append8", "bf16", (32, 32), 128, 1, (1000, 1000), (1, 1), 4), name="append8_token"),
        # A decode step of a full batch.
        dict(_append("append8", "bf16", (64, 8), 128, 64, (512, 2048), (1, 1), 5), name="append8_steps"),
        # Freshly computed documents and questions of a loaded server.
        dict(_append("append8", "bf16", (32, 8), 128, 16, (256, 4096), (64, 768), 6), name="append8_prompts"),
        # The first answer token over one short document: latency alone.
        dict(_attn((32, 8), 128, 1, (300, 300), (1, 1), 7), name="attn8_token"),
        # A decode step over one very long context.
        dict(_attn((64, 8), 128, 1, (100003, 100003), (1, 1), 8), name="attn8_long_step"),
        # A decode step of a full batch of ragged requests, 70B-shaped layer.
        dict(_attn((64, 8), 128, 64, (512, 2048), (1, 1), 9), name="attn8_steps"),
        # A loaded server: ragged requests, one to many documents, some of them just computed.
        dict(_attn((32, 8), 128, 16, (256, 4096), (64, 768), 10), name="attn8_ragged"),
        # Questions over long cached prefixes, 70B-shaped layer.
        dict(_attn((64, 8), 128, 4, (4096, 4096), (128, 128), 11), name="attn8_long_prefix"),
        # Models with head dimension 64, ragged.
        dict(_attn((32, 8), 64, 8, (300, 2000), (50, 300), 12), name="attn8_d64"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    """A range of lengths: one length for all requests, or up to a factor of four between them."""
    top = _log_int(rng, lo, hi)
    return (top, top) if rng.random() < 0.4 else (max(lo, top // rng.randint(2, 4)), top)


def draw(rng):
    most = {op: max(work(c)[unit] for c in listed() if c["op"] == op)
            for op, unit in (("append", "bytes"), ("append8", "bytes"), ("attn8", "flops"))}
    op = rng.choice(["append", "append8", "attn8", "attn8"])
    decode = rng.random() < 0.5
    while True:
        heads = rng.choice([(32, 32), (32, 8), (64, 8), (8, 2), (16, 16), (12, 4), (28, 4), (16, 1)])
        head_dim = rng.choice([64, 128, 128])
        lengths = rng.randint(100, 10**6)
        requests = _log_int(rng, 1, 128 if decode else 32)
        cached = (0, 0) if not decode and rng.random() < 0.15 else _span(rng, 16, 100000 if decode else 8192)
        new = (1, 1) if decode else _span(rng, 2, 4096)
        if op == "attn8":
            case = _attn(heads, head_dim, requests, cached, new, lengths)
            fits = work(case)["flops"] <= most[op] and _plain_bytes(case) <= 8 << 30
        else:
            case = _append(op, "bf16" if op == "append8" else rng.choice(["bf16", "bf16", "f32"]), heads, head_dim, requests,
                           cached, new, lengths, rng.choice([head_dim, head_dim, head_dim // 2, 16]), rng.random() < 0.3)
            fits = work(case)["bytes"] <= most[op]
        if fits and _pool_bytes(case) <= MAX_POOL_BYTES:
            return case


# ---- the batch of a case --------------------------------------------------------------------
def _lens(case):
    rng = random.Random(case["lengths"])
    cached = [rng.randint(case["cached_min"], case["cached_max"]) for _ in range(case["requests"])]
    new = [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["requests"])]
    return cached, new


def _esize(case):
    return 1 if case["op"] != "append" else 2 if case["dtype"] == "bf16" else 4


def _blocks(case):
    return sum(-(-(p + n) // BLOCK) for p, n in zip(*_lens(case)))


def _pool_bytes(case):
    return int(_blocks(case) * POOL_SLACK) * 2 * case["kv_heads"] * BLOCK * case["head_dim"] * _esize(case)


def _plain_bytes(case):
    """The scores of the plain form, padded to the longest request."""
    cached, new = _lens(case)
    return 4 * case["requests"] * case["q_heads"] * max(new) * max(p + n for p, n in zip(cached, new))


def work(case):
    """append, append8: K, V, Q and a row of cos and sin per token read once, K, V (with a scale byte per block and head in 8
    bits) and Q written once, one table entry per block; 6 flop per pair.  attn8: the cache, its scales, Q and the table
    read once, the output written once; two products of 2 flop per visible (query, key) pair and element."""
    cached, new = _lens(case)
    d, hq, hkv, total = case["head_dim"], case["q_heads"], case["kv_heads"], sum(new)
    if case["op"] == "attn8":
        named = _blocks(case)
        nbytes = 2 * hkv * d * (sum(cached) + total) + 2 * hkv * named + 4 * named + 2 * 2 * hq * d * total
        pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(cached, new))
        return {"bytes": nbytes, "flops": 4 * d * hq * pairs}
    e = 2 if case["dtype"] == "bf16" else 4
    touched = sum(-(-(p + n) // BLOCK) - p // BLOCK for p, n in zip(cached, new))
    nbytes = total * (2 * hkv * d * (e + _esize(case)) + 2 * hq * d * e + 4 * case["rot_dim"]) + 4 * touched
    if case["op"] == "append8":
        nbytes += 2 * hkv * touched
    return {"bytes": nbytes, "flops": 3 * case["rot_dim"] * (hq + hkv) * total}


# ---- inputs ---------------------------------------------------------------------------------
class _State:
    """What a server has in hand before the call: the pool, the packed tensors, the batch and its host copies."""


def _scale_of(amax):
    """The scale byte for a largest value in 64 bits: 448 = 1.75 * 2^8, amax = m * 2^x with 1 <= m < 2."""
    m, x = torch.frexp(amax.double())  # 0.5 <= m < 1
    s = x - 1 - 8 + (m > 0.875).int() + 127
    return torch.where(amax > 0, s.clamp(1, 254), 1)


def _to_e4m3(x):
    """Nearest e4m3 number in 64 bits, ties to the even one, |x| <= 448; not finite: NaN."""
    fine = torch.isfinite(x)
    x = torch.where(fine, x, 0.0).double()
    step = torch.exp2((torch.frexp(x).exponent - 1).clamp(min=-6).double() - 3)
    return torch.where(fine, torch.round(x / step) * step, float("nan"))


def _tiles(plane, case):
    """The code bytes of a plane, [blocks, kv_heads, 16 * head_dim], and its scale bytes, [blocks, kv_heads]."""
    h, tile = case["kv_heads"], BLOCK * case["head_dim"]
    return plane[:, :h * tile].unflatten(1, (h, tile)), plane[:, h * tile:h * tile + h]


def _pack(x, is_k):
    """[..., token, head_dim] -> [..., 16 * head_dim] in a tile's order."""
    d = x.shape[-1]
    if is_k:
        return x.unflatten(-1, (d // 16, 16)).transpose(-3, -2).flatten(-3)
    x = x.unflatten(-1, (d // 64, 4, 16)).unflatten(-4, (4, 4))  # [..., token / 4, token % 4, d / 64, d % 64 / 16, d % 16]
    return x.movedim((-3, -5, -1, -2, -4), (-5, -4, -3, -2, -1)).flatten(-5)


def _unpack(tile, is_k):
    """[..., 16 * head_dim] in a tile's order -> [..., token, head_dim]."""
    d = tile.shape[-1] // BLOCK
    if is_k:
        return tile.unflatten(-1, (d // 16, 16, 16)).transpose(-3, -2).flatten(-2)
    x = tile.unflatten(-1, (d // 64, 4, 16, 4, 4))
    return x.movedim((-5, -4, -3, -2, -1), (-3, -5, -1, -2, -4)).flatten(-3).flatten(-3, -2)


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    place = np.random.Generator(np.random.PCG64(seed))
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    cached, new = _lens(case)
    num_blocks = int(_blocks(case) * POOL_SLACK) + 2
    if case["op"] == "append":
        s.planes = [normal(num_blocks, hkv, BLOCK, d).to(dtype) for _ in range(2)]
    else:
        stride = hkv * BLOCK * d + -(-hkv // 16) * 16
        s.planes = [torch.zeros(num_blocks, stride, dtype=torch.uint8, device="cuda") for _ in range(2)]
        for plane in s.planes:
            codes, scales = _tiles(plane, case)
            x = normal(num_blocks, hkv, BLOCK * d)
            scale = _scale_of(x.abs().amax(-1))
            scales.copy_(scale)
            codes.copy_((x * torch.exp2(127.0 - scale)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8))
    ids = place.permutation(num_blocks).astype(np.int32)
    stride = max(-(-(p + n) // BLOCK) for p, n in zip(cached, new))
    table = np.zeros((len(cached), stride), np.int32)
    at = 0
    for r, (p, n) in enumerate(zip(cached, new)):
        need = -(-(p + n) // BLOCK)
        table[r, :need] = ids[at:at + need]
        at += need
    s.h = [np.asarray(cached, np.int32), np.asarray(new, np.int32), np.concatenate([[0], np.cumsum(new)]).astype(np.int32), table]
    s.d = [torch.from_numpy(a).cuda() for a in s.h]
    total = sum(new)
    s.q = (2.0 * normal(total, hq, d)).to(dtype)
    s.out = torch.empty_like(s.q)
    if case["op"] == "attn8":
        s.scale = 1.0 / math.sqrt(d)
    else:
        s.k_new, s.v_new = normal(total, hkv, d).to(dtype), normal(total, hkv, d).to(dtype)
        last = max(p + n for p, n in zip(cached, new))
        freq = ROPE_BASE ** (-torch.arange(0, case["rot_dim"], 2, dtype=torch.float64) / case["rot_dim"])
        angle = torch.arange(last, dtype=torch.float64)[:, None] * freq
        s.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
    if own:
        from paper_2404_12457_amd import binding

        wide = binding.RAGC_DTYPE_BF16 if case["dtype"] == "bf16" else binding.RAGC_DTYPE_F32
        code = wide if case["op"] == "append" else binding.RAGC_DTYPE_E4M3
        s.pool = binding.make_pool(*s.planes, num_blocks, hkv, d, code, s.planes[0].stride(0))
        s.batch = binding.make_batch(len(cached), stride, *s.d, *s.h)
        if case["op"] == "attn8":
            need = binding.ragc_kv8_attn_workspace(s.pool, s.batch, hq)
            s.workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        else:
            s.rope = binding.make_rope(s.cos_sin, last, case["rot_dim"], case["interleaved"])
    return s


# ---- the plain forms ------------------------------------------------------------------------
def _rotate(x, pos, cos_sin, interleaved):
    """x [rows, heads, head_dim] turned by the angles of its rows' positions."""
    rot = cos_sin.shape[1]
    cos, sin = cos_sin[pos].to(x.dtype)[:, None].chunk(2, -1)
    turned, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, rest], -1)


def _rows(s):
    """Request, position and block of every packed row."""
    prefix, new, start, table = s.d
    req = torch.repeat_interleave(torch.arange(len(s.h[0]), device="cuda"), new.long(), output_size=len(s.q))
    pos = prefix.long()[req] + torch.arange(len(s.q), device="cuda") - start.long()[req]
    return req, pos, table[req, pos // BLOCK].long()


def _plain_append(s):
    _, pos, block = _rows(s)
    inter = s.case["interleaved"]
    s.out.copy_(_rotate(s.q.float(), pos, s.cos_sin, inter))
    s.planes[0][block, :, pos % BLOCK] = _rotate(s.k_new.float(), pos, s.cos_sin, inter).to(s.q.dtype)
    s.planes[1][block, :, pos % BLOCK] = s.v_new


def _plain_append8_plane(s, plane, x, is_k, pos, block, page, pages, held):
    """x [rows, kv_heads, head_dim] in 64 bits into the 8-bit plane.  page: which of the written blocks a row joins;
    pages: those blocks; held: how many tokens each of them holds already."""
    codes, scales = _tiles(plane, s.case)
    tile = torch.zeros(len(pages), x.shape[1], BLOCK, x.shape[2], dtype=torch.float64, device="cuda")
    tile[page, :, pos % BLOCK] = x
    fresh = torch.zeros(len(pages), BLOCK, dtype=torch.bool, device="cuda")
    fresh[page, pos % BLOCK] = True
    old = torch.arange(BLOCK, device="cuda") < held[:, None]
    before = scales[pages].int()
    scale = _scale_of(torch.where(tile.isfinite(), tile, 0.0).abs().amax((-2, -1)))
    scale = torch.where(held[:, None] > 0, torch.maximum(scale, before), scale)
    was = _unpack(codes[pages].view(torch.float8_e4m3fn).double(), is_k) * torch.exp2((before - scale).double())[..., None, None]
    tile = torch.where(old[:, None, :, None], was, tile * torch.exp2((127 - scale).double())[..., None, None])
    packed = _pack(_to_e4m3(tile), is_k).float().to(torch.float8_e4m3fn).view(torch.uint8)
    touched = _pack((old | fresh)[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[2]), is_k)
    codes[pages] = torch.where(touched, packed, codes[pages])
    scales[pages] = scale.to(torch.uint8)


def _plain_append8(s):
    prefix, new, _, table = s.d
    req, pos, block = _rows(s)
    count = (prefix + new + BLOCK - 1) // BLOCK - prefix // BLOCK  # blocks that a request writes
    first = torch.cumsum(count, 0) - count
    total = int(sum(-(-(int(p) + int(n)) // BLOCK) - int(p) // BLOCK for p, n in zip(s.h[0], s.h[1])))
    page = first[req] + pos // BLOCK - prefix[req] // BLOCK
    owner = torch.repeat_interleave(torch.arange(len(s.h[0]), device="cuda"), count.long(), output_size=total)
    nth = torch.arange(total, device="cuda") - first[owner]
    pages = table[owner, prefix[owner] // BLOCK + nth].long()
    held = torch.where(nth == 0, prefix[owner] % BLOCK, 0)
    inter = s.case["interleaved"]
    s.out.copy_(_rotate(s.q.float(), pos, s.cos_sin, inter))
    k = _rotate(s.k_new.double(), pos, s.cos_sin, inter)
    _plain_append8_plane(s, s.planes[0], k, True, pos, block, page, pages, held)
    _plain_append8_plane(s, s.planes[1], s.v_new.double(), False, pos, block, page, pages, held)


def _plain_attn8(s):
    prefix, new, start, table = s.d
    case = s.case
    hq, hkv, d, group = case["q_heads"], case["kv_heads"], case["head_dim"], case["q_heads"] // case["kv_heads"]
    most = int(s.h[1].max())
    keys = table.shape[1] * BLOCK

    def values(plane, is_k):  # [requests, kv_heads, keys, head_dim]
        codes, scales = _tiles(plane, case)
        x = _unpack(codes[table.long()].view(torch.float8_e4m3fn).float(), is_k)
        x = x * torch.exp2(scales[table.long()].float() - 127.0)[..., None, None]
        return x.transpose(1, 2).flatten(2, 3)

    tok = torch.arange(most, device="cuda")
    row = torch.minimum(start[:-1, None] + tok, start[1:, None] - 1)  # rows past a request's end repeat its last one
    q = s.q[row].float().unflatten(2, (hkv, group)).transpose(1, 2).flatten(2, 3)  # [requests, kv_heads, tokens * group, head_dim]
    scores = torch.matmul(q, values(s.planes[0], True).transpose(-1, -2).contiguous()) * s.scale
    seen = torch.arange(keys, device="cuda") <= (prefix[:, None] + tok)[:, None, :, None, None]
    scores = scores.unflatten(2, (most, group)).masked_fill_(~seen, -math.inf).flatten(2, 3)
    scores = torch.exp(scores.sub_(scores.amax(-1, keepdim=True)))
    v = values(s.planes[1], False)
    v = torch.where((torch.arange(keys, device="cuda") < (prefix + new)[:, None])[:, None, :, None], v, 0.0)
    out = torch.matmul(scores, v) / scores.sum(-1, keepdim=True)
    out = out.unflatten(2, (most, group)).transpose(1, 2).flatten(2, 3)  # [requests, tokens, q_heads, head_dim]
    s.out.copy_(out[tok < new[:, None]])


def _outputs(s):
    if s.case["op"] == "attn8":
        return {"out": s.out}
    if s.case["op"] == "append":
        return {"q": s.out, "k": s.planes[0], "v": s.planes[1]}
    k, k_scale = _tiles(s.planes[0], s.case)
    v, v_scale = _tiles(s.planes[1], s.case)
    e4m3 = torch.float8_e4m3fn
    return {"q": s.out, "k": k.view(e4m3), "v": v.view(e4m3), "k_scale": k_scale, "v_scale": v_scale}


def run(s):
    case = s.case
    if not own:
        {"append": _plain_append, "append8": _plain_append8, "attn8": _plain_attn8}[case["op"]](s)
        return _outputs(s)
    from paper_2404_12457_amd import binding

    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "attn8":
        w = s.workspace
        binding.ragc_kv8_attn(s.pool, s.batch, s.q, s.out, case["q_heads"], s.scale, 0, w, w.numel() if w is not None else 0, stream)
    elif case["op"] == "append8":
        binding.ragc_kv8_append(s.pool, s.batch, s.rope, s.q, s.k_new, s.v_new, s.out, case["q_heads"], stream)
    else:
        binding.ragc_kv_append_rope(s.pool, s.batch, s.rope, s.q, s.k_new, s.v_new, s.out, None, case["q_heads"], stream)
    return _outputs(s)


# ---- the definition in 64 bits --------------------------------------------------------------
def _exact_turn(x, pos, cos_sin, interleaved):
    """One request's rows as complex numbers times cos + i sin."""
    rot = cos_sin.shape[1]
    unit = torch.complex(*[t.double() for t in cos_sin[pos].split(rot // 2, 1)])[:, None]
    y = x.double().clone()
    if interleaved:
        z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:2], rot // 2, 2).contiguous()) * unit
        y[..., :rot] = torch.view_as_real(z).reshape(*y.shape[:2], rot)
    else:
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * unit
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def _e4m3_values():
    """The 256 numbers by their codes, from sign, four bits of exponent and three of mantissa."""
    got = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if e == 15 and m == 7 else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        got.append(-v if c & 128 else v)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _exact_round(x):
    """The e4m3 number nearest to each |x| <= 448 by search among all of them; of two as near the one with an even code."""
    grid = _e4m3_values()[:127]
    a = x.abs().contiguous()
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(grid[pick], x)


def _exact_order(d, is_k):
    """Byte of a tile for each (token, element)."""
    t, e = np.meshgrid(np.arange(BLOCK), np.arange(d), indexing="ij")
    at = (e // 16 * 16 + t) * 16 + e % 16 if is_k else (((e // 64 * 4 + t // 4) * 16 + e % 16) * 4 + e % 64 // 16) * 4 + t % 4
    return torch.from_numpy(at).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    cached, new = _lens(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    start, table = s.h[2], s.h[3]
    grid = _e4m3_values()
    spans = [(r, p, n, slice(int(start[r]), int(start[r]) + n)) for r, (p, n) in enumerate(zip(cached, new))]

    def planes8():
        """codes as values [blocks, heads, token, element] and scale exponents, of both planes"""
        got = []
        for plane, is_k in zip(s.planes, (True, False)):
            b = plane.long()
            tile = b[:, :hkv * BLOCK * d].reshape(len(b), hkv, BLOCK * d)[..., _exact_order(d, is_k).reshape(-1)]
            got.append([grid[tile].reshape(len(b), hkv, BLOCK, d), b[:, hkv * BLOCK * d:hkv * BLOCK * d + hkv].double() - 127])
        return got

    if case["op"] == "attn8":
        (kc, ke), (vc, ve) = planes8()
        out = torch.empty(len(s.q), hq, d, dtype=torch.float64, device="cuda")
        for r, p, n, rows in spans:
            ids = torch.from_numpy(table[r, :-(-(p + n) // BLOCK)].astype(np.int64)).cuda()
            k = (kc[ids] * torch.pow(2.0, ke[ids])[..., None, None]).permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :p + n]
            v = (vc[ids] * torch.pow(2.0, ve[ids])[..., None, None]).permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :p + n]
            hidden = torch.arange(p + n, device="cuda")[None] > p + torch.arange(n, device="cuda")[:, None]
            for h in range(hq):
                g = h // (hq // hkv)
                a = (s.q[rows, h].double() @ k[g].T.contiguous()) * s.scale
                a[hidden] = -math.inf
                out[rows, h] = torch.softmax(a, -1) @ v[g]
        return {"out": out}

    q = torch.cat([_exact_turn(s.q[rows], torch.arange(p, p + n, device="cuda"), s.cos_sin, case["interleaved"]) for _, p, n, rows in spans])
    turned = [_exact_turn(s.k_new[rows], torch.arange(p, p + n, device="cuda"), s.cos_sin, case["interleaved"]) for _, p, n, rows in spans]
    fresh = [turned, [s.v_new[rows].double() for _, _, _, rows in spans]]
    if case["op"] == "append":
        got = [p.double() for p in s.planes]
        for plane, x in zip(got, fresh):
            for (r, p, n, _), y in zip(spans, x):
                at = np.arange(p, p + n)
                ids = torch.from_numpy(table[r, at // BLOCK].astype(np.int64)).cuda()
                plane[ids, :, torch.from_numpy(at % BLOCK).cuda()] = y
        return {"q": q, "k": got[0], "v": got[1]}
    got = planes8()
    for (codes, exps), x in zip(got, fresh):
        for (r, p, n, _), y in zip(spans, x):
            have = p % BLOCK  # tokens in the first block already
            blocks = torch.from_numpy(table[r, p // BLOCK:-(-(p + n) // BLOCK)].astype(np.int64)).cuda()
            wide = torch.zeros(len(blocks) * BLOCK, hkv, d, dtype=torch.float64, device="cuda")
            wide[have:have + n] = y
            wide = wide.reshape(len(blocks), BLOCK, hkv, d).transpose(1, 2)
            top = wide.abs().amax((2, 3))
            e = torch.full_like(top, -126)
            some = top > 0
            e[some] = torch.ceil(torch.log2(top[some] / 448.0)).clamp(min=-126)
            e = torch.where(top > 448.0 * torch.pow(2.0, e), e + 1, torch.where((top <= 448.0 * torch.pow(2.0, e - 1)) & (e > -126), e - 1, e))
            if have:
                e[0] = torch.maximum(e[0], exps[blocks[0]])
                old = codes[blocks[0], :, :have] * torch.pow(2.0, exps[blocks[0]])[:, None, None]
                wide[0, :, :have] = old
            rounded = _exact_round(wide / torch.pow(2.0, e)[..., None, None])
            last = BLOCK - (len(blocks) * BLOCK - have - n)  # tokens in the last block
            if last < BLOCK:
                rounded[-1, :, last:] = codes[blocks[-1], :, last:]
            codes[blocks], exps[blocks] = rounded, e
    packed = []
    for (codes, _), is_k in zip(got, (True, False)):
        flat = torch.empty(codes.shape[0], hkv, BLOCK * d, dtype=torch.float64, device="cuda")
        flat[..., _exact_order(d, is_k).reshape(-1)] = codes.reshape(codes.shape[0], hkv, BLOCK * d)
        packed.append(flat)
    return {"q": q, "k": packed[0], "v": packed[1], "k_scale": None, "v_scale": None}
