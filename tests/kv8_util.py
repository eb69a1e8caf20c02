"""Batches for the GPU tests of the rotation and of the 8-bit cache: a pool with every byte of it random, blocks in random
order, lengths as given."""
import numpy as np
import torch

from oracle import kv8 as O
from paper_2404_12457_amd import binding as B


class Case:
    def __init__(self, lens, q_heads, kv_heads, head_dim, dtype="e4m3", seed=0, pad=0, spare=3, first_row=0, gain=1.0, room=0, device="cuda"):
        g = self.rng = np.random.Generator(np.random.PCG64(seed))
        self.hq, self.hkv, self.d, self.dtype, self.first = q_heads, kv_heads, head_dim, dtype, first_row
        self.h_prefix, self.h_new = (np.asarray(x, np.int32) for x in zip(*lens))
        self.h_start = (first_row + np.concatenate([[0], np.cumsum(self.h_new)])).astype(np.int32)
        need = [-(-(int(p) + int(n) + room) // 16) for p, n in lens]  # room: tokens that later steps add
        self.blocks = sum(need) + spare
        ids = g.permutation(self.blocks).astype(np.int32)
        self.h_table = np.full((len(lens), max(max(need), 1) + 2), 0, np.int32)
        at = 0
        for r, k in enumerate(need):
            self.h_table[r, :k] = ids[at:at + k]
            at += k
        self.rows = int(self.h_start[-1])
        rows = lambda h, s: torch.from_numpy((s * g.standard_normal((self.rows, h, head_dim))).astype(np.float32)).to(device)  # noqa: E731
        self.io = torch.float32 if dtype == "f32" else torch.bfloat16
        self.q, self.k_new, self.v_new = rows(q_heads, 2.0 * gain).to(self.io), rows(kv_heads, gain).to(self.io), rows(kv_heads, gain).to(self.io)
        if dtype == "e4m3":
            self.stride = O.block_bytes(kv_heads, head_dim) + 16 * pad
            planes = g.integers(0, 256, (2, self.blocks, self.stride), np.uint8)
            sat = kv_heads * 16 * head_dim
            planes[:, :, sat:sat + kv_heads] = g.integers(110, 124, (2, self.blocks, kv_heads))
            code = B.RAGC_DTYPE_E4M3
            self.planes = [torch.from_numpy(p).to(device) for p in planes]
        else:
            self.stride = kv_heads * 16 * head_dim + 16 * pad
            self.planes = [torch.from_numpy(g.standard_normal((self.blocks, self.stride)).astype(np.float32)).to(device).to(self.io) for _ in range(2)]
            code = B.RAGC_DTYPE_BF16 if dtype == "bf16" else B.RAGC_DTYPE_F32
        self.dev = [torch.from_numpy(a).to(device) for a in (self.h_prefix, self.h_new, self.h_start, self.h_table)]
        self.pool = B.make_pool(*self.planes, self.blocks, kv_heads, head_dim, code, self.stride)
        self.batch = B.make_batch(len(lens), self.h_table.shape[1], *self.dev, self.h_prefix, self.h_new, self.h_start, self.h_table)

    def fill_prefixes(self, x=None):
        """The cached tokens of every request, of unit variance, in an 8-bit pool: both planes."""
        for plane, is_k in zip(self.planes, (True, False)):
            host = plane.cpu().numpy()
            for r, p in enumerate(self.h_prefix):
                O.write_tokens(host, self.h_table[r], 0, self.rng.standard_normal((int(p), self.hkv, self.d)), is_k)
            plane.copy_(torch.from_numpy(host))

    def spans(self):
        for r, (p, n) in enumerate(zip(self.h_prefix, self.h_new)):
            if n:
                yield r, int(p), int(n), slice(int(self.h_start[r]), int(self.h_start[r]) + int(n))

    def host(self, t):
        return t.detach().double().cpu().numpy()

    def appended8(self, k, v):
        """What the planes hold after k, v (float64 rows) have joined them, by the oracle."""
        out = []
        for plane, is_k, x in zip(self.planes, (True, False), (k, v)):
            b = plane.cpu().numpy().copy()
            for r, p, n, rows in self.spans():
                O.write_tokens(b, self.h_table[r], p, x[rows], is_k)
            out.append(b)
        return out

    def rotated(self, x, cos_sin, interleaved):
        out = np.array(x, np.float64)
        for _, p, n, rows in self.spans():
            out[rows] = O.rotate(x[rows], p, cos_sin, interleaved)
        return out
