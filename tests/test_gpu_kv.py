"""Append to, and read from, the paged cache of 4-bit codes on the GPU. The
format is defined bit for bit, so the whole cache, the turned queries and what
is read back must equal the oracle's."""
import numpy as np
import pytest
import torch

import paper_1911_08076_amd as P
from oracle import serve as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, P.IFQ_TYPE_BF16), "f16": (torch.float16, P.IFQ_TYPE_F16)}


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device=DEV)


class Batch:
    """A cache of anything, a page table of distinct pages, and new tokens."""

    def __init__(self, rng, new, lens, heads, kv_heads, dim, page, kind, rot=0, adjacent=False,
                 rot_len=None, spare=3):
        self.new, self.lens, self.heads, self.kv_heads = new, lens, heads, kv_heads
        self.dim, self.page, self.adjacent = dim, page, adjacent
        self.dtype, code = TYPES[kind]
        most = max(1, -(-max(max(lens), 1) // page))
        pages = len(new) * most + spare
        self.table = rng.permutation(pages)[:len(new) * most].reshape(len(new), most)
        self.cache = rng.integers(0, 256, (pages, kv_heads, page * (dim + 8)), dtype=np.uint8)
        self.offs = np.concatenate([[0], np.cumsum(new)])
        total = int(self.offs[-1])
        width = heads + 2 * kv_heads
        x = rng.standard_normal((total, width, dim)) * np.exp(rng.standard_normal((1, width, dim)))
        self.rows = torch.from_numpy(x).to(self.dtype).to(DEV)
        self.rot_len = most * page if rot_len is None else rot_len
        ang = rng.uniform(-3, 3, (max(self.rot_len, 1), max(rot // 2, 1)))
        self.cos, self.sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
        self.rot = rot
        self.desc = P.kv_desc(len(new), total, max(new), max(lens), heads, kv_heads, dim, page,
                              pages, most, code, rot_dim=rot, rot_adjacent=adjacent,
                              rot_len=self.rot_len, q_stride=width * dim, k_stride=width * dim,
                              v_stride=width * dim)

    def append(self, with_q=True):
        h, hk = self.heads, self.kv_heads
        total = self.rows.shape[0]
        cache = torch.from_numpy(self.cache).to(DEV)
        q = torch.full((total, h, self.dim), 77.0, dtype=self.dtype, device=DEV)
        cos, sin = (torch.from_numpy(t).to(DEV) if self.rot else None
                    for t in (self.cos, self.sin))
        args = (i32(self.offs), i32(self.lens), i32(self.table), cache)
        P.ifq_kv_append(self.desc, self.rows if with_q else None, self.rows[:, h:],
                        self.rows[:, h + hk:], cos, sin, *args, q if with_q else None)
        k = torch.full((total, hk, self.dim), 77.0, dtype=self.dtype, device=DEV)
        v = torch.full_like(k, 77.0)
        P.ifq_kv_read(self.desc, *args, k, v)
        return [t.float().cpu().numpy() if t.dtype != torch.uint8 else t.cpu().numpy()
                for t in (cache, q, k, v)]

    def expected(self):
        h, hk, dim = self.heads, self.kv_heads, self.dim
        x = self.rows.float().cpu().numpy()
        cache = self.cache.copy()
        q = x[:, :h].copy()
        k, v = np.zeros((2, len(x), hk, dim), np.float32)
        most = self.table.shape[1]
        for b, n in enumerate(self.new):
            for i in range(n):
                t, p = self.offs[b] + i, self.lens[b] - n + i
                turned = x[t, :h + hk]
                if self.rot and 0 <= p < self.rot_len:
                    turned = S.rotate(turned, self.cos[p], self.sin[p], self.adjacent)
                q[t] = turned[:h]
                inside = 0 <= p < most * self.page
                page = self.table[b, p // self.page] if inside else -1
                if not 0 <= page < len(cache):
                    continue
                store = not self.rot or p < self.rot_len
                kw, kc = S.row_codes(turned[h:])
                vw, vc = S.row_codes(x[t, h + hk:])
                for g in range(hk):
                    head = S.head_of(cache, page, g, self.page, dim)
                    s = p % self.page
                    if store:
                        head.put(s, kw[g], kc[g], vw[g], vc[g])
                        k[t, g], v[t, g] = S.row_values(kw[g], kc[g]), S.row_values(vw[g], vc[g])
                    else:
                        c = [a[s] for a in head.codes()]
                        k[t, g] = S.row_values(head.kw[s], c[0])
                        v[t, g] = S.row_values(head.vw[s], c[1])
        half = [torch.from_numpy(a).to(self.dtype).float().numpy() for a in (q, k, v)]
        return [cache] + half

    def check(self, with_q=True):
        got, want = self.append(with_q), self.expected()
        assert np.array_equal(got[0], want[0])
        if with_q:
            assert np.array_equal(got[1], want[1])
        else:
            assert (got[1] == 77).all()
        for g, w in zip(got[2:], want[2:]):
            assert np.array_equal(g, w, equal_nan=True)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens,heads,kv_heads,dim,page,rot,adjacent", [
    ([1], [1], 1, 1, 64, 32, 64, False),
    ([1, 1, 1], [1, 33, 100], 4, 2, 128, 32, 128, False),
    ([1, 1], [64, 65], 3, 1, 256, 64, 256, True),
    ([1, 0, 1], [9, 40, 8], 2, 2, 64, 32, 16, True),
    ([5, 1, 40], [5, 70, 71], 4, 2, 128, 64, 64, False),
    ([33, 64, 2], [33, 96, 34], 2, 1, 64, 96, 0, False),
    ([100], [131], 2, 2, 256, 32, 96, False),
    ([31, 32, 70], [31, 63, 130], 5, 5, 128, 128, 32, True)])
def test_append_and_read(kind, new, lens, heads, kv_heads, dim, page, rot, adjacent, rng):
    Batch(rng, new, lens, heads, kv_heads, dim, page, kind, rot, adjacent).check()


def test_append_without_queries(rng):
    Batch(rng, [3, 1], [7, 40], 2, 1, 64, 32, "bf16", 64).check(with_q=False)


def test_append_token_by_token_equals_at_once(rng):
    a = Batch(rng, [40], [75], 2, 2, 128, 32, "bf16", 128)
    want = a.append()[0]
    rows, lens = a.rows, a.lens
    for i in range(40):
        a.rows, a.new, a.lens, a.offs = rows[i:i + 1], [1], [36 + i], np.array([0, 1])
        a.desc.total_q = a.desc.max_q = 1
        a.cache = a.append()[0]
    assert np.array_equal(a.cache, want)


def test_rows_that_hold_nan_infinity_or_one_value(rng):
    a = Batch(rng, [12], [12], 1, 1, 64, 32, "bf16")
    a.rows[1, 1, 3] = float("nan")
    a.rows[2, 2, 5] = float("inf")
    a.rows[3, 1] = 0.0
    a.rows[4, 2] = -3.25
    a.rows[5, 1] = float("-inf")
    a.rows[6, 1, ::2], a.rows[6, 1, 1::2] = 3.3e38, -3.3e38         # the spread overflows
    a.rows[7, 1] = 1e-40
    a.rows[8, 2, :32], a.rows[8, 2, 32:] = 2.0 ** -130, 2.0 ** -126
    a.rows[9, 1], a.rows[9, 1, 0] = 100.0, 100.5
    a.check()


def test_positions_outside_the_tables(rng):
    """Before the sequence, past the page table, past the rotation's tables, on
    pages that the cache does not have: nothing is stored there."""
    a = Batch(rng, [6, 40, 5, 4], [3, 33, 30, 64], 2, 1, 64, 32, "f16", 32, rot_len=60)
    a.table[1, 1], a.table[2, 0], a.table[3, 0] = -1, len(a.cache), 2 ** 30
    a.check()
    b = Batch(rng, [10], [30], 1, 1, 64, 32, "bf16")
    b.lens = [38]                                   # positions 28 .. 37 of a table of 32
    b.check()
    b.lens = [2 ** 31 - 1]
    b.check()
    b.lens = [-2 ** 31]
    b.check()


def test_pages_past_4_gib(rng):
    """A cache of 5 GiB, its last pages in use."""
    dim, page, hk = 128, 64, 2
    size = hk * page * (dim + 8)
    pages = (5 << 30) // size
    new, lens = [1, 3], [65, 67]
    small = Batch(rng, new, lens, 2, hk, dim, page, "bf16", 128)
    want = small.expected()
    big = torch.zeros(pages, hk, page * (dim + 8), dtype=torch.uint8, device=DEV)
    first = pages - len(small.cache)
    big[first:] = torch.from_numpy(small.cache).to(DEV)
    small.desc.num_pages = pages
    table = i32(small.table + first)
    q = torch.empty(4, 2, dim, dtype=torch.bfloat16, device=DEV)
    cos, sin = torch.from_numpy(small.cos).to(DEV), torch.from_numpy(small.sin).to(DEV)
    args = (i32(small.offs), i32(lens), table, big)
    P.ifq_kv_append(small.desc, small.rows, small.rows[:, 2:], small.rows[:, 4:], cos, sin, *args,
                    q)
    assert np.array_equal(big[first:].cpu().numpy(), want[0])
    assert not big[:64].any() and not big[first - 64:first].any()
    k, v = torch.empty(2, 4, hk, dim, dtype=torch.bfloat16, device=DEV)
    P.ifq_kv_read(small.desc, *args, k, v)
    assert np.array_equal(k.float().cpu().numpy(), want[2])
    assert np.array_equal(v.float().cpu().numpy(), want[3])
