"""The page cache against the same calls made one row after the other on Python lists."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from model_ops_reference import PlainCache

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Both:
    def __init__(self, layers, pages, page, heads, d, rows, width, dtype, seed):
        self.rng = np.random.default_rng(seed)
        shape = (layers, 2, pages, heads, page, d)
        self.bits = torch.int16
        start = self.rng.integers(-2 ** 15, 2 ** 15, shape).astype(np.int16)       # contents are only moved: any bits will do
        self.gpu = disc.DiscCache(torch.as_tensor(start).to(DEV).view(dtype), rows, width)
        self.cpu = PlainCache(start, rows, width)
        self.dtype = dtype

    def check(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.gpu.table.cpu().numpy(), self.cpu.table())
        assert self.gpu.len.cpu().tolist() == self.cpu.len
        assert np.array_equal(self.gpu.ref.cpu().numpy(), self.cpu.ref())
        assert np.array_equal(self.gpu.pool.view(torch.int16).cpu().numpy(), self.cpu.pool)

    def extend(self, add=None):
        a = None if add is None else torch.as_tensor(np.asarray(add, np.int32)).to(DEV)
        st = disc.disc_cache_extend(self.gpu, a)
        want = self.cpu.extend([1] * self.cpu.rows if add is None else list(add))
        assert np.array_equal(st.cpu().numpy(), want)
        return want

    def fork(self, parent):
        disc.disc_cache_fork(self.gpu, torch.as_tensor(np.asarray(parent, np.int32)).to(DEV))
        self.cpu.fork(parent)

    def free(self, rows):
        f = np.zeros(self.cpu.rows, np.uint8)
        f[list(rows)] = 1
        disc.disc_cache_free(self.gpu, torch.as_tensor(f).to(DEV))
        self.cpu.fork([-1 if f[r] else r for r in range(self.cpu.rows)])

    def write(self, layer, seqs):
        """seqs: (row, tokens)"""
        lens = [n for _, n in seqs]
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        h, d = self.gpu.n_kv_heads, self.gpu.head_dim
        kv = self.rng.integers(-2 ** 15, 2 ** 15, (int(cu[-1]), 2 * h + 1, d)).astype(np.int16)
        both = torch.as_tensor(kv).to(DEV).view(self.dtype)
        disc.disc_cache_write(self.gpu, layer, both[:, :h], both[:, h + 1:], cu=torch.as_tensor(cu).to(DEV),
                              rows=torch.as_tensor(np.array([r for r, _ in seqs], np.int32)).to(DEV))
        self.cpu.write(layer, kv[:, :h], kv[:, h + 1:], [(r, int(c), n) for (r, n), c in zip(seqs, cu)])

    def compact(self):
        assert int(disc.disc_cache_compact(self.gpu)) == self.cpu.compact()


@pytest.mark.parametrize("layers,pages,page,heads,d,rows,width,dtype", [
    (2, 40, 16, 2, 64, 8, 6, torch.bfloat16), (1, 9, 32, 1, 8, 5, 3, torch.float16), (3, 130, 16, 3, 40, 33, 7, torch.bfloat16),
    (1, 5000, 16, 1, 8, 70, 20, torch.float16), (1, 64, 128, 2, 128, 12, 4, torch.bfloat16), (1, 1, 16, 1, 8, 1, 1, torch.bfloat16)])
def test_a_random_life(layers, pages, page, heads, d, rows, width, dtype):
    b = Both(layers, pages, page, heads, d, rows, width, dtype, rows + pages)
    rng = b.rng
    for step in range(30):
        what = rng.choice(["extend", "extend", "one", "fork", "free", "compact"])
        if what == "extend":
            add = rng.integers(-1, 2 * page, rows) * (rng.random(rows) < 0.5)
            st = b.extend(add)
            todo = [(r, int(add[r])) for r in range(rows) if add[r] > 0 and st[r] == 0]
            if todo:
                b.write(int(rng.integers(layers)), todo)
        elif what == "one":
            st = b.extend()
            todo = [(r, 1) for r in range(rows) if st[r] == 0]
            if todo:
                b.write(layers - 1, todo)
        elif what == "fork":
            parent = np.where(rng.random(rows) < 0.5, np.arange(rows), rng.integers(-2, rows + 1, rows))
            b.fork([int(x) for x in parent])
        elif what == "free":
            b.free(np.nonzero(rng.random(rows) < 0.3)[0])
        else:
            b.compact()
        b.check()


def test_candidates_of_a_query_share_the_prompt_and_part_at_its_last_page():
    K, P = 5, 16
    b = Both(2, 64, P, 2, 16, 2 * K, 6, torch.bfloat16, 3)
    b.extend([37 if r == 0 else 48 if r == K else 0 for r in range(2 * K)])
    b.write(0, [(0, 37), (K, 48)])
    b.fork([0] * K + [K] * K)
    b.check()
    assert b.gpu.ref.max() == K
    for t in range(18):
        b.extend()
        b.write(t % 2, [(r, 1) for r in range(2 * K)])
        b.check()
    # 2 full pages of the first prompt and 3 of the second stay shared
    assert int((b.gpu.ref == K).sum()) == 5
    b.fork([3, -1, -1, -1, -1, K + 1, -1, -1, -1, -1])
    b.compact()
    b.check()


def test_rows_beyond_the_free_pages_are_left_alone():
    b = Both(1, 6, 16, 1, 8, 6, 3, torch.bfloat16, 4)
    st = b.extend([16, 20, 16, 17, 0, 16])               # 1 + 2 + 1 = 4 pages, row 3 wants 2 more: fits; row 5 does not
    assert st.tolist() == [0, 0, 0, 0, 0, 32]
    b.check()
    st = b.extend([0, 12, 16, 15, 0, 0])                 # room in their pages but row 2
    assert st.tolist() == [0, 0, 32, 0, 0, 0]
    b.check()
    st = b.extend([40, 0, 0, 17, 49, 0])                 # beyond the table
    assert st.tolist() == [32, 0, 0, 32, 32, 0]
    b.check()
    # a refused row that goes on sharing a page keeps its tokens when the others write on
    c = Both(1, 3, 16, 1, 8, 3, 2, torch.bfloat16, 5)
    c.extend([5, 0, 0])
    c.write(0, [(0, 5)])
    c.fork([0, 0, 0])
    d = Both(1, 2, 16, 1, 8, 3, 2, torch.bfloat16, 6)
    d.extend([5, 0, 0])
    d.write(0, [(0, 5)])
    d.fork([0, 0, 0])
    for x, want in ((c, [0, 0, 0]), (d, [0, 0, 32])):
        assert x.extend().tolist() == want
        x.write(0, [(r, 1) for r in range(3) if want[r] == 0])
        x.check()
        x.extend([0, 0, 1])
        x.check()


@pytest.mark.parametrize("rows,pages", [(9000, 12000), (40000, 45000)])
def test_many_rows(rows, pages):
    """More rows than threads: four of a thread in registers, and more."""
    b = Both(1, pages, 16, 1, 8, rows, 3, torch.bfloat16, rows)
    b.extend((b.rng.integers(0, 24, rows) * (b.rng.random(rows) < 0.6)).astype(np.int32))
    b.check()
    parent = np.arange(rows)
    pick = b.rng.random(rows) < 0.4
    parent[pick] = b.rng.integers(-1, rows, int(pick.sum()))
    b.fork([int(x) for x in parent])
    b.check()
    b.extend((b.rng.integers(0, 10, rows)).astype(np.int32))
    b.check()
    b.free(np.nonzero(b.rng.random(rows) < 0.5)[0])
    b.compact()
    b.check()


def test_one_token_each_without_offsets_and_skipped_rows():
    b = Both(1, 16, 16, 2, 8, 4, 2, torch.float16, 7)
    b.extend([3, 0, 16, 1])
    kv = b.rng.integers(-2 ** 15, 2 ** 15, (2, 4, 2, 8)).astype(np.int16)
    k, v = (torch.as_tensor(x).to(DEV).view(torch.float16) for x in kv)
    status = torch.tensor([0, 0, 32, 0], dtype=torch.uint8, device=DEV)
    disc.disc_cache_write(b.gpu, 0, k, v, status=status)
    b.cpu.write(0, kv[0], kv[1], [(0, 0, 1), (3, 3, 1)])     # row 1 is empty, row 2 is skipped
    b.check()


def test_refusals():
    pool = torch.zeros((1, 2, 4, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    c = disc.DiscCache(pool, 3, 2)
    with pytest.raises(disc.DiscError):
        disc.DiscCache(pool.float(), 3, 2)
    with pytest.raises(TypeError):
        disc.DiscCache(pool[:, :, :, :, ::2], 3, 2)
    with pytest.raises(TypeError):
        disc.DiscCache(pool, 3, 2, book=torch.zeros(5, dtype=torch.int32, device=DEV))
    for shape in ((1, 2, 4, 2, 24, 64), (1, 2, 4, 2, 8, 64), (1, 2, 4, 2, 256, 64), (1, 2, 4, 2, 16, 136), (1, 2, 4, 2, 16, 12)):
        bad = disc.DiscCache(torch.zeros(shape, dtype=torch.bfloat16, device=DEV), 3, 2)
        with pytest.raises(disc.DiscError):
            disc.disc_cache_extend(bad)
    with pytest.raises(TypeError):
        disc.disc_cache_fork(c, torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        disc.disc_cache_fork(c, torch.zeros(3, dtype=torch.int64, device=DEV))
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(TypeError):
        disc.disc_cache_write(c, 0, k, k[:2])
    with pytest.raises(disc.DiscError):
        disc.disc_cache_write(c, 1, k, k)
    odd = torch.zeros((3, 2, 68), dtype=torch.bfloat16, device=DEV)[:, :, :64]
    with pytest.raises(disc.DiscError):
        disc.disc_cache_write(c, 0, odd, odd)
