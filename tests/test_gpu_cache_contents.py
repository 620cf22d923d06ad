"""Rows of the page cache keep their tokens, whatever the rows do that they share pages with.  The contents are followed row by
row as lists of tokens, without pages: how pages are given out is not assumed."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"
P = 16


class Rows:
    """A cache and, for every row, the numbers of its tokens.  Token n has n in every key and -n in every value."""

    def __init__(self, rows, pages, width, *, layers=2, heads=2, d=8):
        self.cache = disc.DiscCache.empty(layers, pages, P, heads, d, rows, width)
        self.rows, self.tokens, self.last = rows, [[] for _ in range(rows)], 0

    def extend(self, add):
        st = disc.disc_cache_extend(self.cache, torch.as_tensor(np.asarray(add, np.int32)).to(DEV)).cpu().tolist()
        new = [list(range(self.last + sum(max(a, 0) for a in add[:r]) + 1, self.last + sum(max(a, 0) for a in add[:r + 1]) + 1)) for r in range(self.rows)]
        self.last += sum(max(a, 0) for a in add)
        todo = [r for r in range(self.rows) if add[r] > 0 and st[r] == 0]
        for r in todo:
            self.tokens[r] = self.tokens[r] + new[r]
        if todo:
            n = torch.as_tensor(np.array([x for r in todo for x in new[r]], np.int16)).to(DEV)
            k = n[:, None, None].expand(-1, self.cache.n_kv_heads, self.cache.head_dim).contiguous()
            cu = torch.as_tensor(np.concatenate([[0], np.cumsum([len(new[r]) for r in todo])]).astype(np.int32)).to(DEV)
            rows = torch.as_tensor(np.array(todo, np.int32)).to(DEV)
            for layer in range(self.cache.n_layers):
                disc.disc_cache_write(self.cache, layer, k.view(torch.bfloat16), (-k).view(torch.bfloat16), cu=cu, rows=rows)
        self.check()
        return st

    def fork(self, parent):
        disc.disc_cache_fork(self.cache, torch.as_tensor(np.asarray(parent, np.int32)).to(DEV))
        old = self.tokens
        self.tokens = [list(old[p]) if 0 <= p < self.rows else [] for p in parent]
        self.check()

    def compact(self):
        disc.disc_cache_compact(self.cache)
        self.check()

    def check(self):
        c = self.cache
        table, lens, ref = c.table.cpu().numpy(), c.len.cpu().tolist(), c.ref.cpu().numpy()
        assert lens == [len(t) for t in self.tokens]
        used = [-(-n // P) for n in lens]
        named = np.concatenate([table[r, :used[r]] for r in range(self.rows)])
        assert np.array_equal(ref, np.bincount(named, minlength=c.n_pages))
        pool = c.pool.view(torch.int16).cpu().numpy()
        for r, t in enumerate(self.tokens):
            if not t:
                continue
            at = np.arange(len(t))
            got = pool[:, :, table[r, at // P], :, at % P]           # [tokens, layers, 2, heads, d]
            want = np.asarray(t, np.int16)[:, None, None, None, None] * np.array([1, -1], np.int16)[None, None, :, None, None]
            assert np.array_equal(got, np.broadcast_to(want, got.shape)), (r, t)


def test_the_longest_of_the_rows_on_a_page_goes_on_in_place():
    """Two rows of one page, one of them longer because the other found no page, in the other order: the shorter one, lower now,
    must not write over the longer one's last token."""
    x = Rows(2, 1, 1)
    assert x.extend([5, 0]) == [0, 0]
    x.fork([0, 0])
    st = x.extend([1, 1])
    assert sorted(st) == [0, 32]
    longer = st.index(0)
    x.fork([1 - longer, longer] if longer == 1 else [1, 0])          # row 0: 5 tokens, row 1: 6
    assert [len(t) for t in x.tokens] == [5, 6]
    x.extend([1, 1])


@pytest.mark.parametrize("rows,pages,width,seed", [(2, 1, 2, 9), (2, 2, 2, 1), (3, 3, 2, 20), (5, 5, 2, 2), (8, 8, 3, 0), (20, 16, 3, 1)])
def test_a_random_life_in_few_pages(rows, pages, width, seed):
    rng = np.random.default_rng(seed)
    x = Rows(rows, pages, width)
    for _ in range(80):
        what = rng.choice(["few", "one", "mix", "turn", "turn", "compact"])
        if what == "few":
            x.extend([int(a) for a in rng.integers(0, 5, rows) * (rng.random(rows) < 0.8)])
        elif what == "one":
            x.extend([1] * rows)
        elif what == "compact":
            x.compact()
        elif what == "turn":
            x.fork([int(a) for a in rng.permutation(rows)])
        else:
            x.fork([int(a) for a in np.where(rng.random(rows) < 0.2, -1, rng.integers(0, rows, rows))])


def test_writing_more_tokens_than_threads_can_be_counted_in_32_bits():
    """2^27 tokens take 2^32 threads.  The row holds the last 16 of them; the tokens before have no place and are skipped."""
    n = (1 << 27) + 16
    cache = disc.DiscCache.empty(1, 1, P, 1, 8, 1, 1)
    disc.disc_cache_extend(cache, torch.tensor([16], dtype=torch.int32, device=DEV))
    k = torch.full((1, 1, 8), 3.0, dtype=torch.bfloat16, device=DEV).expand(n, 1, 8)
    disc.disc_cache_write(cache, 0, k, k, cu=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    assert torch.all(cache.pool == 3.0)
