"""Batches of rows over paged and contiguous caches, for the GPU tests of the
operators around a round."""
import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def half_step(dt):
    """Largest relative error of one rounding to dt."""
    return torch.finfo(dt).eps / 2


class Batch:
    """Rows of several requests and the pages of their caches.

    rows, prefix: per request; page: page size, 0 for a contiguous cache;
    gap: rows of no request between and behind the requests' rows."""

    def __init__(self, rows, prefix, page, seed=0, gap=0, spare=3):
        rng = np.random.default_rng(seed)
        self.rows, self.prefix = np.asarray(rows, np.int32), np.asarray(prefix, np.int32)
        self.batch = len(rows)
        self.start = (np.cumsum([0] + [n + gap for n in rows[:-1]])).astype(np.int32)
        self.total = max(1, int(sum(rows)) + gap * self.batch)
        slots = [p + n for p, n in zip(prefix, rows)]
        if page == 0:
            self.page_size, self.n_pages, self.max_pages = max(slots + [1]) + 5, self.batch, 1
            self.table = None
        else:
            need = [-(-s // page) for s in slots]
            self.page_size, self.n_pages = page, sum(need) + spare
            self.max_pages = max(need + [1])
            order = rng.permutation(self.n_pages).astype(np.int32)
            # entries past a request's pages are no pages at all
            self.table = np.full((self.batch, self.max_pages), -7, np.int32)
            at = 0
            for r, n in enumerate(need):
                self.table[r, :n] = order[at:at + n]
                at += n

    def dev(self):
        d = lambda a: None if a is None else torch.from_numpy(a).cuda()
        return dict(row_start=d(self.start), n_rows=d(self.rows), prefix_len=d(self.prefix),
                    page_table=d(self.table))

    def places(self, r, first, last):
        from oracle.kv_oracle import place_of
        return np.array([place_of(s, r, self.page_size, self.table) for s in range(first, last)],
                        np.int64)

    def used_rows(self):
        m = np.zeros(self.total, bool)
        for a, n in zip(self.start, self.rows):
            m[a:a + n] = True
        return m


def f64(t):
    return t.double().cpu().numpy()
