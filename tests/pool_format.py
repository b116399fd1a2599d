"""The cache's tile format, for tests that look at whole pools: element numbers of token rows (see aspd.h: the order inside a
tile is private to the library; this is csrc/aspd_internal.cuh's, stated once more)."""
import numpy as np


def elements(page, row, n_kv_heads, page_size, head_dim, esize):
    """[tokens][KV heads][head_dim] element numbers in a pool of the rows `row` of pages `page`."""
    page, row = (np.asarray(x, dtype=np.int64).reshape(-1, 1, 1) for x in (page, row))
    head, b = np.arange(n_kv_heads).reshape(1, -1, 1), np.arange(head_dim) * esize
    inside = (row // 8) * (8 * head_dim * esize) + (b // 128) * 1024 + (row % 8) * 128 + (((b % 128) // 16) ^ (row % 8)) * 16 + b % 16
    return ((page * n_kv_heads + head) * (page_size * head_dim * esize) + inside) // esize
