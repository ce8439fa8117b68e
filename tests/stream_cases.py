"""Batches of the stream operators' tests: sequences with any number of rows and any length, pages in any order."""
import numpy as np

from paper_2411_16102_amd import workloads as W


def make_batch(seqs, seed=0, spare=3, given_up=None):
    """seqs: (rows, kv_len) each.  given_up: page numbers of every table that become -1."""
    q = np.array([s[0] for s in seqs], dtype=np.int64)
    kv = np.array([s[1] for s in seqs], dtype=np.int64)
    start = np.concatenate([[0], np.cumsum(-(-kv // 16))])
    n_pages = int(start[-1]) + spare
    pages = np.random.default_rng([seed, 7]).permutation(n_pages)[:int(start[-1])]
    for s, gone in (given_up or {}).items():
        pages[start[s] + np.asarray(gone, dtype=np.int64)] = -1
    none = np.zeros(0, dtype=np.int32)
    i32 = lambda a: np.asarray(a, dtype=np.int32)
    return W.Batch(page_size=16, n_seq=len(seqs), n_prefill=0, n_rows=int(q.sum()), row_start=i32(np.concatenate([[0], np.cumsum(q)])),
                   kv_len=i32(kv), page_start=i32(start), page_ids=i32(pages), n_nodes=0, node_parent=none, node_page_start=i32([0]),
                   node_page_ids=none, node_seq_first=none, node_seq_count=none, seq_leaf_node=np.full(len(seqs), -1, dtype=np.int32),
                   n_pages=n_pages)
