"""Shared by the 4-bit cache's GPU tests."""
import numpy as np
import torch

from paper_2607_20940_gb300 import msf


def ints(x):
    return None if x is None else torch.tensor(list(x), dtype=torch.int32, device="cuda")


def make(layers=1, kv_heads=2, head_dim=64, page_tokens=16, pages=64, sequences=4, sequence_pages=16, k_exponent=0,
         v_exponent=0):
    c = msf.Cache(msf.make_cache_desc(layers, kv_heads, head_dim, page_tokens, pages, sequences, sequence_pages,
                                      k_exponent, v_exponent))
    c.bind(c.pool().fill_(0xff), c.state(), c.workspace().fill_(0xa5))  # a pool of NaN scales
    return c


def ok(cache, want=msf.MSF_OK):
    assert cache.device_status() == want


def f64(t):
    return t.detach().double().cpu().numpy()


def rows(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16).cuda()


def same_tables(cache, model):
    assert np.array_equal(cache.table.cpu().numpy(), model.table_array())
    assert cache.lengths.tolist() == model.lengths
    assert cache.refs.tolist() == model.refs()
