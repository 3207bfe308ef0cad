"""Inputs of the tests of the operators over a paged cache."""
import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def ints(values):
    return torch.tensor(np.ascontiguousarray(values), dtype=torch.int32).cuda()


def pages(rng, n_pages, P, Hkv, dh, dtype, heads_first=False, layers=None):
    """Pages [(layers,) n_pages, P, Hkv, dh], their slots in the order of tokens or of heads."""
    lead = (n_pages,) if layers is None else (layers, n_pages)
    shape = lead + ((Hkv, P, dh) if heads_first else (P, Hkv, dh))
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DT[dtype]).cuda()
    return t.transpose(-3, -2) if heads_first else t


def batch(rng, lens, news, P, spare=2, extra_columns=1):
    """(n_pages, table [B, M], cu) of sequences whose pages lie anywhere in the pool."""
    counts = [-(-n // P) for n in lens]
    n_pages = sum(counts) + spare
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max(counts + [1]) + extra_columns), -1, np.int32)
    for b, n in enumerate(counts):
        table[b, :n] = ids[sum(counts[:b]):sum(counts[:b]) + n]
    return n_pages, table, np.concatenate([[0], np.cumsum(news)]).astype(np.int32)


def rows(rng, N, H, dh, dtype, scale=1.0, packed=False):
    """[N, H, dh]; packed: a view into wider rows, as out of one projection."""
    x = torch.from_numpy((scale * rng.standard_normal((N, H + (3 if packed else 0), dh))).astype(np.float32)).to(DT[dtype]).cuda()
    return x[:, 1:1 + H] if packed else x


def f64(t):
    return t.detach().cpu().double().numpy()
