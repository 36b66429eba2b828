"""Caches and tables for the GPU tests of the cache operators."""
import torch

from paper_2607_16784_amd import api


def make_cache(lengths, kv_heads, page, dim, codes, seed, spare=2):
    """A cache of random codes in which every sequence's pages are scattered,
    its table (unused entries -1) and lengths."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    most = max([1] + need)
    table = torch.full((len(lengths), most), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    top = 127.0 if codes == torch.int8 else 448.0
    cache = api.new_cache(pages, kv_heads, page, dim, codes)
    for name in ("k", "v"):
        x = torch.randn(cache[name].shape, generator=g) * (top / 3)
        x = x.clamp(-top, top)
        x = x.round().to(torch.int8) if codes == torch.int8 else x.to(codes)
        cache[name].view(torch.uint8).copy_(x.view(torch.uint8))
        s = (torch.rand((pages, kv_heads), generator=g) + 0.5) * 3 / top
        cache[name + "_scale"].copy_(s)
    return cache, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), order[at:]


def offsets_of(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out
