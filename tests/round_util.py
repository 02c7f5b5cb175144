"""Batches for the tests of the paged cache and its attention: seeded numpy data, pages in a shuffled pool, uploads."""
import numpy as np

from oracle import round_oracle as RO

NAMES = {"bf16": 1, "fp16": 2, "int8": 3, "e4m3": 4}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn, "fp32": torch.float32}[name]


def rounded(x, dtype):
    """x rounded to a 16-bit type, as a torch CPU tensor and as fp32 values."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch_dtype(dtype))
    return t, t.float().numpy()


class Batch:
    """Sequences of `length` tokens of which the last `new` are the rows of the call; `pad` rows behind the last sequence."""

    def __init__(self, rng, new, length, page, spare=3, pad=0, extra_width=0):
        self.new, self.length, self.page, self.S = list(new), list(length), page, len(new)
        need = [max(0, -(-n // page)) for n in length]
        self.width = max(max(need), 1) + extra_width
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.pages = rng.integers(0, self.n_pages, (self.S, self.width)).astype(np.int32)
        at = 0
        for s, n in enumerate(need):
            self.pages[s, :n] = order[at:at + n]
            at += n
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = int(self.start[-1]) + pad

    def places(self):
        return RO.places(self.start, self.length, self.pages, self.page, self.n_pages, self.T)

    def params(self, H, D, dtype, kept):
        import paper_2605_02218_amd as C
        return C.CacheParams(n_seq=self.S, n_tokens=self.T, n_kv_heads=H, head_dim=D, page_size=self.page, n_pages=self.n_pages, max_pages=self.width,
                             dtype=NAMES[dtype], cache_dtype=NAMES[kept])

    def device(self):
        import torch
        return [torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda() for a in (self.start, self.length, self.pages)]


def pool_of(x, kept, dtype):
    """A pool tensor pair (codes, scale or None) on the CPU from values [n_pages, H, page, D], and the fp64 values it stands for."""
    import torch
    if kept == dtype:
        t, v = rounded(x, dtype)
        return t, None, v.astype(np.float64)
    c, s = RO.quantise(rounded(x, dtype)[1], kept)
    return torch.from_numpy(c).to(torch_dtype(kept)), torch.from_numpy(s), c.astype(np.float64) * s[..., None].astype(np.float64)
