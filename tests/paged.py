"""A paged cache for the tests: filled with values for the tokens that its rows hold and with NaN everywhere else, on the device and for the oracle."""
import numpy as np
import torch

from oracle import generation as og
from synth import inputs as si
from synth.device import dev_bf16


def bits(rng, shape, std=1.0, mean=0.0):
    return si.f32_to_bf16_bits((rng.standard_normal(shape) * std + mean).astype(np.float32))


def i64(values):
    return None if values is None else torch.tensor(values, dtype=torch.int64, device="cuda")


def garbage(shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def workspace(nbytes):
    return torch.full((max(int(nbytes), 16),), 0xFF, dtype=torch.uint8, device="cuda")


class Pages:
    """held[b]: tokens of row b that the cache holds.  Rows get their pages from a shuffled pool with a few to spare; the table names pages that do not
    exist behind a row's last."""

    def __init__(self, rng, held, n_kv_heads, head_dim, page, e4m3, columns=None, spare=3, std=1.0, mean=0.0):
        need = [-(-max(n, 0) // page) for n in held]
        columns = columns or max(max(need), 1)
        n_pages = sum(need) + spare
        pool = list(rng.permutation(n_pages))
        table = np.full((len(held), columns), -1, np.int32)
        table[1::2] = n_pages + 7
        for b, n in enumerate(need):
            table[b, :n] = [pool.pop() for _ in range(n)]
        shape = (n_pages, n_kv_heads, page, head_dim)
        self.e4m3, self.table, self.shape = e4m3, table, shape
        self.codes = [np.full(shape, 0xFF if e4m3 else 0xFFFF, np.uint8 if e4m3 else np.uint16) for _ in range(2)]
        self.scales = [np.full(shape[:3], 0xFF, np.uint8) for _ in range(2)] if e4m3 else [None, None]
        for b, n in enumerate(held):
            for p in range(n):
                for w in range(2):
                    self.put(w, b, p, bits(rng, (n_kv_heads, head_dim), std, mean))

    def put(self, w, b, p, bf16_bits):
        """The vectors of position p of row b (w: 0 key, 1 value), from bf16 bits [n_kv_heads, head_dim]."""
        page = self.shape[2]
        at = self.table[b, p // page], slice(None), p % page
        if self.e4m3:
            code, e = og.quantise(si.bf16_bits_to_f64(bf16_bits))
            self.codes[w][at], self.scales[w][at] = code, e + 127
        else:
            self.codes[w][at] = bf16_bits

    def oracle(self):
        if self.e4m3:
            values = [og.dequantise(c, s.astype(np.int64) - 127) for c, s in zip(self.codes, self.scales)]
        else:
            values = [si.bf16_bits_to_f64(c) for c in self.codes]
        return {"k": values[0], "v": values[1], "page_table": self.table}

    def device(self, K):
        """The library's handle; the tensors are its .tensors."""
        if self.e4m3:
            x = [torch.from_numpy(c.copy()).cuda() for c in self.codes]
            s = [torch.from_numpy(c.copy()).cuda() for c in self.scales]
        else:
            x, s = [dev_bf16(c) for c in self.codes], [None, None]
        return K.KVCache.of(x[0], x[1], torch.from_numpy(self.table).cuda(), *s)
