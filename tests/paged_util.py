"""A batch of sequences over a paged cache, on the host in fp64 and on the device: shared by the tests of its operators."""
import numpy as np
import torch

from oracle import quasar_paged_ref as pg
from oracle import quasar_ref as ref
from paper_2603_01399_amd import synth
from gpu_util import bf16_to_dev, f32_to_dev, i32_to_dev

D, BLOCK = 128, 32


def rnd_bits(shape, seed, scale=1.0):
    r = np.random.Generator(np.random.Philox(seed))
    return synth.to_bf16_bits((r.standard_normal(shape) * scale).astype(np.float32))


class Batch:
    """`lengths` cached positions and `news` new rows of each sequence; pages scattered over a pool that holds NaN patterns
    wherever no position lies.  keys, values: [total, Hkv, 128] fp64 of each sequence, as the pages hold them."""

    def __init__(self, qb, kv, page_len, hq, hk, lengths, news, *, layers=1, layer=0, seed=1, spare=3, scaled=True, empty_rows=0, more_columns=1):
        self.kv, self.page_len, self.hq, self.hk, self.lengths, self.news, self.layer = kv, page_len, hq, hk, list(lengths), list(news), layer
        n = len(lengths)
        r = np.random.Generator(np.random.Philox(seed))
        totals = [a + b for a, b in zip(lengths, news)]
        held = [-(-t // page_len) for t in totals]
        columns = max(max(held), 1) + more_columns
        n_pages = sum(held) + spare
        ids = r.permutation(n_pages)[:sum(held)]
        table, at = np.full((n + empty_rows, columns), -1, np.int32), 0
        for s in range(n):
            table[s, :held[s]] = ids[at:at + held[s]]
            at += held[s]
        self.table = table
        dtype = torch.bfloat16 if kv == "bf16" else torch.float8_e4m3fn
        self.scales = [None, None]
        if kv == "e4m3" and scaled:
            self.scales = [(0.02 + 0.08 * r.random((layers, hk))).astype(np.float32) for _ in range(2)]
        self.cache = qb.PagedKvCache(layers, hk, n_pages, page_len=page_len, max_seqs=n + empty_rows, max_pages=columns, dtype=dtype,
                                     **{k: None if s is None else f32_to_dev(s) for k, s in zip(("k_scale", "v_scale"), self.scales)})
        c = self.cache
        c.refs.copy_(i32_to_dev((np.bincount(ids, minlength=n_pages) > 0).astype(np.int32)))
        c.lengths.copy_(i32_to_dev(np.concatenate([lengths, np.zeros(empty_rows)])))
        c.table.copy_(i32_to_dev(table))
        raw = np.full((n_pages, hk, page_len // BLOCK, 2, BLOCK * D), 0xFF7F if kv == "bf16" else 0xFF, np.uint16 if kv == "bf16" else np.uint8)
        places = pg.block_places(kv)
        self.keys, self.values = [], []
        for s in range(n):
            j = np.arange(totals[s])
            for half, to in ((0, self.keys), (1, self.values)):
                bits = rnd_bits((totals[s], hk, D), (seed, s, half))
                if kv == "e4m3":
                    bits = pg.f64_to_e4m3(ref.bf16_bits_to_f64(bits) * 20.0)
                for h in range(hk):
                    raw[table[s, j // page_len][:, None], h, (j % page_len // BLOCK)[:, None], half, places[half][j % BLOCK]] = bits[:, h]
                to.append(self.decoded(bits, half))
        pool = torch.from_numpy(raw.view(np.int16) if kv == "bf16" else raw).cuda()
        c.pool[layer].view(pool.dtype).copy_(pool)
        self.row_start = i32_to_dev(np.concatenate([[0], np.cumsum(news)]))
        self.rows = int(sum(news))
        self.q_bits = rnd_bits((self.rows, hq, D), (seed, 777), 1.3)

    def decoded(self, bits, half):
        """[.., Hkv, 128] bit patterns of the pages -> fp64."""
        if self.kv == "bf16":
            return ref.bf16_bits_to_f64(bits)
        scale = self.scales[half]
        return pg.e4m3_to_f64(bits) * (1.0 if scale is None else scale[self.layer].astype(np.float64)[:, None])

    def read(self, s, count, half):
        """Bit patterns of the first `count` positions of a sequence, from the device: [count, Hkv, 128]."""
        c = self.cache
        raw = c.pool[self.layer].view(torch.int16 if self.kv == "bf16" else torch.uint8).cpu().numpy()
        raw = raw.view(np.uint16) if self.kv == "bf16" else raw
        table, j = c.table.cpu().numpy(), np.arange(count)
        return raw[table[s, j // self.page_len][:, None, None], np.arange(self.hk)[None, :, None], (j % self.page_len // BLOCK)[:, None, None], half,
                   pg.block_places(self.kv)[half][j % BLOCK][:, None, :]]

    def expected(self):
        """(out, tolerance) [rows, Hq, 128] of the attention, fp64.

        A score is off by the fp32 rounding of 128 products and their sum, the scale and the exponent's argument: at most 132 roundings of 2^-24
        of sum |q k| / sqrt(128), so a weight, before it is divided by the sum, by twice that relatively.  It is then rounded to bf16 (2^-8
        relatively), and the sum is one of the rounded weights: what is applied is w (1 + e) / sum w (1 + e), off by at most twice 2^-8 plus twice the
        scores' part, of sum w |v|.  One bf16 rounding of the output (2^-8 of it).  fp32 sums and the exponential are covered by 1 % more."""
        out, tol = [], []
        q = ref.bf16_bits_to_f64(self.q_bits)
        at = 0
        for s, n in enumerate(self.news):
            rows = q[at:at + n]
            at += n
            if not n:
                continue
            o, size = pg.attention(rows, self.keys[s], self.values[s], self.lengths[s])
            most = np.linalg.norm(rows, axis=2).max() * np.linalg.norm(self.keys[s], axis=2).max() / np.sqrt(D)      # >= sum |q k| / sqrt(128)
            out.append(o)
            tol.append(1.01 * (2.0 ** -8 * np.abs(o) + (2.0 ** -7 + 4 * 132 * 2.0 ** -24 * most) * size) + 1e-30)
        return np.concatenate(out), np.concatenate(tol)

    def q(self):
        return bf16_to_dev(self.q_bits.reshape(self.rows, -1))
