"""Plain references of the key/value cache's operators and the bounds that their
results are held to."""
import numpy as np
import torch

TORCH_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


class PlanReference:
    """The tables of a batch, planned sequence by sequence on the host."""

    def __init__(self, batch, num_pages, page_size, max_pages, first_page=0):
        self.P, self.M, self.N = page_size, max_pages, num_pages
        self.lengths, self.counts = [0] * batch, [0] * batch
        self.rows = [[] for _ in range(batch)]
        self.free = list(range(num_pages - 1, first_page - 1, -1))
        self.below = [-1] * num_pages      # the stack's whole array, popped entries as they were
        self.below[:len(self.free)] = self.free

    def plan(self, n, accepted=None, new_tokens=None, release=None, base=0):
        batch = len(self.rows)
        for b in range(batch):
            if release is not None and release[b] != 0:
                for page in self.rows[b]:
                    self.below[len(self.free)] = page
                    self.free.append(page)
                self.rows[b], self.lengths[b], self.counts[b] = [], 0, 0
        slots, positions = np.full((batch, n), -1, np.int32), np.full((batch, n), -1, np.int32)
        wanted, depth = 0, len(self.free)
        for b in range(batch):
            ok = True
            if self.counts[b] > 0:
                kept = self.counts[b] if accepted is None else accepted[b] + 1
                if 0 <= kept <= self.counts[b]:
                    self.lengths[b] += kept
                else:
                    ok = False
            want = n if new_tokens is None else new_tokens[b]
            ok = ok and 0 <= want <= n
            need = -(-(self.lengths[b] + want) // self.P) if ok else 0
            if ok and need <= self.M:
                extra = max(0, need - len(self.rows[b]))
                wanted += extra
                if extra and wanted > depth:
                    ok = False
                else:
                    for _ in range(extra):
                        self.rows[b].append(self.free.pop())
            else:
                ok = False
            self.counts[b] = want if ok else -1
            for i in range(want if ok else 0):
                at = self.lengths[b] + i
                slots[b, i] = self.rows[b][at // self.P] * self.P + at % self.P
                positions[b, i] = base + at
        return slots, positions

    def table(self):
        t = np.full((len(self.rows), self.M), -1, np.int32)
        for b, row in enumerate(self.rows):
            t[b, :len(row)] = row
        return t


def gather(cache, table, count):
    """The first ``count`` tokens' rows of one sequence, [kv_heads, count, D], fp64 on the host."""
    P = cache.shape[2]
    if count == 0:
        return np.zeros((cache.shape[1], 0, cache.shape[3]))
    pages = torch.as_tensor([int(table[j // P]) for j in range(0, count, P)], device=cache.device)
    x = cache[pages].double().cpu().numpy()           # [pages, H, P, D]
    return x.transpose(1, 0, 2, 3).reshape(cache.shape[1], -1, cache.shape[3])[:, :count]


def attend_reference(q, k_cache, v_cache, table, lengths, counts, prefix_table, prefix_len, scale):
    """softmax(scale q k) v in 64 bits, and the same with |v| and the largest sum of |q k| (for the bound)."""
    B, n, H, D = q.shape
    K = k_cache.shape[1]
    G = H // K
    q64 = q.double().cpu().numpy()
    out, size = np.zeros((B, n, H, D)), np.zeros((B, n, H, D))
    product = 0.0
    pk = gather(k_cache, prefix_table, prefix_len) if prefix_len else np.zeros((K, 0, D))
    pv = gather(v_cache, prefix_table, prefix_len) if prefix_len else np.zeros((K, 0, D))
    for b in range(B):
        m = counts[b]
        if m <= 0:
            continue
        k = np.concatenate([pk, gather(k_cache, table[b], lengths[b] + m)], 1)
        v = np.concatenate([pv, gather(v_cache, table[b], lengths[b] + m)], 1)
        seen = np.arange(k.shape[1])[None] <= prefix_len + lengths[b] + np.arange(m)[:, None]
        for h in range(H):
            z = scale * (q64[b, :m, h] @ k[h // G].T)
            product = max(product, scale * (np.abs(q64[b, :m, h]) @ np.abs(k[h // G]).T).max())
            z = np.where(seen, z, -np.inf)
            w = np.exp(z - z.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            out[b, :m, h] = w @ v[h // G]
            size[b, :m, h] = w @ np.abs(v[h // G])
    return out, size, product


def attend_bound(size, product, dtype, head_dim, keys, v_max):
    """How far an output may be from the 64-bit one.

    With A = sum w |v| / sum w (``size``), each term relative to A:
    * the weights are rounded to the storage type, half a step u: u;
    * the output is rounded to it, and |out| <= A: u (1 + small);
    * a score is a sum of head_dim products in fp32, off by at most head_dim + 2 roundings of 2^-24 of sum |q k| scale
      (``product``), and the exponential by 2^-21 of itself: the weights and their sum move by that, relatively, so
      twice;
    * sums over the keys in fp32: one rounding of 2^-24 an addition, in the product and in the sum of the weights,
      and the joining of parts: 2 (keys + 64) 2^-24.
    fp16 weights below 2^-14 (of the largest one, or of one at most 2^8 times smaller) are off by up to 2^-25 each,
    not relatively; the sum is at least 1 there: keys 2^-25 v_max more.
    """
    t = TORCH_DTYPES[dtype]
    u = torch.finfo(t).eps / 2
    relative = 2 * u * (1 + 2 * u) + 2 * ((head_dim + 2) * 2.0 ** -24 * product + 2.0 ** -21) + \
        2 * (keys + 64) * 2.0 ** -24
    tiny = keys * 2.0 ** -25 * v_max + 2.0 ** -25 if dtype == "f16" else 0.0
    return relative * size + tiny
