"""fp64 CPU oracles for rotary positions, page means, page selection and attention over listed pages -- TEST INFRASTRUCTURE ONLY.

The paper notes that sparse attention flattens the growth of the attention cost with the prefix (its "Impact of Sparse
Attention" paragraph) without defining a selection for models with ordinary key/value heads.  What these functions fix:

  * rotation: pair (a, b) of a row at position p turns by p * inv_freq[j]; "half" pairs feature j with j + rot / 2 of the rotated part,
    "interleaved" 2 j with 2 j + 1; both results are multiplied by the amplitude; other features are copied;
  * the mean key of a page is the mean over its block_size keys;
  * the score of page b for token t and kv-head g is the sum over the q-heads h of g of <q_h(t), mean_b>; a token of position p lists pages 0 .. c,
    c = p // block_size: all of them if there are at most topk, else the first num_first, the last num_last and the best of the others,
    ties to the lowest index, NaN below everything; ascending, -1 behind;
  * attention over listed pages is Eq. 1 over the keys at or before the token's position in the pages of its list (a set: listed twice counts
    once; entries outside 0 .. c are skipped); a token with no page left has out = 0 and lse = -inf.

Plain numpy in float64, one row at a time.  Nothing here imports or shares code with the CUDA library.
"""
import numpy as np


def rows_of(prefix_len, chunk_len):
    """(request, position) of every packed row."""
    return [(r, int(p) + i) for r, (p, c) in enumerate(zip(prefix_len, chunk_len)) for i in range(int(c))]


def ref_rope(x, positions, inv_freq, layout="half", offset=0, amplitude=1.0):
    """x float64 [T, H, D] -> float64 [T, H, D]."""
    y = np.array(x, np.float64)
    half = len(inv_freq)
    for t, p in enumerate(positions):
        for j in range(half):
            angle = float(p) * float(inv_freq[j])
            c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
            ia, ib = (offset + j, offset + j + half) if layout == "half" else (offset + 2 * j, offset + 2 * j + 1)
            a, b = np.array(x[t, :, ia], np.float64), np.array(x[t, :, ib], np.float64)
            y[t, :, ia] = a * c - b * s
            y[t, :, ib] = b * c + a * s
    return y


def completed_pages(prefix_len, chunk_len, block_size):
    """(request, logical page) of every page whose last position is in the chunk."""
    return [(r, j) for r, (p, c) in enumerate(zip(prefix_len, chunk_len)) for j in range(int(p) // block_size, (int(p) + int(c)) // block_size)]


def ref_block_means(k_cache, block_table, prefix_len, chunk_len, block_size):
    """{physical page: float64 [Hkv, D]} of the pages that the chunk completes; k_cache float64 [num_blocks, block_size, Hkv, D]."""
    return {int(block_table[r, j]): k_cache[int(block_table[r, j])].sum(axis=0) / block_size
            for r, j in completed_pages(prefix_len, chunk_len, block_size)}


def ref_block_select(q, k_means, block_table, prefix_len, chunk_len, block_size, topk, num_first, num_last):
    """q float64 [T, Hq, D], k_means float64 [num_blocks, Hkv, D] -> int32 [T, Hkv, topk]."""
    hkv = k_means.shape[1]
    group = q.shape[1] // hkv
    out = np.full((q.shape[0], hkv, topk), -1, np.int32)
    for t, (r, p) in enumerate(rows_of(prefix_len, chunk_len)):
        c = p // block_size
        for g in range(hkv):
            if c + 1 <= topk:
                out[t, g, :c + 1] = np.arange(c + 1)
                continue
            sure = list(range(num_first)) + list(range(c + 1 - num_last, c + 1))
            rest = np.arange(num_first, c + 1 - num_last)
            with np.errstate(all="ignore"):
                ask = q[t, g * group:(g + 1) * group].sum(axis=0)
                score = (k_means[block_table[r, rest], g] * ask).sum(axis=1)
            score = np.where(np.isnan(score), -np.inf, score)
            best = np.lexsort((rest, -score))[:topk - num_first - num_last]
            out[t, g] = np.sort(np.concatenate([sure, rest[best]]))
    return out


def ref_block_attn(q, k_cache, v_cache, lists, block_table, prefix_len, chunk_len, block_size, scale):
    """q float64 [T, Hq, D], caches float64 [num_blocks, block_size, Hkv, D], lists int [T, Hkv, topk].  Returns (out [T, Hq, D], lse [T, Hq],
    weighted mean of |v| [T, Hq, D]: what a relative error of the weights is multiplied by)."""
    T, hq, d = q.shape
    hkv = k_cache.shape[2]
    group = hq // hkv
    out, lse, mag = np.zeros((T, hq, d)), np.full((T, hq), -np.inf), np.zeros((T, hq, d))
    for t, (r, p) in enumerate(rows_of(prefix_len, chunk_len)):
        for g in range(hkv):
            pages = sorted({int(e) for e in lists[t, g] if 0 <= e <= p // block_size})
            if not pages:
                continue
            at = np.concatenate([np.arange(e * block_size, min((e + 1) * block_size, p + 1)) for e in pages])
            blk = block_table[r, at // block_size]
            k, v = k_cache[blk, at % block_size, g], v_cache[blk, at % block_size, g]
            heads = slice(g * group, (g + 1) * group)
            s = scale * (q[t, heads] @ k.T)
            m = s.max(axis=1, keepdims=True)
            w = np.exp(s - m)
            total = w.sum(axis=1, keepdims=True)
            out[t, heads] = (w / total) @ v
            mag[t, heads] = (w / total) @ np.abs(v)
            lse[t, heads] = (m + np.log(total))[:, 0]
    return out, lse, mag
