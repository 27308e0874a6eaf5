"""Plain 64-bit forms of the operators of branching decoding, written from their definitions (include/del.h), and makers of inputs."""
import math

import numpy as np
import torch

PAGE = 16


def pool(n_pages, layers, nkv, hd, seed, device="cpu"):
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(n_pages, layers, nkv, PAGE, hd, generator=g).to(torch.bfloat16)
    v = torch.randn(n_pages, layers, nkv, hd, PAGE, generator=g).to(torch.bfloat16)
    return k.to(device), v.to(device)


def tables(lengths, cols, n_pages, seed, shared=()):
    """Distinct pages for every row in random order; entries that no position needs hold ids far outside the pool."""
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    t = torch.full((len(lengths), cols), 0x7ffffff0, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lengths):
        m = min(cols, -(-n // PAGE))
        t[b, :m] = torch.tensor(order[at:at + m], dtype=torch.int32)
        at += m
    assert at <= n_pages
    return t


def random_masks(batch, n, seed, empty=True):
    """Ancestor bits of random trees; with `empty` some rows that see no node and some that do not see themselves."""
    rng = np.random.default_rng(seed)
    m = np.zeros((batch, n), dtype=np.uint64)
    for b in range(batch):
        for i in range(n):
            up = 0 if i == 0 else int(m[b, rng.integers(0, i)])
            m[b, i] = up | (1 << i)
            if empty and i and rng.random() < 0.1:
                m[b, i] = 0 if rng.random() < 0.5 else up
    return torch.from_numpy(m.view(np.int64))


def tree_attention_ref(q, k, v, layer, table, lens, nodes, mask, scale=None):
    """(output fp64, A = softmax-weighted sum of |v|, largest sum of |q k| times the scale); rows that are not computed are NaN."""
    batch, n, nh, hd = q.shape
    nkv, n_pages, cols = k.shape[2], k.shape[0], table.shape[1]
    scale = scale or hd ** -0.5
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    out = torch.full((batch, n, nh, hd), math.nan, dtype=torch.float64)
    mass = torch.zeros_like(out)
    dots = 0.0
    for b in range(batch):
        length = min(max(int(lens[b]), 0), cols * PAGE)
        live = n if nodes is None else min(max(int(nodes[b]), 0), n)
        for i in range(live):
            bits = (1 << (i + 1)) - 1 if mask is None else int(mask[b, i]) & (2 ** 64 - 1)
            pos = list(range(length)) + [length + j for j in range(live) if bits >> j & 1]
            pos = [p for p in pos if p < cols * PAGE and 0 <= int(table[b, p // PAGE]) < n_pages]
            if not pos:
                out[b, i] = 0.0
                continue
            p = torch.tensor(pos)
            pg, sl = table[b].cpu().long()[p // PAGE], p % PAGE
            keys, vals = k[pg, layer - 1, :, sl], v[pg, layer - 1, :, :, sl]          # [positions][nkv][hd]
            for h in range(nh):
                c = h // (nh // nkv)
                s = keys[:, c] @ q[b, i, h] * scale
                w = torch.softmax(s, 0)
                out[b, i, h] = (w[:, None] * vals[:, c]).sum(0)
                mass[b, i, h] = (w[:, None] * vals[:, c].abs()).sum(0)
                dots = max(dots, float((keys[:, c].abs() @ q[b, i, h].abs()).nan_to_num(0, 0, 0).max()) * scale)
    return out, mass, dots


def tree_attention_bound(ref, mass, dots, hd, n_keys, low=False):
    """What an output may be off, element by element.  Scores are fp32 sums of hd products, their error at most
    hd * 2^-24 * sum |q k|, plus the conversions to powers of two: e_s.  A probability is off by a factor within 1 +- 2 e_s (its
    own and the normaliser's) and rounded to bf16 (2^-8); sums of up to n_keys terms and a few rescalings in fp32.  The result is
    rounded to bf16 (2^-8), or to a pair of bf16 (2^-16)."""
    e_s = (hd + 4) * 2.0 ** -24 * dots + 2.0 ** -22
    rel = 2.0 ** -8 + 2 * e_s + (n_keys + 64) * 2.0 ** -24
    return mass * rel * 1.01 + ref.abs() * (2.0 ** -16 if low else 2.0 ** -8) + 1e-30


def compact_ref(k, v, src_table, src_pos, counts, dst_table, dst_start):
    k0, v0 = k.clone(), v.clone()
    n_pages = k.shape[0]
    for b in range(src_pos.shape[0]):
        for i in range(min(max(int(counts[b]), 0), src_pos.shape[1])):
            s, d = int(src_pos[b, i]), int(dst_start[b]) + i
            if not (0 <= s < src_table.shape[1] * PAGE and 0 <= d < dst_table.shape[1] * PAGE):
                continue
            sp, dp = int(src_table[b, s // PAGE]), int(dst_table[b, d // PAGE])
            if 0 <= sp < n_pages and 0 <= dp < n_pages:
                k[dp, :, :, d % PAGE] = k0[sp, :, :, s % PAGE]
                v[dp, :, :, :, d % PAGE] = v0[sp, :, :, :, s % PAGE]


def fork_ref(k, v, table, lens, parents, spare, n_spare, new_table, new_lens, counts, room=0, free_pages=None):
    n_pages, n_old, old_cols, new_cols = k.shape[0], table.shape[0], table.shape[1], new_table.shape[1]
    n_spare = min(max(int(n_spare[0]), 0), spare.shape[0])
    k0, v0 = k.clone(), v.clone()
    held, first, at, missing = set(), {}, 0, 0

    def take():
        nonlocal at
        at += 1
        page = int(spare[at - 1]) if at <= n_spare else -1
        return page if 0 <= page < n_pages else -1

    for b in range(parents.shape[0]):
        a = int(parents[b])
        if not 0 <= a < n_old:
            new_lens[b] = 0
            continue
        length = min(max(int(lens[a]), 0), min(old_cols, new_cols) * PAGE)
        new_lens[b] = length
        pages = table[a, : length // PAGE].tolist()
        if length % PAGE:
            src = int(table[a, length // PAGE])
            if first.setdefault(a, b) == b:
                pages.append(src)
            else:
                dst = take()
                if dst >= 0 and 0 <= src < n_pages:
                    k[dst], v[dst] = k0[src], v0[src]
                else:
                    dst, missing = -1, missing + 1
                pages.append(dst)
        while len(pages) < min(new_cols, -(-(length + room) // PAGE)):
            pages.append(take())
            missing += pages[-1] < 0
        new_table[b, : len(pages)] = torch.tensor(pages, dtype=torch.int32)
        held |= set(pages)
    counts[0], counts[1] = 0, missing
    if free_pages is not None:
        free = [p for p in range(n_pages) if p not in held]
        free_pages[: len(free)] = torch.tensor(free, dtype=torch.int32)
        counts[0] = len(free)


def beam_ref(logits, scores, k, finished=None, eos=0):
    """(scores fp64, tokens, rows): the k best of every item by (score descending, row, logit descending, token)."""
    batch, beams, vocab = logits.shape
    x = logits.detach().cpu().double().numpy()
    out = []
    for item in range(batch):
        cands = []
        for b in range(beams):
            cum, row = float(scores[item, b]), x[item, b]
            s = np.full(vocab, -np.inf)
            if math.isfinite(cum):
                if finished is not None and bool(finished[item, b]):
                    s[eos] = cum
                else:
                    with np.errstate(all="ignore"):
                        m = row.max() if not np.isnan(row).any() else np.nan
                        s = cum + (row - (m + np.log(np.exp(row - m).sum())))
                    s[~(s < np.inf)] = -np.inf
            order = np.lexsort((np.arange(vocab), np.where(s > -np.inf, -row, 0), -s))[:k]
            cands += [(-s[t], b, i, int(t)) for i, t in enumerate(order)]
        best = sorted(cands)[:k]
        out.append(([-c[0] for c in best], [c[3] for c in best], [item * beams + c[1] for c in best]))
    return tuple(np.array([o[j] for o in out]) for j in range(3))
