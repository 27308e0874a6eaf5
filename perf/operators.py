"""Operators of branching decoding over the paged cache: what is measured of each, and its plain form.

A case is one call of one operator.  Kinds:
  "tree"     attention of a tree of drafted tokens (or of single tokens) over a paged cache
  "path"     the accepted path of a draft tree moved together behind the committed positions, in place
  "keep"     the kept positions of long contexts compacted into fresh pages
  "fork"     rows that share pages reordered: tables, copies of part-filled last pages, the list of free pages
  "beam"     the best continuations over beams and vocabulary

The cache is the framework's: keys [page][layer][kv head][16 tokens][head dim], values [page][layer][kv head][head dim][16 tokens],
bf16.  Shapes (layers, heads, head dimension, vocabulary) are those of the repository's configurations.
"""
import math

import torch

own = False
PAGE = 16

# layers, query heads, kv heads, head dimension of the repository's configurations
SHAPES = {
    "tiny": (4, 4, 4, 64),
    "1b": (16, 32, 8, 64),
    "7b": (32, 32, 32, 128),
    "8b": (32, 32, 8, 128),
    "13b": (40, 40, 40, 128),
}
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _tree(name, model, batch, nodes, length, layers=2):
    return dict(name=name, kind="tree", model=model, batch=batch, nodes=nodes, length=length, layers=layers)


def _path(name, model, batch, nodes, accepted, length):
    return dict(name=name, kind="path", model=model, batch=batch, nodes=nodes, accepted=accepted, length=length)


def _keep(name, model, batch, length, kept):
    return dict(name=name, kind="keep", model=model, batch=batch, length=length, kept=kept)


def _fork(name, model, groups, beams, length, own_tokens):
    return dict(name=name, kind="fork", model=model, groups=groups, beams=beams, length=length, own_tokens=own_tokens)


def _beam(name, batch, beams, k, vocab, dtype, finished):
    return dict(name=name, kind="beam", batch=batch, beams=beams, k=k, vocab=vocab, dtype=dtype, finished=finished)


def listed():
    return [
        # one user early in a conversation, a small draft tree: launch and latency
        _tree("tree 8b x1 short", "8b", 1, 8, 200),
        # the four-sequence workload of the repository in mid-generation, trees of 33 nodes (132 rows per kv head)
        _tree("tree 8b x4 1.3k", "8b", 4, 33, 1300),
        # one user behind a long prompt on a model without shared heads
        _tree("tree 13b x1 3.1k", "13b", 1, 26, 3100),
        # beam search: single tokens of 32 rows over their caches
        _tree("tokens 1b x32 1.1k", "1b", 32, 1, 1100),
        # long contexts, the widest trees: the most of both bytes and operations
        _tree("tree 8b x8 32k", "8b", 8, 64, 32700),
        # four sequences commit what a draft tree of 32 nodes got accepted
        _path("path 8b x4", "8b", 4, 32, 5, 1200),
        # two contexts of 8 000 positions cut down to half
        _keep("keep 1b x2 8k", "1b", 2, 8001, 4003),
        # one step of a four-beam search on the small model
        _fork("fork 1b 1x4", "1b", 1, 4, 1060, 36),
        # one step of sixteen four-beam searches on the large one
        _fork("fork 8b 16x4", "8b", 16, 4, 500, 117),
        # the selection of the same small search, with one finished beam
        _beam("beam 1x4 32000", 1, 4, 4, 32000, "float32", 1),
        # candidates for four searches, twice as many as beams, bf16 logits
        _beam("beam 4x4 128256 bf16", 4, 4, 8, 128256, "bfloat16", 0),
        # the largest step: sixteen searches of eight beams over the large vocabulary
        _beam("beam 16x8 128256", 16, 8, 16, 128256, "float32", 9),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "path", "keep", "fork", "beam"])
    if kind == "tree":
        model = rng.choice(sorted(SHAPES))
        layers, nh, nkv, hd = SHAPES[model]
        batch = _log(rng, 1, 32)
        most = 8 * 32700 * 8 * 128 // (batch * nkv * hd)            # no more cache than the largest listed case reads
        length = _log(rng, 1, max(1, min(32700, most)))
        nodes = _log(rng, 1, max(1, min(64, 8 * 64 * 32 * 128 * 32700 // (batch * nh * hd * length))))
        return dict(kind="tree", model=model, batch=batch, nodes=nodes, length=length, layers=rng.choice([1, 2, 3]))
    model = rng.choice(["tiny", "1b", "8b"])
    layers, nh, nkv, hd = SHAPES[model]
    row = 4 * layers * nkv * hd                                     # bytes of one position
    if kind == "path":
        nodes = rng.randint(2, 64)
        return dict(kind="path", model=model, batch=rng.randint(1, 8), nodes=nodes, accepted=rng.randint(1, max(1, nodes // 2)),
                    length=_log(rng, 1, 1500))
    if kind == "keep":
        batch = rng.randint(1, 4)
        length = _log(rng, 16, min(8001, 2 * 8001 * 32768 // (batch * row)))
        return dict(kind="keep", model=model, batch=batch, length=length, kept=rng.randint(1, max(1, length // 2)))
    if kind == "fork":
        groups, beams = rng.randint(1, 16), rng.randint(2, 4)
        length = _log(rng, 1, 500)
        return dict(kind="fork", model=model, groups=groups, beams=beams, length=length, own_tokens=rng.randint(0, min(length, 117)))
    batch, beams = _log(rng, 1, 16), rng.randint(1, 8)
    vocab = _log(rng, 1000, 128256)
    return dict(kind="beam", batch=batch, beams=beams, k=rng.randint(1, 2 * beams), vocab=vocab, dtype=rng.choice(sorted(DTYPES)),
                finished=rng.randint(0, batch * beams // 2))


def _pages(length):
    return -(-length // PAGE)


def _pool(n_pages, layers, nkv, hd, gen):
    k = torch.randn(n_pages, layers, nkv, PAGE, hd, device="cuda", dtype=torch.bfloat16, generator=gen)
    v = torch.randn(n_pages, layers, nkv, hd, PAGE, device="cuda", dtype=torch.bfloat16, generator=gen)
    return k, v


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = torch.Generator().manual_seed(seed)

    def below(n, *shape):
        return torch.randint(0, n, shape, generator=rnd)

    def random_tree(n):
        """Bits of the nodes that each node of a random tree sees: its ancestors and itself.  Node 0 is the root."""
        seen = []
        for i in range(n):
            up = 0 if i == 0 else seen[int(torch.randint(max(0, i - 8), i, (1,), generator=rnd))]
            bits = up | (1 << i)
            seen.append(bits)
        return [b - (1 << 64) if b >> 63 else b for b in seen]

    kind = case["kind"]
    if kind == "beam":
        n, vocab = case["batch"] * case["beams"], case["vocab"]
        logits = 2.5 * torch.randn(case["batch"], case["beams"], vocab, device="cuda", generator=gen)
        logits += 8.0 * (torch.rand(logits.shape, device="cuda", generator=gen) < 8.0 / vocab)      # a few likely tokens
        scores = -10.0 - 8.0 * torch.rand(case["batch"], case["beams"], device="cuda", generator=gen)
        finished = torch.zeros(n, dtype=torch.bool)
        finished[torch.randperm(n, generator=rnd)[: case["finished"]]] = True
        k = case["k"]
        return dict(case=case, logits=logits.to(DTYPES[case["dtype"]]), scores=scores, eos=2,
                    finished=finished.view(case["batch"], -1).cuda(), out_scores=torch.empty(case["batch"], k, device="cuda"),
                    out_tokens=torch.empty(case["batch"], k, dtype=torch.int32, device="cuda"),
                    out_rows=torch.empty(case["batch"], k, dtype=torch.int32, device="cuda"))

    layers, nh, nkv, hd = SHAPES[case["model"]]
    if kind == "tree":
        batch, n = case["batch"], case["nodes"]
        least = max(1, case["length"] * 7 // 8)
        lens = [case["length"]] + [int(x) + least for x in below(case["length"] - least + 1, batch - 1)]
        nodes = [n] + [max(1, n - int(x)) for x in below(1 + n // 8, batch - 1)]
        per_row = _pages(case["length"] + n)
        n_pages = sum(_pages(a + b) for a, b in zip(lens, nodes)) + 3
        k, v = _pool(n_pages, case["layers"], nkv, hd, gen)
        order, table, at = torch.randperm(n_pages, generator=rnd), torch.zeros(batch, per_row, dtype=torch.int32), 0
        for b in range(batch):
            m = _pages(lens[b] + nodes[b])
            table[b, :m] = order[at:at + m]
            at += m
        mask = torch.tensor([random_tree(n) for _ in range(batch)], dtype=torch.int64).cuda()
        q = 1.5 * torch.randn(batch, n, nh, hd, device="cuda", generator=gen)
        return dict(case=case, q=q.to(torch.bfloat16), k=k, v=v, table=table.cuda(), lens=_int32(lens), nodes=_int32(nodes), mask=mask,
                    layer=case["layers"], max_len=case["length"], out=torch.zeros(batch, n, nh, hd, device="cuda", dtype=torch.bfloat16))

    if kind == "path":
        batch, n, acc = case["batch"], case["nodes"], case["accepted"]
        lens = [case["length"] - int(x) for x in below(max(1, case["length"] // 8), batch)]
        counts = [acc] + [1 + int(x) for x in below(acc, batch - 1)]
        per_row = _pages(case["length"] + n)
        k, v = _pool(batch * per_row, layers, nkv, hd, gen)
        table = torch.randperm(batch * per_row, generator=rnd).to(torch.int32).view(batch, per_row).cuda()
        src = torch.zeros(batch, acc, dtype=torch.int32)
        for b in range(batch):          # the root stays; the other accepted nodes come from behind where the path will lie
            tail = torch.randperm(n - counts[b], generator=rnd)[: counts[b] - 1].sort().values + counts[b]
            src[b, : counts[b]] = lens[b] + torch.cat([torch.zeros(1, dtype=torch.int64), tail])
        return dict(case=case, k=k, v=v, src_table=table, dst_table=table, src=src.cuda(), counts=_int32(counts), start=_int32(lens))

    if kind == "keep":
        batch, length, kept = case["batch"], case["length"], case["kept"]
        counts = [kept] + [kept - int(x) for x in below(1 + kept // 8, batch - 1)]
        old, new = _pages(length), _pages(kept)
        k, v = _pool(batch * (old + new), layers, nkv, hd, gen)
        ids = torch.randperm(batch * (old + new), generator=rnd).to(torch.int32).cuda()
        src = torch.zeros(batch, kept, dtype=torch.int32)
        for b in range(batch):
            src[b, : counts[b]] = torch.randperm(length, generator=rnd)[: counts[b]].sort().values
        return dict(case=case, k=k, v=v, src_table=ids[: batch * old].view(batch, old).contiguous(),
                    dst_table=ids[batch * old:].view(batch, new).contiguous(), src=src.cuda(), counts=_int32(counts),
                    start=_int32([0] * batch))

    groups, beams, length, tail = case["groups"], case["beams"], case["length"], case["own_tokens"]
    rows = groups * beams
    lens = [length - int(x) for x in below(1 + min(tail, 15), groups)]
    shared = [(n - min(tail, n)) // PAGE for n in lens]
    per_row = _pages(length + 1)
    n_pages = groups * (_pages(length) + (beams - 1) * (tail // PAGE + 2)) + rows * 2 + 5      # room for any of these lengths
    k, v = _pool(n_pages, layers, nkv, hd, gen)
    order, table, at = torch.randperm(n_pages, generator=rnd).to(torch.int32), torch.zeros(rows, per_row, dtype=torch.int32), 0
    for g in range(groups):
        prefix = order[at:at + shared[g]]
        at += shared[g]
        for b in range(beams):
            m = _pages(lens[g]) - shared[g]
            table[g * beams + b, : shared[g]] = prefix
            table[g * beams + b, shared[g]: shared[g] + m] = order[at:at + m]
            at += m
    parents = below(beams, groups, beams) + beams * torch.arange(groups)[:, None]
    parents = parents.reshape(-1)
    if groups > 8:
        parents[-beams:] = -1           # the last search is over: its rows are given up
    return dict(case=case, k=k, v=v, table=table.cuda(), lens=_int32([n for n in lens for _ in range(beams)]),
                parents=parents.to(torch.int32).cuda(), spare=order[at:].cuda(), n_spare=_int32([n_pages - at]), room=1,
                new_table=torch.zeros(rows, per_row, dtype=torch.int32, device="cuda"),
                new_lens=torch.zeros(rows, dtype=torch.int32, device="cuda"),
                free=torch.full((n_pages,), -1, dtype=torch.int32, device="cuda"), counts=torch.zeros(2, dtype=torch.int32, device="cuda"))


def _visible(lens, nodes, mask, n, width):
    """[batch][node][position]: committed positions, then the tree's nodes by the bits of the mask."""
    pos = torch.arange(width, device=lens.device)
    j = pos[None, :] - lens[:, None].long()
    bit = (mask[:, :, None] >> j.clamp(0, 63)[:, None, :]) & 1
    in_tree = (j >= 0) & (j < nodes[:, None])
    return (j < 0)[:, None, :] | (in_tree[:, None, :] & (bit == 1))


def _plain_tree(s):
    q, table, layer = s["q"], s["table"].long(), s["layer"] - 1
    batch, n, nh, hd = q.shape
    nkv, width = s["k"].shape[2], table.shape[1] * PAGE
    k = s["k"][table, layer].float().permute(0, 2, 1, 3, 4).reshape(batch, nkv, width, hd)
    v = s["v"][table, layer].float().permute(0, 2, 3, 1, 4).reshape(batch, nkv, hd, width)
    qg = q.float().view(batch, n, nkv, nh // nkv, hd).permute(0, 2, 3, 1, 4).reshape(batch, nkv, -1, hd)
    scores = torch.matmul(qg, k.transpose(2, 3)) / math.sqrt(hd)
    see = _visible(s["lens"], s["nodes"], s["mask"], n, width)[:, None, None]
    scores = scores.view(batch, nkv, nh // nkv, n, width).masked_fill(~see, -math.inf)
    p = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p.view(batch, nkv, -1, width), v.transpose(2, 3))
    o = o.view(batch, nkv, nh // nkv, n, hd).permute(0, 3, 1, 2, 4).reshape(batch, n, nh, hd)
    live = torch.arange(n, device=q.device)[None, :] < s["nodes"][:, None]
    s["out"].copy_(torch.where(live[:, :, None, None], o.to(q.dtype), s["out"]))
    return s["out"]


def _plain_compact(s):
    b, i = torch.nonzero(torch.arange(s["src"].shape[1], device="cuda")[None, :] < s["counts"][:, None], as_tuple=True)
    src, dst = s["src"][b, i].long(), s["start"][b].long() + i
    sp, dp = s["src_table"][b, src // PAGE].long(), s["dst_table"][b, dst // PAGE].long()
    rows_k, rows_v = s["k"][sp, :, :, src % PAGE], s["v"][sp, :, :, :, src % PAGE]
    s["k"][dp, :, :, dst % PAGE] = rows_k
    s["v"][dp, :, :, :, dst % PAGE] = rows_v
    return s["k"], s["v"]


def _plain_fork(s):
    parents, width = s["parents"].long(), s["table"].shape[1]
    rows = torch.arange(parents.shape[0], device="cuda")
    live = parents >= 0
    old = parents.clamp(min=0)
    lens = torch.where(live, s["lens"][old].long(), 0)
    full, part = lens // PAGE, lens % PAGE > 0
    first = torch.full((s["table"].shape[0],), parents.shape[0], device="cuda").scatter_reduce(0, old, torch.where(live, rows, parents.shape[0]), "amin")
    keeps = live & (first[old] == rows)
    copies = (part & ~keeps).long()
    wanted = torch.where(live, ((lens + s["room"] + PAGE - 1) // PAGE).clamp(max=width), 0)
    fresh = copies + (wanted - (lens + PAGE - 1) // PAGE).clamp(min=0)
    base = torch.cumsum(fresh, 0) - fresh
    page = torch.arange(width, device="cuda")[None, :]
    first_new = full + (part & keeps).long()                              # the row's first page that is not its parent's
    from_spare = base[:, None] + page - first_new[:, None]
    spare = s["spare"][from_spare.clamp(0, s["spare"].shape[0] - 1)]
    table = torch.where(page < first_new[:, None], s["table"][old], spare)
    used = page < wanted[:, None]
    s["new_table"].copy_(torch.where(used, table, s["new_table"]))
    s["new_lens"].copy_(lens)
    c = torch.nonzero(copies).flatten()
    source, target = s["table"][old[c], full[c]].long(), s["new_table"][c, full[c]].long()
    s["k"][target], s["v"][target] = s["k"][source], s["v"][source]
    taken = torch.zeros(s["k"].shape[0], dtype=torch.bool, device="cuda")
    taken[s["new_table"][used].long()] = True
    free = torch.nonzero(~taken).flatten()
    s["free"][: free.shape[0]] = free.to(torch.int32)
    s["counts"].copy_(torch.tensor([free.shape[0], 0], device="cuda"))
    return s["k"], s["v"], s["new_table"], s["new_lens"], s["free"], s["counts"]


def _plain_beam(s):
    logits = s["logits"].double()                        # in 64 bits: the order of near candidates hangs on it
    batch, beams, vocab = logits.shape
    top = logits.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(-1, keepdim=True))
    each = s["scores"].double()[:, :, None] + (logits - lse)
    at_eos = torch.arange(vocab, device="cuda") == s["eos"]
    done = torch.where(at_eos, s["scores"].double()[:, :, None], -math.inf)
    each = torch.where(s["finished"][:, :, None], done, each)
    each = torch.where(each < math.inf, each, -math.inf)
    best, at = torch.sort(each.view(batch, -1), dim=1, descending=True, stable=True)
    best, at = best[:, : s["case"]["k"]], at[:, : s["case"]["k"]]
    s["out_scores"].copy_(best)
    s["out_tokens"].copy_(at % vocab)
    s["out_rows"].copy_(at // vocab + beams * torch.arange(batch, device="cuda")[:, None])
    return s["out_scores"], s["out_tokens"], s["out_rows"]


def _own(s):
    import paper_2504_05598_b200 as dl
    kind = s["case"]["kind"]
    if kind == "tree":
        dl.tree_attention(s["q"], s["k"], s["v"], s["layer"], s["table"], s["lens"], s["nodes"], s["mask"], out=s["out"], max_len=s["max_len"])
        return s["out"]
    if kind in ("path", "keep"):
        dl.kv_compact(s["k"], s["v"], s["src_table"], s["src"], s["counts"], s["dst_table"], s["start"])
        return s["k"], s["v"]
    if kind == "fork":
        dl.kv_fork(s["k"], s["v"], s["table"], s["lens"], s["parents"], s["spare"], s["n_spare"], s["new_table"], s["new_lens"],
                   room=s["room"], free_pages=s["free"], counts=s["counts"])
        return s["k"], s["v"], s["new_table"], s["new_lens"], s["free"], s["counts"]
    dl.beam_select(s["logits"], s["scores"], s["out_scores"], s["out_tokens"], s["out_rows"], finished=s["finished"], eos=s["eos"])
    return s["out_scores"], s["out_tokens"], s["out_rows"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    plain = {"tree": _plain_tree, "path": _plain_compact, "keep": _plain_compact, "fork": _plain_fork, "beam": _plain_beam}
    return plain[kind](state)


def work(case):
    kind = case["kind"]
    if kind == "beam":
        values = case["batch"] * case["beams"] * case["vocab"]
        return {"bytes": values * DTYPES[case["dtype"]].itemsize + 12 * case["batch"] * case["k"], "flops": 4 * values}
    layers, nh, nkv, hd = SHAPES[case["model"]]
    if kind == "tree":
        rows, length = case["batch"] * case["nodes"], case["length"] * 15 / 16
        cache = case["batch"] * (length + case["nodes"]) * nkv * hd * 4
        return {"bytes": cache + rows * (nh * hd * 4 + 8), "flops": rows * nh * hd * 4 * (length + 4)}
    row = 4 * layers * nkv * hd
    if kind == "path":
        return {"bytes": 2 * row * max(1, case["batch"] * (case["accepted"] - 1) * 3 // 4), "flops": 0}
    if kind == "keep":
        return {"bytes": 2 * row * case["batch"] * case["kept"] * 15 / 16, "flops": 0}
    rows, beams = case["groups"] * case["beams"], case["beams"]
    copied = rows * (1 - 1 / beams) ** beams            # rows that are not their parent's first child
    return {"bytes": 2 * PAGE * row * copied * 15 / 16 + 8 * rows * _pages(case["length"] + 1), "flops": 0}


def exact(case, seed):
    def tree(s):
        q, out = s["q"].double(), s["out"].double()
        batch, n, nh, hd = q.shape
        nkv = s["k"].shape[2]
        for b in range(batch):
            length, live = int(s["lens"][b]), int(s["nodes"][b])
            pages = s["table"][b, : _pages(length + live)].long()
            bits = [[(int(m) >> j) & 1 for j in range(live)] for m in s["mask"][b, :live]]
            bias = torch.zeros(live, length + live, dtype=torch.float64, device="cuda")
            bias[:, length:] = torch.where(torch.tensor(bits, device="cuda") == 1, 0.0, -math.inf)
            for h in range(nkv):
                keys = s["k"][pages, s["layer"] - 1, h].double().reshape(-1, hd)[: length + live]
                values = s["v"][pages, s["layer"] - 1, h].double().transpose(1, 2).reshape(-1, hd)[: length + live]
                for g in range(h * nh // nkv, (h + 1) * nh // nkv):
                    out[b, :live, g] = torch.softmax(q[b, :live, g] @ keys.T * hd ** -0.5 + bias, -1) @ values
        return out

    def beam(s):
        beams, vocab = s["logits"].shape[1:]
        best = []
        for item, scores, finished in zip(s["logits"], s["scores"], s["finished"]):
            each = torch.log_softmax(item.double(), -1) + scores.double()[:, None]
            for b in torch.nonzero(finished).flatten().tolist():
                each[b] = -math.inf
                each[b, s["eos"]] = scores[b].double()
            best.append(torch.topk(each.flatten(), s["case"]["k"]).values)
        return torch.stack(best), None, None

    if case["kind"] not in ("tree", "beam"):
        return None                                     # nothing is computed: bits are moved
    s = prepare(case, seed)
    return tree(s) if case["kind"] == "tree" else beam(s)
