"""Speculative decoding over the KV cache, as cases that can be timed and compared: attention of a
tree of drafted tokens, verification of the drafts, moving the accepted path's rows into place, and
the pages of the cache (fork, grow with copy on write, free, defragment).

`run` computes a case in plain torch operations, or, where `own` is true, with the library."""
import math

import numpy as np
import torch

own = False

HEADS = 40      # the paper's 13B-class layer: 40 heads of 128
KINDS = ("attention", "verify", "keep", "pages", "defragment")


# ---------------------------------------------------------------- cases
def listed():
    return [
        # the smallest step: one sequence, eight drafted tokens, a short contiguous cache (latency)
        dict(name="tree_short", kind="attention", batch=1, q_heads=HEADS, kv_heads=HEADS, head_dim=128, nodes=8,
             ragged_nodes=False, len_lo=1024, len_hi=1024, block_tokens=0),
        # the 13B-class step: ragged 4k-8k contexts in 32-token pages, 64 drafted tokens a sequence
        dict(name="tree_64_ragged", kind="attention", batch=16, q_heads=HEADS, kv_heads=HEADS, head_dim=128, nodes=64,
             ragged_nodes=False, len_lo=4096, len_hi=8192, block_tokens=32),
        # grouped heads over a long context: 256 query rows share every cached key
        dict(name="tree_grouped_long", kind="attention", batch=8, q_heads=64, kv_heads=8, head_dim=128, nodes=32,
             ragged_nodes=True, len_lo=32768, len_hi=32768, block_tokens=64),
        # wide heads, odd counts: 25 nodes of 3 heads a group, trees of several sizes, lengths from a few tokens on
        dict(name="tree_d256_odd", kind="attention", batch=7, q_heads=15, kv_heads=5, head_dim=256, nodes=25,
             ragged_nodes=True, len_lo=33, len_hi=20011, block_tokens=16),
        # one sequence's drafts from a 32000-token vocabulary (latency)
        dict(name="verify_one", kind="verify", batch=1, nodes=8, vocab=32000, dtype="float32", drafted=True, noise=0.5),
        # a full batch, wide trees, an odd vocabulary, probabilities in bf16
        dict(name="verify_batch", kind="verify", batch=64, nodes=32, vocab=50257, dtype="bfloat16", drafted=True, noise=1.0),
        # one sequence of one layer: a few rows (latency)
        dict(name="keep_one", kind="keep", layers=1, batch=1, heads=HEADS, head_dim=128, nodes=8, kept=4, length=600,
             block_tokens=0),
        # every layer of the 13B-class model at once, 32-token pages
        dict(name="keep_40_layers", kind="keep", layers=40, batch=16, heads=HEADS, head_dim=128, nodes=64, kept=7, length=110,
             block_tokens=32),
        # one sequence forked into four continuations, one layer
        dict(name="pages_fork_4", kind="pages", layers=1, heads=HEADS, head_dim=128, block_tokens=16, parents=1, children=4,
             length=1000, grow=17, blocks=512),
        # sixteen prompts, three samples each, many layers; a pool of which most is in use
        dict(name="pages_fork_48", kind="pages", layers=16, heads=HEADS, head_dim=128, block_tokens=32, parents=16, children=3,
             length=240, grow=40, blocks=320),
        # a small pool, one layer (latency)
        dict(name="defragment_small", kind="defragment", layers=1, heads=8, head_dim=128, block_tokens=16, sequences=5,
             length=300, blocks=400),
        # half of a pool of 64-token pages in all layers moves
        dict(name="defragment_large", kind="defragment", layers=8, heads=HEADS, head_dim=128, block_tokens=64, sequences=12,
             length=1500, blocks=640),
    ]


def log_int(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(KINDS + ("attention", "attention"))
    if kind == "attention":
        while True:
            kv = log_int(rng, 1, 40)
            group = rng.choice([1, 1, 2, 3, 4, 5, 8])
            hi = log_int(rng, 1, 40000)
            c = dict(kind=kind, batch=log_int(rng, 1, 24), q_heads=kv * group, kv_heads=kv,
                     head_dim=rng.choice([64, 128, 128, 256]), nodes=log_int(rng, 1, 128), ragged_nodes=rng.random() < 0.5,
                     len_lo=0, len_hi=hi, block_tokens=rng.choice([0, 16, 32, 48, 64, 128, 256]))
            c["len_hi"] = max(c["len_hi"], c["nodes"])
            c["len_lo"] = max(c["nodes"], int(c["len_hi"] * rng.choice([0.1, 0.5, 1.0])))
            w = work(c)
            if w["bytes"] < 2.0e9 and w["flops"] < 1.2e11:
                return c
    if kind == "verify":
        while True:
            c = dict(kind=kind, batch=log_int(rng, 1, 96), nodes=log_int(rng, 1, 128), vocab=log_int(rng, 30, 140000),
                     dtype=rng.choice(["float32", "float16", "bfloat16"]), drafted=rng.random() < 0.7,
                     noise=rng.choice([0.1, 0.5, 1.0, 2.0]))
            if c["batch"] * c["nodes"] * c["vocab"] <= 64 * 32 * 50257 and c["batch"] * c["vocab"] <= 64 * 50257:
                return c
    if kind == "keep":
        while True:
            nodes = log_int(rng, 2, 128)
            c = dict(kind=kind, layers=log_int(rng, 1, 40), batch=log_int(rng, 1, 24), heads=log_int(rng, 1, 40),
                     head_dim=rng.choice([64, 128, 256]), nodes=nodes, kept=max(1, min(nodes // 2, log_int(rng, 1, 12))),
                     length=nodes + log_int(rng, 1, 300), block_tokens=rng.choice([0, 8, 16, 32, 64]))
            if work(c)["bytes"] <= 1.5e8 and c["layers"] * c["batch"] * c["heads"] * c["head_dim"] * c["length"] <= 5e8:
                return c
    if kind == "pages":
        while True:
            c = dict(kind=kind, layers=log_int(rng, 1, 24), heads=log_int(rng, 1, 40), head_dim=rng.choice([64, 128, 256]),
                     block_tokens=rng.choice([8, 16, 32, 64]), parents=log_int(rng, 1, 16), children=rng.randint(1, 4),
                     length=log_int(rng, 1, 1000), grow=log_int(rng, 1, 100), blocks=0)
            per = -(-(c["length"] + c["grow"]) // c["block_tokens"])
            c["blocks"] = c["parents"] * (c["children"] + 1) * per + rng.randint(1, 40)
            size = c["layers"] * c["blocks"] * c["heads"] * c["head_dim"] * c["block_tokens"]
            if size <= 8.0e8 and work(c)["bytes"] <= 9e8:
                return c
    while True:
        c = dict(kind="defragment", layers=log_int(rng, 1, 16), heads=log_int(rng, 1, 40), head_dim=rng.choice([64, 128, 256]),
                 block_tokens=rng.choice([8, 16, 32, 64]), sequences=log_int(rng, 1, 24), length=log_int(rng, 1, 1500), blocks=0)
        per = -(-c["length"] // c["block_tokens"])
        c["blocks"] = 2 * c["sequences"] * per + rng.randint(1, 40)
        if c["layers"] * c["blocks"] * c["heads"] * c["head_dim"] * c["block_tokens"] <= 1.0e9:
            return c


def lengths_of(c):
    """The sequences' lengths: spread evenly from len_lo to len_hi, the longest first."""
    n = c["batch"]
    return [c["len_hi"] - (c["len_hi"] - c["len_lo"]) * i // max(1, n - 1) for i in range(n)]


def nodes_of(c):
    return [max(1, c["nodes"] - (i % 3) * (c["nodes"] // 4)) if c["ragged_nodes"] else c["nodes"] for i in range(c["batch"])]


def work(c):
    if c["kind"] == "attention":
        rows = c["q_heads"] * c["nodes"] * c["batch"]
        keys = sum(lengths_of(c))
        live = sum(n * length for n, length in zip(nodes_of(c), lengths_of(c)))
        return dict(bytes=keys * c["kv_heads"] * c["head_dim"] * 4 + rows * c["head_dim"] * 4 + rows * 4,
                    flops=4 * c["q_heads"] * c["head_dim"] * live)
    if c["kind"] == "verify":
        # a row of the target's probabilities for the last draw, one of the draft's for a residual
        size = 4 if c["dtype"] == "float32" else 2
        return dict(bytes=c["batch"] * (c["vocab"] * size * (2 if c["drafted"] else 1) + c["nodes"] * 24),
                    flops=c["batch"] * c["vocab"] * 4)
    row = 2 * c["layers"] * c["heads"] * c["head_dim"] * 2      # K and V of one token in all layers
    if c["kind"] == "keep":
        return dict(bytes=2 * row * c["batch"] * (c["kept"] - 1) + 8 * c["batch"] * (c["nodes"] + 2), flops=0)
    if c["kind"] == "pages":
        copies = c["parents"] * c["children"] if c["length"] % c["block_tokens"] else 0
        entries = c["parents"] * (1 + c["children"]) * -(-(c["length"] + c["grow"]) // c["block_tokens"])
        return dict(bytes=2 * row * c["block_tokens"] * copies + 12 * entries + 8 * c["blocks"], flops=0)
    used = c["sequences"] * -(-c["length"] // c["block_tokens"])
    # half of the used blocks lie behind the used count, where every second block is in use
    return dict(bytes=2 * row * c["block_tokens"] * (used // 2) + 8 * used + 8 * c["blocks"], flops=0)


# ---------------------------------------------------------------- inputs
def normal(g, *shape, dtype=torch.float16):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32 if math.prod(shape) < 1 << 26 else dtype).to(dtype)


def random_parents(rng, nodes):
    """A tree in which a parent comes before its children: -1 for the root, mostly recent nodes."""
    t = np.arange(nodes)
    back = np.minimum(rng.geometric(0.35, nodes), t)
    return np.where(t == 0, -1, t - np.maximum(back, 1)).astype(np.int32)


def ancestor_bits(parents, words):
    """Row t: the bits of t and of all nodes on its way to the root."""
    bits = np.zeros((len(parents), words), dtype=np.uint64)
    for t, up in enumerate(parents):
        if up >= 0:
            bits[t] = bits[up]
        bits[t, t // 64] |= np.uint64(1) << np.uint64(t % 64)
    return bits


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    on_gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    state = dict(PREPARE[case["kind"]](case, g, rng, on_gpu))
    state.update(kind=case["kind"], flags=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return state


def prepare_attention(c, g, rng, on_gpu):
    lens, nodes, T = lengths_of(c), nodes_of(c), c["block_tokens"]
    words = -(-c["nodes"] // 64)
    bits = np.zeros((c["batch"], c["nodes"], words), dtype=np.uint64)
    for b, n in enumerate(nodes):
        bits[b, :n] = ancestor_bits(random_parents(rng, n), words)
    kv, d = c["kv_heads"], c["head_dim"]
    if T:
        per = -(-c["len_hi"] // T)
        blocks = sum(-(-n // T) for n in lens)
        table = np.zeros((c["batch"], per), dtype=np.int32)
        ids, at = rng.permutation(blocks), 0
        for b, n in enumerate(lens):
            need = -(-n // T)
            table[b, :need] = ids[at:at + need]
            at += need
        shape, table = (blocks, kv, T, d), on_gpu(table)
    else:
        shape, table = (c["batch"], kv, c["len_hi"], d), None
    q = normal(g, c["batch"], c["nodes"], c["q_heads"], d)
    return dict(q=q, k=normal(g, *shape), v=normal(g, *shape), table=table, lens=on_gpu(np.array(lens, dtype=np.int32)),
                nodes=on_gpu(np.array(nodes, dtype=np.int32)), mask=on_gpu(bits.view(np.int64)), max_len=c["len_hi"],
                scale=1.0 / math.sqrt(d), out=torch.empty_like(q),
                lse=torch.empty(q.shape[:3], dtype=torch.float32, device="cuda"), scratch={})


def prepare_verify(c, g, rng, on_gpu):
    B, N, V = c["batch"], c["nodes"], c["vocab"]
    logits = 3.0 * torch.randn(B, N, V, generator=g, device="cuda")
    target = torch.softmax(logits, dim=-1)
    draft = torch.softmax(logits.add_(torch.randn(B, N, V, generator=g, device="cuda"), alpha=c["noise"]), dim=-1)
    del logits
    parents = on_gpu(np.stack([random_parents(rng, N) for _ in range(B)]))
    # a node's token is drawn from the draft's distribution at its parent; the root's is any
    rows = draft.gather(1, parents.clamp(min=0).long()[:, :, None].expand(B, N, V)).reshape(B * N, V)
    tokens = torch.multinomial(rows, 1, generator=g).reshape(B, N).int()
    dtype = getattr(torch, c["dtype"])
    new = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(target=target.to(dtype), draft=draft.to(dtype) if c["drafted"] else None, tokens=tokens, parents=parents,
                uniforms=torch.rand(B, N, generator=g, device="cuda"),
                nodes=on_gpu(np.array([max(1, N - (i % 3) * (N // 4)) for i in range(B)], dtype=np.int32)),
                path=new(B, N), path_lens=new(B), emitted=new(B, N))


def caches(g, c, shape):
    both = [normal(g, c["layers"], *shape) for _ in range(2)]
    return dict(k=both[0], v=both[1], k_layers=list(both[0].unbind(0)), v_layers=list(both[1].unbind(0)))


def prepare_keep(c, g, rng, on_gpu):
    B, T, N = c["batch"], c["block_tokens"], c["nodes"]
    per = -(-c["length"] // T) if T else 0
    shape = (B * per, c["heads"], T, c["head_dim"]) if T else (B, c["heads"], c["length"], c["head_dim"])
    path = np.full((B, N), -1, dtype=np.int32)
    for b in range(B):      # the root stays; the others all move
        rest = np.arange(2, N) if N > c["kept"] else np.arange(1, N)
        path[b, :c["kept"]] = [0, *sorted(rng.choice(rest, c["kept"] - 1, replace=False))]
    full = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(caches(g, c, shape), table=on_gpu(rng.permutation(B * per).astype(np.int32).reshape(B, per)) if T else None,
                path=on_gpu(path), path_lens=full(c["kept"]), nodes=full(N), lens=full(c["length"]), new_lens=full(0))


def prepare_pages(c, g, rng, on_gpu):
    T, n, kids = c["block_tokens"], c["parents"], c["children"]
    B, per, all_per = n * (1 + kids), -(-c["length"] // T), -(-(c["length"] + c["grow"]) // T)
    table = np.full((B, all_per), -1, dtype=np.int32)
    table[:n, :per] = rng.permutation(c["blocks"])[:n * per].reshape(n, per)
    refs = np.zeros(c["blocks"], dtype=np.int32)
    refs[table[:n, :per].ravel()] = 1
    base = np.where(np.arange(B) < n, c["length"], 0).astype(np.int32)
    want = np.where(np.arange(B) < n, c["length"], c["length"] + c["grow"]).astype(np.int32)
    return dict(caches(g, c, (c["blocks"], c["heads"], T, c["head_dim"])), table=on_gpu(table), refs=on_gpu(refs),
                lens=on_gpu(base), base=on_gpu(base), want=on_gpu(want), grown=on_gpu(want * 0), block_tokens=T,
                src=on_gpu((np.arange(n * kids) // kids).astype(np.int32)),
                dst=on_gpu(n + np.arange(n * kids).astype(np.int32)), scratch={})


def prepare_defragment(c, g, rng, on_gpu):
    T, S = c["block_tokens"], c["sequences"]
    per = -(-c["length"] // T)
    ids = np.arange(0, 2 * S * per, 2) + rng.integers(0, 2, S * per)       # one of each two neighbours is in use
    table = rng.permutation(ids).astype(np.int32).reshape(S, per)
    refs = np.zeros(c["blocks"], dtype=np.int32)
    refs[table.ravel()] = 1
    return dict(caches(g, c, (c["blocks"], c["heads"], T, c["head_dim"])), table=on_gpu(table), refs=on_gpu(refs),
                lens=torch.full((S,), c["length"], dtype=torch.int32, device="cuda"), new_table=on_gpu(table * 0 - 1),
                new_refs=on_gpu(refs * 0), used=torch.zeros(1, dtype=torch.int32, device="cuda"), block_tokens=T, scratch={})


PREPARE = dict(attention=prepare_attention, verify=prepare_verify, keep=prepare_keep, pages=prepare_pages,
               defragment=prepare_defragment)


# ---------------------------------------------------------------- one pass
def run(state):
    return (OWN if own else PLAIN)[state["kind"]](state)


# The plain forms: torch operations on whole tensors.
def rows_of(cache, table):
    """[B, H, L, D] in 32 bits from a contiguous cache, or from the pages that the table lists."""
    if table is None:
        return cache.float()
    pages = cache[table.long()]                                   # [B, M, H, T, D]
    B, M, H, T, D = pages.shape
    return pages.permute(0, 2, 1, 3, 4).reshape(B, H, M * T, D).float()


def plain_attention(s):
    B, N, Hq, D = s["q"].shape
    k, v = rows_of(s["k"], s["table"])[:, :, :s["max_len"]], rows_of(s["v"], s["table"])[:, :, :s["max_len"]]
    H, L = k.shape[1:3]
    group = Hq // H
    at = torch.arange(L, device="cuda")
    prefix = (s["lens"] - s["nodes"])[:, None]
    node = (at - prefix).clamp(0, N - 1)                          # [B, L]
    bits = s["mask"].gather(2, (node // 64)[:, None, :].expand(B, N, L)) if s["mask"].shape[2] > 1 else s["mask"]
    sees = ((bits >> (node % 64)[:, None, :]) & 1).bool() | (at < prefix)[:, None, :]
    sees &= (at < s["lens"][:, None])[:, None, :]
    sees &= (torch.arange(N, device="cuda") < s["nodes"][:, None])[:, :, None]
    q = s["q"].float().reshape(B, N, H, group, D).permute(0, 2, 1, 3, 4).reshape(B, H, N * group, D)
    logits = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(B, H, N, group, L)
    logits.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = logits.sub_(top.clamp(min=-1e30)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = (weights.view(B, H, N * group, L) @ v).view(B, H, N, group, D) / total.clamp(min=1e-37)
    lse = top + total.log()
    return (out.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D).half(), lse[..., 0].permute(0, 2, 1, 3).reshape(B, N, Hq))


def plain_verify(s):
    """One step per node, since whether a node is tried follows from the nodes before it; all sequences at once."""
    B, N, V = s["target"].shape
    row = torch.arange(B, device="cuda")
    target, draft = s["target"], s["draft"]
    at = torch.zeros(B, dtype=torch.long, device="cuda")          # the node that each sequence stands at
    w, total = target[:, 0].double(), torch.ones(B, dtype=torch.float64, device="cuda")
    kept = torch.zeros(B, N, dtype=torch.bool, device="cuda")
    kept[:, 0] = s["nodes"] > 0
    for t in range(1, N):
        tried = (s["parents"][:, t] == at) & (t < s["nodes"])
        x = s["tokens"][:, t].long()
        q = torch.zeros_like(w).scatter_(1, x[:, None], 1.0) if draft is None else draft[row, at].double()
        taken = tried & (s["uniforms"][:, t].double() * q[row, x] * total < w[row, x])
        left = (w - total[:, None] * q).clamp_(min=0)
        left_total = left.sum(1)
        shrunk = tried & ~taken & (left_total > 0)
        w = torch.where(shrunk[:, None], left, w)
        total = torch.where(shrunk, left_total, total)
        w = torch.where(taken[:, None], target[:, t].double(), w)
        total = torch.where(taken, 1.0, total)
        at = torch.where(taken, t, at)
        kept[:, t] = taken
    sums = w.cumsum(1)
    last = torch.where(sums > s["uniforms"][:, :1].double() * sums[:, -1:], 1, 0).argmax(1)
    count = kept.sum(1)
    order = torch.argsort((~kept).int(), dim=1, stable=True)
    place = torch.arange(N, device="cuda")
    path = torch.where(place < count[:, None], order, -1)
    token = s["tokens"].gather(1, order.roll(-1, 1)).long()       # the token of the path's next node
    emitted = torch.where(place < count[:, None] - 1, token, torch.where(place == count[:, None] - 1, last[:, None], -1))
    return path.int(), count.int(), emitted.int()


def plain_keep(s):
    B, N = s["path"].shape
    prefix = (s["lens"] - s["nodes"]).long()[:, None]
    place = torch.arange(N, device="cuda")
    moves = place < s["path_lens"][:, None]
    src, dst = prefix + torch.where(moves, s["path"].long(), place), prefix + place
    new_lens = (prefix[:, 0] + s["path_lens"]).int()
    row = torch.arange(B, device="cuda")[:, None]
    for cache in (s["k"], s["v"]):
        if s["table"] is None:
            cache[:, row, :, dst] = cache[:, row, :, src]
        else:
            T = cache.shape[3]
            there, here = s["table"][row, dst // T].long(), s["table"][row, src // T].long()
            cache[:, there, :, dst % T] = cache[:, here, :, src % T]
    return s["k"], s["v"], new_lens


def plain_fork(s):
    src, dst, T = s["src"].long(), s["dst"].long(), s["block_tokens"]
    entry = torch.arange(s["table"].shape[1], device="cuda")
    held = entry < (-(-s["lens"][src] // T))[:, None]
    s["table"][dst] = torch.where(held, s["table"][src], s["table"][dst])
    s["refs"].index_add_(0, s["table"][src].clamp(min=0).long().reshape(-1), held.int().reshape(-1))
    s["lens"][dst] = s["lens"][src]


def plain_resize(s, lens, want):
    """Frees what the shorter lengths do not need, then gives the growing sequences, in order, the lowest free
    blocks: their copy of a shared partial block first, then the new blocks.  The pool is large enough here."""
    table, refs, T = s["table"], s["refs"], s["block_tokens"]
    B, M = table.shape
    entry = torch.arange(M, device="cuda")
    have, need = -(-lens // T), -(-want // T)
    drop = (entry >= need[:, None]) & (entry < have[:, None])
    refs.index_add_(0, table.clamp(min=0).long().reshape(-1), -drop.int().reshape(-1))
    partial = (want > lens) & (lens % T != 0)
    spot = (lens // T).clamp(max=M - 1).long()[:, None]
    block = torch.where(partial, table.gather(1, spot)[:, 0], 0).long()
    shared = partial & (refs[block] > 1)
    growing = torch.zeros_like(refs).index_add_(0, block, shared.int())
    last = torch.full_like(refs, -1).scatter_reduce_(0, block, torch.where(shared, torch.arange(B, device="cuda").int(), -1), "amax")
    copies = shared & ~((growing[block] == refs[block]) & (last[block] == torch.arange(B, device="cuda")))
    count = (need - have).clamp(min=0) + copies.int()
    first = (count.cumsum(0) - count)[:, None]
    free = torch.argsort((refs > 0).int(), stable=True).int()      # the free blocks come first, lowest id first
    fresh = (entry >= have[:, None]) & (entry < need[:, None]) | ((entry == spot) & copies[:, None])
    rank = (first + fresh.int().cumsum(1) - 1).clamp(min=0)
    refs.index_add_(0, block, -copies.int())
    new = torch.where(fresh, free[rank.clamp(max=refs.numel() - 1).long()], table)
    refs.index_add_(0, new.clamp(min=0).long().reshape(-1), fresh.int().reshape(-1))
    table.copy_(new)
    who = copies.nonzero()[:, 0]
    to = new.gather(1, spot)[who, 0].long()
    s["k"][:, to] = s["k"][:, block[who]]
    s["v"][:, to] = s["v"][:, block[who]]
    return want


def plain_pages(s):
    """Children forked, grown, and freed again: the counts end as they began."""
    plain_fork(s)
    s["grown"].copy_(plain_resize(s, s["lens"], s["want"]))
    s["lens"].copy_(plain_resize(s, s["grown"], s["base"]))
    return s["table"], s["refs"], s["grown"], s["lens"], s["k"], s["v"]


def plain_defragment(s):
    refs, table = s["refs"], s["table"]
    used_here = refs > 0
    used = used_here.sum()
    ids = torch.arange(refs.numel(), device="cuda")
    moved = used_here & (ids >= used)
    holes = torch.argsort((used_here | (ids >= used)).int(), stable=True)
    to = torch.where(moved, holes[(moved.cumsum(0) - 1).clamp(min=0)], ids)
    held = torch.arange(table.shape[1], device="cuda") < (-(-s["lens"] // s["block_tokens"]))[:, None]
    s["new_table"].copy_(torch.where(held, to[table.clamp(min=0).long()].int(), table))
    s["new_refs"].zero_().index_add_(0, to, refs)
    src = moved.nonzero()[:, 0]
    s["k"][:, to[src]] = s["k"][:, src]
    s["v"][:, to[src]] = s["v"][:, src]
    s["used"].copy_(used)
    return s["new_table"], s["new_refs"], s["used"], s["k"], s["v"]


PLAIN = dict(attention=plain_attention, verify=plain_verify, keep=plain_keep, pages=plain_pages, defragment=plain_defragment)


# The library's calls.
def scratch(s, size):
    """The workspace that the program keeps between its calls."""
    if "bytes" not in s["scratch"]:
        s["scratch"]["bytes"] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return s["scratch"]["bytes"]


def own_attention(s):
    from paper_2409_04992_b200 import binding
    B, N, Hq, D = s["q"].shape
    room = scratch(s, lambda: binding.tree_workspace_bytes(B, N, Hq, s["k"].shape[1], D, s["max_len"]))
    binding.decode_attention_tree(s["out"], s["lse"], s["q"], s["k"], s["v"], s["table"], s["lens"], s["nodes"], s["mask"],
                                  s["max_len"], s["scale"], room, s["flags"])
    return s["out"], s["lse"]


def own_verify(s):
    from paper_2409_04992_b200 import binding
    binding.verify_tree(s["path"], s["path_lens"], s["emitted"], s["target"], s["draft"], s["tokens"], s["parents"], s["nodes"],
                        s["uniforms"], s["flags"])
    return s["path"], s["path_lens"], s["emitted"]


def own_keep(s):
    from paper_2409_04992_b200 import binding
    binding.kv_keep_path(s["k_layers"], s["v_layers"], s["path"], s["path_lens"], s["nodes"], s["lens"], s["new_lens"],
                         s["table"], s["flags"])
    return s["k"], s["v"], s["new_lens"]


def own_pages(s):
    from paper_2409_04992_b200 import binding
    room = scratch(s, lambda: binding.kv_resize_workspace_bytes(s["table"].shape[0], s["refs"].numel()))
    binding.kv_fork(s["table"], s["refs"], s["lens"], s["src"], s["dst"], s["block_tokens"], s["flags"])
    for have, want, new in ((s["lens"], s["want"], s["grown"]), (s["grown"], s["base"], s["lens"])):
        binding.kv_resize(s["k_layers"], s["v_layers"], s["table"], s["refs"], have, want, new, room, s["flags"])
    return s["table"], s["refs"], s["grown"], s["lens"], s["k"], s["v"]


def own_defragment(s):
    from paper_2409_04992_b200 import binding
    room = scratch(s, lambda: binding.kv_defragment_workspace_bytes(s["refs"].numel()))
    binding.kv_defragment(s["k_layers"], s["v_layers"], s["table"], s["refs"], s["lens"], s["new_table"], s["new_refs"], s["used"],
                          room, s["flags"])
    return s["new_table"], s["new_refs"], s["used"], s["k"], s["v"]


OWN = dict(attention=own_attention, verify=own_verify, keep=own_keep, pages=own_pages, defragment=own_defragment)


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    """Attention head by head, verification token by token; the other operators only move bits."""
    if case["kind"] == "attention":
        return exact_attention(case, prepare(case, seed))
    if case["kind"] == "verify":
        return exact_verify(case, prepare(case, seed))
    return None


def exact_attention(c, s):
    B, N, Hq, D = s["q"].shape
    group = Hq // c["kv_heads"]
    out = torch.zeros(B, N, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, N, Hq), -math.inf, dtype=torch.float64, device="cuda")
    bits = s["mask"].cpu().numpy().view(np.uint64)
    for b, (length, nodes) in enumerate(zip(lengths_of(c), nodes_of(c))):
        see = torch.ones(nodes, length, dtype=torch.bool)
        for t in range(nodes):
            for j in range(nodes):
                see[t, length - nodes + j] = bool(int(bits[b, t, j // 64]) >> (j % 64) & 1)
        hide = torch.where(see, 0.0, -math.inf).double().cuda()
        for h in range(c["kv_heads"]):
            if s["table"] is None:
                k, v = s["k"][b, h, :length], s["v"][b, h, :length]
            else:
                pages = s["table"][b, :-(-length // c["block_tokens"])].long()
                k, v = s["k"][pages, h].flatten(0, 1)[:length], s["v"][pages, h].flatten(0, 1)[:length]
            for j in range(h * group, (h + 1) * group):
                score = s["q"][b, :nodes, j].double() @ k.double().T * s["scale"] + hide
                lse[b, :nodes, j] = torch.logsumexp(score, 1)
                out[b, :nodes, j] = torch.softmax(score, 1) @ v.double()
    return out, lse


def exact_verify(c, s):
    B, N, V = s["target"].shape
    parents, tokens, nodes = (s[n].cpu().tolist() for n in ("parents", "tokens", "nodes"))
    uniforms = s["uniforms"].double().cpu().tolist()
    read = lambda p, b, t: p[b, t].double().cpu().numpy()  # noqa: E731
    paths, counts, emitted = [], [], []
    for b in range(B):
        path, again = [0], True
        while again:
            v = path[-1]
            again, w, total = False, read(s["target"], b, v), 1.0
            for child in (t for t in range(1, nodes[b]) if parents[b][t] == v):
                q = np.eye(1, V, tokens[b][child])[0] if s["draft"] is None else read(s["draft"], b, v)
                if uniforms[b][child] * q[tokens[b][child]] * total < w[tokens[b][child]]:
                    path.append(child)
                    again = True
                    break
                left = np.maximum(w - total * q, 0)
                if left.sum() > 0:
                    w, total = left, left.sum()
        sums = np.cumsum(w)
        said = [tokens[b][t] for t in path[1:]] + [int(np.searchsorted(sums, uniforms[b][0] * sums[-1], side="right"))]
        pad = [-1] * (N - len(path))
        paths.append(path + pad)
        counts.append(len(path))
        emitted.append(said + pad)
    return tuple(torch.tensor(x, dtype=torch.int32) for x in (paths, counts, emitted))
