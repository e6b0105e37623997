"""A decode step around the attention, as cases that can be timed and compared: rotary positions applied on
the way into the cache, a cache of one latent vector a token with the attention that reads it, and the way
from the last layer's logits to the probabilities that verification and sampling take.

`run` computes a case in plain torch operations, or, where `own` is true, with the library."""
import math

import numpy as np
import torch

own = False

KINDS = ("rope", "latent_append", "latent", "latent", "logits")
LATENT, ROPE = 512, 64          # a latent cache row: 512 values that are keys and values, 64 rotated key dims


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one sequence, one new token of the 13B-class layer, contiguous cache (latency)
        dict(name="rope_one", kind="rope", batch=1, tokens=1, ragged=False, q_heads=40, kv_heads=40, head_dim=128, rope_dim=128,
             interleaved=False, dtype="float16", scaled=False, length=1024, block_tokens=0, fused=False),
        # a decode batch with grouped heads, half of each head rotated, a bf16 model's fused projection, 32-token pages
        dict(name="rope_batch", kind="rope", batch=128, tokens=1, ragged=False, q_heads=64, kv_heads=8, head_dim=128, rope_dim=64,
             interleaved=True, dtype="bfloat16", scaled=False, length=1000, block_tokens=32, fused=True),
        # ragged prompts of four sequences into 32-token pages at far positions of a stretched context
        dict(name="rope_prompts", kind="rope", batch=4, tokens=4096, ragged=True, q_heads=40, kv_heads=40, head_dim=128, rope_dim=128,
             interleaved=False, dtype="float16", scaled=True, length=4500, block_tokens=32, fused=False),
        # a decode batch's latent rows and rotated query parts, 128 heads
        dict(name="latent_append_batch", kind="latent_append", batch=64, tokens=1, ragged=False, q_heads=128, interleaved=True,
             dtype="bfloat16", scaled=True, length=1000, block_tokens=64),
        # prompts' latent rows
        dict(name="latent_append_prompts", kind="latent_append", batch=8, tokens=2048, ragged=True, q_heads=16, interleaved=False,
             dtype="float16", scaled=False, length=2100, block_tokens=16),
        # one sequence, a model's heads split over eight GPUs, a short contiguous cache (latency)
        dict(name="latent_one", kind="latent", batch=1, q_tokens=1, q_heads=16, tree=False, dtype="float16", len_lo=1000, len_hi=1000,
             block_tokens=0),
        # a full serving batch of that GPU: ragged contexts in 64-token pages, memory bound
        dict(name="latent_16_heads", kind="latent", batch=64, q_tokens=1, q_heads=16, tree=False, dtype="bfloat16", len_lo=4096,
             len_hi=16384, block_tokens=64),
        # all 128 heads on one GPU: 242 operations for every byte of the cache
        dict(name="latent_128_heads", kind="latent", batch=32, q_tokens=1, q_heads=128, tree=False, dtype="float16", len_lo=4096,
             len_hi=8192, block_tokens=32),
        # trees of eight drafted tokens, odd lengths from a few tokens on
        dict(name="latent_tree", kind="latent", batch=7, q_tokens=8, q_heads=16, tree=True, dtype="bfloat16", len_lo=33, len_hi=30011,
             block_tokens=16),
        # one row of logits to probabilities, a short history (latency)
        dict(name="logits_one", kind="logits", batch=1, nodes=1, vocab=32000, dtype="float32", out="float32", history=300, bias=4,
             mask=False, greedy=0),
        # a decode batch with everything on: penalties, biases and grammar masks, some rows greedy, an odd vocabulary
        dict(name="logits_batch", kind="logits", batch=192, nodes=1, vocab=50257, dtype="bfloat16", out="float32", history=4000, bias=32,
             mask=True, greedy=5),
        # the nodes of draft trees, each with its own ancestors' penalties, a large vocabulary
        dict(name="logits_tree", kind="logits", batch=16, nodes=32, vocab=131072, dtype="bfloat16", out="bfloat16", history=2000, bias=0,
             mask=True, greedy=0),
    ]


def log_int(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(KINDS)
    while True:
        if kind == "rope":
            kv, d = log_int(rng, 1, 64), rng.choice([64, 128, 128, 256])
            tokens = rng.choice([1, log_int(rng, 1, 4096)])
            c = dict(kind=kind, batch=log_int(rng, 1, 256), tokens=tokens, ragged=rng.random() < 0.5,
                     q_heads=kv * rng.choice([1, 1, 2, 3, 4, 8]), kv_heads=kv, head_dim=d,
                     rope_dim=rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)]), interleaved=rng.random() < 0.5,
                     dtype=rng.choice(["float16", "bfloat16", "float32"]), scaled=rng.random() < 0.5,
                     length=tokens + log_int(rng, 1, 600), block_tokens=rng.choice([0, 8, 16, 32, 48, 64]), fused=rng.random() < 0.5)
            size = c["batch"] * kv * d * (c["length"] + 64)
            if work(c)["bytes"] <= 9e8 and size <= 1.5e8:
                return c
        elif kind == "latent_append":
            tokens = rng.choice([1, log_int(rng, 1, 4096)])
            c = dict(kind=kind, batch=log_int(rng, 1, 256), tokens=tokens, ragged=rng.random() < 0.5, q_heads=log_int(rng, 1, 128),
                     interleaved=rng.random() < 0.5, dtype=rng.choice(["float16", "bfloat16"]), scaled=rng.random() < 0.5,
                     length=tokens + log_int(rng, 1, 600), block_tokens=rng.choice([0, 8, 16, 32, 48, 64]))
            if c["batch"] * tokens * c["q_heads"] <= 2.7e5 and c["batch"] * c["length"] <= 1.5e5:
                return c
        elif kind == "latent":
            hi = log_int(rng, 1, 60000)
            c = dict(kind=kind, batch=log_int(rng, 1, 96), q_tokens=rng.choice([1, 1, 2, log_int(rng, 1, 64)]),
                     q_heads=rng.choice([1, 5, 8, 16, 16, 20, 32, 64, 128]), tree=rng.random() < 0.4,
                     dtype=rng.choice(["float16", "bfloat16"]), len_lo=0, len_hi=hi, block_tokens=rng.choice([0, 8, 16, 32, 48, 64, 128]))
            c["len_hi"] = max(hi, c["q_tokens"])
            c["len_lo"] = max(c["q_tokens"], int(c["len_hi"] * rng.choice([0.1, 0.5, 1.0])))
            w = work(c)
            if w["bytes"] <= 7e8 and w["flops"] <= 5.5e10 and c["batch"] * c["q_tokens"] * c["q_heads"] * c["len_hi"] <= 1.2e8 and \
                    c["batch"] * c["len_hi"] <= 1.0e6:
                return c
        else:
            c = dict(kind=kind, batch=log_int(rng, 1, 256), nodes=rng.choice([1, 1, log_int(rng, 1, 128)]), vocab=log_int(rng, 30, 260000),
                     dtype=rng.choice(["float32", "float16", "bfloat16"]), out=rng.choice(["float32", "float16", "bfloat16"]),
                     history=log_int(rng, 1, 40000), bias=rng.choice([0, 3, 32, 256]), mask=rng.random() < 0.5,
                     greedy=rng.choice([0, 0, 3, 5]))
            if c["batch"] * c["nodes"] * c["vocab"] <= 16 * 32 * 131072 and c["batch"] * c["history"] <= 1e6:
                return c


def lengths_of(c):
    """The sequences' lengths: spread evenly from len_lo to len_hi, the longest first."""
    n = c["batch"]
    return [c["len_hi"] - (c["len_hi"] - c["len_lo"]) * i // max(1, n - 1) for i in range(n)]


def fresh_of(c):
    """New tokens of each sequence."""
    return [max(1, c["tokens"] - (i % 4) * (c["tokens"] // 5)) if c["ragged"] else c["tokens"] for i in range(c["batch"])]


def size_of(name):
    return 4 if name == "float32" else 2


def work(c):
    if c["kind"] == "rope":
        n = sum(fresh_of(c)) * c["head_dim"]
        return dict(bytes=n * (c["q_heads"] + 2 * c["kv_heads"]) * (size_of(c["dtype"]) + 2),
                    flops=3 * sum(fresh_of(c)) * c["rope_dim"] * (c["q_heads"] + c["kv_heads"]))
    if c["kind"] == "latent_append":
        n = sum(fresh_of(c))
        return dict(bytes=n * (LATENT + ROPE + c["q_heads"] * ROPE) * 4, flops=3 * n * ROPE * (c["q_heads"] + 1))
    if c["kind"] == "latent":
        rows, keys = c["q_tokens"] * c["q_heads"], sum(lengths_of(c))
        return dict(bytes=2 * keys * (LATENT + ROPE) + 2 * c["batch"] * rows * (2 * LATENT + ROPE) + 4 * c["batch"] * rows,
                    flops=2 * rows * keys * (2 * LATENT + ROPE))
    rows = c["batch"] * c["nodes"]
    return dict(bytes=rows * c["vocab"] * (size_of(c["dtype"]) + size_of(c["out"])) + c["batch"] * c["history"] * 4 +
                (rows * c["vocab"] // 8 if c["mask"] else 0), flops=8 * rows * c["vocab"])


# ---------------------------------------------------------------- inputs
def normal(g, *shape, dtype):
    if math.prod(shape) < 1 << 26:
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float16 if dtype == torch.float32 else dtype).to(dtype)


def frequencies(dim, scaled):
    """Radians per position of each pair of dims, and the factor on the rotated values: plain, or stretched eight times by
    parts (pairs that turn often over the trained 4096 positions keep their frequency, slow ones are divided)."""
    f = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    if not scaled:
        return f, 1.0
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
    return keep * f + (1 - keep) * f / 8, 0.1 * math.log(8) + 1


def pages(rng, lens, T):
    """A block table for sequences of these lengths, blocks in random order, and the number of blocks."""
    blocks = sum(-(-n // T) for n in lens)
    table = np.zeros((len(lens), max(1, -(-max(lens) // T))), dtype=np.int32)
    ids, at = rng.permutation(blocks), 0
    for b, n in enumerate(lens):
        need = -(-n // T)
        table[b, :need] = ids[at:at + need]
        at += need
    return table, blocks


def random_tree(rng, nodes):
    """Parents (-1 for the root, before their children, mostly recent nodes) and every node's bits: its ancestors and itself."""
    t = np.arange(nodes)
    parents = np.where(t == 0, -1, t - np.maximum(np.minimum(rng.geometric(0.35, nodes), t), 1)).astype(np.int32)
    bits = np.zeros((nodes, -(-nodes // 64)), dtype=np.uint64)
    for n, up in enumerate(parents):
        if up >= 0:
            bits[n] = bits[up]
        bits[n, n // 64] |= np.uint64(1) << np.uint64(n % 64)
    return parents, bits


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    on_gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    state = dict(PREPARE[case["kind"]](case, g, rng, on_gpu))
    state.update(kind=case["kind"], flags=torch.zeros(1, dtype=torch.int32, device="cuda"), scratch={})
    return state


def prepare_append(c, rng, on_gpu):
    """What both appends have: lengths after them, the new tokens' number and positions, pages, the pairs' frequencies."""
    B, T, N = c["batch"], c["block_tokens"], c["tokens"]
    fresh = fresh_of(c)
    lens = [c["length"] - b % 3 if c["length"] - b % 3 >= fresh[b] else c["length"] for b in range(B)]
    table, blocks = pages(rng, lens, T) if T else (None, 0)
    offset = 100000 if c["scaled"] else 0                          # the context before these tokens was dropped
    at = offset + np.array(lens)[:, None] - np.array(fresh)[:, None] + np.arange(N)[None, :]
    f, magnitude = frequencies(c.get("rope_dim", ROPE), c["scaled"])
    return dict(lens=on_gpu(np.array(lens, dtype=np.int32)), fresh=on_gpu(np.array(fresh, dtype=np.int32)),
                positions=on_gpu(at.astype(np.int32)), table=None if table is None else on_gpu(table), frequencies=f.cuda(),
                magnitude=magnitude, interleaved=c["interleaved"]), blocks


def prepare_rope(c, g, rng, on_gpu):
    s, blocks = prepare_append(c, rng, on_gpu)
    B, N, Hq, H, D, T = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"], c["head_dim"], c["block_tokens"]
    dtype = getattr(torch, c["dtype"])
    if c["fused"]:                                                 # slices of one projection's output
        q, k, v = normal(g, B, N, Hq + 2 * H, D, dtype=dtype).split([Hq, H, H], dim=2)
    else:
        q, k, v = (normal(g, B, N, h, D, dtype=dtype) for h in (Hq, H, H))
    shape = (blocks, H, T, D) if T else (B, H, c["length"], D)
    cache = lambda: torch.zeros(shape, dtype=torch.float16, device="cuda")  # noqa: E731
    return dict(s, q=q, k_new=k, v_new=v, k=cache(), v=cache(), q_out=torch.zeros(B, N, Hq, D, dtype=torch.float16, device="cuda"))


def prepare_latent_append(c, g, rng, on_gpu):
    s, blocks = prepare_append(c, rng, on_gpu)
    B, N, H, T = c["batch"], c["tokens"], c["q_heads"], c["block_tokens"]
    dtype = getattr(torch, c["dtype"])
    new = normal(g, B, N, LATENT + ROPE, dtype=dtype)              # one projection makes the latent vector and the shared key part
    q = normal(g, B, N, H, 128 + ROPE, dtype=dtype)                # the queries' projection: 128 dims as they are, 64 to rotate
    shape = (blocks, T, LATENT + ROPE) if T else (B, c["length"], LATENT + ROPE)
    return dict(s, latent=new[..., :LATENT], key=new[..., LATENT:], q=q[..., 128:], cache=torch.zeros(shape, dtype=dtype, device="cuda"),
                q_out=torch.zeros(B, N, H, LATENT + ROPE, dtype=dtype, device="cuda"))


def prepare_latent(c, g, rng, on_gpu):
    lens, T, N = lengths_of(c), c["block_tokens"], c["q_tokens"]
    table, blocks = pages(rng, lens, T) if T else (None, 0)
    dtype = getattr(torch, c["dtype"])
    shape = (blocks, T, LATENT + ROPE) if T else (c["batch"], c["len_hi"], LATENT + ROPE)
    mask = nodes = None
    if c["tree"]:
        nodes = [max(1, N - (b % 3) * (N // 4)) for b in range(c["batch"])]
        bits = np.zeros((c["batch"], N, -(-N // 64)), dtype=np.uint64)
        for b, n in enumerate(nodes):
            bits[b, :n, :-(-n // 64)] = random_tree(rng, n)[1]
        mask, nodes = on_gpu(bits.view(np.int64)), on_gpu(np.array(nodes, dtype=np.int32))
    q = normal(g, c["batch"], N, c["q_heads"], LATENT + ROPE, dtype=dtype)
    return dict(q=q, cache=normal(g, *shape, dtype=dtype), table=None if table is None else on_gpu(table),
                lens=on_gpu(np.array(lens, dtype=np.int32)), nodes=nodes, mask=mask, max_len=c["len_hi"],
                scale=1.0 / math.sqrt(128 + ROPE), out=torch.zeros(*q.shape[:3], LATENT, dtype=dtype, device="cuda"),
                lse=torch.full(q.shape[:3], -math.inf, dtype=torch.float32, device="cuda"))


def prepare_logits(c, g, rng, on_gpu):
    B, N, V, M = c["batch"], c["nodes"], c["vocab"], c["history"]
    logits = (4.0 * torch.randn(B, N, V, generator=g, device="cuda")).to(getattr(torch, c["dtype"]))
    # few tokens of the vocabulary make most of a text
    often = torch.rand(B, M + N, generator=g, device="cuda").pow_(4).mul_(V).long().clamp_(max=V - 1).int()
    lens = np.array([M - (b % 4) * (M // 5) for b in range(B)], dtype=np.int32)
    s = dict(logits=logits, history=often[:, :M].contiguous(), lens=on_gpu(lens), prompts=on_gpu(lens // 2),
             penalties=on_gpu(np.tile(np.array([1.2, 0.3, 0.2], dtype=np.float32), (B, 1)) - 0.01 * (np.arange(B) % 7)[:, None].astype(np.float32)),
             drafts=None, mask=None, bias_tokens=None, bias=None, allowed=None,
             temperatures=on_gpu(np.array([0.0 if c["greedy"] and b % c["greedy"] == 1 else 0.6 + 0.1 * (b % 8) for b in range(B)], dtype=np.float32)),
             out=torch.zeros(B, N, V, dtype=getattr(torch, c["out"]), device="cuda"))
    if N > 1:
        bits = np.stack([random_tree(rng, N)[1] for _ in range(B)])
        s.update(drafts=often[:, M:].contiguous(), mask=on_gpu(bits.view(np.int64)))
    if c["bias"]:
        n = min(c["bias"], V)
        s.update(bias_tokens=on_gpu(np.stack([rng.permutation(V)[:n] for _ in range(min(B, 4))])[np.arange(B) % min(B, 4)].astype(np.int32)),
                 bias=torch.randn(B, n, generator=g, device="cuda").mul_(3))
    if c["mask"]:
        words = torch.randint(-2 ** 31, 2 ** 31, (B, N, -(-V // 32)), generator=g, device="cuda").int()
        words[:, :, 0] |= 1                                        # a grammar leaves something
        s.update(allowed=words)
    return s


PREPARE = dict(rope=prepare_rope, latent_append=prepare_latent_append, latent=prepare_latent, logits=prepare_logits)


# ---------------------------------------------------------------- one pass
def run(state):
    return (OWN if own else PLAIN)[state["kind"]](state)


# The plain forms: torch operations on whole tensors.
def turned(x, s):
    """x [B, N, heads, dims] in 32 bits, its first rotary dims turned by their positions' angles (angles in 64 bits: far
    positions turn fast pairs by many thousand radians)."""
    half = s["frequencies"].numel()
    angle = s["positions"].double()[:, :, None, None] * s["frequencies"]
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    part = x[..., :2 * half]
    a, b = (part[..., ::2], part[..., 1::2]) if s["interleaved"] else (part[..., :half], part[..., half:])
    new = (a * cos - b * sin, a * sin + b * cos)
    new = torch.stack(new, -1).flatten(-2) if s["interleaved"] else torch.cat(new, -1)
    return torch.cat((new, x[..., 2 * half:]), -1)


def places(s):
    """Which new tokens there are, and for each its sequence, its number among the new ones and its position in the cache
    (behind a sequence's last new token that one again: it is written more than once, always alike)."""
    B, N = s["positions"].shape
    t = torch.arange(N, device="cuda")
    last = torch.minimum(t, s["fresh"][:, None] - 1).long()
    b = torch.arange(B, device="cuda")[:, None].expand(B, N)
    return t < s["fresh"][:, None], b, last, (s["lens"] - s["fresh"]).long()[:, None] + last


def plain_rope(s):
    which, b, t, at = places(s)
    q, k = turned(s["q"].float(), s).half(), turned(s["k_new"].float(), s).half()
    s["q_out"].copy_(torch.where(which[:, :, None, None], q, s["q_out"]))
    for cache, new in ((s["k"], k), (s["v"], s["v_new"].half())):
        if s["table"] is None:
            cache[b, :, at] = new[b, t]
        else:
            T = cache.shape[2]
            cache[s["table"][b, at // T].long(), :, at % T] = new[b, t]
    return s["q_out"], s["k"], s["v"]


def plain_latent_append(s):
    which, b, t, at = places(s)
    q = turned(s["q"].float(), s).to(s["q_out"].dtype)
    key = turned(s["key"].float()[:, :, None], s)[:, :, 0].to(s["q_out"].dtype)
    s["q_out"][..., LATENT:].copy_(torch.where(which[:, :, None, None], q, s["q_out"][..., LATENT:]))
    new = torch.cat((s["latent"], key), -1)[b, t]
    if s["table"] is None:
        s["cache"][b, at] = new
    else:
        T = s["cache"].shape[1]
        s["cache"][s["table"][b, at // T].long(), at % T] = new
    return s["q_out"], s["cache"]


def seen_by(s, N, L):
    """[B, N, L]: which positions of the cache each new token attends to; the new tokens are the last ones."""
    at = torch.arange(L, device="cuda")
    nodes = torch.full_like(s["lens"], N) if s["nodes"] is None else s["nodes"]
    node = at - (s["lens"] - nodes)[:, None]                       # [B, L]
    if s["mask"] is None:
        sees = node[:, None, :] <= torch.arange(N, device="cuda")[:, None]
    else:
        word = (node.clamp(0, N - 1) // 64)[:, None, :].expand(-1, N, L)
        sees = ((s["mask"].gather(2, word) >> (node.clamp(0, N - 1) % 64)[:, None, :]) & 1).bool() | (node < 0)[:, None, :]
    sees = sees & (at < s["lens"][:, None])[:, None, :]
    return sees & (torch.arange(N, device="cuda") < nodes[:, None])[:, :, None]


def plain_latent(s):
    B, N, H, D = s["q"].shape
    L = s["max_len"]
    rows = s["cache"] if s["table"] is None else s["cache"][s["table"].long()].flatten(1, 2)[:, :L]
    rows = rows.float()
    sees = seen_by(s, N, L)
    logits = (s["q"].float().reshape(B, N * H, D) @ rows.transpose(1, 2)).mul_(s["scale"]).view(B, N, H, L)
    logits.masked_fill_(~sees[:, :, None, :], -math.inf)
    top = logits.amax(-1, keepdim=True)
    weights = logits.sub_(top.clamp(min=-1e30)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = (weights.view(B, N * H, L) @ rows[..., :LATENT]).view(B, N, H, LATENT) / total.clamp(min=1e-37)
    return out.to(s["q"].dtype), (top + total.log())[..., 0]


def plain_logits(s):
    B, N, V = s["logits"].shape
    M = s["history"].shape[1]
    z = s["logits"].float()
    place = torch.arange(M, device="cuda")
    said = (place < s["lens"][:, None]) & (place >= s["prompts"][:, None])
    token = s["history"].long()
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, token, said.float())[:, None, :]
    asked = torch.zeros(B, V, device="cuda").scatter_add_(1, token, (place < s["prompts"][:, None]).float())[:, None, :]
    if s["drafts"] is not None:                                    # a node has said its ancestors' tokens and its own too
        node = torch.arange(N, device="cuda")
        sees = ((s["mask"].gather(2, (node // 64).expand(B, N, N)) >> (node % 64)) & 1).float()
        own_path = torch.zeros(B, N, V, device="cuda").scatter_add_(2, s["drafts"].long()[:, None, :].expand(B, N, N), sees)
        count = count + own_path
    often, flat, once = (p[:, None, None] for p in s["penalties"].unbind(1))
    z = torch.where((count > 0) | (asked > 0), torch.where(z > 0, z / often, z * often), z)
    z = z - flat * count - once * (count > 0)
    if s["bias"] is not None:
        z = z + torch.zeros(B, V, device="cuda").scatter_add_(1, s["bias_tokens"].long(), s["bias"])[:, None, :]
    if s["allowed"] is not None:
        bit = torch.arange(V, device="cuda")
        z = z.masked_fill(((s["allowed"][:, :, bit // 32] >> (bit % 32)) & 1) == 0, -math.inf)
    hot = s["temperatures"][:, None, None]
    best = z.argmax(-1, keepdim=True)
    z = z / torch.where(hot > 0, hot, 1.0)
    e = (z - z.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    probs = e / e.sum(-1, keepdim=True).clamp(min=1e-37)
    return torch.where(hot > 0, probs, torch.zeros_like(probs).scatter_(2, best, 1.0)).to(s["out"].dtype)


PLAIN = dict(rope=plain_rope, latent_append=plain_latent_append, latent=plain_latent, logits=plain_logits)


# The library's calls.
def own_rope(s):
    from paper_2409_04992_b200 import binding
    binding.rope_append(s["q_out"], s["k"], s["v"], s["q"], s["k_new"], s["v_new"], s["frequencies"], s["lens"], s["fresh"],
                        s["table"], positions=s["positions"], interleaved=s["interleaved"], magnitude=s["magnitude"],
                        status_flags=s["flags"])
    return s["q_out"], s["k"], s["v"]


def own_latent_append(s):
    from paper_2409_04992_b200 import binding
    binding.latent_append(s["q_out"], s["cache"], s["q"], s["latent"], s["key"], s["frequencies"], s["lens"], s["fresh"], s["table"],
                          positions=s["positions"], interleaved=s["interleaved"], magnitude=s["magnitude"], status_flags=s["flags"])
    return s["q_out"], s["cache"]


def own_latent(s):
    from paper_2409_04992_b200 import binding
    B, N, H, _ = s["q"].shape
    if "room" not in s["scratch"]:                                 # the workspace that the program keeps between its calls
        s["scratch"]["room"] = torch.empty(binding.latent_workspace_bytes(B, N, H, LATENT, ROPE, s["max_len"]), dtype=torch.uint8, device="cuda")
    binding.decode_attention_latent(s["out"], s["lse"], s["q"], s["cache"], s["table"], s["lens"], s["nodes"], s["mask"], s["max_len"],
                                    s["scale"], s["scratch"]["room"], s["flags"])
    return s["out"], s["lse"]


def own_logits(s):
    from paper_2409_04992_b200 import binding
    binding.process_logits(s["out"], s["logits"], tokens=s["history"], token_lens=s["lens"], prompt_lens=s["prompts"],
                           penalties=s["penalties"], draft_tokens=s["drafts"], mask=s["mask"], bias_tokens=s["bias_tokens"],
                           bias_values=s["bias"], allowed=s["allowed"], temperatures=s["temperatures"], status_flags=s["flags"])
    return s["out"]


OWN = dict(rope=own_rope, latent_append=own_latent_append, latent=own_latent, logits=own_logits)


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    """The rotated values as complex numbers, attention sequence by sequence, probabilities row by row."""
    return EXACT[case["kind"]](case, prepare(case, seed))


def as_complex(x, s):
    """The pairs of x's rotary dims, turned: e^(i position frequency) on a + i b."""
    half = s["frequencies"].numel()
    x = x.double()
    pair = x[..., :2 * half].unflatten(-1, (half, 2) if s["interleaved"] else (2, half))
    z = torch.complex(*pair.unbind(-1 if s["interleaved"] else -2))
    turn = torch.polar(torch.full_like(s["frequencies"], s["magnitude"]).expand(*s["positions"].shape, half),
                       s["positions"].double()[..., None] * s["frequencies"])
    z = z * turn.reshape(*turn.shape[:2], *[1] * (x.dim() - 3), half)
    pair = torch.stack((z.real, z.imag), -1 if s["interleaved"] else -2)
    return torch.cat((pair.flatten(-2), x[..., 2 * half:]), -1)


def exact_rope(c, s):
    q, k = as_complex(s["q"], s), as_complex(s["k_new"], s)
    q_out, cache = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda")
    T = c["block_tokens"]
    for b, (n, length) in enumerate(zip(fresh_of(c), s["lens"].tolist())):
        q_out[b, :n] = q[b, :n]
        at = torch.arange(length - n, length, device="cuda")
        if T:
            cache[s["table"][b].long()[at // T], :, at % T] = k[b, :n]
        else:
            cache[b][:, at] = k[b, :n].transpose(0, 1)
    return q_out, cache, None


def exact_latent_append(c, s):
    q, key = as_complex(s["q"], s), as_complex(s["key"], s)
    q_out, cache = (torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("q_out", "cache"))
    T = c["block_tokens"]
    for b, (n, length) in enumerate(zip(fresh_of(c), s["lens"].tolist())):
        q_out[b, :n, :, LATENT:] = q[b, :n]
        at = torch.arange(length - n, length, device="cuda")
        row = (s["table"][b].long()[at // T], at % T) if T else (b, at)
        cache[row] = torch.cat((s["latent"][b, :n].double(), key[b, :n]), -1)
    return q_out, cache


def exact_latent(c, s):
    B, N, H, _ = s["q"].shape
    out = torch.zeros(B, N, H, LATENT, dtype=torch.float64, device="cuda")
    lse = torch.full((B, N, H), -math.inf, dtype=torch.float64, device="cuda")
    bits = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    nodes = [N] * B if s["nodes"] is None else s["nodes"].tolist()
    for b, length in enumerate(lengths_of(c)):
        n = nodes[b]
        see = torch.ones(n, length, dtype=torch.bool)
        for t in range(n):
            for j in range(n):
                see[t, length - n + j] = j <= t if bits is None else bool(int(bits[b, t, j // 64]) >> (j % 64) & 1)
        if s["table"] is None:
            rows = s["cache"][b, :length].double()
        else:
            rows = s["cache"][s["table"][b, :-(-length // c["block_tokens"])].long()].flatten(0, 1)[:length].double()
        score = torch.einsum("nhd,ld->nhl", s["q"][b, :n].double(), rows) * s["scale"] + torch.where(see, 0.0, -math.inf).double().cuda()[:, None]
        lse[b, :n] = torch.logsumexp(score, -1)
        out[b, :n] = torch.softmax(score, -1) @ rows[:, :LATENT]
    return out, lse


def exact_logits(c, s):
    B, N, V = s["logits"].shape
    probs = torch.zeros(B, N, V, dtype=torch.float64)
    history, lens, prompts = s["history"].cpu().numpy(), s["lens"].tolist(), s["prompts"].tolist()
    drafts = None if s["drafts"] is None else s["drafts"].cpu().numpy()
    bits = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint64)
    logits, penalties, hot = s["logits"].double().cpu().numpy(), s["penalties"].double().cpu().numpy(), s["temperatures"].double().cpu().numpy()
    for b in range(B):
        before = np.bincount(history[b, :prompts[b]], minlength=V) > 0
        count0 = np.bincount(history[b, prompts[b]:lens[b]], minlength=V).astype(np.float64)
        for t in range(N):
            z, count = logits[b, t].copy(), count0.copy()
            if drafts is not None:
                for j in range(N):
                    if int(bits[b, t, j // 64]) >> (j % 64) & 1:
                        count[drafts[b, j]] += 1
            seen = before | (count > 0)
            z[seen] = np.where(z[seen] > 0, z[seen] / penalties[b, 0], z[seen] * penalties[b, 0])
            z -= penalties[b, 1] * count + penalties[b, 2] * (count > 0)
            if s["bias"] is not None:
                np.add.at(z, s["bias_tokens"][b].cpu().numpy(), s["bias"][b].double().cpu().numpy())
            if s["allowed"] is not None:
                words = s["allowed"][b, t].cpu().numpy().view(np.uint8)
                z[np.unpackbits(words, bitorder="little")[:V] == 0] = -np.inf
            if hot[b] > 0:
                e = np.exp((z - z.max()) / hot[b])
                probs[b, t] = torch.from_numpy(e / e.sum())
            else:
                probs[b, t, int(z.argmax())] = 1.0
    return probs


EXACT = dict(rope=exact_rope, latent_append=exact_latent_append, latent=exact_latent, logits=exact_logits)
