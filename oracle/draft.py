"""Speculative decoding over the cache, in plain loops and 64 bits: attention of a tree of drafted
tokens, its verification, keeping the accepted path, and the blocks of a shared pool.  Written
from the definitions in include/instinfer.h, one sequence, one block, one token at a time; test
infrastructure, no part of the library."""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import numpy as np

FLAG_SEQ_LEN_RANGE, FLAG_BLOCK_RANGE, FLAG_TREE_RANGE, FLAG_POOL = 1, 2, 16, 32


def ancestor_mask(parents: Sequence[int], nodes: int, width: int) -> np.ndarray:
    """bool [width, width]: does node t see node j."""
    see = np.zeros((width, width), dtype=bool)
    for t in range(nodes):
        see[t, t] = True
        if 0 <= parents[t] < t:
            see[t] |= see[parents[t]]
    return see


def pack_mask(see: np.ndarray) -> np.ndarray:
    """bool [..., T, T] -> the int64 words [..., T, ceil(T / 64)] that the library reads."""
    width = see.shape[-1]
    words = np.zeros(see.shape[:-1] + ((width + 63) // 64,), dtype=np.uint64)
    for j in range(width):
        words[..., j // 64] |= see[..., j].astype(np.uint64) << np.uint64(j % 64)
    return words.view(np.int64)


def rows_of(cache: np.ndarray, b: int, length: int, table: Optional[np.ndarray]) -> np.ndarray:
    """The sequence's rows [heads, length, D] in float64."""
    if table is None:
        return cache[b, :, :length].astype(np.float64)
    tokens = cache.shape[2]
    out = np.zeros((cache.shape[1], length, cache.shape[3]))
    for i in range(length):
        out[:, i] = cache[table[b, i // tokens], :, i % tokens]
    return out


def tree_attention(q, k_cache, v_cache, table, seq_lens, tree_lens, see, scale):
    """(out, lse, size, spread): size = softmax . |V| and spread = the largest sum |q||k| * |scale| a row
    meets, from which a test can say how far rounding may move a result.  A row's value is the sum
    over what it sees only, so what is hidden may hold anything."""
    B, T, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    group = Hq // Hkv
    out = np.zeros((B, T, Hq, D))
    size = np.zeros((B, T, Hq, D))
    lse = np.full((B, T, Hq), -np.inf)
    spread = np.zeros((B, T, Hq))
    for b in range(B):
        n, nodes = int(seq_lens[b]), int(tree_lens[b])
        if n <= 0 or nodes > n:
            continue
        k, v = rows_of(k_cache, b, n, table), rows_of(v_cache, b, n, table)
        for t in range(min(nodes, T)):
            seen = [*range(n - nodes), *(n - nodes + j for j in range(nodes) if see[b, t, j])]
            if not seen:
                continue
            for h in range(Hq):
                ks, vs = k[h // group][seen], v[h // group][seen]
                query = q[b, t, h].astype(np.float64)
                s = ks @ query * scale
                top = s.max()
                w = np.exp(s - top)
                lse[b, t, h] = top + np.log(w.sum())
                w = w / w.sum()
                out[b, t, h] = w @ vs
                size[b, t, h] = w @ np.abs(vs)
                spread[b, t, h] = (np.abs(ks) @ np.abs(query)).max() * abs(scale)
    return out, lse, size, spread


def clean(row: np.ndarray) -> np.ndarray:
    row = np.asarray(row, dtype=np.float64)
    return np.where((row > 0) & np.isfinite(row), row, 0.0)


def verify(target, draft, tokens, parents, tree_lens, uniforms) -> Tuple[np.ndarray, np.ndarray, np.ndarray, int]:
    """(path, path_lens, out_tokens, flags); target, draft float64 [B, T, V], draft None: not sampled."""
    B, T, V = target.shape
    path = np.full((B, T), -1, dtype=np.int32)
    said = np.full((B, T), -1, dtype=np.int32)
    counts = np.zeros(B, dtype=np.int32)
    flags = 0
    for b in range(B):
        nodes = int(tree_lens[b])
        if nodes < 0 or nodes > T:
            flags |= FLAG_TREE_RANGE
            continue
        if nodes == 0:
            continue
        usable = [False] * nodes
        for t in range(1, nodes):
            usable[t] = 0 <= parents[b, t] < t and 0 <= tokens[b, t] < V
            flags |= 0 if usable[t] else FLAG_TREE_RANGE
        taken = [0]
        while True:
            at = taken[-1]
            w, total = clean(target[b, at]), 1.0
            step = None
            for c in range(1, nodes):
                if not usable[c] or parents[b, c] != at:
                    continue
                x = tokens[b, c]
                if draft is None:
                    q = np.zeros(V)
                    q[x] = 1.0
                else:
                    q = clean(draft[b, at])
                if float(uniforms[b, c]) * q[x] * total < w[x]:
                    step = c
                    break
                left = np.maximum(w - total * q, 0.0)
                if left.sum() > 0:
                    w, total = left, float(left.sum())
            if step is None:
                break
            taken.append(step)
        running = np.cumsum(w)
        above = np.nonzero((running > float(uniforms[b, 0]) * running[-1]) & (w > 0))[0]
        if running[-1] > 0:
            last = int(above[0]) if len(above) else int(np.nonzero(w > 0)[0][-1])
        else:
            last = -1
            flags |= FLAG_TREE_RANGE
        counts[b] = len(taken)
        path[b, :len(taken)] = taken
        said[b, :len(taken)] = [*(tokens[b, t] for t in taken[1:]), last]
    return path, counts, said, flags


def keep_path(caches: List[np.ndarray], path, path_lens, tree_lens, seq_lens, table) -> Tuple[np.ndarray, int]:
    """Moves the rows in place, in every cache; (new_lens, flags)."""
    new_lens = np.array(seq_lens, dtype=np.int32)
    flags = 0
    for b in range(len(seq_lens)):
        n, nodes, kept = int(seq_lens[b]), int(tree_lens[b]), int(path_lens[b])
        tokens = caches[0].shape[2]
        capacity = tokens if table is None else table.shape[1] * tokens
        if n < 0 or n > capacity:
            flags |= FLAG_SEQ_LEN_RANGE
            continue
        steps = [int(x) for x in path[b, :max(kept, 0)]]
        ok = 0 <= nodes <= min(n, path.shape[1]) and 0 <= kept <= nodes
        ok = ok and all(0 <= x < nodes for x in steps) and all(x < y for x, y in zip(steps, steps[1:]))
        if not ok:
            flags |= FLAG_TREE_RANGE if n != 0 else 0
            continue
        base = n - nodes
        new_lens[b] = base + kept
        for i, node in enumerate(steps):
            if node == i:
                continue
            src, dst = base + node, base + i
            for cache in caches:
                if table is None:
                    cache[b, :, dst] = cache[b, :, src]
                    continue
                there, here = table[b, dst // tokens], table[b, src // tokens]
                if not (0 <= there < cache.shape[0] and 0 <= here < cache.shape[0]):
                    flags |= FLAG_BLOCK_RANGE
                    continue
                cache[there, :, dst % tokens] = cache[here, :, src % tokens]
    return new_lens, flags


def blocks_for(length: int, tokens: int) -> int:
    return -(-int(length) // tokens)


def fork(table, refs, seq_lens, src, dst, tokens) -> int:
    """In place; flags."""
    flags = 0
    before = np.array(seq_lens)
    for i, (s, d) in enumerate(zip(src, dst)):
        if not (0 <= s < len(before) and 0 <= d < len(before)) or d in list(dst[:i]) or s in list(dst):
            flags |= FLAG_POOL
            continue
        if not 0 <= before[s] <= table.shape[1] * tokens or before[d] != 0:
            flags |= FLAG_SEQ_LEN_RANGE
            continue
        held = blocks_for(before[s], tokens)
        for e in range(held):
            table[d, e] = table[s, e]
            if not 0 <= table[s, e] < len(refs):
                flags |= FLAG_BLOCK_RANGE
                continue
            flags |= FLAG_POOL if refs[table[s, e]] <= 0 else 0
            refs[table[s, e]] += 1
        seq_lens[d] = before[s]
    return flags


def resize(caches, table, refs, seq_lens, want_lens, tokens) -> Tuple[np.ndarray, int]:
    """In place; (new_lens, flags)."""
    flags = 0
    B, M = table.shape
    old = np.array(seq_lens, dtype=np.int64)
    want = np.array(want_lens, dtype=np.int64)
    for b in range(B):
        if not (0 <= old[b] <= M * tokens and 0 <= want[b] <= M * tokens):
            flags |= FLAG_SEQ_LEN_RANGE
            want[b] = old[b]
    for b in range(B):
        for e in range(blocks_for(want[b], tokens), blocks_for(old[b], tokens)) if want[b] < old[b] else ():
            block = table[b, e]
            if not 0 <= block < len(refs):
                flags |= FLAG_BLOCK_RANGE
            elif refs[block] <= 0:
                flags |= FLAG_POOL
            else:
                refs[block] -= 1
    # who writes into a block that others list
    writers = {}
    for b in range(B):
        if want[b] > old[b] and old[b] % tokens:
            block = int(table[b, old[b] // tokens])
            if not 0 <= block < len(refs):
                flags |= FLAG_BLOCK_RANGE
            elif refs[block] > 1:
                writers.setdefault(block, []).append(b)
    copies, keeps = set(), set()
    for block, who in writers.items():
        if len(who) == refs[block]:
            keeps.add(who[-1])
            who = who[:-1]
        copies.update(who)
    new_lens = want.astype(np.int32)
    short = False
    moves = []
    for b in range(B):
        more = max(0, blocks_for(want[b], tokens) - blocks_for(old[b], tokens))
        need = more + (b in copies)
        free = [i for i in range(len(refs)) if refs[i] <= 0]
        if need or b in keeps:
            short = short or need > len(free)
        if short and (need or b in keeps):
            flags |= FLAG_POOL
            new_lens[b] = old[b]
            continue
        if b in copies:
            e = old[b] // tokens
            moves.append((int(table[b, e]), free[0]))
            refs[free[0]] = 1
            refs[table[b, e]] -= 1
            table[b, e] = free.pop(0)
        for i in range(more):
            refs[free[i]] = 1
            table[b, blocks_for(old[b], tokens) + i] = free[i]
    for src, dst in moves:
        for cache in caches:
            cache[dst] = cache[src]
    return new_lens, flags


def defragment(caches, table, refs, seq_lens, tokens):
    """(new_table, new_refs, used, flags); the caches in place."""
    flags = 0
    used = int((refs > 0).sum())
    holes = [i for i in range(used) if refs[i] <= 0]
    movers = [i for i in range(used, len(refs)) if refs[i] > 0]
    to = {i: i for i in range(used) if refs[i] > 0}
    to.update(zip(movers, holes))
    new_refs = np.zeros_like(refs)
    for i in range(len(refs)):
        if refs[i] > 0:
            new_refs[to[i]] = refs[i]
    for src, dst in zip(movers, holes):
        for cache in caches:
            cache[dst] = cache[src]
    new_table = np.array(table)
    for b in range(table.shape[0]):
        if not 0 <= seq_lens[b] <= table.shape[1] * tokens:
            flags |= FLAG_SEQ_LEN_RANGE
            continue
        for e in range(blocks_for(seq_lens[b], tokens)):
            block = int(table[b, e])
            if not 0 <= block < len(refs):
                flags |= FLAG_BLOCK_RANGE
            elif block in to:
                new_table[b, e] = to[block]
            else:
                flags |= FLAG_POOL
    return new_table, new_refs, used, flags
