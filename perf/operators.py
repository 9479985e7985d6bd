"""The attention and cache operators of a rollout that samples several answers to a prompt, as cases that can be timed.

A rollout runs its prompts through causal attention (all of a prompt at once, or in chunks against the paged FP8
cache), gives the prompt's cache pages to the samples drawn from it, decodes the samples of a prompt together, reading
the prompt's keys and values once for all of them, and frees and compacts the cache as samples end.

``listed()`` / ``draw(rng)`` give cases, ``prepare`` makes what the program holds before the call, ``run`` is one
pass, ``work`` its unavoidable bytes and operations, ``exact`` the same outputs in 64 bits.  ``own`` chooses between
the operators in plain torch operations and the library's kernels.
"""
import math

import torch

own = False

DIM, PAGE = 128, 16
PAGE_ROWS = 4                                               # value pages: four tokens of a dim side by side
HEADS = [(32, 8), (32, 4), (16, 16), (64, 8), (16, 8)]      # the dense and the expert model's first


def listed():
    return [
        # one short question: nothing but latency
        {"name": "prompt_one", "kind": "prompt", "count": 1, "min_len": 19, "max_len": 19, "q_heads": 32, "kv_heads": 8,
         "fused": False},
        # a rollout step's prompts, ragged and packed, read out of the fused qkv output
        {"name": "prompt_batch", "kind": "prompt", "count": 33, "min_len": 37, "max_len": 1500, "q_heads": 32,
         "kv_heads": 8, "fused": True},
        # long documents: the largest product
        {"name": "prompt_long", "kind": "prompt", "count": 2, "min_len": 8191, "max_len": 16384, "q_heads": 32,
         "kv_heads": 4, "fused": False},
        # a few drafted tokens of every sequence, checked against its cache
        {"name": "chunk_draft", "kind": "chunk", "count": 24, "min_context": 60, "max_context": 4000, "min_new": 1,
         "max_new": 8, "q_heads": 32, "kv_heads": 8},
        # chunks of prompts mixed with single decode tokens
        {"name": "chunk_mixed", "kind": "chunk", "count": 13, "min_context": 0, "max_context": 3001, "min_new": 1,
         "max_new": 777, "q_heads": 32, "kv_heads": 4},
        # 2048-token chunks of prompts whose beginning is cached already
        {"name": "chunk_long", "kind": "chunk", "count": 3, "min_context": 2048, "max_context": 18432, "min_new": 2048,
         "max_new": 2048, "q_heads": 32, "kv_heads": 8},
        # three samples of one short prompt, just begun
        {"name": "shared_few", "kind": "shared", "groups": 1, "samples": 3, "prefix": 208, "min_own": 1, "max_own": 40,
         "q_heads": 32, "kv_heads": 4},
        # a rollout batch: 16 samples of each prompt at all lengths
        {"name": "shared_batch", "kind": "shared", "groups": 16, "samples": 16, "prefix": 1808, "min_own": 1,
         "max_own": 2500, "q_heads": 32, "kv_heads": 8},
        # many samples of long prompts: the prefix is nearly all there is to read
        {"name": "shared_long", "kind": "shared", "groups": 4, "samples": 32, "prefix": 18000, "min_own": 200,
         "max_own": 1500, "q_heads": 32, "kv_heads": 4},
        # shared pages that one layer's decode step is about to write to, copied first
        {"name": "copy_few", "kind": "copy", "layers": 1, "kv_heads": 8, "blocks": 300, "count": 5},
        # samples of a batch of prompts get their tables, all layers of the dense model
        {"name": "fork_batch", "kind": "fork", "layers": 36, "kv_heads": 8, "prompts": 8, "samples": 16, "min_len": 40,
         "max_len": 500},
        # half of the samples have ended: their pages are freed, the others' moved together
        {"name": "release_half", "kind": "release", "layers": 12, "kv_heads": 4, "prompts": 24, "samples": 8,
         "min_len": 100, "max_len": 1000, "max_own": 700, "ended": 0.5},
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "chunk", "chunk", "chunk", "shared", "shared", "shared", "copy", "fork",
                       "release"])
    q_heads, kv_heads = rng.choice(HEADS)
    if kind == "prompt":
        max_len = _logint(rng, 1, 16384 if q_heads <= 32 else 11000)
        most = int(200e6 * 32 / q_heads / max_len ** 2)
        return {"kind": kind, "count": _logint(rng, 1, max(1, min(48, most, 40000 // max_len))),
                "min_len": rng.randint(1, max_len), "max_len": max_len, "q_heads": q_heads, "kv_heads": kv_heads,
                "fused": rng.random() < 0.5}
    if kind == "chunk":
        max_new = _logint(rng, 1, 2048)
        max_context = _logint(rng, 16, 18432 if q_heads <= 32 else 9000)
        most = int(60e6 * 32 / q_heads / max_new / (max_context + max_new))
        return {"kind": kind, "count": _logint(rng, 1, max(1, min(64, most, 200000 // max_context))),
                "min_context": rng.randint(0, max_context), "max_context": max_context,
                "min_new": rng.randint(1, max_new), "max_new": max_new, "q_heads": q_heads, "kv_heads": kv_heads}
    if kind == "shared":
        samples, prefix = rng.randint(2, 32), 16 * _logint(rng, 1, 1125)
        max_own = _logint(rng, 1, 4000)
        most = min(256 // samples, int(600e3 * 8 / kv_heads / (prefix + samples * max_own)), int(2e6 / (samples * prefix)))
        return {"kind": kind, "groups": _logint(rng, 1, max(1, min(16, most))), "samples": samples, "prefix": prefix,
                "min_own": rng.randint(1, max_own), "max_own": max_own, "q_heads": q_heads, "kv_heads": kv_heads}
    kv_heads = rng.choice([4, 8])
    layers = rng.randint(1, 48 // kv_heads if kind == "release" else 24)
    if kind == "copy":
        blocks = _logint(rng, 4, 1000)
        return {"kind": kind, "layers": layers, "kv_heads": kv_heads, "blocks": blocks, "count": rng.randint(1, blocks // 2)}
    max_len = _logint(rng, 16, 1000)
    case = {"kind": kind, "layers": layers, "kv_heads": kv_heads, "prompts": rng.randint(1, 16), "samples": rng.randint(2, 12),
            "min_len": rng.randint(1, max_len), "max_len": max_len}
    return case if kind == "fork" else dict(case, max_own=_logint(rng, 1, 700), ended=round(rng.uniform(0.1, 0.9), 2))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _gen(seed, salt, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 1013 + salt)
    return g


def _spread(count, lo, hi):
    """`count` whole numbers from lo to hi, evenly."""
    return [hi if count == 1 else lo + (hi - lo) * i // (count - 1) for i in range(count)]


def _new(case):
    """The new tokens of each sequence of a chunk case."""
    low = case["min_new"] / case["max_new"]
    return [round(case["max_new"] * low ** (i / max(1, case["count"] - 1))) for i in range(case["count"])]


def _shuffled(values, g):
    return [values[i] for i in torch.randperm(len(values), generator=g).tolist()]


def _normal(shape, std, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(std)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return _i32(at)


def _caches(blocks, kv_heads, g):
    """A layer's key and value pages, all written: E4M3 codes of keys N(0, 1.3), a few channels four times larger, and
    of values N(0, 0.7), at the scales that a calibration pass gives them."""
    out = {}
    for name, shape, std in (("k", (blocks, kv_heads, PAGE, DIM), 1.3), ("v", (blocks, kv_heads, PAGE // PAGE_ROWS, DIM, PAGE_ROWS), 0.7)):
        x = _normal(shape, std, g)
        if name == "k":
            x[..., 5::41] *= 4.0
        amax = 5.7 * std * (4.0 if name == "k" else 1.0)
        out[name + "_scale"] = torch.full((1,), amax / 448.0, dtype=torch.float32, device="cuda")
        out[name + "_cache"] = x.mul_(448.0 / amax).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return out


def _prepare_prompt(case, seed):
    g, h, kv = _gen(seed, 1), case["q_heads"], case["kv_heads"]
    lengths = _shuffled(_spread(case["count"], case["min_len"], case["max_len"]), _gen(seed, 2, "cpu"))
    n = sum(lengths)
    s = {"lengths": lengths, "cu_seqlens": _offsets(lengths)}
    if case["fused"]:
        qkv = _normal((n, h + 2 * kv, DIM), 1.0, g)
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
    else:
        s["q"], s["k"], s["v"] = (_normal((n, x, DIM), std, g) for x, std in ((h, 1.0), (kv, 1.2), (kv, 0.8)))
    return s


def _tables(need, g, blocks=0):
    """A block table of as many random blocks as each row needs (the rest -1), and the blocks of the cache."""
    blocks = max(blocks, sum(need) + 3)
    perm = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, blocks


def _prepare_chunk(case, seed):
    g, c = _gen(seed, 3), _gen(seed, 4, "cpu")
    context = _shuffled(_spread(case["count"], case["min_context"], case["max_context"]), c)
    # from max_new down to min_new by equal factors: a few chunks, and drafts or single tokens behind them
    new = _new(case)
    lengths = [a + b for a, b in zip(context, new)]
    table, blocks = _tables([(n + PAGE - 1) // PAGE for n in lengths], g)
    s = {"lengths": lengths, "new": new, "table": table, "seq_lens": _i32(lengths), "cu_seqlens": _offsets(new),
         "max_len": case["max_context"] + case["max_new"], "q": _normal((sum(new), case["q_heads"], DIM), 1.0, g)}
    s["table"] = torch.nn.functional.pad(table, (0, max(0, -(-s["max_len"] // PAGE) - table.shape[1])), value=-1)
    s.update(_caches(blocks, case["kv_heads"], g))
    if own:
        import paper_2601_18150_amd as fp8rl
        s["workspace"] = torch.empty(max(16, fp8rl.fp8rl_attention_prompt_workspace_size(
            case["count"], sum(new), case["q_heads"], case["kv_heads"], s["max_len"])), dtype=torch.uint8, device="cuda")
    return s


def _prepare_shared(case, seed):
    g, batch = _gen(seed, 5), case["groups"] * case["samples"]
    own_lens = _shuffled(_spread(batch, case["min_own"], case["max_own"]), _gen(seed, 6, "cpu"))
    pages = case["prefix"] // PAGE
    need = [(n + PAGE - 1) // PAGE for n in own_lens]
    table, blocks = _tables([pages] * case["groups"] + need, g)
    first, rest = table[:case["groups"], :pages], table[case["groups"]:, :max(need)]
    max_len = case["prefix"] + case["max_own"]
    s = {"lengths": [case["prefix"] + n for n in own_lens], "max_len": max_len, "prefix": case["prefix"],
         "table": torch.cat([first.repeat_interleave(case["samples"], 0), rest], 1).contiguous(),
         "group_offsets": _i32([case["samples"] * i for i in range(case["groups"] + 1)]),
         "prefix_lens": _i32([case["prefix"]] * case["groups"]), "q": _normal((batch, case["q_heads"], DIM), 1.0, g)}
    s["table"] = torch.nn.functional.pad(s["table"], (0, max(0, -(-max_len // PAGE) - s["table"].shape[1])), value=-1)
    s["seq_lens"] = _i32(s["lengths"])
    s.update(_caches(blocks, case["kv_heads"], g))
    if own:
        import paper_2601_18150_amd as fp8rl
        s["workspace"] = torch.empty(max(16, fp8rl.fp8rl_attention_decode_shared_workspace_size(
            batch, case["groups"], case["q_heads"], case["kv_heads"], case["prefix"], max_len)), dtype=torch.uint8, device="cuda")
    return s


def _pools(case, blocks, g):
    """The key pages and the value pages of all layers, and each layer's as the calls take them."""
    k, v = (torch.randint(0, 256, (case["layers"], blocks, case["kv_heads"]) + page, generator=g, device="cuda",
                          dtype=torch.uint8) for page in ((PAGE, DIM), (PAGE // PAGE_ROWS, DIM, PAGE_ROWS)))
    return {"k_pool": k, "v_pool": v, "caches": [c for pair in zip(k, v) for c in pair]}


def _prepare_copy(case, seed):
    g = _gen(seed, 7)
    perm = torch.randperm(case["blocks"], generator=g, device="cuda").to(torch.int32)
    return dict(_pools(case, case["blocks"], g), src=perm[:case["count"]].contiguous(),
                dst=perm[case["count"]:2 * case["count"]].contiguous())


def _prepare_fork(case, seed):
    """Prompts in the first rows of the table, their samples' rows behind them and still empty."""
    g, p, n = _gen(seed, 8), case["prompts"], case["prompts"] * case["samples"]
    lengths = _shuffled(_spread(p, case["min_len"], case["max_len"]), _gen(seed, 9, "cpu"))
    need = [(x + PAGE - 1) // PAGE for x in lengths]
    table, blocks = _tables(need + [1] * n, g)
    s = dict(_pools(case, blocks, g), new_blocks=table[p:, 0].contiguous())
    table[p:] = -1
    refs = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    refs[table[:p][table[:p] >= 0].long()] = 1
    s["parents"] = torch.arange(p, dtype=torch.int32, device="cuda").repeat_interleave(case["samples"])
    s["children"] = (torch.randperm(n, generator=g, device="cuda") + p).to(torch.int32)
    s["before"] = {"table": table, "seq_lens": _i32(lengths + [0] * n), "refs": refs}
    s["now"] = {k: v.clone() for k, v in s["before"].items()}
    return s


def _prepare_release(case, seed):
    """Samples that share their prompt's whole pages, each with pages of its own; a part of them has ended."""
    g, c, p, m = _gen(seed, 10), _gen(seed, 11, "cpu"), case["prompts"], case["samples"]
    prompts = _shuffled(_spread(p, case["min_len"], case["max_len"]), c)
    lengths = [prompts[i // m] + n for i, n in enumerate(_shuffled(_spread(p * m, 1, case["max_own"]), c))]
    shared = [x // PAGE for x in prompts]
    mine = [(x + PAGE - 1) // PAGE - shared[i // m] for i, x in enumerate(lengths)]
    most = sum(shared) + p + p * m * (2 + case["max_own"] // PAGE)   # (the same for every seed)
    pages, blocks = _tables([x if x else 1 for x in shared] + mine, g, most)
    width = (case["max_len"] + case["max_own"]) // PAGE + 1
    table = torch.full((p * m, width), -1, dtype=torch.int32, device="cuda")
    for i in range(p * m):
        a = shared[i // m]
        table[i, :a] = pages[i // m, :a]
        table[i, a:a + mine[i]] = pages[p + i, :mine[i]]
    refs = torch.bincount(table[table >= 0].long(), minlength=blocks).to(torch.int32)
    ended = max(1, int(case["ended"] * p * m))
    s = dict(_pools(case, blocks, g), blocks=blocks,
             ended=torch.randperm(p * m, generator=g, device="cuda")[:ended].to(torch.int32),
             before={"table": table, "seq_lens": _i32(lengths), "refs": refs})
    s["now"] = {k: v.clone() for k, v in s["before"].items()}
    s["live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2601_18150_amd as fp8rl
        s["workspace"] = torch.empty(max(16, fp8rl.fp8rl_kv_compact_workspace_size(blocks)), dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    s = {"prompt": _prepare_prompt, "chunk": _prepare_chunk, "shared": _prepare_shared, "copy": _prepare_copy,
         "fork": _prepare_fork, "release": _prepare_release}[case["kind"]](case, seed)
    s["kind"], s["sm_scale"] = case["kind"], 1.0 / math.sqrt(DIM)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def _attend(q, k, v, at, sm_scale):
    """Queries q [n][heads][128] at positions at, at + 1, .. against keys and values [m][kv_heads][128], causal."""
    n, heads, _ = q.shape
    m, kv_heads, _ = k.shape
    group = heads // kv_heads
    rows = q.float().view(n, kv_heads, group, DIM).permute(1, 0, 2, 3).reshape(kv_heads, n * group, DIM)
    k, v = k.float().permute(1, 2, 0).contiguous(), v.float().permute(1, 0, 2).contiguous()
    position = torch.arange(n, device=q.device).repeat_interleave(group) + at
    key = torch.arange(m, device=q.device)
    out = torch.empty_like(rows)
    step = max(1, (1 << 28) // m)                                   # at most 1 GiB of scores at a time
    for h in range(kv_heads):
        for r in range(0, n * group, step):
            x = torch.matmul(rows[h, r:r + step], k[h]) * sm_scale
            x = x.masked_fill(key[None, :] > position[r:r + step, None], -math.inf)
            x = torch.exp(x - x.amax(1, keepdim=True))
            out[h, r:r + step] = torch.matmul(x, v[h]) / x.sum(1, keepdim=True)
    return out.view(kv_heads, n, group, DIM).permute(1, 0, 2, 3).reshape(n, heads, DIM).to(torch.bfloat16)


def _tokens(s, b, n):
    """Keys and values of sequence b's n tokens, [n][kv_heads][128] in 32 bits."""
    blocks = s["table"][b, :(n + PAGE - 1) // PAGE].long()
    k = s["k_cache"][blocks].view(torch.float8_e4m3fn).float() * s["k_scale"]
    v = s["v_cache"][blocks].view(torch.float8_e4m3fn).float() * s["v_scale"]
    kv_heads = k.shape[1]
    return (k.permute(0, 2, 1, 3).reshape(-1, kv_heads, DIM)[:n],
            v.permute(0, 2, 4, 1, 3).reshape(-1, kv_heads, DIM)[:n])


def _prompt(s):
    if own:
        import paper_2601_18150_amd as fp8rl
        return {"out": fp8rl.fp8rl_attention_prompt_bf16(s["q"], s["k"], s["v"], s["cu_seqlens"], s["sm_scale"])}
    out, at = [], 0
    for n in s["lengths"]:
        r = slice(at, at + n)
        out.append(_attend(s["q"][r], s["k"][r], s["v"][r], 0, s["sm_scale"]))
        at += n
    return {"out": torch.cat(out)}


def _chunk(s):
    if own:
        import paper_2601_18150_amd as fp8rl
        return {"out": fp8rl.fp8rl_attention_prompt_fp8kv(
            s["q"], s["k_cache"], s["v_cache"], s["table"], s["seq_lens"], s["cu_seqlens"], s["max_len"], s["k_scale"],
            s["v_scale"], s["sm_scale"], workspace=s["workspace"])}
    out, at = [], 0
    for b, (n, m) in enumerate(zip(s["lengths"], s["new"])):
        out.append(_attend(s["q"][at:at + m], *_tokens(s, b, n), n - m, s["sm_scale"]))
        at += m
    return {"out": torch.cat(out)}


def _shared(s):
    if own:
        import paper_2601_18150_amd as fp8rl
        return {"out": fp8rl.fp8rl_attention_decode_shared_fp8kv(
            s["q"], s["k_cache"], s["v_cache"], s["table"], s["seq_lens"], s["group_offsets"], s["prefix_lens"],
            s["prefix"], s["max_len"], s["k_scale"], s["v_scale"], s["sm_scale"], workspace=s["workspace"])}
    return {"out": torch.cat([_attend(s["q"][b:b + 1], *_tokens(s, b, n), n - 1, s["sm_scale"])
                              for b, n in enumerate(s["lengths"])])}


def _pages(s):
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _copy(s):
    if own:
        import paper_2601_18150_amd as fp8rl
        fp8rl.fp8rl_kv_copy_blocks(s["caches"], s["src"], s["dst"])
    else:
        for c in s["caches"]:
            c[s["dst"].long()] = c[s["src"].long()]
    return _pages(s)


def _restore(s):
    """The tables as the program's scheduler left them before the call."""
    for name, x in s["now"].items():
        x.copy_(s["before"][name])
    return s["now"]["table"], s["now"]["seq_lens"], s["now"]["refs"]


def _fork(s):
    table, lens, refs = _restore(s)
    if own:
        import paper_2601_18150_amd as fp8rl
        fp8rl.fp8rl_kv_fork_sequences(s["caches"], table, lens, refs, s["parents"], s["children"], s["new_blocks"])
    else:
        parents, children = s["parents"].long(), s["children"].long()
        n = lens[parents]
        page = torch.arange(table.shape[1], device="cuda")[None, :]
        whole, tail = page < (n // PAGE)[:, None], n % PAGE != 0
        rows = table[parents]
        refs.index_add_(0, rows[whole].long(), torch.ones_like(rows[whole]))
        at = (n // PAGE).long().clamp(max=table.shape[1] - 1)[:, None]
        src, dst = rows.gather(1, at)[:, 0][tail].long(), s["new_blocks"][tail].long()
        for c in s["caches"]:
            c[dst] = c[src]
        refs.index_add_(0, dst, torch.ones_like(dst, dtype=torch.int32))
        rows = torch.where(whole, rows, table[children])
        last = (page == (n // PAGE)[:, None]) & tail[:, None]
        table[children] = torch.where(last, s["new_blocks"][:, None], rows)
        lens[children] = n
    return dict(_pages(s), **s["now"])


def _release(s):
    table, lens, refs = _restore(s)
    if own:
        import paper_2601_18150_amd as fp8rl
        fp8rl.fp8rl_kv_free_sequences(table, lens, refs, s["ended"])
        fp8rl.fp8rl_kv_compact(s["caches"], table, lens, refs, live=s["live"], workspace=s["workspace"])
    else:
        page, ended = torch.arange(table.shape[1], device="cuda")[None, :], s["ended"].long()
        gone = table[ended][page < ((lens[ended] + PAGE - 1) // PAGE)[:, None]].long()
        refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
        lens[ended] = 0
        live = refs > 0
        total = int(live.sum())
        holes = torch.nonzero(~live[:total])[:, 0]
        movers = total + torch.nonzero(live[total:])[:, 0].flip(0)
        for c in s["caches"]:
            c[holes] = c[movers]
        refs[holes] = refs[movers]
        refs[movers] = 0
        to = torch.arange(s["blocks"], dtype=torch.int32, device="cuda")
        to[movers] = holes.to(torch.int32)
        used = page < ((lens + PAGE - 1) // PAGE)[:, None]
        table.copy_(torch.where(used, to[table.clamp(min=0).long()], table))
        s["live"].fill_(total)
    return dict(_pages(s), live=s["live"], **s["now"])


def run(state):
    return {"prompt": _prompt, "chunk": _chunk, "shared": _shared, "copy": _copy, "fork": _fork,
            "release": _release}[state["kind"]](state)


# --------------------------------------------------------------------------
# unavoidable work, 64-bit outputs
# --------------------------------------------------------------------------
def work(case):
    kind, kv = case["kind"], case["kv_heads"]
    if kind in ("prompt", "chunk", "shared"):
        h = case["q_heads"]
        if kind == "prompt":
            lengths = _spread(case["count"], case["min_len"], case["max_len"])
            pairs = sum(n * (n + 1) // 2 for n in lengths)
            size = sum(lengths) * DIM * 2 * (2 * h + 2 * kv)
        elif kind == "chunk":
            new, context = _new(case), _spread(case["count"], case["min_context"], case["max_context"])
            mean = sum(context) / len(context)                      # (which context meets which chunk is the seed's)
            pairs = sum(n * mean + n * (n + 1) / 2 for n in new)
            size = sum(new) * DIM * 2 * 2 * h + (sum(context) + sum(new)) * DIM * 2 * kv
        else:
            lengths = _spread(case["groups"] * case["samples"], case["min_own"], case["max_own"])
            pairs = sum(lengths) + len(lengths) * case["prefix"]
            size = len(lengths) * DIM * 2 * 2 * h + (sum(lengths) + case["groups"] * case["prefix"]) * DIM * 2 * kv
        return {"bytes": int(size), "flops": int(4 * DIM * h * pairs)}
    page = 2 * case["layers"] * kv * PAGE * DIM                     # of all caches
    if kind == "copy":
        return {"bytes": 2 * page * case["count"], "flops": 0}
    prompts = _spread(case["prompts"], case["min_len"], case["max_len"])
    if kind == "fork":
        return {"bytes": 2 * page * case["samples"] * sum(n % PAGE != 0 for n in prompts), "flops": 0}
    # the samples' pages that stay, and the prompts' of which a sample stays; the holes below the number of pages that
    # stay are as frequent as anywhere in the pool, and each takes a page
    samples = case["prompts"] * case["samples"]
    own_pages = sum((n % PAGE + m + PAGE - 1) // PAGE for n, m in
                    zip(prompts * case["samples"], _spread(samples, 1, case["max_own"])))
    shared = sum(n // PAGE for n in prompts) * (1.0 - case["ended"] ** case["samples"])
    live = own_pages * (1.0 - case["ended"]) + shared
    total = sum(n // PAGE for n in prompts) + case["prompts"] + samples * (2 + case["max_own"] // PAGE)
    return {"bytes": int(2 * page * live * (1.0 - live / total)), "flops": 0}


def _exact_rows(q, k, v, at, sm_scale):
    """One sequence in 64 bits, query head by query head, a block of rows at a time."""
    n, heads, _ = q.shape
    group = heads // k.shape[1]
    out = torch.empty((n, heads, DIM), dtype=torch.float64, device=q.device)
    for h in range(heads):
        kh, vh = k[:, h // group].double().t().contiguous(), v[:, h // group].double().contiguous()
        for r in range(0, n, 4096):
            e = min(n, r + 4096)
            last = at + e                                           # keys that any row of the block sees
            x = torch.matmul(q[r:e, h].double(), kh[:, :last].contiguous()) * sm_scale
            x += torch.triu(torch.full((e - r, last), -math.inf, dtype=torch.float64, device=q.device), at + r + 1)
            out[r:e, h] = torch.matmul(torch.softmax(x, 1), vh[:last])
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind not in ("prompt", "chunk", "shared"):
        return None                                                 # bytes and whole numbers, moved and counted
    s = prepare(case, seed)
    out, at = [], 0
    for b, n in enumerate(s["lengths"]):
        m = n if kind == "prompt" else s["new"][b] if kind == "chunk" else 1
        if kind == "prompt":
            k, v = s["k"][at:at + n], s["v"][at:at + n]
        else:
            t = torch.arange(n, device="cuda")
            blk, off = s["table"][b].long()[t // PAGE], t % PAGE
            k = s["k_cache"].view(torch.float8_e4m3fn)[blk, :, off].double() * s["k_scale"].double()
            v = s["v_cache"].view(torch.float8_e4m3fn)[blk, :, off // PAGE_ROWS, :, off % PAGE_ROWS].double() * s["v_scale"].double()
        out.append(_exact_rows(s["q"][at:at + m], k, v, n - m, s["sm_scale"]))
        at += m
    return {"out": torch.cat(out)}
