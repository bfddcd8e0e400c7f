"""Operators on many tokens a sequence over the paged cache: insertion, attention of prompts, of drafted tokens.

Tokens come packed: sequence b owns rows [cu[b], cu[b + 1]) of the packed arrays.

  append  new tokens go into the pages of the cache and into the pages' min/max metadata; token i of
          sequence b is row `rows`[cu[b] + i] of the keys and values (or row cu[b] + i) and takes position
          L_b - n_b + i of the L_b tokens that the sequence then has
  prompt  causal attention: query i of sequence b stands at position p = L_b - n_b + i of the cached tokens,
          z_j = scale q.k_j for j <= p, out = sum_j exp(z_j - lse) v_j, lse = log sum_j exp(z_j)
  tree    attention of drafted tokens: node i of sequence b attends to the L_b cached tokens, or to those of the listed
          pages of its KV head, and to the drafted nodes j of its sequence whose bit j % 64 of mask word j / 64 is set

Fields of a case: op; batch; heads and kv_heads (query and KV heads of 128 channels); page (tokens per page); new and
shortest_new (most and fewest packed tokens of a sequence); past and shortest_past (most and fewest tokens
that a sequence has in the cache before them); listed (pages listed per KV head; 0: all); half_out (fp16 output
instead of fp32); shuffled (physical pages in random order); picked (append: the new tokens are rows picked
from a larger packed array).
"""
import math

import numpy as np
import torch

own = False

HEAD_DIM = 128
SCALE = 1.0 / math.sqrt(HEAD_DIM)
OUTLIERS, OUTLIER_SCALE = 4, 8.0     # channels of a head whose keys are much larger than the others'
MAX_FLOPS = 8.0e12                   # of a drawn case
MAX_BYTES = 2.6e9


def _case(name, op, new, past, **more):
    case = dict(name=name, op=op, batch=1, heads=32, kv_heads=32, page=16, new=new, shortest_new=new, past=past,
                shortest_past=past, listed=0, half_out=True, shuffled=False, picked=False)
    case.update(more)
    return case


def listed():
    return [
        # a short question to an idle server: launches and latency
        _case("prompt 77", "prompt", 77, 0),
        # a page of text, multi-head attention
        _case("prompt 4k", "prompt", 4096, 0),
        # several users' prompts of different lengths, prefilled together
        _case("prompt ragged groups", "prompt", 4999, 0, batch=6, kv_heads=8, page=64, shortest_new=301, shuffled=True),
        # the next part of a long prompt that is prefilled in parts, between decode steps
        _case("prompt part 512 at 32k", "prompt", 512, 32256, kv_heads=8, shuffled=True),
        # a long document at once, grouped heads
        _case("prompt 32k groups", "prompt", 32749, 0, kv_heads=8),
        # a second turn of two chats, outputs kept in fp32
        _case("prompt turn fp32", "prompt", 1500, 2600, batch=2, heads=40, kv_heads=40, shortest_new=700,
              shortest_past=35, page=32, half_out=False),
        # the smallest check of drafts: one head, 4k tokens of context
        _case("tree 1 head 4k", "tree", 8, 4096, heads=1, kv_heads=1, half_out=False),
        # one user's drafts at 32k tokens, multi-head attention
        _case("tree 32k", "tree", 26, 32768, shuffled=True),
        # sixteen users, grouped heads, ragged contexts of 8k to 64k tokens, trees of 5 to 60 nodes
        _case("tree batch 16 groups", "tree", 60, 65519, batch=16, heads=64, kv_heads=8, shortest_new=5,
              shortest_past=8209, shuffled=True),
        # drafts over selected pages: 128 pages of 16 tokens, a 2048-token budget
        _case("tree selected", "tree", 16, 32768, batch=4, kv_heads=8, shortest_past=20011, listed=128, half_out=False,
              shuffled=True),
        # after a check of drafts: the accepted ones of 16 users go into the cache
        _case("append accepted", "append", 5, 30000, batch=16, kv_heads=8, shortest_new=1, shortest_past=900, shuffled=True,
              picked=True),
        # a 32k prompt goes into the cache
        _case("append 32k", "append", 32749, 0),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "tree", "tree", "append"])
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (8, 8), (1, 1), (32, 8), (64, 8), (16, 8)])
    batch = _spread(rng, 1, 16)
    if op == "prompt":
        new, past = _spread(rng, 1, 32000), rng.choice([0, 0, _spread(rng, 1, 60000)])
    elif op == "tree":
        new, past = _spread(rng, 1, 100), _spread(rng, 1, 100000)
    else:
        new, past = rng.choice([_spread(rng, 1, 8), _spread(rng, 1, 32000)]), rng.choice([0, _spread(rng, 1, 30000)])
    case = _case("", op, new, past, batch=batch, heads=heads, kv_heads=kv_heads, page=rng.choice([8, 16, 16, 16, 32, 64]),
                 half_out=rng.random() < 0.6, shuffled=rng.random() < 0.6)
    del case["name"]
    if op == "tree" and rng.random() < 0.4:
        case["listed"] = max(1, _spread(rng, 256, 4096) // case["page"])
    if op == "append":
        case["picked"] = rng.random() < 0.5
    ragged = rng.uniform(0.05, 1.0) if batch > 1 else 1.0
    while True:
        case["shortest_new"] = max(1, int(case["new"] * ragged))
        case["shortest_past"] = int(case["past"] * ragged)
        cost = work(case)
        if cost["flops"] <= MAX_FLOPS and cost["bytes"] <= MAX_BYTES and _cached(case) <= 800000:
            return case
        if case["batch"] > 1:
            case["batch"] -= 1
        else:
            case["new"] = max(1, case["new"] * 3 // 4)
            case["past"] = case["past"] * 3 // 4


def _between(longest, shortest, n, turn):
    """n lengths from shortest to longest, evenly spaced, in mixed order."""
    order = sorted(range(n), key=lambda i: (i * turn) % 1.0)
    lens = [longest] * n
    for rank, b in enumerate(order):
        if rank:
            lens[b] -= (longest - shortest) * rank // (n - 1)
    return lens


def _new(case):
    return _between(case["new"], case["shortest_new"], case["batch"], 0.618034)


def _past(case):
    return _between(case["past"], case["shortest_past"], case["batch"], 0.414214)


def _cached(case):
    return sum(_past(case)) + (0 if case["op"] == "tree" else sum(_new(case)))


def work(case):
    H, Hkv, S = case["heads"], case["kv_heads"], case["page"]
    row = 2 * HEAD_DIM                                            # one fp16 vector
    new, past = _new(case), _past(case)
    total = sum(new)
    if case["op"] == "append":
        opened = sum((p + n - 1) // S - -(-p // S) + 1 for n, p in zip(new, past))
        folded = sum(p % S > 0 for p in past)                     # pages that held tokens before
        entries = (opened + 2 * folded) * Hkv * 2 * row
        return {"bytes": 4 * total * Hkv * row + entries, "flops": 0}
    outs = total * H * (HEAD_DIM * (2 if case["half_out"] else 4) + 4)
    if case["op"] == "prompt":
        pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
        tokens = sum(new) + sum(past)
        more = 0
    else:
        seen = [min(p, case["listed"] * S) if case["listed"] else p for p in past]
        depth = [min(n, 1 + int(math.log2(n))) for n in new]      # ancestors of a node, about
        pairs = sum(n * (s + d) for n, s, d in zip(new, seen, depth))
        tokens = sum(seen) + total
        more = 8 * total * -(-case["new"] // 64) + 4 * case["batch"] * Hkv * case["listed"]
    return {"bytes": total * H * row + 2 * tokens * Hkv * row + outs + more, "flops": 4 * HEAD_DIM * H * pairs}


def _trees(rng, new, words):
    """A random tree per sequence, a node behind its parent: which nodes a node attends to, as 64-bit words."""
    mask = np.zeros((sum(new), words), np.uint64)
    at = 0
    for n in new:
        rows = mask[at:at + n]
        for i in range(n):
            parent = int(rng.integers(-1, i)) if i else -1        # -1: the context
            if parent >= 0:
                rows[i] = rows[parent]
            rows[i, i // 64] |= np.uint64(1 << (i % 64))
        at += n
    return mask.view(np.int64)


def prepare(case, seed):
    dev = "cuda:0"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, H, Hkv, S, op = case["batch"], case["heads"], case["kv_heads"], case["page"], case["op"]
    new, past = _new(case), _past(case)
    lens = past if op == "tree" else [n + p for n, p in zip(new, past)]
    pages = [-(-n // S) for n in lens]
    width, count = max(max(pages), 1), max(sum(pages), 1)
    ids = rng.permutation(count) if case["shuffled"] else np.arange(count)
    table = np.zeros((B, width), np.int32)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = ids[at:at + pages[b]]
        at += pages[b]

    def normal(*shape):
        return torch.randn(*shape, device=dev, dtype=torch.float16, generator=gen)

    size = torch.ones(Hkv, HEAD_DIM, device=dev, dtype=torch.float16)
    for h in range(Hkv):
        size[h, torch.from_numpy(rng.choice(HEAD_DIM, OUTLIERS, replace=False)).to(dev)] = OUTLIER_SCALE
    total = sum(new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    s = dict(case=case, new=new, lens=lens, pages=pages, total=total,
             table=torch.from_numpy(table).to(dev), seq_lens=torch.tensor(lens, dtype=torch.int32, device=dev),
             cu=torch.from_numpy(cu).to(dev),
             k_pool=normal(count, Hkv, S, HEAD_DIM).mul_(size[:, None]), v_pool=normal(count, Hkv, S, HEAD_DIM),
             meta=torch.zeros(Hkv, count, 2, HEAD_DIM, device=dev, dtype=torch.float16))
    if op == "append":
        for b in range(B):                                        # metadata of the tokens before the new ones
            full, rest = past[b] // S, past[b] % S
            phys = s["table"][b].long()
            if full:
                keys = s["k_pool"][phys[:full]]
                s["meta"][:, phys[:full], 0] = keys.amin(2).transpose(0, 1)
                s["meta"][:, phys[:full], 1] = keys.amax(2).transpose(0, 1)
            if rest:
                keys = s["k_pool"][phys[full], :, :rest]
                s["meta"][:, phys[full], 0] = keys.amin(1)
                s["meta"][:, phys[full], 1] = keys.amax(1)
        given = total if not case["picked"] else total * 3 + 5
        s["k_new"], s["v_new"] = normal(given, Hkv, HEAD_DIM).mul_(size), normal(given, Hkv, HEAD_DIM)
        s["rows"] = torch.from_numpy(rng.permutation(given)[:total].astype(np.int32)).to(dev) if case["picked"] else None
    else:
        s["q"] = normal(total, H, HEAD_DIM)
        s["out"] = torch.empty(total, H, HEAD_DIM, device=dev, dtype=torch.float16 if case["half_out"] else torch.float32)
        s["lse"] = torch.empty(total, H, device=dev, dtype=torch.float32)
    if op == "tree":
        s["k_new"], s["v_new"] = normal(total, Hkv, HEAD_DIM).mul_(size), normal(total, Hkv, HEAD_DIM)
        s["mask"] = torch.from_numpy(_trees(rng, new, -(-case["new"] // 64))).to(dev)
        s["pages_of"] = None
        if case["listed"]:                                        # as a selection leaves them: ascending, -1 behind
            lists = np.full((B, Hkv, case["listed"]), -1, np.int32)
            for b in range(B):
                for h in range(Hkv):
                    n = min(case["listed"], pages[b])
                    lists[b, h, :n] = np.sort(rng.permutation(pages[b])[:n])
            s["pages_of"] = torch.from_numpy(lists).to(dev)
    if own:
        from paper_2406_10774_amd import binding as Q
        s["cache"] = Q.Cache(s["k_pool"], s["v_pool"], s["meta"], s["table"], s["seq_lens"], num_heads=H)
        if op != "append":
            s["workspace"] = torch.zeros(max(Q.quest_tokens_workspace_bytes(s["cache"], total), 4) // 4, device=dev,
                                         dtype=torch.int32)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2406_10774_amd import binding as Q
        if op == "append":
            Q.quest_append_tokens(s["cache"], s["k_new"], s["v_new"], s["cu"], rows=s["rows"])
            return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "meta": s["meta"]}
        if op == "prompt":
            Q.quest_prompt_attention(s["cache"], s["q"], s["cu"], SCALE, s["out"], lse=s["lse"], workspace=s["workspace"])
        else:
            Q.quest_tree_attention(s["cache"], s["q"], s["k_new"], s["v_new"], s["cu"], s["mask"], SCALE, s["out"],
                                   topk_idx=s["pages_of"], lse=s["lse"], workspace=s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "append":
        _append(s)
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "meta": s["meta"]}
    (_prompt if op == "prompt" else _tree)(s)
    return {"out": s["out"], "lse": s["lse"]}


# ---- the plain forms

def _append(s):
    S = s["case"]["page"]
    at = 0
    for b, (n, length) in enumerate(zip(s["new"], s["lens"])):
        src = torch.arange(at, at + n, device=s["cu"].device)
        if s["rows"] is not None:
            src = s["rows"][src].long()
        at += n
        position = torch.arange(length - n, length, device=src.device)
        phys = s["table"][b].long()[position // S]
        s["k_pool"][phys, :, position % S] = s["k_new"][src]
        s["v_pool"][phys, :, position % S] = s["v_new"][src]
        first, last = (length - n) // S, (length - 1) // S
        touched = s["table"][b, first:last + 1].long()
        keys = s["k_pool"][touched].transpose(0, 1).float()                       # [Hkv][pages][S][D]
        there = torch.arange(first * S, (last + 1) * S, device=src.device).view(1, -1, S, 1) < length
        s["meta"][:, touched, 0] = torch.where(there, keys, math.inf).amin(2).half()
        s["meta"][:, touched, 1] = torch.where(there, keys, -math.inf).amax(2).half()


def _cached_kv(s, b):
    """Keys and values of sequence b as [Hkv][tokens][D], in 32 bits."""
    phys = s["table"][b, :s["pages"][b]].long()
    return [pool[phys].transpose(0, 1).flatten(1, 2)[:, :s["lens"][b]].float() for pool in (s["k_pool"], s["v_pool"])]


def _softmax(z, v):
    """Weights of z against the values v: outputs and lse; a row of -inf gives 0 and -inf."""
    top = z.amax(-1, keepdim=True).clamp(min=-3.0e38)
    p = (z - top).exp()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total.clamp(min=1e-38), (top + total.log()).squeeze(-1)


def _prompt(s):
    H, Hkv = s["case"]["heads"], s["case"]["kv_heads"]
    G = H // Hkv
    at = 0
    for b, (n, length) in enumerate(zip(s["new"], s["lens"])):
        k, v = _cached_kv(s, b)
        step = max(64, min(2048, (1 << 28) // (G * length)))
        for i in range(0, n, step):
            m = min(step, n - i)
            end = length - n + i + m                                              # keys that the last of them sees
            position = torch.arange(end - m, end, device=k.device)
            hidden = torch.arange(end, device=k.device) > position[:, None]
            q = s["q"][at + i:at + i + m].float()
            for h in range(Hkv):
                qh = q[:, h * G:(h + 1) * G].transpose(0, 1)                      # [G][m][D]
                z = torch.matmul(qh, k[h, :end].t()) * SCALE
                z.masked_fill_(hidden, -math.inf)
                o, lse = _softmax(z, v[h, :end])
                s["out"][at + i:at + i + m, h * G:(h + 1) * G] = o.transpose(0, 1).to(s["out"].dtype)
                s["lse"][at + i:at + i + m, h * G:(h + 1) * G] = lse.t()
        at += n


def _tree(s):
    H, Hkv, S = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["page"]
    G = H // Hkv
    at = 0
    for b, (n, length) in enumerate(zip(s["new"], s["lens"])):
        j = torch.arange(n, device=s["mask"].device)
        sees = (s["mask"][at:at + n][:, j // 64] >> (j % 64)) & 1                 # [n][n]
        kd, vd = (t[at:at + n].transpose(0, 1).float() for t in (s["k_new"], s["v_new"]))
        if s["pages_of"] is None:
            k, v = _cached_kv(s, b)
            there = torch.ones(Hkv, k.shape[1], dtype=torch.bool, device=k.device)
        else:
            pages = s["pages_of"][b].long()                                       # [Hkv][K]
            position = pages[..., None] * S + torch.arange(S, device=pages.device)
            there = ((pages[..., None] >= 0) & (position < length)).flatten(1)
            phys = s["table"][b].long()[pages.clamp(min=0)]
            head = torch.arange(Hkv, device=pages.device)[:, None]
            k, v = (torch.where(there[..., None], pool[phys, head].flatten(1, 2).float(), 0.0)
                    for pool in (s["k_pool"], s["v_pool"]))
        k, v = torch.cat([k, kd], 1), torch.cat([v, vd], 1)
        q = s["q"][at:at + n].float().view(n, Hkv, G, HEAD_DIM).permute(1, 2, 0, 3).reshape(Hkv, G * n, HEAD_DIM)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) * SCALE
        z = z.view(Hkv, G, n, -1)
        z[..., :-n].masked_fill_(~there[:, None, None], -math.inf)
        z[..., -n:].masked_fill_(sees == 0, -math.inf)
        o, lse = _softmax(z.view(Hkv, G * n, -1), v)
        s["out"][at:at + n] = o.view(Hkv, G, n, HEAD_DIM).permute(2, 0, 1, 3).reshape(n, H, HEAD_DIM).to(s["out"].dtype)
        s["lse"][at:at + n] = lse.view(Hkv, G, n).permute(2, 0, 1).reshape(n, H)
        at += n


# ---- the same from the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    H, Hkv, S = case["heads"], case["kv_heads"], case["page"]
    table, cu = s["table"].cpu().numpy(), s["cu"].cpu().numpy()
    if case["op"] == "append":
        k_pool, v_pool, meta = (s[name].double() for name in ("k_pool", "v_pool", "meta"))
        rows = np.arange(s["total"]) if s["rows"] is None else s["rows"].cpu().numpy()
        page, slot, changed = [], [], []
        for b in range(case["batch"]):
            n = cu[b + 1] - cu[b]
            for position in range(s["lens"][b] - n, s["lens"][b]):
                page.append(table[b, position // S])
                slot.append(position % S)
                if not changed or changed[-1][0] != page[-1]:
                    changed.append([page[-1], 0])
                changed[-1][1] = slot[-1] + 1                     # tokens that the page holds
        page, slot, rows = (torch.from_numpy(np.asarray(a, np.int64)).to(k_pool.device) for a in (page, slot, rows))
        k_pool[page, :, slot] = s["k_new"].double()[rows]
        v_pool[page, :, slot] = s["v_new"].double()[rows]
        for held in sorted({c[1] for c in changed}):
            at = torch.tensor([int(c[0]) for c in changed if c[1] == held], device=k_pool.device)
            keys = k_pool[at, :, :held]
            meta[:, at, 0] = keys.min(2).values.transpose(0, 1)
            meta[:, at, 1] = keys.max(2).values.transpose(0, 1)
        return {"k_pool": k_pool, "v_pool": v_pool, "meta": meta}
    if work(case)["flops"] > 2.0e13:
        return None
    device = s["table"].device
    out = torch.zeros(s["total"], H, HEAD_DIM, dtype=torch.float64, device=device)
    lse = torch.zeros(s["total"], H, dtype=torch.float64, device=device)
    mask = s["mask"].tolist() if case["op"] == "tree" else None
    for b in range(case["batch"]):
        first, last, length = int(cu[b]), int(cu[b + 1]), s["lens"][b]
        where = torch.arange(length, device=device)
        phys = torch.from_numpy(table[b].astype(np.int64)).to(device)[where // S]
        if mask:
            unseen = torch.tensor([[(words[j // 64] >> (j % 64)) & 1 == 0 for j in range(last - first)]
                                   for words in mask[first:last]], device=device)
        for g in range(Hkv):
            k, v = s["k_pool"][phys, g, where % S].double(), s["v_pool"][phys, g, where % S].double()
            if mask:
                if s["pages_of"] is not None:
                    pages = s["pages_of"][b, g]
                    chosen = torch.isin(where // S, pages[pages >= 0].long())
                    k, v = k[chosen], v[chosen]
                k = torch.cat([k, s["k_new"][first:last, g].double()])
                v = torch.cat([v, s["v_new"][first:last, g].double()])
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                for i in range(first, last, 4096):
                    e = min(i + 4096, last)
                    keys = k.shape[0] if mask else length - last + e
                    logits = s["q"][i:e, h].double() @ k[:keys].t() * SCALE
                    if mask:
                        logits[:, keys - (last - first):][unseen[i - first:e - first]] = -math.inf
                    else:
                        logits[torch.triu(torch.ones_like(logits, dtype=torch.bool), keys - (e - i) + 1)] = -math.inf
                    total = torch.logsumexp(logits, -1)
                    out[i:e, h] = (logits - total[:, None]).exp() @ v[:keys]
                    lse[i:e, h] = total
    return {"out": out, "lse": lse}
