"""Operators of drafting and of cache eviction over the paged KV cache, and the cases they are measured on.

Four operators: attention of a tree of drafted tokens over the cache (`tree`), attention that also adds up how much weight
every cached token gets (`weighted`), the choice of the tokens to keep by that weight (`select`), and the move of kept
tokens to the front, in place, in the pages of one or of all layers (`compact`: the accepted path of a tree, or an eviction).

`run` computes them in their plain form, or, where `own` is true, with the library's entry points.  Lengths, page tables
and drafted trees' sizes come from the case alone, values from the seed; K/V and queries are N(0,1) as in the repository's
other workloads, pages a random permutation of the pool.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
FP8_SCALE = 2.0 ** -5  # K and V scale of the FP8 pages: N(0,1) values / scale stay far below 448


def _case(name, op, hq, hkv, dim, pages, batch, ctx, shape, new=(1, 1), layers=1, budget=0, sinks=0, recent=0):
    case = dict(op=op, hq=hq, hkv=hkv, dim=dim, pages=pages, batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1],
                layers=layers, budget=budget, sinks=sinks, recent=recent, shape=shape)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: one conversation of a small model, a handful of drafted tokens
        _case("tree_tiny", "tree", 8, 2, 64, "bf16", 1, (37, 256), 1, new=(5, 5)),
        # a few conversations of an 8B-class layer, a usual tree of some tens of nodes each
        _case("tree_few", "tree", 32, 8, 128, "bf16", 6, (700, 6000), 2, new=(26, 64)),
        # a decode batch of a 70B-class layer with small trees, as a loaded node drafts
        _case("tree_batch", "tree", 64, 8, 128, "bf16", 32, (1024, 8192), 3, new=(8, 24)),
        # long contexts on quantised pages, full trees
        _case("tree_long_fp8", "tree", 32, 8, 128, "fp8", 4, (30000, 90000), 4, new=(60, 64)),
        # one running answer whose cache is watched
        _case("weighted_one", "weighted", 32, 8, 128, "bf16", 1, (4000, 4000), 5),
        # a decode batch whose cache is watched
        _case("weighted_batch", "weighted", 32, 8, 128, "bf16", 64, (1024, 8192), 6),
        # the last rows of long prompts choose what stays of them, five query heads to a KV head
        _case("weighted_window", "weighted", 40, 8, 128, "bf16", 4, (4096, 32768), 7, new=(16, 33)),
        # one conversation is cut down
        _case("select_one", "select", 32, 8, 128, "bf16", 1, (1500, 1500), 8, budget=512, sinks=4, recent=64),
        # a whole batch, some contexts still below the budget
        _case("select_batch", "select", 32, 8, 128, "bf16", 64, (1024, 8192), 9, budget=2048, sinks=4, recent=256),
        # very long prompts, few of them
        _case("select_long", "select", 32, 8, 128, "bf16", 3, (40000, 131072), 10, budget=8192, sinks=16, recent=1024),
        # the accepted paths of a batch of trees, every layer of a model in one call
        _case("compact_accepted", "compact", 32, 8, 128, "bf16", 16, (300, 2000), 11, new=(16, 64), layers=32),
        # an eviction: every KV head keeps tokens of its own
        _case("compact_evicted", "compact", 32, 8, 128, "bf16", 32, (1024, 8192), 12, budget=1024, sinks=4, recent=128),
    ]


MOST_BYTES, MOST_FLOPS, MOST_SCORES = 1.4e9, 3.0e11, 1.0e9  # of a drawn case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["tree", "tree", "weighted", "weighted", "select", "compact"])
        hq, hkv, dim = rng.choice([(8, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (40, 8, 128), (32, 4, 128)])
        pages = rng.choice(["bf16", "bf16", "fp8"])
        batch, low = _log_int(rng, 1, 64), _log_int(rng, 20, 30000)
        ctx = (low, _log_int(rng, low, 8 * low))
        new, layers, budget, sinks, recent = (1, 1), 1, 0, 0, 0
        if op == "tree" or op == "weighted" and rng.random() < 0.4:
            few = _log_int(rng, 2, 64)
            new = (few, rng.randint(few, 64))
        if op == "select" or op == "compact" and rng.random() < 0.6:
            budget = max(8, min(16384, int(low * rng.uniform(0.1, 1.2))))
            sinks, recent = rng.randint(0, min(16, budget // 4)), rng.randint(0, budget // 2)
        elif op == "compact":
            few = _log_int(rng, 2, 64)
            new, layers = (few, rng.randint(few, 64)), rng.choice([1, 16, 32])
        case = _case(None, op, hq, hkv, dim, pages, batch, ctx, rng.randrange(1 << 20), new, layers, budget, sinks, recent)
        L, n = _lengths(case)
        w = work(case)
        scores = float(batch) * hq * float(n.max()) * float((L + n).max())  # the plain form's padded scores
        pool = 2.0 * hkv * dim * float((L + n).sum()) * layers * 2
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and (op not in ("tree", "weighted") or scores <= MOST_SCORES) and pool <= 8e9:
            return case


def _lengths(case):
    """Cached and new tokens of every sequence."""
    r = np.random.default_rng(case["shape"])
    lo, hi = math.log(max(1, case["ctx_lo"])), math.log(max(1, case["ctx_hi"]))
    L = np.rint(np.exp(r.uniform(lo, hi, case["batch"]))).astype(np.int64)
    n = r.integers(case["new_lo"], case["new_hi"] + 1, case["batch"])
    return L, n


def _counts(case):
    """Compaction: where the moved tokens go (first[i] ..), and how many they are."""
    L, n = _lengths(case)
    if case["budget"]:
        return np.zeros_like(L), np.minimum(L, case["budget"])
    r = np.random.default_rng(case["shape"] + 2)
    return L, np.minimum(n, r.integers(1, 9, case["batch"]))


def _page_tables(case, tokens):
    """Page ids of sequences of `tokens` tokens: disjoint slices of one permutation of a pool with some room."""
    r = np.random.default_rng(case["shape"] + 1)
    need = (tokens + PAGE - 1) // PAGE
    num_pages = int(need.sum()) + 64
    perm = r.permutation(num_pages).astype(np.int32)
    table = np.full((len(need), int(need.max())), -1, np.int32)
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = perm[at:at + c]
        at += int(c)
    return table, num_pages


def _trees(case, seed):
    """Who descends from whom: word j of a sequence has the bits of node j and of its ancestors."""
    r = np.random.default_rng([case["shape"], seed])
    rows = []
    for count in _lengths(case)[1]:
        masks = []
        for j in range(int(count)):
            parent = int(r.integers(max(-1, j - 12), j)) if j else -1
            masks.append((masks[parent] if parent >= 0 else 0) | (1 << j))
        rows += masks
    return np.array(rows, np.uint64).view(np.int64).reshape(-1, 1)


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _filled_pools(gen, layers, elems, fp8):
    """Resident K/V of every layer's pool: N(0,1) values, or the FP8 codes of such values over the scale."""
    pools = torch.empty((layers, elems), dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
    flat = pools.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        part = flat[a:a + (1 << 28)]
        if fp8:
            x = torch.empty(part.shape, dtype=torch.float32, device="cuda").normal_(generator=gen)
            part.copy_((x / FP8_SCALE).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            part.normal_(generator=gen)
    return pools


def _gathered(weights, spread=2.0):
    """Weights as attention leaves them: heavy-tailed, many of them next to nothing, some exactly zero."""
    w = weights.normal_().mul_(spread).exp_()
    return w.masked_fill_(torch.rand_like(w) < 0.03, 0.0)


def prepare(case, seed):
    torch.manual_seed(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    fp8 = case["pages"] == "fp8"
    hq, hkv, dim, op = case["hq"], case["hkv"], case["dim"], case["op"]
    L, n = _lengths(case)
    state = dict(op=op, hq=hq, hkv=hkv, dim=dim, fp8=fp8, layers=case["layers"], budget=case["budget"], sinks=case["sinks"], recent=case["recent"],
                 scale=1.0 / math.sqrt(dim), L=L.astype(np.int32), n=n.astype(np.int32), L_dev=torch.from_numpy(L).cuda(), n_dev=torch.from_numpy(n).cuda())
    total = L if op == "select" or op == "compact" and case["budget"] else L + n
    table, num_pages = _page_tables(case, total)
    state.update(num_pages=num_pages, table=torch.from_numpy(table).cuda(), longest=int(total.max()))
    if own:
        import paper_2603_13358_amd as ppd
        state["stream"] = torch.cuda.current_stream().cuda_stream
        state["ctx"] = ppd.Context(hq, hkv, dim, num_pages)
        if fp8:
            state["ctx"].set_kv_format(ppd.PPD_KV_FP8_E4M3, FP8_SCALE, FP8_SCALE)
    if op == "select":
        state["weights"] = _gathered(torch.empty((case["batch"], hkv, int(L.max())), device="cuda"))
        state["keep"] = torch.full((case["batch"], hkv, case["budget"]), -1, dtype=torch.int32, device="cuda")
        return state
    elems = num_pages * 2 * hkv * PAGE * dim
    state["pools"] = _filled_pools(gen, case["layers"], elems, fp8)
    state["elems"] = elems
    if op == "compact":
        first, count = _counts(case)
        state.update(first=first.astype(np.int32), count=count.astype(np.int32), first_dev=torch.from_numpy(first).cuda(), count_dev=torch.from_numpy(count).cuda())
        if case["budget"]:  # every head's own choice, and the weights that go along with the tokens
            state["weights"] = _gathered(torch.empty((case["batch"], hkv, int(L.max())), device="cuda"))
            empty = torch.full((case["batch"], hkv, case["budget"]), -1, dtype=torch.int32, device="cuda")
            state["keep"] = _select(state["weights"], state["L_dev"], case["budget"], case["sinks"], case["recent"], empty)
        else:  # accepted nodes of every tree, the same in all heads and layers
            r = np.random.default_rng([case["shape"], seed])
            keep = np.full((case["batch"], int(count.max())), -1, np.int32)
            for i, c in enumerate(count):
                keep[i, :c] = L[i] + np.sort(r.permutation(int(n[i]))[:c])
            state["keep"], state["weights"] = torch.from_numpy(keep).cuda(), None
        return state
    rows = int(n.sum())
    at = np.cumsum(n) - n
    of = np.repeat(np.arange(case["batch"]), n)
    state.update(q=_normal(gen, rows, hq, dim), out=torch.zeros((rows, hq, dim), dtype=torch.bfloat16, device="cuda"), max_new=int(n.max()),
                 of=torch.from_numpy(of).cuda(), within=torch.from_numpy(np.arange(rows) - at[of]).cuda())
    if op == "tree":
        state["mask"] = torch.from_numpy(_trees(case, seed)).cuda()
    else:
        # as a few earlier rows left them: of the size of what this pass adds
        state["weights"] = _gathered(torch.empty((case["batch"], hkv, state["longest"]), device="cuda"), 1.0).mul_(int(n.max()) * hq / hkv / state["longest"])
    return state


def _views(pool, s):
    """K and V of a pool as [page, head, d / 8, token, d % 8] and [page, head, token / 8, d, token % 8]."""
    hkv, dim = s["hkv"], s["dim"]
    halves = pool.view(s["num_pages"], 2, hkv * PAGE * dim)
    return halves[:, 0].view(-1, hkv, dim // 8, PAGE, 8), halves[:, 1].view(-1, hkv, PAGE // 8, dim, 8)


def _values(x, fp8):
    """What gathered pool elements stand for (every FP8 code times a power of two is a bf16 number)."""
    return x.view(torch.float8_e4m3fn).to(torch.bfloat16) * FP8_SCALE if fp8 else x


def _dense(s):
    """K and V of every sequence in 32 bits, padded to the longest: [sequence, head, token, d]."""
    k, v = _views(s["pools"][0], s)
    ids = s["table"].clamp(min=0).long()
    k, v = _values(k[ids], s["fp8"]).float(), _values(v[ids], s["fp8"]).float()
    B, P = ids.shape
    k = k.permute(0, 2, 1, 4, 3, 5).reshape(B, s["hkv"], P * PAGE, s["dim"])
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, s["hkv"], P * PAGE, s["dim"])
    valid = torch.arange(P * PAGE, device="cuda") < (s["L_dev"] + s["n_dev"])[:, None]  # what lies behind was never written
    return k, v.masked_fill(~valid[:, None, :, None], 0.0)


def _attend(s, sees):
    """Attention of padded rows; `sees`: [sequence, row, token].  Results and probabilities, [sequence, KV head, group * row, .]."""
    k, v = _dense(s)
    B, N, group = k.shape[0], s["max_new"], s["hq"] // s["hkv"]
    q = torch.zeros((B, N, s["hq"], s["dim"]), device="cuda")
    q[s["of"], s["within"]] = s["q"].float()
    q = q.view(B, N, s["hkv"], group, s["dim"]).permute(0, 2, 3, 1, 4).reshape(B, s["hkv"], group * N, s["dim"])
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    scores = scores.view(B, s["hkv"], group, N, -1).masked_fill(~sees[:, None, None], -math.inf).view(B, s["hkv"], group * N, -1)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = torch.matmul(p, v).view(B, s["hkv"], group, N, s["dim"]).permute(0, 3, 1, 2, 4).reshape(B, N, s["hq"], s["dim"])
    return out[s["of"], s["within"]].to(torch.bfloat16), p


def _sees(s, tree):
    """What every padded row may look at: the cached tokens, and of the new ones its ancestors, or those up to itself."""
    P = s["table"].shape[1]
    t = torch.arange(P * PAGE, device="cuda")[None, None]
    L, n = s["L_dev"][:, None, None], s["n_dev"][:, None, None]
    j = torch.arange(s["max_new"], device="cuda")[None, :, None]
    if tree:
        words = torch.zeros((L.shape[0], s["max_new"], 1), dtype=torch.int64, device="cuda")
        words[s["of"], s["within"]] = s["mask"]
        mine = (words >> (t - L).clamp(0, 63)) & 1 == 1
        return (t < L) | ((t < L + n) & mine)
    return (t <= L + j) & (t < L + n) & (j < n)


def _select(weights, lengths, budget, sinks, recent, keep):
    """Positions of the first `sinks`, the last `recent` and the heaviest other tokens, `budget` in all, ascending."""
    t = torch.arange(weights.shape[-1], device="cuda")[None, None]
    n = lengths[:, None, None]
    kind = torch.where(t >= n, 2, torch.where((t < sinks) | (t >= n - recent), 0, 1)).expand(weights.shape)
    order = torch.sort(weights, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(kind.gather(-1, order), dim=-1, stable=True).indices)
    width = min(budget, weights.shape[-1])
    i = torch.arange(width, device="cuda")[None, None]
    count = n.clamp(max=budget)
    chosen = torch.where(i < count, order[..., :width], weights.shape[-1])
    chosen = torch.sort(chosen, dim=-1).values
    keep[..., :width] = torch.where(i < count, chosen.int(), keep[..., :width])
    return keep


def _compact(s):
    """Token keep[i] of every sequence and head goes to position first + i, in the pages of all layers, and its weight along."""
    keep = s["keep"].long()
    keep = (keep if keep.dim() == 3 else keep[:, None].expand(-1, s["hkv"], -1))[..., :int(s["count"].max())]
    i = torch.minimum(torch.arange(keep.shape[-1], device="cuda")[None], s["count_dev"][:, None] - 1)[:, None].expand(keep.shape)
    src = keep.gather(-1, i)
    dst = s["first_dev"][:, None, None] + i
    b = torch.arange(keep.shape[0], device="cuda")[:, None, None]
    h = torch.arange(s["hkv"], device="cuda")[None, :, None]
    from_page, to_page = s["table"][b, src // PAGE].long(), s["table"][b, dst // PAGE].long()
    pools = s["pools"]
    halves = pools.view(s["layers"], s["num_pages"], 2, -1)
    k = halves[:, :, 0].view(s["layers"], -1, s["hkv"], s["dim"] // 8, PAGE, 8)
    v = halves[:, :, 1].view(s["layers"], -1, s["hkv"], PAGE // 8, s["dim"], 8)
    new_k = k[:, from_page, h, :, src % PAGE]
    new_v = v[:, from_page, h, src % PAGE // 8, :, src % 8]
    k[:, to_page, h, :, dst % PAGE] = new_k
    v[:, to_page, h, dst % PAGE // 8, :, dst % 8] = new_v
    if s["weights"] is not None:
        s["weights"].scatter_(-1, dst, s["weights"].gather(-1, src))


def _outputs(s):
    op = s["op"]
    if op == "select":
        return s["keep"]
    if op == "compact":
        pools = s["pools"].view(torch.float8_e4m3fn) if s["fp8"] else s["pools"]
        return {"pools": pools, "weights": s["weights"]} if s["weights"] is not None else {"pools": pools}
    return {"out": s["out"]} if op == "tree" else {"out": s["out"], "weights": s["weights"]}


def run(s):
    op = s["op"]
    if own:
        ctx, stream = s["ctx"], s["stream"]
        if op == "tree":
            ctx.tree_attention(s["q"], s["pools"], s["table"], s["L"], s["n"], s["mask"], s["scale"], s["out"], stream=stream)
        elif op == "weighted":
            ctx.weighted_attention(s["q"], s["pools"], s["table"], s["L"], s["n"], s["scale"], s["out"], s["weights"], stream=stream)
        elif op == "select":
            ctx.kv_select(s["weights"], s["L"], s["budget"], s["sinks"], s["recent"], s["keep"], stream=stream)
        else:
            ctx.kv_compact(s["pools"], s["table"], s["keep"], s["first"], s["count"], layer_stride_elems=s["elems"], num_layers=s["layers"],
                           weights=s["weights"], stream=stream)
    elif op == "tree":
        s["out"], _ = _attend(s, _sees(s, True))
    elif op == "weighted":
        s["out"], p = _attend(s, _sees(s, False))
        B, width = p.shape[0], s["longest"]
        j = torch.arange(s["max_new"], device="cuda")[None] < s["n_dev"][:, None]
        got = (p.view(B, s["hkv"], -1, s["max_new"], p.shape[-1]) * j[:, None, None, :, None]).sum((2, 3))[..., :width]
        t = torch.arange(width, device="cuda")[None, None]
        old = s["weights"].masked_fill(t >= s["L_dev"][:, None, None], 0.0)
        s["weights"] = torch.where(t < (s["L_dev"] + s["n_dev"])[:, None, None], old + got, s["weights"])
    elif op == "select":
        _select(s["weights"], s["L_dev"], s["budget"], s["sinks"], s["recent"], s["keep"])
    else:
        _compact(s)
    return _outputs(s)


def work(case):
    L, n = (x.astype(np.float64) for x in _lengths(case))
    hq, hkv, dim, op = case["hq"], case["hkv"], case["dim"], case["op"]
    token = 2 * hkv * dim * (1 if case["pages"] == "fp8" else 2)
    if op == "select":
        return {"bytes": float((L + np.minimum(L, case["budget"])).sum()) * hkv * 4, "flops": 0.0}
    if op == "compact":
        first, count = _counts(case)
        listed = count.sum() * 4.0 * (hkv if case["budget"] else 1)
        moved = np.where(count < L if case["budget"] else count > 0, count - case["sinks"], 0).sum()
        return {"bytes": float(listed + moved * (2 * token * case["layers"] + (8 * hkv if case["budget"] else 0))), "flops": 0.0}
    nbytes = (L + n).sum() * token + n.sum() * hq * dim * 2 * 2
    # a drafted node sees the cache, itself and, on average over such trees, few others; a causal row those before it
    seen = (n * L + n).sum() if op == "tree" else (n * L + n * (n + 1) / 2).sum()
    nbytes += n.sum() * 8 if op == "tree" else (2 * L + n).sum() * hkv * 4
    return {"bytes": float(nbytes), "flops": float(4.0 * hq * dim * seen)}


def _token_offsets(case, table, b, h, positions, value):
    """Element offsets of [position, d] of one head in a pool, from the layout's index formulas."""
    hkv, dim = case["hkv"], case["dim"]
    t = torch.as_tensor(positions, device="cuda").long()[:, None]
    d = torch.arange(dim, device="cuda")[None]
    page, tok = torch.as_tensor(table[b], device="cuda").long()[t // PAGE], t % PAGE
    base = page * (2 * hkv * PAGE * dim) + h * PAGE * dim
    if value:
        return base + hkv * PAGE * dim + tok // 8 * (dim * 8) + d * 8 + tok % 8
    return base + d // 8 * (PAGE * 8) + tok * 8 + d % 8


def exact(case, seed):
    s = prepare(case, seed)
    L, n = _lengths(case)
    hkv, op, group = case["hkv"], case["op"], case["hq"] // case["hkv"]
    table = s["table"].cpu().numpy()
    if op == "select":
        w, keep = s["weights"].double().cpu().numpy(), s["keep"].cpu().numpy()
        for b in range(case["batch"]):
            t = np.arange(L[b])
            held = (t < case["sinks"]) | (t >= L[b] - case["recent"])
            for h in range(hkv):
                best = np.lexsort((t, -w[b, h, :L[b]], ~held))[:case["budget"]]
                keep[b, h, :len(best)] = np.sort(best)
        return torch.from_numpy(keep)
    if op == "compact":
        first, count = _counts(case)
        keep = s["keep"].cpu().numpy()
        before = s["pools"].clone()
        for b in range(case["batch"]):
            for h in range(hkv):
                src = keep[b, h] if keep.ndim == 3 else keep[b]
                src, dst = src[:count[b]], first[b] + np.arange(count[b])
                for value in (False, True):
                    s["pools"][:, _token_offsets(case, table, b, h, dst, value)] = before[:, _token_offsets(case, table, b, h, src, value)]
                if s["weights"] is not None:
                    s["weights"][b, h, :count[b]] = s["weights"][b, h][torch.from_numpy(src).long().cuda()]
        return _outputs(s)
    pool = s["pools"][0]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if op == "weighted" else None
    at = 0
    for b in range(case["batch"]):
        keys = int(L[b] + n[b])
        new = torch.arange(int(n[b]), device="cuda")
        seen = torch.ones((int(n[b]), keys), dtype=torch.bool, device="cuda")
        if op == "tree":
            seen[:, int(L[b]):] = (s["mask"][at:at + int(n[b])] >> new[None]) & 1 == 1
        else:
            seen[:, int(L[b]):] = new[None] <= new[:, None]
        for h in range(hkv):
            k, v = (pool[_token_offsets(case, table, b, h, np.arange(keys), value)] for value in (False, True))
            k, v = ((x.view(torch.float8_e4m3fn).double() * FP8_SCALE if s["fp8"] else x.double()) for x in (k, v))
            q = s["q"][at:at + int(n[b]), h * group:(h + 1) * group].double().reshape(-1, case["dim"])
            e = (q @ k.T) * s["scale"]
            e = torch.where(seen.repeat_interleave(group, 0), e, -math.inf)
            p = torch.softmax(e, -1)
            out[at:at + int(n[b]), h * group:(h + 1) * group] = (p @ v).view(int(n[b]), group, -1)
            if weights is not None:
                weights[b, h, int(L[b]):keys] = 0.0
                weights[b, h, :keys] += p.sum(0)
        at += int(n[b])
    return {"out": out} if weights is None else {"out": out, "weights": weights}
