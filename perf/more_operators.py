"""Operators of positions and of shared prefixes over the paged KV cache, and the cases they are measured on.

Three operators: the rotation of queries or keys by their positions and its transpose, which is its gradient (`rope`), the
append of a step's keys and values with the rotation applied on the way, queries rotated in the same pass (`append`), and
attention of a batch whose sequences share leading tokens, each shared range read once for all that have it (`prefix`).

`run` computes them in their plain form, or, where `own` is true, with the library's entry points.  Lengths, page tables,
what is shared and positions come from the case alone, values from the seed; queries, keys and values are N(0,1) as in the
repository's other workloads, pages a random permutation of the pool.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
FP8_SCALE = 2.0 ** -5  # K and V scale of the FP8 pages: N(0,1) values / scale stay far below 448


def _rotation(layout="half", part=1.0, base=10000.0, scaling="none", factor=1.0, original=8192.0, amplitude=1.0):
    return dict(layout=layout, part=part, base=base, scaling=scaling, factor=factor, original=original, amplitude=amplitude)


def _case(name, op, hq, hkv, dim, pages="bf16", rotation=None, batch=1, ctx=(0, 0), new=(1, 1), shape=0, packed=False, transpose=False,
          all_share=0, fan=0, document=(0, 0), alone=0):
    case = dict(op=op, hq=hq, hkv=hkv, dim=dim, pages=pages, batch=batch, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], shape=shape,
                packed=packed, transpose=transpose, all_share=all_share, fan=fan, doc_lo=document[0], doc_hi=document[1], alone=alone,
                **(rotation or _rotation()))
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: one token's queries of a small model
        _case("rope_one", "rope", 8, 2, 64, ctx=(37, 37), shape=1),
        # a decode batch's queries, far along in long contexts that frequencies were stretched for
        _case("rope_decode", "rope", 32, 8, 128, batch=64, ctx=(8000, 500000), shape=2,
              rotation=_rotation(base=500000.0, scaling="by_parts", factor=8.0, amplitude=1.2)),
        # the queries of a few long prompts, straight out of a packed projection
        _case("rope_prompts", "rope", 32, 8, 128, batch=5, new=(900, 3500), shape=3, packed=True, rotation=_rotation("interleaved")),
        # gradients of a training batch's queries, five query heads to a KV head, half of every head rotated
        _case("rope_gradient", "rope", 40, 8, 128, batch=9, new=(1000, 2500), shape=4, transpose=True, rotation=_rotation(part=0.5, scaling="linear", factor=4.0)),
        # one decoded token of a small model
        _case("append_one", "append", 8, 2, 64, ctx=(300, 300), shape=5),
        # a decode step of a loaded node
        _case("append_decode", "append", 32, 8, 128, batch=128, ctx=(100, 30000), shape=6, packed=True, rotation=_rotation(base=500000.0)),
        # first prompts of odd lengths
        _case("append_prompts", "append", 32, 8, 128, batch=7, new=(700, 2300), shape=7, packed=True, rotation=_rotation(scaling="base", factor=4.0)),
        # a step of decodes and next turns on quantised pages, a quarter of every head rotated pair by pair
        _case("append_mixed_fp8", "append", 64, 8, 128, pages="fp8", batch=40, ctx=(500, 9000), new=(1, 200), shape=8, rotation=_rotation("interleaved", part=0.25)),
        # three answers sampled from one short prompt of a small model
        _case("prefix_samples", "prefix", 8, 2, 64, batch=3, ctx=(5, 40), shape=9, all_share=200),
        # a decode batch behind one system prompt
        _case("prefix_decode", "prefix", 32, 8, 128, batch=64, ctx=(60, 700), shape=10, all_share=8000),
        # next turns of some users over the same documents, all behind a system prompt, a few requests of other kinds between them
        _case("prefix_turns", "prefix", 40, 8, 128, batch=18, ctx=(10, 900), new=(20, 150), shape=11, all_share=1500, fan=5, document=(2000, 9000), alone=2),
        # many decodes over long documents on quantised pages
        _case("prefix_documents_fp8", "prefix", 64, 8, 128, pages="fp8", batch=96, ctx=(50, 2000), shape=12, all_share=1000, fan=32, document=(12000, 24000)),
    ]


MOST_BYTES, MOST_FLOPS, MOST_SCORES, MOST_DENSE = 2.5e8, 7.0e10, 2.0e8, 2.4e6  # of a drawn case; dense: tokens of the plain form's padded K, times KV heads over 8


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "append", "prefix", "prefix"])
        hq, hkv, dim = rng.choice([(8, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (40, 8, 128), (32, 4, 128), (6, 6, 64)])
        scaling = rng.choice(["none", "linear", "base", "by_parts"])
        rotation = _rotation(rng.choice(["half", "interleaved"]), rng.choice([0.25, 0.3125, 0.5, 1.0, 1.0, 1.0]), rng.choice([10000.0, 500000.0]), scaling,
                             1.0 if scaling == "none" else rng.choice([2.0, 8.0]), 8192.0, rng.choice([1.0, 1.0, 1.1]))
        pages = rng.choice(["bf16", "bf16", "fp8"])
        batch, low = _log_int(rng, 1, 128), _log_int(rng, 1, 3000)
        ctx = (low, _log_int(rng, low, 8 * low))
        few = _log_int(rng, 1, 3000 if op != "prefix" else 200)
        new = (1, 1) if rng.random() < 0.5 else (few, _log_int(rng, few, 3 * few))
        packed, transpose = rng.random() < 0.5, op == "rope" and rng.random() < 0.5
        all_share, fan, document, alone = 0, 0, (0, 0), 0
        if op == "prefix":
            batch = max(2, batch)
            all_share = _log_int(rng, 16, 30000)
            if rng.random() < 0.4:
                fan, deep = _log_int(rng, 2, 32), _log_int(rng, 30, 20000)
                document = (deep, _log_int(rng, deep, 3 * deep))
            alone = rng.choice([0, 0, batch // 4])
        case = _case(None, op, hq, hkv, dim, pages, rotation, batch, ctx, new, rng.randrange(1 << 20), packed, transpose, all_share, fan, document, alone)
        w, (L, n, _) = work(case), _lengths(case)
        fits = w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS
        if op == "prefix":
            most = float((L + n).max())
            fits = fits and batch * hq * float(n.max()) * most <= MOST_SCORES and batch * most * hkv / 8 <= MOST_DENSE
        if fits:
            return case


def _lengths(case):
    """Cached and new tokens of every sequence, and the leading tokens that it has in common with the sequence before."""
    r = np.random.default_rng(case["shape"])

    def spread(lo, hi, size):
        return np.rint(np.exp(r.uniform(math.log(max(1, lo)), math.log(max(1, hi)), size))).astype(np.int64)
    B = case["batch"]
    L = spread(case["ctx_lo"], case["ctx_hi"], B) if case["ctx_hi"] else np.zeros(B, np.int64)
    n = spread(case["new_lo"], case["new_hi"], B)
    common = np.zeros(B, np.int64)
    if case["op"] == "prefix":
        together = B - case["alone"]  # the others come last and share nothing
        common[1:together] = case["all_share"]
        L[:together] += case["all_share"]
        if case["fan"]:
            document = np.arange(together) // case["fan"]
            tokens = spread(case["doc_lo"], case["doc_hi"], int(document[-1]) + 1)
            L[:together] += tokens[document]
            common[1:together] += np.where(document[1:] == document[:-1], tokens[document[1:]], 0)
    return L, n, common


def _page_tables(case):
    """Page ids of every sequence out of one permutation of a pool with some room; whole pages of common tokens are the same pages.
    An append has those that new tokens go into alone."""
    L, n, common = _lengths(case)
    r = np.random.default_rng(case["shape"] + 1)
    need = (L + n + PAGE - 1) // PAGE
    same = common // PAGE if case["op"] == "prefix" else L // PAGE
    num_pages = int((need - same).sum()) + 64
    perm = r.permutation(num_pages).astype(np.int32)
    table = np.full((len(need), int(need.max())), -1, np.int32)
    at = 0
    for i, c in enumerate(need):
        s = int(same[i])
        if case["op"] == "prefix" and i:
            table[i, :s] = table[i - 1, :s]
        table[i, s:c] = perm[at:at + int(c) - s]
        at += int(c) - s
    return table, num_pages


def _rotary_dim(case):
    return int(case["dim"] * case["part"])


def _frequencies(case):
    """Radians per position of every pair."""
    dim, factor = _rotary_dim(case), case["factor"]
    base = case["base"] * factor ** (dim / (dim - 2)) if case["scaling"] == "base" else case["base"]
    f = base ** (-np.arange(0, dim, 2, dtype=np.float64) / dim)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "by_parts":  # pairs that turn often within the original context keep their frequency, slow ones are stretched
        turns = case["original"] * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = keep * f + (1 - keep) * f / factor
    return f


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _filled_pool(gen, elems, fp8):
    """Resident K/V: N(0,1) values, or the FP8 codes of such values over the scale."""
    pool = torch.empty(elems, dtype=torch.uint8 if fp8 else torch.bfloat16, device="cuda")
    for a in range(0, elems, 1 << 28):
        part = pool[a:a + (1 << 28)]
        if fp8:
            x = torch.empty(part.shape, dtype=torch.float32, device="cuda").normal_(generator=gen)
            part.copy_((x / FP8_SCALE).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            part.normal_(generator=gen)
    return pool


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    fp8, op = case["pages"] == "fp8", case["op"]
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    L, n, common = _lengths(case)
    rows = int(n.sum())
    of = np.repeat(np.arange(case["batch"]), n)
    within = np.arange(rows) - (np.cumsum(n) - n)[of]
    position = L[of] + within
    state = dict(op=op, hq=hq, hkv=hkv, dim=dim, fp8=fp8, scale=1.0 / math.sqrt(dim), layout=case["layout"], rotary=_rotary_dim(case),
                 amplitude=case["amplitude"], transpose=case["transpose"], position=torch.from_numpy(position).cuda())
    if op != "prefix":
        state["frequency"] = torch.from_numpy(_frequencies(case)).cuda()
        if case["packed"]:  # rows of a projection that gives queries, keys and values side by side
            whole = _normal(gen, rows, hq + 2 * hkv, dim)
            q, k, v = whole[:, :hq], whole[:, hq:hq + hkv], whole[:, hq + hkv:]
        else:
            q = _normal(gen, rows, hq, dim)
            k, v = (_normal(gen, rows, hkv, dim) if op == "append" else None for _ in range(2))
    else:
        q, k, v = _normal(gen, rows, hq, dim), None, None
    state.update(q=q, k=k, v=v, out=torch.zeros((rows, hq, dim), dtype=torch.bfloat16, device="cuda"))
    table, num_pages = _page_tables(case) if op != "rope" else (None, 1)
    state["num_pages"] = num_pages
    if own:
        import paper_2603_13358_amd as ppd
        state["stream"] = torch.cuda.current_stream().cuda_stream
        state["ctx"] = ppd.Context(hq, hkv, dim, num_pages)
        if fp8:
            state["ctx"].set_kv_format(ppd.PPD_KV_FP8_E4M3, FP8_SCALE, FP8_SCALE)
        if op != "prefix":
            scaling = dict(none=ppd.PPD_ROPE_SCALE_NONE, linear=ppd.PPD_ROPE_SCALE_LINEAR, base=ppd.PPD_ROPE_SCALE_BASE, by_parts=ppd.PPD_ROPE_SCALE_BY_PARTS)
            frequency = ppd.ppd_rope_frequencies(state["rotary"], case["base"], scaling[case["scaling"]], case["factor"], case["original"], 1.0, 32.0)
            state["ctx"].set_rope(frequency, ppd.PPD_ROPE_HALF if case["layout"] == "half" else ppd.PPD_ROPE_INTERLEAVED, case["amplitude"])
    if op == "rope":
        return state
    state["pool"] = _filled_pool(gen, num_pages * 2 * hkv * PAGE * dim, fp8)
    if op == "append":
        state["slots"] = torch.from_numpy(table[of, position // PAGE].astype(np.int64) * PAGE + position % PAGE).cuda()
        return state
    state.update(table=torch.from_numpy(table).cuda(), shared=(common // PAGE * PAGE).astype(np.int32), L=L.astype(np.int32), n=n.astype(np.int32),
                 L_dev=torch.from_numpy(L).cuda(), n_dev=torch.from_numpy(n).cuda(), max_new=int(n.max()), of=torch.from_numpy(of).cuda(),
                 within=torch.from_numpy(within).cuda())
    return state


def _rotated(s, x):
    """x [row, head, d] rotated by its row's position, in 32 bits."""
    angle = s["position"].double()[:, None] * s["frequency"][None]
    cos, sin = (s["amplitude"] * t.float()[:, None] for t in (torch.cos(angle), torch.sin(angle)))
    sin = -sin if s["transpose"] else sin
    r = s["rotary"]
    x = x.float()
    y = x.clone()
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if s["layout"] == "half" else (x[..., :r:2], x[..., 1:r:2])
    first, second = a * cos - b * sin, b * cos + a * sin
    if s["layout"] == "half":
        y[..., :r // 2], y[..., r // 2:r] = first, second
    else:
        y[..., :r:2], y[..., 1:r:2] = first, second
    return y


def _views(pool, s):
    """K and V of a pool as [page, head, d / 8, token, d % 8] and [page, head, token / 8, d, token % 8]."""
    hkv, dim = s["hkv"], s["dim"]
    halves = pool.view(s["num_pages"], 2, hkv * PAGE * dim)
    return halves[:, 0].view(-1, hkv, dim // 8, PAGE, 8), halves[:, 1].view(-1, hkv, PAGE // 8, dim, 8)


def _stored(x, s):
    """What pages hold of 32-bit values."""
    if not s["fp8"]:
        return x.to(torch.bfloat16)
    return (x * (1.0 / FP8_SCALE)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _append(s):
    k, v = _views(s["pool"], s)
    page, tok = s["slots"] // PAGE, s["slots"] % PAGE
    rows = len(s["slots"])
    k[page, :, :, tok] = _stored(_rotated(s, s["k"]), s).view(rows, s["hkv"], s["dim"] // 8, 8)
    v[page, :, tok // 8, :, tok % 8] = _stored(s["v"].float(), s)
    s["out"] = _rotated(s, s["q"]).to(torch.bfloat16)


def _dense(s):
    """K and V of every sequence in 32 bits, padded to the longest: [sequence, head, token, d]."""
    k, v = _views(s["pool"], s)
    ids = s["table"].clamp(min=0).long()
    k, v = ((x[ids].view(torch.float8_e4m3fn).float() * FP8_SCALE if s["fp8"] else x[ids].float()) for x in (k, v))
    B, P = ids.shape
    k = k.permute(0, 2, 1, 4, 3, 5).reshape(B, s["hkv"], P * PAGE, s["dim"])
    v = v.permute(0, 2, 1, 3, 5, 4).reshape(B, s["hkv"], P * PAGE, s["dim"])
    return k, v


def _attend(s):
    k, v = _dense(s)
    B, N, group = k.shape[0], s["max_new"], s["hq"] // s["hkv"]
    q = torch.zeros((B, N, s["hq"], s["dim"]), device="cuda")
    q[s["of"], s["within"]] = s["q"].float()
    q = q.view(B, N, s["hkv"], group, s["dim"]).permute(0, 2, 3, 1, 4).reshape(B, s["hkv"], group * N, s["dim"])
    t = torch.arange(k.shape[2], device="cuda")[None, None]
    j = torch.arange(N, device="cuda")[None, :, None]
    sees = t <= s["L_dev"][:, None, None] + j
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    scores = scores.view(B, s["hkv"], group, N, -1).masked_fill(~sees[:, None, None], -math.inf).view(B, s["hkv"], group * N, -1)
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    out = torch.matmul(p / p.sum(-1, keepdim=True), v)
    out = out.view(B, s["hkv"], group, N, s["dim"]).permute(0, 3, 1, 2, 4).reshape(B, N, s["hq"], s["dim"])
    s["out"] = out[s["of"], s["within"]].to(torch.bfloat16)


def _outputs(s):
    if s["op"] == "append":
        return {"q": s["out"], "pool": s["pool"].view(torch.float8_e4m3fn) if s["fp8"] else s["pool"]}
    return {"out": s["out"]}


def run(s):
    op = s["op"]
    if own:
        ctx, stream = s["ctx"], s["stream"]
        if op == "rope":
            ctx.rope(s["q"], s["position"], s["out"], transpose=s["transpose"], stream=stream)
        elif op == "append":
            ctx.kv_append_rotated(s["q"], s["k"], s["v"], s["position"], s["pool"], s["slots"], s["out"], stream=stream)
        else:
            ctx.prefix_attention(s["q"], s["pool"], s["table"], s["shared"], s["L"], s["n"], s["scale"], s["out"], stream=stream)
    elif op == "rope":
        s["out"] = _rotated(s, s["q"]).to(torch.bfloat16)
    elif op == "append":
        _append(s)
    else:
        _attend(s)
    return _outputs(s)


def work(case):
    L, n, common = (x.astype(np.float64) for x in _lengths(case))
    hq, hkv, dim, op, rows = case["hq"], case["hkv"], case["dim"], case["op"], n.sum()
    token = 2 * hkv * dim * (1 if case["pages"] == "fp8" else 2)
    pairs = 6.0 * _rotary_dim(case) / 2  # of one head
    if op == "rope":
        return {"bytes": float(rows * (hq * dim * 4 + 8)), "flops": float(rows * hq * pairs)}
    if op == "append":
        return {"bytes": float(rows * (hq * dim * 4 + 2 * hkv * dim * 2 + token + 16)), "flops": float(rows * (hq + hkv) * pairs)}
    nbytes = (L + n - common // PAGE * PAGE).sum() * token + rows * hq * dim * 2 * 2
    return {"bytes": float(nbytes), "flops": float(4.0 * hq * dim * (n * L + n * (n + 1) / 2).sum())}


def _token_offsets(case, pages, h, positions, value):
    """Element offsets of [position, d] of one head in a pool, from the layout's index formulas."""
    hkv, dim = case["hkv"], case["dim"]
    t = torch.as_tensor(positions, device="cuda").long()[:, None]
    d = torch.arange(dim, device="cuda")[None]
    page, tok = torch.as_tensor(pages, device="cuda").long()[t // PAGE], t % PAGE
    base = page * (2 * hkv * PAGE * dim) + h * PAGE * dim
    if value:
        return base + hkv * PAGE * dim + tok // 8 * (dim * 8) + d * 8 + tok % 8
    return base + d // 8 * (PAGE * 8) + tok * 8 + d % 8


def _turned(case, s, x):
    """x [row, head, d] times unit complex numbers, pair by pair, in 64 bits."""
    r = _rotary_dim(case)
    where = np.arange(r).reshape(2, r // 2) if case["layout"] == "half" else np.arange(r).reshape(r // 2, 2).T
    where = torch.from_numpy(where.copy()).cuda()
    turn = torch.polar(torch.full((1,), case["amplitude"], dtype=torch.float64, device="cuda"),
                       (-1.0 if case["transpose"] else 1.0) * s["position"].double()[:, None] * torch.from_numpy(_frequencies(case)).cuda())
    y = x.double()
    z = torch.complex(y[..., where[0]], y[..., where[1]]) * turn[:, None]
    y = y.clone()
    y[..., where[0]], y[..., where[1]] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    op, hkv, group = case["op"], case["hkv"], case["hq"] // case["hkv"]
    if op == "rope":
        return {"out": _turned(case, s, s["q"])}
    table, _ = _page_tables(case)
    L, n, _ = _lengths(case)
    scale = FP8_SCALE if s["fp8"] else 1.0
    pool = s["pool"].view(torch.float8_e4m3fn).double() if s["fp8"] else s["pool"].double()
    at = 0
    if op == "append":
        k, v = _turned(case, s, s["k"]) / scale, s["v"].double() / scale
        for b in range(case["batch"]):
            tokens = np.arange(L[b], L[b] + n[b])
            for h in range(hkv):
                pool[_token_offsets(case, table[b], h, tokens, False)] = k[at:at + int(n[b]), h]
                pool[_token_offsets(case, table[b], h, tokens, True)] = v[at:at + int(n[b]), h]
            at += int(n[b])
        return {"q": _turned(case, s, s["q"]), "pool": pool}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        keys, rows = int(L[b] + n[b]), int(n[b])
        seen = torch.arange(keys, device="cuda")[None] <= int(L[b]) + torch.arange(rows, device="cuda")[:, None]
        for h in range(hkv):
            k, v = (pool[_token_offsets(case, table[b], h, np.arange(keys), value)] * scale for value in (False, True))
            q = s["q"][at:at + rows, h * group:(h + 1) * group].double().reshape(-1, case["dim"])
            e = torch.where(seen.repeat_interleave(group, 0), (q @ k.T) * s["scale"], -math.inf)
            out[at:at + rows, h * group:(h + 1) * group] = (torch.softmax(e, -1) @ v).view(rows, group, -1)
        at += rows
    return {"out": out}
