"""The serving-side operators beside the attention forward pass, as measured cases.

Four operators, the steps of one pass of a server (or, the third, of a trainer) around an attention kernel:

  plan     block tables, slot maps and positions of a step, built on the GPU from the requests' lengths and a pool of free pages
  rope     RMS norm of every query and key head, the position rotation, and the append of keys and values to a paged cache
  rope_bwd the gradients of that norm and rotation
  decode   attention of one new token per request over the paged cache

`own` chooses the side: the operators written out in elementary torch operations (False), or the package's kernels (True).
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # One step of a server that only decodes: every request grows by a token, a few of them onto a new page.
        dict(name="plan-decode-64", op="plan", requests=64, page=16, longest=8192, prefilling=0, chunk=0, leaving=0),
        # A step that decodes for some requests, takes in pieces of new prompts and gives back the pages of finished requests.
        dict(name="plan-mixed-256", op="plan", requests=256, page=16, longest=8192, prefilling=16, chunk=1024, leaving=12),
        # The new tokens of a decode step, in 16-token pages.
        dict(name="rope-decode-64", op="rope", tokens=64, heads=32, kv_heads=8, d=128, type="bf16", rot=128, interleaved=False,
             page=16, heads_first=False, dense_k=False, far=131072),
        # A prefill of 8192 tokens: queries and keys go on to the attention kernel, keys and values to the cache as well.
        dict(name="rope-prefill-8192", op="rope", tokens=8192, heads=32, kv_heads=8, d=128, type="bf16", rot=128, interleaved=False,
             page=16, heads_first=False, dense_k=True, far=65536),
        # Head dimension 64, as many key heads as query heads, half of each head rotated in adjacent pairs, an odd number of tokens.
        dict(name="rope-partial-4001", op="rope", tokens=4001, heads=16, kv_heads=16, d=64, type="f16", rot=32, interleaved=True,
             page=64, heads_first=True, dense_k=False, far=8192),
        # A training step's gradients: 8192 tokens, grouped heads.
        dict(name="rope-bwd-8192", op="rope_bwd", tokens=8192, heads=32, kv_heads=8, d=128, type="bf16", rot=128, interleaved=False, far=8192),
        # The same at head dimension 64 with an odd, small number of tokens.
        dict(name="rope-bwd-1001", op="rope_bwd", tokens=1001, heads=16, kv_heads=16, d=64, type="f16", rot=64, interleaved=True, far=4096),
        # One user, a short conversation: latency.
        dict(name="decode-1x1000", op="decode", requests=1, longest=1000, even=True, heads=32, kv_heads=8, d=128, type="bf16",
             page=16, heads_first=False),
        # One user, a very long context: the length has to be split over the GPU.
        dict(name="decode-1x131072", op="decode", requests=1, longest=131072, even=True, heads=32, kv_heads=8, d=128, type="bf16",
             page=16, heads_first=False),
        # A busy server: 64 requests of very different lengths, some of them empty places of a padded batch.
        dict(name="decode-64x8192", op="decode", requests=64, longest=8192, even=False, heads=32, kv_heads=8, d=128, type="bf16",
             page=16, heads_first=False),
        # Many short requests, one key head for all query heads.
        dict(name="decode-200x700-mqa", op="decode", requests=200, longest=700, even=False, heads=32, kv_heads=1, d=128, type="f16",
             page=32, heads_first=False),
        # The largest: 8 requests of 131072 tokens, every query head with keys of its own, heads outside tokens within a page.
        dict(name="decode-8x131072-mha", op="decode", requests=8, longest=131072, even=True, heads=16, kv_heads=16, d=64, type="f16",
             page=64, heads_first=True),
    ]


HEADS = [(1, 1), (5, 1), (7, 7), (8, 8), (12, 4), (16, 4), (16, 16), (24, 8), (32, 1), (32, 4), (32, 8), (40, 8), (32, 32)]


def draw(rng):
    def spread(low, high):
        """A whole number between low and high, even over its logarithm."""
        return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))

    op = rng.choice(["plan", "rope", "rope_bwd", "decode", "decode"])
    if op == "plan":
        requests = spread(1, 1024)
        prefilling = rng.randint(0, max(1, requests // 8))
        leaving = rng.randint(0, (requests - prefilling) // 4)
        chunk = spread(1, max(1, min(4096, 16384 // max(1, prefilling))))
        return dict(op=op, requests=requests, page=rng.choice([1, 8, 16, 24, 32, 64, 128]), longest=spread(1, 8192), prefilling=prefilling,
                    chunk=chunk, leaving=leaving)
    heads, kv_heads = rng.choice(HEADS)
    d, kind = rng.choice([64, 128]), rng.choice(["bf16", "f16"])
    if op == "decode":
        page = rng.choice([1, 8, 16, 24, 32, 64, 128])
        longest = spread(1, 131072)
        # 4 GiB of keys and values at most, and of pages as small as a token no more than 2^20 table entries
        most = min((1 << 32) // (longest * kv_heads * d * 4), (1 << 20) // max(1, longest // page))
        requests = spread(1, max(1, min(256, most)))
        return dict(op=op, requests=requests, longest=longest, even=rng.random() < 0.3, heads=heads, kv_heads=kv_heads, d=d, type=kind, page=page,
                    heads_first=rng.random() < 0.5)
    tokens = spread(1, 8192)
    rot = rng.choice([d, d, d // 2])
    case = dict(op=op, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, type=kind, rot=rot, interleaved=rng.random() < 0.5, far=spread(128, 1 << 20))
    if op == "rope":
        case.update(page=rng.choice([1, 8, 16, 24, 32, 64, 128]), heads_first=rng.random() < 0.5, dense_k=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------------------------------------------------------ inputs
def _generators(seed):
    gpu = torch.Generator(device=DEVICE)
    gpu.manual_seed(seed)
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    return gpu, cpu


def _cache(pages, case, gpu):
    """K and V of a paged cache: [page, token, head, d], or [page, head, token, d] with heads outside tokens."""
    inner = (case["kv_heads"], case["page"]) if case["heads_first"] else (case["page"], case["kv_heads"])
    kind = TYPES[case["type"]]
    return [torch.randn((pages, *inner, case["d"]), generator=gpu, device=DEVICE, dtype=kind) for _ in range(2)]


def prepare(case, seed):
    gpu, cpu = _generators(seed)
    state = dict(case)
    if case["op"] == "plan":
        n, page, longest, chunk = case["requests"], case["page"], case["longest"], case["chunk"]
        cached = torch.randint(0, longest + 1, (n,), generator=cpu)
        cached[0] = longest
        added = torch.ones(n, dtype=torch.int64)
        order = torch.randperm(n, generator=cpu)
        some = order[: case["prefilling"]]
        added[some] = torch.randint(1, max(1, chunk) + 1, (some.numel(),), generator=cpu)
        added[order[case["prefilling"]: case["prefilling"] + case["leaving"]]] = -1
        width = -(-(longest + max(1, chunk)) // page)
        held = (cached + page - 1) // page
        pages = n * width + 7
        names = torch.randperm(pages, generator=gpu, device=DEVICE).to(torch.int32)
        column = torch.arange(width, device=DEVICE)[None]
        first = (held.cumsum(0) - held).to(DEVICE)[:, None]
        mine = column < held.to(DEVICE)[:, None]
        table = torch.where(mine, names[(first + column).clamp_max(pages - 1)], torch.full_like(names[:1], -1))
        taken = int(held.sum())
        free = torch.full((pages,), -1, dtype=torch.int32, device=DEVICE)
        free[: pages - taken] = names[taken:]
        state.update(cached=cached.to(DEVICE, torch.int32), added=added.to(DEVICE, torch.int32), table=table.contiguous(), free=free,
                     count=torch.tensor([pages - taken], dtype=torch.int32, device=DEVICE),
                     count_after=torch.empty(1, dtype=torch.int32, device=DEVICE),
                     room=n - case["prefilling"] - case["leaving"] + case["prefilling"] * max(1, chunk))
        return state
    kind = TYPES[case["type"]]
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "decode":
        n, page, longest = case["requests"], case["page"], case["longest"]
        lengths = torch.full((n,), longest) if case["even"] else torch.randint(1, longest + 1, (n,), generator=cpu)
        lengths[0] = longest
        if not case["even"] and n >= 8:
            lengths[-(n // 16 + 1):] = 0      # empty places of a padded batch
        width = -(-longest // page)
        held = (lengths + page - 1) // page
        pages = int(held.sum()) + 3
        names = torch.randperm(pages, generator=gpu, device=DEVICE).to(torch.int32)
        column = torch.arange(width, device=DEVICE)[None]
        first = (held.cumsum(0) - held).to(DEVICE)[:, None]
        table = torch.where(column < held.to(DEVICE)[:, None], names[(first + column).clamp_max(pages - 1)], torch.full_like(names[:1], -1))
        k, v = _cache(pages, case, gpu)
        q = torch.randn((n, heads, d), generator=gpu, device=DEVICE, dtype=kind)
        state.update(q=q, k=k, v=v, table=table.contiguous(), lengths=lengths.to(DEVICE, torch.int32), scale=1.0 / math.sqrt(d),
                     workspace=torch.zeros(32 << 20, dtype=torch.uint8, device=DEVICE))
        return state
    tokens, rot, far = case["tokens"], case["rot"], case["far"]
    # The projection leaves queries, keys and values of a token side by side.
    qkv = torch.randn((tokens, heads + 2 * kv_heads, d), generator=gpu, device=DEVICE, dtype=kind)
    state.update(q=qkv[:, :heads], k=qkv[:, heads: heads + kv_heads], v=qkv[:, heads + kv_heads:],
                 q_weight=(1 + 0.1 * torch.randn(d, generator=gpu, device=DEVICE)).to(kind),
                 k_weight=(1 + 0.1 * torch.randn(d, generator=gpu, device=DEVICE)).to(kind),
                 position=torch.randint(0, far, (tokens,), generator=gpu, device=DEVICE, dtype=torch.int32),
                 inv_freq=(1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(DEVICE))
    if case["op"] == "rope":
        pages = -(-tokens // case["page"]) + 3
        state["k_cache"], state["v_cache"] = _cache(pages, case, gpu)
        # Each token has a slot of its own; a request's tokens lie in pages here and there.
        where = torch.randperm(pages, generator=gpu, device=DEVICE)
        token = torch.arange(tokens, device=DEVICE)
        state["slot"] = where[token // case["page"]] * case["page"] + token % case["page"]
        state["k_out"] = torch.empty((tokens, kv_heads, d), dtype=kind, device=DEVICE) if case["dense_k"] else None
    else:
        state["dq_out"] = torch.randn((tokens, heads, d), generator=gpu, device=DEVICE, dtype=kind)
        state["dk_out"] = torch.randn((tokens, kv_heads, d), generator=gpu, device=DEVICE, dtype=kind)
        state["workspace"] = torch.zeros(4 << 20, dtype=torch.uint8, device=DEVICE)
    return state


# ------------------------------------------------------------------------------------------------------------------ one pass
def run(state):
    return {"plan": _plan, "rope": _rope, "rope_bwd": _rope_bwd, "decode": _decode}[state["op"]](state)


def _plan(s):
    if own:
        import paper_2601_16032_b200 as sa
        p = sa.page_plan(s["cached"], s["added"], s["page"], s["table"], s["free"], s["count"], s["room"], free_count_out=s["count_after"])
        return [s["table"], s["free"], p.free_count, p.seq_len, p.q_start, p.slot, p.position, p.request, p.info]
    page, table, free, room = s["page"], s["table"], s["free"], s["room"]
    cached, added, count = s["cached"].long(), s["added"].long(), s["count"].long()
    width, device = table.shape[1], table.device
    leaves = added < 0
    held = (cached + page - 1) // page
    length = torch.where(leaves, 0, cached + added)
    needed = (length + page - 1) // page
    taken = torch.where(leaves, 0, needed - held)
    given = torch.where(leaves, held, 0)
    taken_to, given_to = taken.cumsum(0), given.cumsum(0)
    # The stack of free pages with the returned ones on top, in the order of requests and of their tables.
    place = torch.arange(free.shape[0], device=device)
    back = (place - count).clamp_min(0)
    giver = torch.searchsorted(given_to, back, right=True).clamp_max(cached.shape[0] - 1)
    entry = (back - (given_to - given)[giver]).clamp(0, width - 1)
    stack = torch.where(place < count, free, table[giver, entry])
    top = count + given_to[-1]
    count_after = top - taken_to[-1]
    free = torch.where((place >= count) & (place < count_after), stack, free)
    column = torch.arange(width, device=device)[None]
    fresh = (column >= held[:, None]) & (column < needed[:, None])
    at = top - 1 - ((taken_to - taken)[:, None] + column - held[:, None])
    table = torch.where(fresh, stack[at.clamp(0, free.shape[0] - 1)], table)
    tokens = torch.where(leaves, 0, added)
    end = tokens.cumsum(0)
    start = torch.cat([torch.zeros_like(end[:1]), end])
    token = torch.arange(room, device=device)
    used = token < end[-1]
    owner = torch.searchsorted(end, token, right=True).clamp_max(cached.shape[0] - 1)
    position = cached[owner] + token - start[owner]
    slot = table[owner, (position // page).clamp(0, width - 1)].long() * page + position % page
    info = torch.stack([torch.zeros_like(end[-1]), end[-1], taken_to[-1], given_to[-1]])
    whole = torch.int32
    return [table, free, count_after.to(whole), length.to(whole), start.to(whole), torch.where(used, slot, -1),
            torch.where(used, position, 0).to(whole), torch.where(used, owner, -1).to(whole), info.to(whole)]


def _turn(s):
    """cos and sin of every token's angles, from 64-bit angles: [tokens, 1, rot / 2]."""
    angle = s["position"].double()[:, None, None] * s["inv_freq"]
    return angle.cos().float(), angle.sin().float()


def _pairs(x, s):
    """The two halves of each rotated pair of the last dimension."""
    part = x[..., : s["rot"]]
    if s["interleaved"]:
        return part[..., 0::2], part[..., 1::2]
    return part[..., : s["rot"] // 2], part[..., s["rot"] // 2:]


def _unpair(a, b, x, s):
    """Puts rotated pairs back in front of the dimensions of x that do not turn."""
    both = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([both, x[..., s["rot"]:]], -1)


def _norm_turn(x, weight, s):
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    cos, sin = _turn(s)
    a, b = _pairs(x, s)
    return _unpair(a * cos - b * sin, b * cos + a * sin, x, s)


def _norm_turn_gradient(dy, x, weight, s):
    dy, x, weight = dy.float(), x.float(), weight.float()
    cos, sin = _turn(s)
    a, b = _pairs(dy, s)
    dn = _unpair(a * cos + b * sin, b * cos - a * sin, dy, s)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    g = dn * weight
    return r * (g - x * r.square() * (g * x).mean(-1, keepdim=True)), (dn * x * r).double().sum((0, 1)).float()


def _store(cache, rows, s):
    page, slot = s["page"], s["slot"]
    if s["heads_first"]:
        cache[slot // page, :, slot % page] = rows
    else:
        cache[slot // page, slot % page] = rows


def _rope(s):
    if own:
        import paper_2601_16032_b200 as sa
        q_out, k_out = sa.qk_norm_rope(s["q"], s["k"], s["v"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, position=s["position"],
                                       inv_freq=s["inv_freq"], interleaved=s["interleaved"], k_cache=s["k_cache"], v_cache=s["v_cache"],
                                       cache_layout=sa.LAYOUT_BHND if s["heads_first"] else sa.LAYOUT_BNHD, slot=s["slot"], k_out=s["k_out"])
    else:
        kind = s["q"].dtype
        q_out = _norm_turn(s["q"], s["q_weight"], s).to(kind)
        k_new = _norm_turn(s["k"], s["k_weight"], s).to(kind)
        _store(s["k_cache"], k_new, s)
        _store(s["v_cache"], s["v"], s)
        k_out = k_new if s["dense_k"] else None
    return [q_out, s["k_cache"], s["v_cache"]] + ([k_out] if s["dense_k"] else [])


def _rope_bwd(s):
    if own:
        import paper_2601_16032_b200 as sa
        return list(sa.qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                             position=s["position"], inv_freq=s["inv_freq"], interleaved=s["interleaved"], workspace=s["workspace"]))
    kind = s["q"].dtype
    dq, dq_weight = _norm_turn_gradient(s["dq_out"], s["q"], s["q_weight"], s)
    dk, dk_weight = _norm_turn_gradient(s["dk_out"], s["k"], s["k_weight"], s)
    return [dq.to(kind), dk.to(kind), dq_weight, dk_weight]


def _decode(s):
    if own:
        import paper_2601_16032_b200 as sa
        return list(sa.decode_paged(s["q"], s["k"], s["v"], s["table"], s["lengths"], scale=s["scale"],
                                    cache_layout=sa.LAYOUT_BHND if s["heads_first"] else sa.LAYOUT_BNHD, return_lse=True, workspace=s["workspace"]))
    q, table, lengths = s["q"], s["table"].long().clamp_min(0), s["lengths"].long()
    n, heads, d = q.shape
    group = heads // s["kv_heads"]

    def gather(cache):                                             # [requests, kv_heads, tokens, d]
        pages = cache[table]
        pages = pages.permute(0, 2, 1, 3, 4) if s["heads_first"] else pages.permute(0, 3, 1, 2, 4)
        return pages.flatten(2, 3).float()

    score = torch.matmul(q.float().view(n, s["kv_heads"], group, d), gather(s["k"]).transpose(2, 3)) * s["scale"]
    hidden = torch.arange(score.shape[-1], device=q.device) >= lengths[:, None, None, None]
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(-1, keepdim=True).clamp_min(-1e30)            # an empty request has no largest score
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, gather(s["v"]).masked_fill(hidden.transpose(2, 3), 0)) / total.clamp_min(1e-30)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    return [out.view(n, heads, d).to(q.dtype), lse.view(n, heads)]


# ------------------------------------------------------------------------------------------------------------------ what a pass costs at least
def work(case):
    if case["op"] == "plan":
        n, room = case["requests"], case["requests"] - case["prefilling"] - case["leaving"] + case["prefilling"] * max(1, case["chunk"])
        pages = room / case["page"] + case["leaving"] * case["longest"] / 2 / case["page"]
        return {"bytes": 20 * n + 16 * room + 8 * pages, "flops": 0}
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "decode":
        n, longest = case["requests"], case["longest"]
        tokens = n * longest
        if not case["even"]:
            filled = n - (n // 16 + 1 if n >= 8 else 0)
            tokens = longest + (filled - 1) * (longest + 1) / 2
        return {"bytes": tokens * (4 * kv_heads * d + 4 / case["page"]) + n * heads * (4 * d + 4), "flops": 4 * tokens * heads * d}
    tokens = case["tokens"]
    both = (heads + kv_heads) * d
    if case["op"] == "rope":
        return {"bytes": tokens * (4 * both + 4 * kv_heads * d + (2 * kv_heads * d if case["dense_k"] else 0) + 12), "flops": 10 * tokens * both}
    return {"bytes": tokens * (6 * both + 4) + 12 * d, "flops": 20 * tokens * both}


# ------------------------------------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_rows(x, weight, case, position, inv_freq, back=None):
    """Norm and rotation of [tokens, heads, d] rows; with `back`, gradients with respect to x and weight. One pair of dimensions after the other."""
    x, weight = x.double(), weight.double()
    d, rot = case["d"], case["rot"]
    size = (x.pow(2).sum(-1) / d + EPS).sqrt()
    unit = x / size[..., None]
    y = unit * weight if back is None else back.double().clone()
    for i in range(rot // 2):
        m, n = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
        turn = torch.polar(torch.ones_like(position, dtype=torch.float64), position.double() * inv_freq[i])[:, None]
        z = torch.complex(y[..., m].clone(), y[..., n].clone()) * (turn if back is None else turn.conj())
        y[..., m], y[..., n] = z.real, z.imag
    if back is None:
        return y
    scaled = y * weight
    along = (scaled * unit).sum(-1, keepdim=True) / d
    return (scaled - unit * along) / size[..., None], (y * unit).sum((0, 1))


def exact(case, seed):
    if case["op"] == "plan":
        return None        # whole numbers
    s = prepare(case, seed)
    if case["op"] == "rope":
        q = _exact_rows(s["q"], s["q_weight"], case, s["position"], s["inv_freq"])
        k = _exact_rows(s["k"], s["k_weight"], case, s["position"], s["inv_freq"])
        caches = []
        for cache, rows in ((s["k_cache"].double(), k), (s["v_cache"].double(), s["v"].double())):
            by_token = cache.transpose(1, 2) if case["heads_first"] else cache
            by_token[s["slot"] // case["page"], s["slot"] % case["page"]] = rows
            caches.append(cache)
        return [q, *caches] + ([k] if case["dense_k"] else [])
    if case["op"] == "rope_bwd":
        dq, dq_weight = _exact_rows(s["q"], s["q_weight"], case, s["position"], s["inv_freq"], s["dq_out"])
        dk, dk_weight = _exact_rows(s["k"], s["k_weight"], case, s["position"], s["inv_freq"], s["dk_out"])
        return [dq, dk, dq_weight, dk_weight]
    n, heads, d = s["q"].shape
    group = heads // case["kv_heads"]
    out = torch.zeros((n, heads, d), dtype=torch.float64, device=DEVICE)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device=DEVICE)
    for b, length in enumerate(s["lengths"].tolist()):
        if length == 0:
            continue
        mine = s["table"][b, : -(-length // case["page"])].long()
        k, v = s["k"][mine], s["v"][mine]
        if case["heads_first"]:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        k, v = (x.reshape(-1, case["kv_heads"], d)[:length].double() for x in (k, v))
        for h in range(case["kv_heads"]):
            score = s["q"][b, h * group: (h + 1) * group].double() @ k[:, h].T * s["scale"]
            total = score.logsumexp(-1)
            lse[b, h * group: (h + 1) * group] = total
            out[b, h * group: (h + 1) * group] = (score - total[:, None]).exp() @ v[:, h]
    return [out, lse]
