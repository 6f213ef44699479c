"""Drafted tokens and a bounded memory over the paged cache, as cases that a program can time and check.

A backbone that writes text or plan tokens over a long memory of frames drafts several tokens at a time as a tree, checks
them in one pass and keeps those that it agrees with; and it keeps its memory within a budget by dropping the tokens that
its attention hardly looks at.  Each case is one call as its program makes it:

* ``tree``: which drafted tokens see which, and their positions, from the parent of each.
* ``verify``: the drafted tokens' attention over the cached tokens and their own ancestors.
* ``accept``: the accepted tokens' keys and values moved to where the next tokens follow.
* ``weigh``: the attention of new tokens, which also adds up the weight that every key got.
* ``evict``: long sequences cut to a budget by these weights, the kept tokens moved together.

Sequence b of a batch has ``length_b`` tokens in the cache, the last ``new_b`` of them new (or drafted): rows
cu[b] .. cu[b + 1] of the packed inputs.  Both are fixed by the case; what fills them is drawn from the seed.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
_SIZE = {"f32": 4, "bf16": 2, "fp8": 1, "int8": 1}
_GOLDEN = 0.6180339887498949


def _case(name, op, seqs, new, length, new_spread=0.0, length_spread=0.0, page=16, **more):
    return dict(name=name, op=op, seqs=seqs, new=new, new_spread=new_spread, length=length, length_spread=length_spread,
                page=page, **more)


def _pages(kv_heads, head_dim, dtype, store):
    return dict(kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, store=store)


def listed():
    pi0, wide = _pages(1, 256, "bf16", "bf16"), _pages(8, 128, "bf16", "bf16")
    return [
        # one robot's drafted tokens: the smallest call, all latency
        _case("tree_robot", "tree", 1, 16, 833),
        # a fleet of 64 with large ragged trees
        _case("tree_fleet64", "tree", 64, 256, 15409, new_spread=0.7, length_spread=0.8),
        # one robot checks 16 drafted tokens over its prompt and one frame
        _case("verify_robot", "verify", 1, 16, 833, q_heads=8, **pi0),
        # a fleet of 32 checks ragged trees over long memories in fp8
        _case("verify_fleet32_fp8", "verify", 32, 64, 15409, new_spread=0.6, length_spread=0.8, page=64, q_heads=8,
              **_pages(1, 256, "bf16", "fp8")),
        # eight long prompts of a backbone with 32 heads of 128 on eight K/V heads
        _case("verify_prompts8", "verify", 8, 128, 8192, new_spread=0.3, page=64, q_heads=32, **wide),
        # a small float32 policy with odd sizes over an 8-bit cache
        _case("verify_ragged_f32", "verify", 5, 37, 1900, new_spread=0.9, length_spread=0.6, q_heads=6,
              **_pages(2, 64, "f32", "int8")),
        # the fleet of 32 goes on from its accepted tokens
        _case("accept_fleet32", "accept", 32, 64, 900, new_spread=0.6, accepted=6, **pi0),
        # eight long prompts whose drafts were long and mostly right
        _case("accept_prompts8", "accept", 8, 128, 8192, new_spread=0.3, page=64, accepted=90, **wide),
        # a fleet generating over long memories in fp8, one token each, the memory's weights kept
        _case("weigh_tokens64_fp8", "weigh", 64, 1, 15409, length_spread=0.8, page=64, q_heads=8, causal=True, window=0,
              **_pages(1, 256, "bf16", "fp8")),
        # a piece of two long prompts, all of whose rows weigh the memory: the largest case
        _case("weigh_prompts", "weigh", 2, 4096, 8192, page=64, q_heads=32, causal=True, window=0, **wide),
        # the memories of 32 robots cut from up to twenty frames to about nine
        _case("evict_fleet32", "evict", 32, 1, 15408, length_spread=0.6, page=64, keep=7000, sinks=48, recent=768, **pi0),
        # eight long prompts of the 32-head backbone cut to an odd budget
        _case("evict_prompts8", "evict", 8, 1, 8192, length_spread=0.2, page=64, keep=2501, sinks=4, recent=333, **wide),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    most["verify"] = most["weigh"]
    while True:
        op = rng.choice(["tree", "verify", "verify", "verify", "accept", "weigh", "weigh", "weigh", "evict", "evict"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        seqs = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, 300)
        if op == "weigh":
            new = 1 if rng.random() < 0.5 else _log_int(rng, 1, 4096)
        length = new + _log_int(rng, 1, 16384) - 1
        case = _case("", op, seqs, new, length, new_spread=rng.choice([0.0, 0.5, 0.9]),
                     length_spread=rng.choice([0.0, 0.4, 0.8]), page=2 ** rng.randint(3, 7))
        if op != "tree":
            kv = rng.choice([1, 1, 2, 3, 8])
            store = rng.choice([dtype, dtype, "fp8", "int8"]) if op in ("verify", "weigh") else dtype
            case.update(_pages(kv, rng.choice([64, 128, 256]), dtype, store))
            if op in ("verify", "weigh"):
                case.update(q_heads=kv * rng.choice([1, 2, 4, 5, 8]))
            if op == "weigh":
                case.update(causal=rng.random() < 0.8, window=0 if rng.random() < 0.7 else _log_int(rng, 16, 4096))
            if op == "accept":
                case.update(accepted=rng.randint(0, new))
            if op == "evict":
                case.update(new=1, new_spread=0.0)
                keep = _log_int(rng, 1, length)
                sinks = rng.choice([0, min(4, keep)])
                case.update(keep=keep, sinks=sinks, recent=rng.randint(0, keep - sinks))
            n, l = _lengths(case)
            # the plain form's padded batch fits the card, and so do a few copies of the cache
            if len(n) * max(n) * max(l) * case.get("q_heads", 0) > 2.5e9 or len(l) * max(l) * kv * case["head_dim"] > 3e8:
                continue
        if _cost(case) <= most[op]:
            del case["name"]
            return case


def _cost(case):
    """A rough time of the plain form: operations in float32, and bytes at a tenth of what they move."""
    w = work(case)
    return w["flops"] / 50e12 + w["bytes"] / 2e11


def _spread(most, spread, b):
    """Sequence b's share of `most`: the largest first, the others spread below it."""
    return round(most * (1 - spread * ((b * _GOLDEN) % 1.0)))


def _lengths(case):
    """(new tokens, cached tokens) of each sequence."""
    new, length = [], []
    for b in range(case["seqs"]):
        n = max(1, _spread(case["new"], case["new_spread"], b))
        new.append(n)
        length.append(max(n, _spread(case["length"], case["length_spread"], b)))
    return new, length


def _accepted(case):
    """How many drafted tokens of each sequence are accepted."""
    return [min(n, _spread(case["accepted"], 0.8, b)) for b, n in enumerate(_lengths(case)[0])]


def _visible(case):
    """Query-key pairs per head, and the keys that any of a sequence's queries sees."""
    pairs = keys = 0
    for n, l in zip(*_lengths(case)):
        w = case["window"] or l + n
        for i in ([0] if not case["causal"] and w >= l else range(n)):
            p = l - n + i
            hi = p + 1 if case["causal"] else l
            pairs += (hi - max(0, p + 1 - w)) * (n if not case["causal"] and w >= l else 1)
        keys += l - max(0, l - n + 1 - w)
    return pairs, keys


def work(case):
    new, length = _lengths(case)
    rows = sum(new)
    if case["op"] == "tree":
        return {"bytes": rows * (4 + 8 + 8 * _words(case)), "flops": rows}
    hk, dh, es, cs = case["kv_heads"], case["head_dim"], _SIZE[case["dtype"]], _SIZE[case["store"]]
    slot = 2 * (dh * cs + (4 if cs == 1 else 0))  # a token's K and V of one head
    if case["op"] == "accept":
        return {"bytes": 2 * sum(_accepted(case)) * hk * slot + 4 * (sum(_accepted(case)) + 3 * len(new)), "flops": 0}
    if case["op"] == "evict":
        cut = [l for l in length if l > case["keep"]]
        # the kept tokens after the first ones are read and written with their weights
        moved = len(cut) * (case["keep"] - case["sinks"])
        return {"bytes": hk * (4 * sum(cut) + moved * (2 * slot + 8)) + 8 * len(new), "flops": hk * sum(cut)}
    if case["op"] == "verify":  # (a node sees some of the others, at least itself)
        pairs, keys = sum((l - n + 1) * n for n, l in zip(new, length)), sum(length)
    else:
        pairs, keys = _visible(case)
    moved = 2 * rows * case["q_heads"] * dh * es + keys * hk * slot + (8 * keys * hk if case["op"] == "weigh" else 0)
    return {"bytes": moved, "flops": 4 * pairs * case["q_heads"] * dh}


def _words(case):
    """64-bit words of a row's visibility bits."""
    return -(-max(_lengths(case)[0]) // 64)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE)

    s = dict(case=case)
    new, length = _lengths(case)
    B, ps, rows = len(new), case["page"], sum(new)
    need = [-(-l // ps) for l in length]
    pool = sum(need) + 8
    order = torch.randperm(pool, generator=g, device=DEVICE).to(torch.int32)
    table = torch.zeros(B, max(need), dtype=torch.int32, device=DEVICE)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table
    s["lengths"] = torch.tensor(length, dtype=torch.int32, device=DEVICE)
    s["cu"] = torch.tensor([0] + new, device=DEVICE).cumsum(0).to(torch.int32)
    if case["op"] in ("tree", "verify"):
        # a drafted token's parent is any earlier one, mostly a recent one; some follow the cached tokens themselves
        i = _rows(s, rows)[1]
        back = 1 + (uniform(rows) ** 3 * (i + 1)).long()
        s["parents"] = torch.clamp(i - back, min=-1).to(torch.int32)
    if case["op"] == "tree":
        # the positions say where the sequences are
        s["lengths"] += torch.randint(0, 100000, (B,), generator=g, device=DEVICE).to(torch.int32)
        return s
    dt, dh, hk = _DT[case["dtype"]], case["head_dim"], case["kv_heads"]
    # keys have a few strong channels, values do not
    k = normal(pool, hk, ps, dh) * torch.exp(0.5 * normal(hk, dh))[:, None]
    v = normal(pool, hk, ps, dh)
    if case["store"] in ("fp8", "int8"):
        s["k"], s["k_scale"] = _encode(k, case["store"])
        s["v"], s["v_scale"] = _encode(v, case["store"])
    else:
        s["k"], s["v"] = k.to(_CODES[case["store"]]), v.to(_CODES[case["store"]])
    del k, v
    if case["op"] in ("verify", "weigh"):
        s["q"] = normal(rows, case["q_heads"], dh).to(dt)
    if case["op"] == "verify":
        s["mask"] = _plain_tree(s)[0]  # what the program has from its draft
    if case["op"] == "weigh":
        # about what one such call gave before
        s["weights"] = uniform(pool, hk, ps) * (rows * (case["q_heads"] // hk) / sum(length))
    if case["op"] == "accept":
        s["full"] = s["lengths"].clone()
        most = max(new)
        pick = uniform(B, most).masked_fill_(torch.arange(most, device=DEVICE)[None] >= torch.tensor(new, device=DEVICE)[:, None],
                                             2.0).argsort(1)
        s["counts"] = torch.tensor(_accepted(case), dtype=torch.int32, device=DEVICE)
        pick = pick.masked_fill_(torch.arange(most, device=DEVICE)[None] >= s["counts"][:, None], most).sort(1).values
        s["path"] = pick.to(torch.int32).contiguous()
    if case["op"] == "evict":
        s["full"] = s["lengths"].clone()
        # sums of probabilities spread over a few powers of ten; tokens that nothing has looked at yet have none
        s["grown"] = torch.exp(1.5 * normal(pool, hk, ps)) * (uniform(pool, hk, ps) < 0.9)
        s["weights"] = s["grown"].clone()
    return s


def _encode(x, store):
    """(codes, scales) of the rows of x as an 8-bit cache holds them."""
    most = x.abs().amax(-1, keepdim=True)
    if store == "int8":
        scale = torch.clamp(most / 127.0, min=2.0 ** -126)
        return torch.clamp(torch.round(x / scale), -127, 127).to(torch.int8), scale[..., 0].contiguous()
    scale = torch.exp2(torch.ceil(torch.log2(most / 448.0)))
    return (x / scale).to(torch.float8_e4m3fn), scale[..., 0].contiguous()


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _rows(s, n):
    """(sequence, index in its chunk) of every packed row."""
    i = torch.arange(n, device=DEVICE)
    b = (i[:, None] >= s["cu"][None, 1:]).sum(1)
    return b, i - s["cu"][b]


def _bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def _plain_tree(s):
    """(bits of the rows that each row sees, positions): the closure of "is the parent of" by squaring."""
    case = s["case"]
    n, B, nmax, words = s["parents"].shape[0], case["seqs"], max(_lengths(case)[0]), _words(case)
    b, i = _rows(s, n)
    sees = torch.zeros(B, nmax, nmax + 1, device=DEVICE)
    sees[b, i, torch.where(s["parents"] < 0, nmax, s["parents"]).long()] = 1.0
    sees = sees[..., :nmax] + torch.eye(nmax, device=DEVICE)
    for _ in range(max(1, math.ceil(math.log2(nmax)))):
        sees = (torch.matmul(sees, sees) > 0).float()
    sees = sees[b, i].long()
    depth = sees.sum(1) - 1
    sees = torch.nn.functional.pad(sees, (0, 64 * words - nmax)).view(n, words, 64)
    mask = (sees << torch.arange(64, device=DEVICE)).sum(-1)
    return mask, (s["lengths"][b] - (s["cu"][b + 1] - s["cu"][b])).long() + depth


def _plain_attend(s):
    case = s["case"]
    q, hk, dh, ps = s["q"], case["kv_heads"], case["head_dim"], case["page"]
    new, length = _lengths(case)
    B, nmax, lmax, n, grp = len(new), max(new), max(length), q.shape[0], case["q_heads"] // case["kv_heads"]
    j = torch.arange(lmax, device=DEVICE)
    page, slot = s["table"][:, j // ps].long(), (j % ps)[None].expand(B, -1)

    def gathered(name):  # [B, Hkv, lmax, dh] in float32
        x = _bits(s[name])[page, :, slot].view(s[name].dtype).float()
        if name + "_scale" in s:
            x = x * s[name + "_scale"][page, :, slot][..., None]
        return x.transpose(1, 2).contiguous()

    count = s["cu"][1:] - s["cu"][:-1]
    i = torch.arange(nmax, device=DEVICE)
    at = torch.clamp(s["cu"][:-1, None] + i, max=n - 1).long()
    real = i[None] < count[:, None]
    qb = q[at].float().view(B, nmax, hk, grp, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, grp * nmax, dh).contiguous()
    scores = torch.matmul(qb, gathered("k").transpose(2, 3).contiguous()).view(B, hk, grp, nmax, lmax)
    scores *= 1.0 / math.sqrt(dh)
    first = s["lengths"] - count
    if case["op"] == "verify":
        drafted = j[None] - first[:, None]  # [B, lmax]
        word = torch.clamp(drafted // 64, min=0, max=s["mask"].shape[1] - 1).long()
        bit = torch.gather(s["mask"][at], 2, word[:, None].expand(-1, nmax, -1)) >> (drafted % 64)[:, None] & 1
        seen = (drafted < 0)[:, None] | ((bit == 1) & (drafted < count[:, None])[:, None])
    else:
        pos = first[:, None] + i  # [B, nmax]
        seen = j[None, None] < s["lengths"][:, None, None]
        if case["causal"]:
            seen = seen & (j[None, None] <= pos[..., None])
        if case["window"]:
            seen = seen & (j[None, None] > pos[..., None] - case["window"])
    seen = seen & real[..., None]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = torch.clamp(scores.amax(-1, keepdim=True), min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    o = torch.matmul(p.view(B, hk, grp * nmax, lmax), gathered("v")).view(B, hk, grp, nmax, dh)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, nmax, hk * grp, dh)
    b, r = _rows(s, n)
    out = o[b, r].to(q.dtype)
    if case["op"] == "verify":
        return out
    got = p.view(B, hk, grp * nmax, lmax).sum(2).transpose(1, 2)  # [B, lmax, Hkv]
    # what lies past a sequence adds nothing to its first token
    page = torch.where(j[None] < s["lengths"][:, None], page, page[:, :1])
    slot = torch.where(j[None] < s["lengths"][:, None], slot, slot[:, :1])
    head = torch.arange(hk, device=DEVICE)[None, None]
    s["weights"].index_put_((page[..., None], head, slot[..., None]), got, accumulate=True)
    return [out, s["weights"]]


def _plain_accept(s):
    case = s["case"]
    ps, most = case["page"], s["path"].shape[1]
    i = torch.arange(most, device=DEVICE)
    first = (s["lengths"] - (s["cu"][1:] - s["cu"][:-1]))[:, None]
    # entries past the count stand for their own place
    src = first + torch.where(i[None] < s["counts"][:, None], s["path"], i[None].to(torch.int32))
    dst = first + i[None]
    inside = dst < s["lengths"][:, None]
    src, dst = torch.where(inside, src, first), torch.where(inside, dst, first)
    # (places past the sequence repeat what the first entry does)
    src = torch.where(inside, src, src[:, :1])
    b = torch.arange(src.shape[0], device=DEVICE)[:, None]
    for name in ("k", "v"):
        x = s[name][s["table"][b, src // ps].long(), :, (src % ps).long()]
        s[name][s["table"][b, dst // ps].long(), :, (dst % ps).long()] = x
    s["lengths"].copy_(first[:, 0] + s["counts"])


def _plain_evict(s):
    case = s["case"]
    ps, keep, hk, sinks, recent = case["page"], case["keep"], case["kv_heads"], case["sinks"], case["recent"]
    L, lmax = s["lengths"][:, None], max(_lengths(case)[1])
    j = torch.arange(lmax, device=DEVICE)[None]
    b = torch.arange(L.shape[0], device=DEVICE)[:, None]
    page, slot = s["table"][b, j // ps].long(), (j % ps).expand(L.shape[0], -1)
    head = torch.arange(hk, device=DEVICE)[None, :, None]
    w = s["weights"][page, :, slot].transpose(1, 2)  # [B, Hkv, lmax]
    # first the tokens that stay anyway, then by weight and index
    stays = (j < sinks) | (j >= L - recent)
    rank = torch.where(j < L, torch.where(stays, math.inf, 0.0), -math.inf)[:, None] + w
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    i = torch.arange(keep, device=DEVICE)
    cut = L[..., None] > keep
    kept = torch.where(cut, torch.nn.functional.pad(order, (0, keep - order.shape[-1])).sort(-1).values, i[None, None])
    valid = cut | (i[None, None] < L[..., None])
    src, dst = torch.where(valid, kept, 0), torch.where(valid, i[None, None].expand_as(kept), 0)
    bb = b[..., None]
    from_, to = (s["table"][bb, src // ps].long(), head, src % ps), (s["table"][bb, dst // ps].long(), head, dst % ps)
    for name in ("k", "v", "weights"):
        s[name][to] = s[name][from_]
    # the places that are left have no weight (what lies past a sequence stands for its first token)
    gone = ((j >= keep) & (j < L))[:, None]
    p3, s3 = torch.where(j < L, page, page[:, :1])[:, None], torch.where(j < L, slot, slot[:, :1])[:, None]
    s["weights"][p3, head, s3] = torch.where(gone, 0.0, s["weights"][p3, head, s3])
    s["lengths"].clamp_(max=keep)
    return torch.where(valid, kept, -1).to(torch.int32)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _handles(s):
    """The cache over the state's own buffers and the batch, kept as a program keeps them."""
    from paper_2607_14695_amd.paged import PagedBatch, PagedCache

    case = s["case"]
    if case["op"] != "tree":
        s["cache"] = PagedCache(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"))
    new, length = _lengths(case)
    s["batch"] = PagedBatch(s["cu"], s["lengths"], s["table"], max_length=max(length))
    s["most"] = max(new)


def run(state):
    s, op = state, state["case"]["op"]
    if op in ("accept", "evict"):
        s["lengths"].copy_(s["full"])  # the tokens have come in again
    if op == "evict":
        s["weights"].copy_(s["grown"])
    if own:
        if "batch" not in s:
            _handles(s)
        if op == "tree":
            return list(s["batch"].tree(s["parents"], max_rows=s["most"]))
        if op == "verify":
            return s["cache"].attend_tree(s["batch"], s["q"], s["mask"])
        if op == "weigh":
            return [s["cache"].attend(s["batch"], s["q"], causal=s["case"]["causal"], window=s["case"]["window"],
                                      weights=s["weights"]), s["weights"]]
        if op == "accept":
            s["cache"].accept(s["batch"], s["path"], s["counts"])
            return [s["lengths"], s["k"], s["v"]]
        kept = s["cache"].evict(s["batch"], s["weights"], s["case"]["keep"], sinks=s["case"]["sinks"],
                                recent=s["case"]["recent"])
        return [kept, s["lengths"], s["k"], s["v"], s["weights"]]
    if op == "tree":
        return list(_plain_tree(s))
    if op in ("verify", "weigh"):
        return _plain_attend(s)
    if op == "accept":
        _plain_accept(s)
        return [s["lengths"], s["k"], s["v"]]
    kept = _plain_evict(s)
    return [kept, s["lengths"], s["k"], s["v"], s["weights"]]


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_tree(s):
    """Every token by itself: its parent's ancestors and itself."""
    new, words = _lengths(s["case"])[0], _words(s["case"])
    parents, lengths = s["parents"].tolist(), s["lengths"].tolist()
    masks, positions, r = [], [], 0
    for n, l in zip(new, lengths):
        sets, depths = [], []
        for i in range(n):
            p = parents[r + i]
            sets.append((sets[p] if p >= 0 else 0) | 1 << i)
            depths.append(depths[p] + 1 if p >= 0 else 0)
        for x, d in zip(sets, depths):
            words_ = [x >> (64 * w) & (2 ** 64 - 1) for w in range(words)]
            masks.append([w - 2 ** 64 if w >= 2 ** 63 else w for w in words_])
            positions.append(l - n + d)
        r += n
    return [torch.tensor(masks, dtype=torch.int64, device=DEVICE), torch.tensor(positions, dtype=torch.int64, device=DEVICE)]


def _exact_attend(s):
    case = s["case"]
    new, length = _lengths(case)
    ps, cu = case["page"], s["cu"].tolist()
    grp, dh, hk = case["q_heads"] // case["kv_heads"], case["head_dim"], case["kv_heads"]
    out = torch.zeros(sum(new), case["q_heads"], dh, dtype=torch.float64, device=DEVICE)
    weights = s["weights"].double() if case["op"] == "weigh" else None
    for b, (n, l) in enumerate(zip(new, length)):
        pages = s["table"][b, :-(-l // ps)].long()
        j = torch.arange(l, device=DEVICE)
        for h in range(hk):
            kv = []
            for name in ("k", "v"):
                x = _bits(s[name])[pages, h].view(s[name].dtype).double()
                if name + "_scale" in s:
                    x = x * s[name + "_scale"][pages, h].double()[..., None]
                kv.append(x.reshape(-1, dh)[:l])
            got = torch.zeros(l, dtype=torch.float64, device=DEVICE)
            step = max(1, 100_000_000 // l)
            for i0 in range(0, n, step):
                m = min(step, n - i0)
                pos = torch.arange(l - n + i0, l - n + i0 + m, device=DEVICE)[:, None]
                hidden = torch.zeros(m, l, dtype=torch.bool, device=DEVICE)
                if case["op"] == "verify":
                    for d in range(n):  # drafted token d, at l - n + d
                        word = s["mask"][cu[b] + i0:cu[b] + i0 + m, d // 64]
                        hidden[:, l - n + d] = (word >> (d % 64)) % 2 == 0
                elif case["causal"]:
                    hidden |= j[None] > pos
                if case["op"] == "weigh" and case["window"]:
                    hidden |= j[None] <= pos - case["window"]
                for q in range(h * grp, (h + 1) * grp):
                    sc = s["q"][cu[b] + i0:cu[b] + i0 + m, q].double() @ kv[0].t() / math.sqrt(dh)
                    p = sc.masked_fill_(hidden, -math.inf).softmax(-1)
                    out[cu[b] + i0:cu[b] + i0 + m, q] = p @ kv[1]
                    got += p.sum(0)
            if weights is not None:
                weights[pages[j // ps], h, j % ps] += got
    return out if weights is None else [out, weights]


def _exact_accept(s):
    case, ps = s["case"], s["case"]["page"]
    table, path = s["table"].tolist(), s["path"].tolist()
    k, v, lengths = s["k"].double(), s["v"].double(), []
    for b, (n, l, c) in enumerate(zip(*_lengths(case), _accepted(case))):
        at = [(table[b][(l - n + d) // ps], (l - n + d) % ps) for d in range(n)]
        for i in range(c):  # a node's index is at least its place on the path: nothing is read after it was written
            (p0, s0), (p1, s1) = at[path[b][i]], at[i]
            k[p1, :, s1], v[p1, :, s1] = k[p0, :, s0], v[p0, :, s0]
        lengths.append(l - n + c)
    return [torch.tensor(lengths, dtype=torch.int32, device=DEVICE), k, v]


def _exact_evict(s):
    case, ps = s["case"], s["case"]["page"]
    keep, sinks, recent, hk = case["keep"], case["sinks"], case["recent"], case["kv_heads"]
    length = _lengths(case)[1]
    kept = torch.full((len(length), hk, keep), -1, dtype=torch.int32)
    k, v, w = s["k"].double(), s["v"].double(), s["weights"].double()
    for b, l in enumerate(length):
        j = torch.arange(l, device=DEVICE)
        page, slot = s["table"][b].long()[j // ps], j % ps
        if l <= keep:
            kept[b, :, :l] = torch.arange(l, dtype=torch.int32)
            continue
        for h in range(hk):
            mine = w[page, h, slot]
            values = mine.tolist()
            middle = sorted(range(sinks, l - recent), key=lambda t: -values[t])[:keep - sinks - recent]
            chosen = list(range(sinks)) + sorted(middle) + list(range(l - recent, l))
            kept[b, h] = torch.tensor(chosen, dtype=torch.int32)
            at = torch.tensor(chosen, device=DEVICE)
            for x in (k, v):
                x[page[:keep], h, slot[:keep]] = x[page[at], h, slot[at]]
            left = torch.zeros_like(mine)
            left[:keep] = mine[at]
            w[page, h, slot] = left
    return [kept.to(DEVICE), torch.tensor([min(l, keep) for l in length], dtype=torch.int32, device=DEVICE), k, v, w]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "tree":
        return _exact_tree(s)
    if case["op"] == "accept":
        return _exact_accept(s)
    if case["op"] == "evict":
        return _exact_evict(s)
    return None if work(case)["flops"] > 3e12 else _exact_attend(s)
