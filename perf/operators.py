"""The backbone's operators as cases that a program can time and check: rotary positions over several axes, the
paged K/V cache (written with quantisation, read back) and the attention of a chunk of new tokens over it.

The action expert's cache takes pre-RoPE K/V of its prefix and frames from a vision-language backbone.  These are
the operators that such a backbone runs to produce them, each case one call as its program makes it:

* ``rotary``: queries or keys rotated by their positions on one axis (text) or on three (time, height, width of
  image tokens); ``inverse`` is the gradient, and what takes a cached key back to its pre-RoPE form.
* ``write``: new keys and values written into their pages, the keys rotated on the way.
* ``store``: the same with a quantised cache, and the same rows read back.
* ``attend``: the new tokens' attention over the pages of their sequences.

Sequence b of a batch has ``length_b`` tokens in the cache, the last ``new_b`` of them new: rows cu[b] .. cu[b + 1]
of the packed inputs.  Both are fixed by the case; what fills them is drawn from the seed.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_CODES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
_SIZE = {"f32": 4, "bf16": 2, "fp8": 1, "int8": 1}
_GOLDEN = 0.6180339887498949


def _rotary(name, tokens, heads, head_dim, axes, dtype, inverse=False, ladder="shared", far=0):
    return dict(name=name, op="rotary", tokens=tokens, heads=heads, head_dim=head_dim, axes=axes, dtype=dtype,
                inverse=inverse, ladder=ladder, far=far)


def _cached(name, op, seqs, new, length, kv_heads, head_dim, dtype, store, page, new_spread=0.0, length_spread=0.0,
            **more):
    return dict(name=name, op=op, seqs=seqs, new=new, new_spread=new_spread, length=length,
                length_spread=length_spread, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, store=store, page=page,
                **more)


def listed():
    return [
        # one token of eight sequences, the heads of the pi0 backbone: all latency
        _rotary("rotary_tokens8", 8, 8, 256, 1, "bf16"),
        # one observation frame of three 256-token views
        _rotary("rotary_frame", 768, 8, 256, 3, "bf16", far=100000),
        # the gradient for a training batch of 32 frames in float32
        _rotary("rotary_batch32_back_f32", 32 * 768, 8, 256, 3, "f32", inverse=True, ladder="per_axis"),
        # a fleet of 32 generating one token each, cache kept in bf16
        _cached("write_tokens32", "write", 32, 1, 900, 1, 256, "bf16", "bf16", 16, length_spread=0.7, axes=1),
        # one frame for each robot of a fleet of 32, cache in fp8
        _cached("store_frames32_fp8", "store", 32, 768, 1584, 1, 256, "bf16", "fp8", 64, axes=3),
        # a batch of long prompts, eight heads of 128, cache in 8-bit integers
        _cached("store_prompts_int8", "store", 8, 8192, 8192, 8, 128, "bf16", "int8", 64, new_spread=0.8, axes=1),
        # a few odd prompts of a small float32 policy
        _cached("store_ragged_f32", "store", 5, 333, 700, 3, 64, "f32", "int8", 8, new_spread=0.9, axes=2),
        # one robot, one token over its prompt and one frame: the smallest attention
        _cached("attend_token1", "attend", 1, 1, 817, 1, 256, "bf16", "bf16", 16, q_heads=8, causal=True, window=0),
        # a fleet generating over long memories in fp8
        _cached("attend_tokens64_fp8", "attend", 64, 1, 15409, 1, 256, "bf16", "fp8", 64, length_spread=0.8, q_heads=8,
                causal=True, window=0),
        # one robot's newest frame, all its tokens seeing each other, over a twenty-frame memory
        _cached("attend_frame_window20", "attend", 1, 768, 15408, 1, 256, "bf16", "bf16", 64, q_heads=8, causal=False,
                window=0),
        # two long prompts of a backbone with 32 heads of 128 on eight K/V heads: the largest case
        _cached("attend_prompts", "attend", 2, 8192, 8192, 8, 128, "bf16", "bf16", 64, q_heads=32, causal=True,
                window=0),
        # a ragged mix of chunks and single tokens in float32 with a sliding window over an 8-bit cache
        _cached("attend_ragged_f32", "attend", 7, 150, 1900, 2, 64, "f32", "int8", 16, new_spread=0.995,
                length_spread=0.6, q_heads=6, causal=True, window=512),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("rotary", "write", "store", "attend")}
    most["write"] = most["store"]
    while True:
        op = rng.choice(["rotary", "write", "store", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        dh = rng.choice([64, 128, 256])
        if op == "rotary":
            dh = rng.choice([64, 80, 96, 128, 256])
            case = _rotary("", _log_int(rng, 1, 40000), _log_int(rng, 1, 40), dh, rng.randint(1, 3), dtype,
                           inverse=rng.random() < 0.4, ladder=rng.choice(["shared", "per_axis"]),
                           far=rng.choice([0, 1000, 1000000]))
        else:
            seqs = _log_int(rng, 1, 64)
            new = 1 if rng.random() < 0.3 else _log_int(rng, 1, 8192)
            length = new + _log_int(rng, 1, 16384) - 1
            store = rng.choice([dtype, "fp8", "int8"] if op == "attend" else
                               [dtype] if op == "write" else ["fp8", "int8"])
            kv = rng.choice([1, 1, 2, 3, 8])
            case = _cached("", op, seqs, new, length, kv, dh, dtype, store, 2 ** rng.randint(3, 7),
                           new_spread=rng.choice([0.0, 0.5, 0.9]), length_spread=rng.choice([0.0, 0.4, 0.8]))
            if op == "attend":
                case.update(q_heads=kv * rng.choice([1, 2, 4, 5, 8]), causal=rng.random() < 0.75,
                            window=0 if rng.random() < 0.7 else _log_int(rng, 16, 4096))
            else:
                case.update(axes=rng.randint(1, 3))
            n, l = _lengths(case)
            pairs = len(n) * max(n) * max(l) * case.get("q_heads", 0)
            # the plain form's padded batch fits the card, and so do a few copies of the cache
            if pairs > 5e9 or sum(l) * kv * dh > 6e8 or len(l) * max(l) * kv * dh > 2e9:
                continue
        if _cost(case) <= most[op]:
            del case["name"]
            return case


def _cost(case):
    """A rough time of the plain form: operations in float32, and bytes at a tenth of what they move."""
    w = work(case)
    return w["flops"] / 50e12 + w["bytes"] / 2e11


def _lengths(case):
    """(new tokens, cached tokens) of each sequence: the largest first, the others spread below it."""
    new, length = [], []
    for b in range(case["seqs"]):
        f = (b * _GOLDEN) % 1.0
        n = max(1, round(case["new"] * (1 - case["new_spread"] * f)))
        new.append(n)
        length.append(max(n, round(case["length"] * (1 - case["length_spread"] * f))))
    return new, length


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
    dh, es = case["head_dim"], _SIZE[case["dtype"]]
    if case["op"] == "rotary":
        n = case["tokens"] * case["heads"] * dh
        return {"bytes": 2 * n * es + 8 * case["tokens"] * case["axes"], "flops": 3 * n}
    new, length = _lengths(case)
    rows, hk, cs = sum(new), case["kv_heads"], _SIZE[case["store"]]
    scales = 4 if cs == 1 else 0
    if case["op"] == "attend":
        pairs, keys = _visible(case)
        return {"bytes": 2 * rows * case["q_heads"] * dh * es + 2 * keys * hk * (dh * cs + scales),
                "flops": 4 * pairs * case["q_heads"] * dh}
    moved = 2 * rows * hk * (dh * (es + cs) + scales) + 8 * rows * case["axes"]
    if case["op"] == "store":
        moved += 2 * rows * hk * (dh * (es + cs) + scales)
    return {"bytes": moved, "flops": 2 * rows * hk * dh * (4 if case["op"] == "store" else 2)}


def _sections(case):
    """The pairs of dimensions that turn with each axis: a quarter with the first of three, else even shares."""
    half, axes = case["head_dim"] // 2, case["axes"]
    if axes == 1:
        return [half]
    first = half // 4 if axes == 3 else half // 2
    rest = half - first
    return [first, rest] if axes == 2 else [first, rest // 2, rest - rest // 2]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    dt, dh = _DT[case["dtype"]], case["head_dim"]
    s = dict(case=case)
    if case["op"] == "rotary":
        n = case["tokens"]
        s["x"] = normal(n, case["heads"], dh).to(dt)
        s["positions"] = _positions(case, n, g, case["far"])
        return s
    new, length = _lengths(case)
    ps, hk = case["page"], case["kv_heads"]
    need = [-(-l // ps) for l in length]
    pool = sum(need) + 8
    order = torch.randperm(pool, generator=g, device=DEVICE).to(torch.int32)
    table = torch.zeros(len(new), max(need), dtype=torch.int32, device=DEVICE)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table
    s["lengths"] = torch.tensor(length, dtype=torch.int32, device=DEVICE)
    s["cu"] = torch.tensor([0] + new, device=DEVICE).cumsum(0).to(torch.int32)
    rows = sum(new)
    # keys have a few strong channels, values do not
    strong = torch.exp(0.5 * normal(hk, dh))
    code = _CODES[case["store"]]
    if case["op"] == "attend":
        s["q"] = (normal(rows, case["q_heads"], dh)).to(dt)
        k = normal(pool, hk, ps, dh) * strong[:, None]
        v = normal(pool, hk, ps, dh)
        if case["store"] in ("fp8", "int8"):
            s["k"], s["k_scale"] = _encode(k.to(dt), case["store"])
            s["v"], s["v_scale"] = _encode(v.to(dt), case["store"])
        else:
            s["k"], s["v"] = k.to(code), v.to(code)
        return s
    s["new_k"] = (normal(rows, hk, dh) * strong).to(dt)
    s["new_v"] = normal(rows, hk, dh).to(dt)
    s["positions"] = _positions(case, rows, g, 1000)
    s["k"] = torch.zeros(pool, hk, ps, dh, dtype=code, device=DEVICE)
    s["v"] = torch.zeros_like(s["k"])
    if code.itemsize == 1:
        s["k_scale"] = torch.zeros(pool, hk, ps, device=DEVICE)
        s["v_scale"] = torch.zeros(pool, hk, ps, device=DEVICE)
    return s


def _positions(case, n, g, far):
    """Text counts on; image tokens have a frame's time and their place on a grid."""
    start = torch.randint(0, far + 1, (1,), generator=g, device=DEVICE)
    i = torch.arange(n, device=DEVICE)
    if case["axes"] == 1:
        return start + i
    t, cell = i // 256, i % 256
    return torch.stack([start + t, cell // 16, cell % 16][:case["axes"]]).contiguous()


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _angles(case, positions, device):
    """cos and sin of every (token, pair), in 64 bits."""
    half, sections = case["head_dim"] // 2, torch.tensor(_sections(case), device=device)
    pair = torch.arange(half, device=device)
    ends = sections.cumsum(0)
    axis = (pair[:, None] >= ends[None]).sum(1)
    if case.get("ladder", "shared") == "shared":
        e = pair.double() / half
    else:
        e = (pair - (ends - sections)[axis]).double() / sections[axis].double()
    freq = torch.exp(e * -math.log(10000.0))
    p = positions.reshape(-1, positions.shape[-1])[axis].double()  # [half, n]
    a = (p * freq[:, None]).t()
    return a.cos()[:, None], a.sin()[:, None]


def _rotate(x, cos, sin):
    a, b = x.double().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _encode(x, store):
    """(codes, scales) of the rows of x: 8 bits each with one scale a row; 64 bits decide what lies on a border."""
    x = x.double()
    most = x.abs().amax(-1).float()
    if store == "int8":
        scale = torch.clamp(most / 127.0, min=2.0 ** -126)
        return torch.clamp(torch.round(x / scale.double()[..., None]), -127, 127).to(torch.int8), scale
    mant, expo = torch.frexp(most)  # most = mant * 2^expo, mant in [0.5, 1); 448 = 0.875 * 2^9
    k = torch.clamp(expo - 9 + (mant > 0.875), min=-126)
    scale = torch.ldexp(torch.ones_like(most), k)
    y = x / scale.double()[..., None]
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), torch.clamp(e - 1, min=-6) - 3)
    y = torch.clamp(torch.round(y / step) * step, -448, 448)
    return y.float().to(torch.float8_e4m3fn), scale


def _rows(s, n):
    """(sequence, index in its chunk) of every packed row."""
    i = torch.arange(n, device=DEVICE)
    b = (i[:, None] >= s["cu"][None, 1:]).sum(1)
    return b, i - s["cu"][b]


def _places(s, n):
    """(page, slot) of every packed row."""
    ps = s["case"]["page"]
    b, i = _rows(s, n)
    p = s["lengths"][b] - (s["cu"][b + 1] - s["cu"][b]) + i
    return s["table"][b, p // ps].long(), p % ps


def _bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def _plain_write(s):
    case, n = s["case"], s["new_k"].shape[0]
    page, slot = _places(s, n)
    k = _rotate(s["new_k"], *_angles(case, s["positions"], DEVICE))
    for name, x in (("k", k), ("v", s["new_v"])):
        if case["store"] in ("fp8", "int8"):
            x, scale = _encode(x, case["store"])
            s[name + "_scale"][page, :, slot] = scale
        else:
            x = x.to(s[name].dtype)
        _bits(s[name])[page, :, slot] = _bits(x)


def _plain_read(s):
    n = s["new_k"].shape[0]
    page, slot = _places(s, n)
    return [(_bits(s[m])[page, :, slot].view(s[m].dtype).float() * s[m + "_scale"][page, :, slot][..., None])
            .to(s["new_k"].dtype) for m in ("k", "v")]


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
    qb = q[at].float().view(B, nmax, hk, grp, dh).permute(0, 2, 3, 1, 4).reshape(B, hk, grp * nmax, dh).contiguous()
    scores = torch.matmul(qb, gathered("k").transpose(2, 3).contiguous()).view(B, hk, grp, nmax, lmax)
    scores *= 1.0 / math.sqrt(dh)
    pos = (s["lengths"] - count)[:, None] + i  # [B, nmax]
    seen = j[None, None] < s["lengths"][:, None, None]
    if case["causal"]:
        seen = seen & (j[None, None] <= pos[..., None])
    if case["window"]:
        seen = seen & (j[None, None] > pos[..., None] - case["window"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = torch.clamp(scores.amax(-1, keepdim=True), min=-3e38)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hk, grp * nmax, lmax), gathered("v")).view(B, hk, grp, nmax, dh)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(B, nmax, hk * grp, dh)
    b, r = _rows(s, n)
    return o[b, r].to(q.dtype)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _handles(s):
    """The rotary plan, the cache over the state's own buffers and the batch, kept as a program keeps them."""
    from paper_2607_14695_amd.paged import PagedBatch, PagedCache, Rotary

    case = s["case"]
    if "axes" in case:
        s["rotary"] = Rotary(case["head_dim"], _sections(case), theta=10000.0, ladder=case.get("ladder", "shared"))
    if case["op"] != "rotary":
        s["cache"] = PagedCache(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"))
        s["batch"] = PagedBatch(s["cu"], s["lengths"], s["table"], max_length=max(_lengths(case)[1]))
    s["made"] = True


def run(state):
    s, case = state, state["case"]
    if own:
        if "made" not in s:
            _handles(s)
        if case["op"] == "rotary":
            return s["rotary"].apply(s["x"], s["positions"], inverse=case["inverse"])
        if case["op"] == "attend":
            return s["cache"].attend(s["batch"], s["q"], causal=case["causal"], window=case["window"])
        s["cache"].write(s["batch"], s["new_k"], s["new_v"], rotary=s["rotary"], positions=s["positions"])
        if case["op"] == "write":
            return [s["k"], s["v"]]
        return list(s["cache"].read(s["batch"], s["new_k"].shape[0], dtype=s["new_k"].dtype))
    if case["op"] == "rotary":
        cos, sin = _angles(case, s["positions"], DEVICE)
        return _rotate(s["x"], cos, -sin if case["inverse"] else sin).to(s["x"].dtype)
    if case["op"] == "attend":
        return _plain_attend(s)
    _plain_write(s)
    return [s["k"], s["v"]] if case["op"] == "write" else _plain_read(s)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_rotated(case, x, positions, sign):
    """Each pair (d, d + half) as a complex number times exp(+-i angle)."""
    half = case["head_dim"] // 2
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    pos = positions.double().reshape(-1, positions.shape[-1])
    first = 0
    for axis, m in enumerate(_sections(case)):
        for d in range(first, first + m):
            e = d / half if case.get("ladder", "shared") == "shared" else (d - first) / m
            a = pos[axis] * (10000.0 ** -e) * sign
            z[..., d] *= torch.polar(torch.ones_like(a), a)[:, None]
        first += m
    return torch.cat([z.real, z.imag], -1)


def _exact_stored(x, store):
    """What the 8-bit cache holds of x: the nearest representable multiple of the row's scale."""
    most = x.abs().max(-1, keepdim=True).values
    if store == "int8":
        scale = (most.float() / 127.0).clamp(min=2.0 ** -126).double()
        return (x / scale).round().clamp(-127, 127) * scale
    grid = torch.arange(0x7F, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()  # 0 .. 448
    scale = 2.0 ** torch.ceil(torch.log2(most.float().double() / 448.0)).clamp(min=-126)
    y = (x / scale).abs()
    hi = torch.searchsorted(grid, y.contiguous()).clamp(max=grid.numel() - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = y - grid[lo], grid[hi] - y
    # ties go to the even code
    at = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return torch.sign(x) * grid[at] * scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_rotated(case, s["x"], s["positions"], -1.0 if case["inverse"] else 1.0)
    new, length = _lengths(case)
    ps, cu = case["page"], s["cu"].tolist()
    if case["op"] in ("write", "store"):
        k = _exact_rotated(case, s["new_k"], s["positions"], 1.0)
        v = s["new_v"].double()
        if case["op"] == "store":
            return [_exact_stored(k, case["store"]), _exact_stored(v, case["store"])]
        outs = [s["k"].double(), s["v"].double()]
        for b, (n, l) in enumerate(zip(new, length)):
            for i in range(n):
                p = l - n + i
                page = int(s["table"][b, p // ps])
                outs[0][page, :, p % ps] = k[cu[b] + i]
                outs[1][page, :, p % ps] = v[cu[b] + i]
        return outs
    if work(case)["flops"] > 3e12:
        return None
    grp, dh = case["q_heads"] // case["kv_heads"], case["head_dim"]
    out = torch.zeros(sum(new), case["q_heads"], dh, dtype=torch.float64, device=DEVICE)
    for b, (n, l) in enumerate(zip(new, length)):
        pages = s["table"][b, :-(-l // ps)].long()
        for h in range(case["kv_heads"]):
            kv = []
            for name in ("k", "v"):
                x = _bits(s[name])[pages, h].view(s[name].dtype).double()
                if name + "_scale" in s:
                    x = x * s[name + "_scale"][pages, h].double()[..., None]
                kv.append(x.reshape(-1, dh)[:l])
            step = max(1, 100_000_000 // l)
            for i0 in range(0, n, step):
                m = min(step, n - i0)
                pos = torch.arange(l - n + i0, l - n + i0 + m, device=DEVICE)[:, None]
                j = torch.arange(l, device=DEVICE)[None]
                hidden = torch.zeros(m, l, dtype=torch.bool, device=DEVICE)
                if case["causal"]:
                    hidden |= j > pos
                if case["window"]:
                    hidden |= j <= pos - case["window"]
                for q in range(h * grp, (h + 1) * grp):
                    sc = s["q"][cu[b] + i0:cu[b] + i0 + m, q].double() @ kv[0].t() / math.sqrt(dh)
                    out[cu[b] + i0:cu[b] + i0 + m, q] = sc.masked_fill(hidden, -math.inf).softmax(-1) @ kv[1]
    return out
