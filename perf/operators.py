"""Performance cases of the operators that serve a decoder's attention block in 8 and 4 bits.

``listed()`` are the standing cases, ``draw(rng)`` gives further ones of the same ranges, ``prepare``
makes what a serving program holds before the call and ``run`` is one pass: with ``own`` false in
elementary torch operations in 32 bits, with ``own`` true through the package's entry points.
``exact`` gives the same outputs from the definition in 64 bits.  Kinds of case:

  linear   y = x W^T + b on 8-bit integers, one factor per row of x (made in the call) and per row of W
  pages    block tables, slots and positions of the tokens that a step adds to its requests
  cache    tokens written into the paged 4-bit cache, and the values that it then holds for them
  attend   attention of new tokens over that cache

The cache is uint8 [pages, heads, page / 16, 18 D]: per 16 tokens of a head 8 D bytes of key codes, 8 D of
value codes, D of key factors and D of value factors (binary16, one for 32 channels of a token).  With
G = D / 32, a nibble holding its code plus 8 and the even or first channel of a byte in its low half:
  key codes      [token][j < 4][g < G][4 bytes]     byte b: channels 32 g + 8 j + 2 b and the one behind it
  value codes    [g < G][r < 16][token]             channels 32 g + r and 32 g + 16 + r
  key factors    [token][g < G]
  value factors  [g < G][token, each four in the order 0, 2, 1, 3]
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
SWAP = [0, 2, 1, 3]


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one token of one request through a square projection: the smallest call, all latency
        dict(name="linear 1 x 4096 x 4096", kind="linear", M=1, K=4096, N=4096, type="bf16", bias=False),
        # a decoding batch through an expanding projection
        dict(name="linear 37 x 4096 x 16384", kind="linear", M=37, K=4096, N=16384, type="f16", bias=False),
        # the classifier behind this package's ResNet-50 (2048 -> 1000, with its bias), on an odd batch
        dict(name="linear 777 x 2048 x 1000", kind="linear", M=777, K=2048, N=1000, type="f32", bias=True),
        # a prompt's tokens through a large square projection: the matrix cores' case
        dict(name="linear 8192 x 8192 x 8192", kind="linear", M=8192, K=8192, N=8192, type="bf16", bias=False),
        # a decoding step: one token for each of a few requests
        dict(name="pages 33 requests", kind="pages", requests=33, page=16, longest=4096, added=1, spare=7, mix=1),
        # a large server's step: prompts in pieces beside decoding requests
        dict(name="pages 4000 requests", kind="pages", requests=4000, page=64, longest=16384, added=257, spare=1000,
             mix=2),
        # a decoding step's keys and values, one token of each request
        dict(name="cache 64 tokens", kind="cache", tokens=64, requests=64, heads=8, D=128, page=64, type="bf16",
             mix=3),
        # the keys and values of several prompts
        dict(name="cache 16001 tokens", kind="cache", tokens=16001, requests=5, heads=8, D=128, page=16,
             type="bf16", mix=4),
        # a few short requests, as many query heads as key heads
        dict(name="attend 5 short", kind="attend", requests=5, added=1, longest=300, heads=12, ratio=1, D=64,
             page=16, window=0, type="bf16", mix=5),
        # one token over one very long context: few rows, one long axis
        dict(name="attend 1 x 131071", kind="attend", requests=1, added=1, longest=131071, heads=8, ratio=4, D=128,
             page=64, window=0, type="bf16", mix=6),
        # a decoding batch of ragged lengths, eight query heads to a key head
        dict(name="attend 48 x 16384", kind="attend", requests=48, added=1, longest=16384, heads=8, ratio=8, D=128,
             page=32, window=0, type="f16", mix=7),
        # prompts in pieces over what the cache already holds
        dict(name="attend 3 pieces", kind="attend", requests=3, added=2048, longest=8192, heads=4, ratio=8, D=128,
             page=64, window=0, type="bf16", mix=8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "pages", "cache", "attend", "attend"])
    mix = rng.randrange(1 << 30)
    if kind == "linear":
        while True:
            M, K, N = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 16, 16384)
            if M * K * N <= 8192 ** 3 and K * N >= 1 << 14:
                return dict(kind=kind, M=M, K=K, N=N, type=rng.choice(sorted(TYPES)), bias=rng.random() < 0.5)
    page = rng.choice([16, 32, 64, 128])
    if kind == "pages":
        return dict(kind=kind, requests=_log(rng, 1, 4000), page=page, longest=_log(rng, 16, 16384),
                    added=rng.choice([1, _log(rng, 1, 257)]), spare=_log(rng, 1, 1000), mix=mix)
    heads, D = rng.choice([1, 2, 3, 4, 6, 8]), 32 * rng.randint(1, 8)
    if kind == "cache":
        tokens = _log(rng, 1, 16001)
        return dict(kind=kind, tokens=tokens, requests=_log(rng, 1, min(tokens, 64)), heads=heads, D=D, page=page,
                    type=rng.choice(sorted(TYPES)), mix=mix)
    ratio, kind_type = rng.choice([1, 2, 3, 4, 5, 8, 12, 16]), rng.choice(["bf16", "f16"])
    window = rng.choice([0, 0, _log(rng, 16, 4096)])
    while True:
        requests, longest = _log(rng, 1, 64), _log(rng, 16, 131071)
        added = rng.choice([1, 1, _log(rng, 1, 2048)])
        # no more than the listed cases: bytes of the cache, and visible pairs
        if requests * longest * heads * D <= 48 * 16384 * 8 * 128 and added <= longest and \
                requests * added * longest * heads * ratio * D <= 3 * 2048 * 8192 * 32 * 128:
            return dict(kind=kind, requests=requests, added=added, longest=longest, heads=heads, ratio=ratio, D=D,
                        page=page, window=window, type=kind_type, mix=mix)


# ------------------------------------------------------------------------------ lengths, by the case alone
def _split(rng, total, parts):
    """`total` tokens over `parts` requests, one at least for each where there are enough."""
    cuts = sorted(rng.sample(range(1, total), parts - 1)) if total > parts > 1 else list(range(1, parts))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _requests(case):
    """(tokens in the cache before the step, tokens added), one of each per request."""
    rng = random.Random(case["mix"])
    n = case["requests"]
    if case["kind"] == "cache":
        added = _split(rng, case["tokens"], n)
        before = [rng.randrange(0, 3 * case["page"]) for _ in range(n)]
    elif case["kind"] == "pages":
        # mostly decoding requests, some idle ones, the others with a piece of a prompt
        kinds = [rng.random() for _ in range(n)]
        added = [0 if u < 0.05 else 1 if u < 0.7 else rng.randint(1, case["added"]) for u in kinds]
        before = [rng.randrange(0, case["longest"] + 1) for _ in range(n)]
    else:
        added = [case["added"]] + [case["added"] if case["added"] == 1 else rng.randint(1, case["added"])
                                   for _ in range(n - 1)]
        total = [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(n - 1)]
        before = [max(0, t - a) for t, a in zip(total, added)]
    return before, added


def _pages(tokens, page):
    return -(-tokens // page)


# ------------------------------------------------------------------------------ what a program holds
def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    return globals()["_prepare_" + case["kind"]](case, g, normal)


def _prepare_linear(case, g, normal):
    M, K, N = case["M"], case["K"], case["N"]
    dtype = TYPES[case["type"]]
    # activations: rows of different size, a few channels far larger than the others
    channel = torch.exp(0.5 * normal(K)) * torch.where(torch.rand(K, generator=g, device=DEVICE) < 0.005, 10.0, 1.0)
    x = (normal(M, K) * channel * torch.exp(0.3 * normal(M, 1))).to(dtype)
    w = normal(N, K) / math.sqrt(K)
    q_w = w.abs().amax(1) / 127
    z_w = torch.clamp(torch.round(w / q_w[:, None]), -128, 127).to(torch.int8)
    s = dict(case=case, x=x, z_w=z_w, q_w=q_w, bias=0.1 * normal(N) if case["bias"] else None,
             y=torch.empty(M, N, dtype=dtype, device=DEVICE))
    if own:
        from paper_1805_08691_amd import binding as B
        s["w"] = B.linear_pack(z_w)
        s["workspace"] = B.linear_workspace(M, N, K, DEVICE)
    return s


def _prepare_pages(case, g, normal):
    before, added = _requests(case)
    page, n = case["page"], case["requests"]
    width = _pages(case["longest"] + max(case["added"], 1), page)
    have = sum(_pages(t, page) for t in before)
    need = sum(_pages(t + a, page) - _pages(t, page) for t, a in zip(before, added))
    order = torch.randperm(have + need + case["spare"], generator=g, device=DEVICE).to(torch.int32)
    lengths, more = _ints(before), _ints(added)
    held = _pages(lengths.long(), page)
    cols = torch.arange(width, device=DEVICE)
    at = (held.cumsum(0) - held)[:, None] + cols
    table = torch.where(cols < held[:, None], order[at.clamp(max=order.numel() - 1)], -1).to(torch.int32)
    tokens = sum(added)
    room = tokens + 1 + tokens // 16           # a fixed number of slots, as a recorded step has it
    return dict(case=case, lengths=lengths, added=more, free=order[have:].contiguous(), table=table.contiguous(),
                slots=torch.empty(room, dtype=torch.int64, device=DEVICE),
                positions=torch.empty(room, dtype=torch.int32, device=DEVICE),
                starts=torch.empty(n + 1, dtype=torch.int32, device=DEVICE),
                grown=torch.empty(n, dtype=torch.int32, device=DEVICE),
                counts=torch.empty(3, dtype=torch.int32, device=DEVICE))


def _tables(total, page, g):
    """Block table of requests of these lengths over a shuffled pool, and the pool's size."""
    held = [_pages(t, page) for t in total]
    pool, width = sum(held) + 3, max(max(held), 1)
    order = torch.randperm(pool, generator=g, device=DEVICE).to(torch.int32)
    h = _ints(held, torch.int64)
    cols = torch.arange(width, device=DEVICE)
    at = (h.cumsum(0) - h)[:, None] + cols
    return torch.where(cols < h[:, None], order[at.clamp(max=pool - 1)], -1).to(torch.int32).contiguous(), pool


def _prepare_cache(case, g, normal):
    before, added = _requests(case)
    page, H, D, T = case["page"], case["heads"], case["D"], case["tokens"]
    table, pool = _tables([t + a for t, a in zip(before, added)], page, g)
    t0, n = _ints(before, torch.int64), _ints(added, torch.int64)
    row = torch.repeat_interleave(torch.arange(len(added), device=DEVICE), n)
    pos = t0[row] + torch.arange(T, device=DEVICE) - (n.cumsum(0) - n)[row]
    slots = table[row, pos // page].long() * page + pos % page
    # keys and values as a joint projection leaves them: slices of its rows, two query heads to a key head
    joint = (normal(T, 4 * H, D) * torch.exp(0.5 * normal(1, 4 * H, D))).to(TYPES[case["type"]])
    return dict(case=case, k=joint[:, 2 * H:3 * H], v=joint[:, 3 * H:], slots=slots,
                cache=torch.zeros(pool, H, page // 16, 18 * D, dtype=torch.uint8, device=DEVICE),
                k_out=torch.empty(T, H, D, dtype=joint.dtype, device=DEVICE),
                v_out=torch.empty(T, H, D, dtype=joint.dtype, device=DEVICE))


def _prepare_attend(case, g, normal):
    before, added = _requests(case)
    total = [t + a for t, a in zip(before, added)]
    page, H, D, R = case["page"], case["heads"], case["D"], case["ratio"]
    table, pool = _tables(total, page, g)
    cache = torch.empty(pool, H, page // 16, 18 * D, dtype=torch.uint8, device=DEVICE)
    channel = torch.exp(0.5 * normal(2, H, 1, 1, D))
    step = max(1, (1 << 27) // (H * page * D))
    for a in range(0, pool, step):                       # (in pieces, for the memory of their fp32 values)
        n = min(step, pool - a)
        kv = normal(2, n, H, page // 16, 16, D) * channel[:, None]
        cache[a:a + n] = _pack(kv[0], kv[1])
    T = sum(added)
    q = (1.5 * normal(T, H * R, D)).to(TYPES[case["type"]])
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    s = dict(case=case, q=q, cache=cache, table=table, lengths=_ints(total), scale=D ** -0.5,
             starts=None if case["added"] == 1 else _ints(starts), added=added, total=total, out=torch.empty_like(q))
    if own:
        from paper_1805_08691_amd import binding as B
        s["workspace"] = B.kv4_attend_workspace(q, cache, len(total), max(total), DEVICE)
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    return globals()[("_own_" if own else "_plain_") + s["case"]["kind"]](s)


def _own_linear(s):
    from paper_1805_08691_amd import binding as B
    return B.linear(s["x"], s["w"], s["q_w"], s["bias"], out=s["y"], workspace=s["workspace"])


def _own_pages(s):
    from paper_1805_08691_amd import binding as B
    return B.page_tables(s["lengths"], s["added"], s["case"]["page"], s["free"], s["table"], s["slots"],
                         s["positions"], s["starts"], s["grown"], s["counts"])


def _own_cache(s):
    from paper_1805_08691_amd import binding as B
    B.kv4_write(s["cache"], s["k"], s["v"], s["slots"])
    return B.kv4_read(s["cache"], s["slots"], s["k_out"], s["v_out"])


def _own_attend(s):
    from paper_1805_08691_amd import binding as B
    return B.kv4_attend(s["q"], s["cache"], s["table"], s["lengths"], s["starts"], s["scale"],
                        window=s["case"]["window"], out=s["out"], workspace=s["workspace"])


# ------------------------------------------------------------------------------ the plain forms
def _plain_linear(s):
    x = s["x"].float()
    q_x = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(1, keepdim=True) / 127
    q_x = torch.where(q_x > 0, q_x, 1.0)
    z = torch.clamp(torch.round(x / q_x), -128, 127)
    z = torch.where(torch.isnan(z), 0.0, z)
    y = (z @ s["z_w"].float().t()) * (q_x * s["q_w"])
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype)


def _plain_pages(s):
    page, table, free = s["case"]["page"], s["table"], s["free"]
    room, width = s["slots"].numel(), table.shape[1]
    length, added = s["lengths"].clamp(min=0).long(), s["added"].clamp(min=0).long()
    ends = added.cumsum(0)
    starts = ends - added
    have, total = _pages(length, page), _pages(length + added, page)
    refused = (total > width) | (ends > room)
    need = torch.where(refused, 0, total - have)
    upto = need.cumsum(0)
    fits = ~refused & ((need == 0) | (upto <= free.numel()))
    cols = torch.arange(width, device=table.device)
    taken = fits[:, None] & (cols >= have[:, None]) & (cols < total[:, None])
    at = (upto - need - have)[:, None] + cols
    table = torch.where(taken, free[at.clamp(0, free.numel() - 1)], table)
    token = torch.arange(room, device=table.device)
    row = torch.searchsorted(ends, token, right=True)
    given = row < ends.numel()
    row = row.clamp(max=ends.numel() - 1)
    given = given & fits[row]
    position = length[row] + token - starts[row]
    slot = table[row, (position // page).clamp(0, width - 1)].long() * page + position % page
    counts = torch.stack([torch.where(fits, need, 0).sum(), ends[-1], (~fits).sum()])
    return dict(table=table, slots=torch.where(given, slot, -1),
                positions=torch.where(given, position, -1).to(torch.int32),
                starts=torch.cat([starts, ends[-1:]]).to(torch.int32),
                lengths=(length + torch.where(fits, added, 0)).to(torch.int32), counts=counts.to(torch.int32))


def _codes(x):
    """fp32 [..., D] -> codes plus 8 (uint8, [..., D / 32, 32]) and factors (binary16, [..., D / 32])."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    q = (torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1) / 7).clamp(max=8188.0).half()
    q = torch.where(q == 0, torch.ones_like(q), q)
    z = torch.clamp(torch.round(x / q.float()[..., None]), -8, 7)
    return (torch.where(torch.isnan(z), 0.0, z) + 8).to(torch.uint8), q


def _as_bytes(f16):
    return f16.contiguous().view(torch.uint8)


def _pack(k, v):
    """Values [..., 16, D] of whole sixteens of tokens -> their bytes [..., 18 D]."""
    zk, qk = _codes(k)
    zv, qv = _codes(v)
    lead, G = k.shape[:-2], k.shape[-1] // 32
    zk = zk.reshape(*lead, 16, G, 4, 4, 2).transpose(-4, -3)                  # token, j, g, byte, half
    kc = (zk[..., 0] | zk[..., 1] << 4).reshape(*lead, -1)
    zv = zv.reshape(*lead, 16, G, 2, 16).movedim(-4, -1)                      # g, half, r, token
    vc = (zv[..., 0, :, :] | zv[..., 1, :, :] << 4).reshape(*lead, -1)
    qv = qv.transpose(-1, -2).reshape(*lead, G, 4, 4)[..., SWAP]
    return torch.cat([kc, vc, _as_bytes(qk).reshape(*lead, -1), _as_bytes(qv).reshape(*lead, -1)], -1)


def _unpack(c):
    """Bytes [..., 18 D] -> fp32 keys and values [..., 16, D]."""
    lead, G = c.shape[:-1], c.shape[-1] // 576
    kc, vc, kf, vf = c.split([256 * G, 256 * G, 32 * G, 32 * G], -1)
    kc = kc.reshape(*lead, 16, 4, G, 4).transpose(-3, -2)                     # token, g, j, byte
    k = torch.stack([kc & 15, kc >> 4], -1).reshape(*lead, 16, G, 32).float() - 8
    k = k * kf.contiguous().view(torch.float16).reshape(*lead, 16, G, 1).float()
    vc = vc.reshape(*lead, G, 1, 16, 16)
    v = torch.cat([vc & 15, vc >> 4], -3).reshape(*lead, G, 32, 16).float() - 8   # g, channel, token
    q = vf.contiguous().view(torch.float16).reshape(*lead, G, 4, 4)[..., SWAP].reshape(*lead, G, 1, 16)
    v = (v * q.float()).movedim(-1, -3)
    return k.reshape(*lead, 16, -1), v.reshape(*lead, 16, -1)


def _plain_cache(s):
    cache, slots, page = s["cache"], s["slots"], s["case"]["page"]
    H, D = s["case"]["heads"], s["case"]["D"]
    G, dev = D // 32, cache.device
    zk, qk = _codes(s["k"].float())
    zv, qv = _codes(s["v"].float())
    T = slots.numel()
    # where the sixteen of a token's head lies, and each of its bytes inside
    token = (slots % 16)[:, None, None]
    base = ((slots // page)[:, None] * H + torch.arange(H, device=dev)) * (page // 16) + (slots % page // 16)[:, None]
    base = (base * 18 * D)[..., None]
    zk = zk.reshape(T, H, G, 4, 4, 2).transpose(2, 3)
    zv = zv.reshape(T, H, G, 2, 16)
    swap = torch.tensor(SWAP, device=dev)
    group, two = torch.arange(G, device=dev), torch.arange(2, device=dev)
    at = [base + token * 16 * G + torch.arange(16 * G, device=dev),
          base + 256 * G + torch.arange(16 * G, device=dev) * 16 + token,
          base + 512 * G + token * 2 * G + torch.arange(2 * G, device=dev),
          base + 544 * G + ((group * 16)[:, None] + two.new_zeros(2)).reshape(-1) * 2 +
          (token - token % 4 + swap[token % 4]) * 2 + two.repeat(G)]
    of = [(zk[..., 0] | zk[..., 1] << 4).reshape(T, H, -1), (zv[..., 0, :] | zv[..., 1, :] << 4).reshape(T, H, -1),
          _as_bytes(qk), _as_bytes(qv)]
    cache.view(-1)[torch.cat(at, -1)] = torch.cat(of, -1)
    # the values that it now holds
    k, v = _unpack(cache.view(-1, H, page // 16, 18 * D)[slots // page, :, slots % page // 16])
    row = torch.arange(T, device=dev)
    return k[row, :, slots % 16].to(s["k"].dtype), v[row, :, slots % 16].to(s["k"].dtype)


def _plain_attend(s):
    case, cache, table = s["case"], s["cache"], s["table"]
    page, H, R, D = case["page"], case["heads"], case["ratio"], case["D"]
    n, most, longest, dev = len(s["total"]), max(s["added"]), max(s["total"]), cache.device
    # keys and values of every request, as long as the longest one
    chunk = torch.arange(0, longest, 16, device=dev)
    at = table[:, chunk // page].clamp(min=0).long()
    k, v = _unpack(cache[at, :, (chunk % page // 16).expand(n, -1)])          # request, sixteen, head, token, D
    k = k.permute(0, 2, 4, 1, 3).reshape(n, H, D, -1)
    v = v.transpose(1, 2).reshape(n, H, -1, D)
    length = s["lengths"].long()
    starts = torch.arange(n + 1, device=dev) if s["starts"] is None else s["starts"].long()
    added = starts[1:] - starts[:-1]
    i = torch.arange(most, device=dev)
    row = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][row].float().reshape(n, most, H, R, D).permute(0, 2, 1, 3, 4).reshape(n, H, most * R, D)
    score = (q @ k).reshape(n, H, most, R, -1) * s["scale"]
    position = (length - added)[:, None, None] + i[:, None]
    j = torch.arange(k.shape[-1], device=dev)
    seen = (j <= position) & (j < length[:, None, None])
    if case["window"]:
        seen = seen & (j > position - case["window"])
    seen = seen[:, None, :, None]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = p.reshape(n, H, most * R, -1) @ v
    o = o.reshape(n, H, most, R, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(n * most, H * R, D)
    given = (i < added[:, None]).reshape(-1)
    return o[given].to(s["q"].dtype)


# ------------------------------------------------------------------------------ work, and the 64-bit outputs
def work(case):
    if case["kind"] == "linear":
        M, K, N, e = case["M"], case["K"], case["N"], BYTES[case["type"]]
        return {"bytes": e * M * K + N * K + 4 * N * (2 if case["bias"] else 1) + e * M * N, "flops": 2 * M * N * K}
    before, added = _requests(case)
    if case["kind"] == "pages":
        page, tokens = case["page"], sum(added)
        taken = sum(_pages(t + a, page) - _pages(t, page) for t, a in zip(before, added))
        room = tokens + 1 + tokens // 16
        return {"bytes": 16 * len(added) + 8 * taken + 12 * room, "flops": 4 * room}
    H, D = case["heads"], case["D"]
    e = BYTES[case["type"]]
    if case["kind"] == "cache":
        values = 2 * case["tokens"] * H * D
        return {"bytes": values * (2 * e) + 2 * values * 9 // 16 + 8 * case["tokens"], "flops": 6 * values}
    keys = pairs = 0
    for t, a in zip(before, added):
        first = max(0, t + 1 - case["window"]) if case["window"] else 0
        keys += t + a - first
        full = [min(t + 1 + i, case["window"] or t + a) for i in range(a)]
        pairs += sum(full)
    R = case["ratio"]
    return {"bytes": keys * H * D * 9 // 8 + 2 * e * sum(added) * H * R * D, "flops": 4 * pairs * H * R * D}


def exact(case, seed):
    if case["kind"] == "pages":
        return None
    return globals()["_exact_" + case["kind"]](prepare(case, seed))


def _exact_linear(s):
    x = s["x"].double()
    largest = x.abs().max(dim=1).values.float() / 127            # the factor is held in 32 bits
    q_x = largest.masked_fill(largest == 0, 1.0).double()
    z = x.div(q_x[:, None]).round_().clamp_(-128, 127)
    y = torch.mm(z, s["z_w"].double().t()).mul_(q_x[:, None]).mul_(s["q_w"].double())
    return y if s["bias"] is None else y.add_(s["bias"].double())


def _grid64(x):
    """What Eq. Q and Eq. D leave of fp64 values [..., D] at p = 3 with a factor for 32 channels in 16 bits."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], 32):
        part = x[..., c:c + 32]
        q = (part.abs().max(dim=-1, keepdim=True).values.float() / 7).clamp(max=8188.0).half().double()
        q = q.masked_fill(q == 0, 1.0)
        out[..., c:c + 32] = part.div(q).round_().clamp_(-8, 7) * q
    return out


def _exact_cache(s):
    return _grid64(s["k"].double()), _grid64(s["v"].double())


def _held64(cache, pages, length, head, D):
    """Keys and values of one request's head in 64 bits, byte by byte from the layout."""
    G, dev = D // 32, cache.device
    page = cache.shape[2] * 16
    t = torch.arange(length, device=dev)
    block = cache[pages.long()[t // page], head, t % page // 16]                 # (a sixteen's bytes for each token)
    t = (t % 16)[:, None]
    c = torch.arange(D, device=dev)[None]
    g, j, i, r = c // 32, c % 32 // 8, c % 8, c % 16

    def half(at):
        lo, hi = block.gather(1, at).to(torch.int16), block.gather(1, at + 1).to(torch.int16)
        return (lo | hi << 8).view(torch.float16).double()

    code = block.gather(1, t * 16 * G + j * 4 * G + 4 * g + i // 2) >> (4 * (i % 2)).to(torch.uint8) & 15
    k = (code.double() - 8) * half(512 * G + 2 * (t * G + g))
    code = block.gather(1, 256 * G + (g * 16 + r) * 16 + t) >> (c % 32 // 16 * 4).to(torch.uint8) & 15
    place = t - t % 4 + torch.tensor(SWAP, device=dev)[t % 4]
    v = (code.double() - 8) * half(544 * G + 2 * (g * 16 + place))
    return k, v


def _exact_attend(s):
    case = s["case"]
    H, R, D = case["heads"], case["ratio"], case["D"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    at = 0
    for b, (n, L) in enumerate(zip(s["added"], s["total"])):
        for h in range(H):
            k, v = _held64(s["cache"], s["table"][b], L, h, D)
            q = s["q"][at:at + n, h * R:(h + 1) * R].double()
            score = torch.matmul(q.reshape(n * R, D), k.t()).mul_(s["scale"]).reshape(n, R, L)
            ahead = torch.arange(L, device=k.device)[None] - (torch.arange(n, device=k.device) + L - n)[:, None]
            hidden = ahead > 0
            if case["window"]:
                hidden |= ahead <= -case["window"]
            score.masked_fill_(hidden[:, None], -math.inf)
            out[at:at + n, h * R:(h + 1) * R] = torch.matmul(torch.softmax(score, -1).reshape(n * R, L), v).reshape(n, R, D)
        at += n
    return out
