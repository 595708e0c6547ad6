"""The trusted half of a decode step, operator by operator, as cases that can be timed.

Between two encrypted products the trusted domain works on plaintext: it appends the new keys and values to a cache held
in 4 bits, attends over that cache, moves its pages about when sequences fork, end or are compacted, and projects the last
hidden state onto the vocabulary with 4-bit weights.  A case is one pass of one of these.  Its fields:

  op       "linear"   y = x W^T, W in 4 bits with group scales
           "attend"   attention over the cache, one token a sequence or a chunk of them
           "store"    new keys and values quantised into the cache, then read back as the values that it holds
           "fork"     pages of the cache, first form: losing branches freed, the surviving sequences forked again
           "compact"  pages of the cache, second form: live pages moved to the front of the pool
  linear:  n (rows of x), d_in, d_out, group, offsets, x and y (types)
  others:  seqs, heads (query heads), kv_heads, head_dim, group, page (tokens), layers, longest and spread (lengths
           lie between longest * spread and longest), tokens (new or querying tokens of a sequence, at most), window, type

Activations are N(0, 1) with a few channels several times larger, as the hidden states of decoders have them.

Layout of the 4-bit matrix: codes [d_out][row_bytes], column c in the low (even c) or high half of byte c/2, rows padded to
16 bytes; scales, and offsets where there are any, fp16 [d_out][groups padded to a multiple of 8]; a weight is
scale * (code - 8) + offset.  Layout of the cache: pool [layers][pages][kv heads][page/16] of sub-blocks of 16 tokens: key codes,
key parameters, value codes, value parameters, in the order in which matrix instructions take them (_keys and _values below);
a value is low + scale * code, both fp16, per token, head and group of channels.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _linear(name, n, d_in, d_out, group, offsets, x, y):
    return dict(name=name, op="linear", n=n, d_in=d_in, d_out=d_out, group=group, offsets=offsets, x=x, y=y)


def _cached(name, op, seqs, heads, kv_heads, head_dim, group, page, layers, longest, spread, tokens, window, type):
    return dict(name=name, op=op, seqs=seqs, heads=heads, kv_heads=kv_heads, head_dim=head_dim, group=group, page=page, layers=layers,
                longest=longest, spread=spread, tokens=tokens, window=window, type=type)


def listed():
    return [
        # one projection of a 124M-parameter decoder for one token: a few microseconds, latency is everything
        _linear("linear_768x2304", 1, 768, 2304, 128, False, "bf16", "bf16"),
        # its vocabulary projection: an odd number of rows, logits in 32 bits
        _linear("linear_768x50257", 1, 768, 50257, 64, False, "bf16", "fp32"),
        # down projection of an 8B model's layer for a batch of eight sequences, asymmetric weights
        _linear("linear_14336x4096_n8", 8, 14336, 4096, 32, True, "fp16", "fp16"),
        # vocabulary projection of that model for 32 sequences: the largest
        _linear("linear_4096x128256_n32", 32, 4096, 128256, 128, False, "bf16", "fp32"),
        # one layer of the 124M decoder, one sequence in the middle of its context
        _cached("attend_12h_64_len700", "attend", 1, 12, 12, 64, 64, 16, 2, 700, 1.0, 1, 0, "bf16"),
        # one layer of a 0.6B model, 32 sequences of very different lengths, finest groups
        _cached("attend_16h_b32_ragged", "attend", 32, 16, 8, 128, 32, 64, 1, 8000, 0.02, 1, 0, "bf16"),
        # one layer of an 8B model, one sequence with the longest context
        _cached("attend_32h_len131072", "attend", 1, 32, 8, 128, 128, 64, 1, 131072, 1.0, 1, 0, "bf16"),
        # chunks of up to 33 tokens (drafts being verified, prompts taken piece by piece) behind a sliding window
        _cached("attend_16h_chunk33_window", "attend", 5, 16, 8, 128, 64, 32, 1, 2500, 0.3, 33, 1000, "fp16"),
        # a decode step's new keys and values, 48 sequences
        _cached("store_b48_step", "store", 48, 16, 8, 128, 32, 64, 1, 2000, 0.1, 1, 0, "bf16"),
        # two prompts at once
        _cached("store_prompts", "store", 2, 32, 8, 128, 64, 64, 1, 4099, 0.9, 4001, 0, "fp16"),
        # sampling in branches: 24 branches end and 24 sequences fork, all layers of the 0.6B model
        _cached("fork_b24", "fork", 24, 16, 8, 128, 64, 32, 28, 1000, 0.2, 0, 0, "bf16"),
        # a pool after many sequences came and went, one in three pages free
        _cached("compact_pool", "compact", 40, 16, 8, 128, 64, 64, 28, 2000, 0.2, 0, 0, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the same ranges."""
    op = rng.choice(["linear", "linear", "linear", "attend", "attend", "attend", "store", "fork", "compact"])
    if op == "linear":
        n, d_in = _log_int(rng, 1, 64), _log_int(rng, 64, 14336)
        if rng.random() < 0.5:
            d_in = max(64, d_in // 64 * 64)
        d_out = _log_int(rng, 16, max(64, min(128256, 16 * 10 ** 9 // (n * d_in), 5 * 10 ** 8 // d_in)))
        case = _linear(None, n, d_in, d_out, rng.choice([32, 64, 128]), rng.random() < 0.4, rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                       rng.choice(["bf16", "fp32", "fp16"]))
    else:
        head_dim = rng.choice([64, 128])
        kv_heads = rng.choice([1, 2, 4, 8, 8, 12])
        heads = kv_heads * rng.choice([1, 2, 4, 7, 8])
        group = rng.choice([g for g in (32, 64, 128) if g <= head_dim])
        page = rng.choice([16, 32, 64, 128])
        seqs = _log_int(rng, 1, 64)
        if op == "attend":
            tokens = rng.choice([1, 1, 1, _log_int(rng, 2, 48)])
            longest = _log_int(rng, 1, max(64, min(131072, 2 ** 24 // (seqs * kv_heads), 2 ** 27 // (seqs * heads * tokens))))
            window = rng.choice([0, 0, 0, _log_int(rng, 1, longest)])
        elif op == "store":
            tokens, window = _log_int(rng, 1, 2000), 0
            seqs = max(1, min(seqs, 8000 // tokens))
            longest = tokens + _log_int(rng, 1, 2000)
        else:
            tokens, window, longest = 0, 0, _log_int(rng, 8, 2000)
        layers = rng.choice([1, 2]) if tokens else _log_int(rng, 1, 28)
        case = _cached(None, op, seqs, heads, kv_heads, head_dim, group, page, layers, longest, rng.choice([1.0, 0.5, 0.05]),
                       min(tokens, longest), window, rng.choice(["bf16", "fp16"]))
    del case["name"]
    return case


def _pad(n, m):
    return -(-n // m) * m


# ---------------------------------------------------------------------------------------------- inputs

def _activations(gen, *shape):
    x = torch.randn(shape, generator=gen, device="cuda")
    big = torch.rand(shape[-1], generator=gen, device="cuda") < 0.02
    return torch.where(big, 6 * x, x)


def _nibbles(c):
    """[..., 2 n] values below 16 -> [..., n] bytes, the even one in the low half."""
    return (c[..., 0::2] | (c[..., 1::2] << 4)).contiguous()


def _groups(x, group):
    """(codes, scale, low) of [..., channels]: what the cache holds for x.  Decided in 64 bits: a value next to a border of two
    codes goes to the same side everywhere.  Values beyond +-61440 are held as that."""
    x = x.double().clamp(-61440.0, 61440.0).unflatten(-1, (-1, group))
    low, high = x.amin(-1), x.amax(-1)
    scale, low = ((high - low) / 15).float().half(), low.float().half()
    s, m = scale.double().unsqueeze(-1), low.double().unsqueeze(-1)
    code = torch.where(s > 0, (x - m) / s, 0.0).round().clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), scale, low


def _sub_blocks(k, v, group):
    """[..., page/16, 16, D] keys and values -> [..., page/16, bytes]: the sub-blocks that hold them."""
    lead, D = k.shape[:-2], k.shape[-1]
    kc, ks, km = _groups(k, group)
    vc, vs, vm = _groups(v, group)
    n = len(lead)
    kc = kc.view(*lead, 2, 8, D // 64, 2, 4, 8).permute(*range(n), n + 2, n + 1, n + 4, n + 3, n, n + 5)
    kp = torch.stack([ks, km], -1).view(*lead, 2, 8, -1, 2).transpose(n, n + 1)
    vc = vc.view(*lead, 2, 4, 2, D // 64, 4, 2, 8).permute(*range(n), n + 3, n + 6, n + 1, n + 4, n + 2, n, n + 5)
    vp = torch.stack([vs, vm], -1).view(*lead, 2, 4, 2, -1, 2).permute(*range(n), n + 3, n + 1, n + 4, n, n + 2)
    parts = [_nibbles(kc).flatten(n), kp.contiguous().flatten(n).view(torch.uint8), _nibbles(vc).flatten(n), vp.contiguous().flatten(n).view(torch.uint8)]
    return torch.cat(parts, -1)


def _block_bytes(case):
    return (16 * case["head_dim"] + 128 * (case["head_dim"] // case["group"])) * (case["page"] // 16)


class _State:
    """What a program keeps between calls."""


def _prepare_linear(s, case, gen):
    n, d_in, d_out, group = case["n"], case["d_in"], case["d_out"], case["group"]
    groups, cols = -(-d_in // group), _pad(d_in, 32)
    s.codes = torch.empty((d_out, cols // 2), dtype=torch.uint8, device="cuda")
    s.scales = torch.zeros((d_out, _pad(groups, 8)), dtype=torch.float16, device="cuda")
    s.offsets = torch.zeros_like(s.scales) if case["offsets"] else None
    for at in range(0, d_out, 16384):                        # in pieces: a vocabulary's weights in 64 bits are large
        rows = min(16384, d_out - at)
        w = torch.randn((rows, groups * group), generator=gen, device="cuda") * 0.02
        w[:, d_in:] = 0
        w = w.view(rows, groups, group)
        if case["offsets"]:
            low, high = w.amin(-1), w.amax(-1)
            scale = ((high - low) / 15).half()
            offset = (low + 8 * scale.float()).half()
            s.offsets[at:at + rows, :groups] = offset
        else:
            scale, offset = (w.abs().amax(-1) / 7).half(), None
        s.scales[at:at + rows, :groups] = scale
        code = (w - offset.float().unsqueeze(-1) if case["offsets"] else w) / scale.float().unsqueeze(-1).clamp(min=1e-7)
        code = (code.round() + 8).clamp(0, 15).to(torch.uint8).flatten(1)
        code = torch.nn.functional.pad(code, (0, max(0, cols - groups * group)))[:, :cols]
        s.codes[at:at + rows] = _nibbles(code)
    s.x = _activations(gen, n, d_in).to(TYPES[case["x"]])
    s.y = torch.empty((n, d_out), dtype=TYPES[case["y"]], device="cuda")


def _spread(low, high, n):
    """n whole numbers between low and high, the last of them high: the same for every seed, so that outputs keep their shapes."""
    return [low + int((0.618 * (i + 1) % 1) * (high - low + 1)) for i in range(n - 1)] + [high]


def _lengths(case):
    return _spread(max(case["tokens"], int(case["longest"] * case["spread"]), 1), case["longest"], case["seqs"])


def _counts(case):
    """New or querying tokens of each sequence."""
    return _spread(1, case["tokens"], case["seqs"]) if case["tokens"] else []


def _prepare_cache(s, case, gen):
    page, op, n = case["page"], case["op"], case["seqs"]
    counts = torch.tensor(_counts(case), device="cuda")
    lens = torch.tensor(_lengths(case), device="cuda")
    s.max_pages = -(-case["longest"] // page)
    need = -(-lens // page)
    used = int(need.sum())
    if op == "compact":                                     # a third of the pool is free, the live pages lie anywhere
        s.n_pages, s.n_seqs = used + used // 2 + 3, n
    elif op == "fork":                                      # parents, and a branch of each
        s.n_pages, s.n_seqs = used + 2 * n + 5, 2 * n
    else:
        s.n_pages, s.n_seqs = used + 3, n
    order = torch.randperm(s.n_pages, generator=gen, device="cuda").int()
    s.tables = torch.full((s.n_seqs, s.max_pages), -1, dtype=torch.int32, device="cuda")
    slot = torch.arange(s.max_pages, device="cuda").expand(n, -1)
    here = slot < need[:, None]
    s.tables[:n][here] = order[:used]
    s.lengths = torch.zeros(s.n_seqs, dtype=torch.int32, device="cuda")
    s.lengths[:n] = lens.int()
    s.refs = torch.zeros(s.n_pages, dtype=torch.int32, device="cuda")
    s.refs[order[:used].long()] = 1
    heads, D = case["kv_heads"], case["head_dim"]
    s.pool = torch.empty((case["layers"], s.n_pages, heads, _block_bytes(case)), dtype=torch.uint8, device="cuda")
    if op == "fork":
        full, rest = lens // page, (lens % page > 0)
        whole = slot < full[:, None]
        s.tables[n:] = torch.where(whole, s.tables[:n], -1)
        s.refs.index_add_(0, s.tables[:n][whole].long(), torch.ones_like(s.tables[:n][whole]))
        tail = order[used:used + int(rest.sum())]
        s.tables[n:][rest, full[rest]] = tail
        s.refs[tail.long()] = 1
        s.lengths[n:] = lens.int()
        s.parents = torch.arange(n, dtype=torch.int32, device="cuda")
        s.children = s.parents + n
    if op in ("fork", "compact"):                           # pages are moved whatever they hold
        s.pool.copy_(torch.randint(0, 256, s.pool.shape, generator=gen, device="cuda", dtype=torch.uint8))
        s.new_tables, s.new_refs = torch.empty_like(s.tables), torch.empty_like(s.refs)
        s.n_live = torch.zeros(1, dtype=torch.int32, device="cuda")
        return
    for layer in range(case["layers"]):
        for at in range(0, s.n_pages, max(1, 2 ** 25 // (heads * page * D))):
            some = s.pool[layer, at:at + max(1, 2 ** 25 // (heads * page * D))]
            k, v = (_activations(gen, some.shape[0], heads, page // 16, 16, D).to(TYPES[case["type"]]) for _ in range(2))
            some.copy_(_sub_blocks(k, v, case["group"]).flatten(-2))
    s.layer = case["layers"] - 1
    s.starts = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).int()
    s.rows = int(counts.sum())
    # queries, keys and values of a token beside each other, as the product before hands them over
    qkv = _activations(gen, s.rows, case["heads"] + 2 * heads, D).to(TYPES[case["type"]])
    s.q, s.k, s.v = qkv.split([case["heads"], heads, heads], 1)
    s.out = torch.empty((s.rows, case["heads"], D), dtype=TYPES[case["type"]], device="cuda")
    s.k_out, s.v_out = (torch.empty((s.rows, heads, D), dtype=torch.float32, device="cuda") for _ in range(2))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = _State()
    s.case, s.device = case, torch.cuda.current_device()
    (_prepare_linear if case["op"] == "linear" else _prepare_cache)(s, case, gen)
    torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------------------------------------- the framework's calls

_trusted = {}


def _context(s):
    """The context that a program's trusted half has on the stream in which its inputs are used: one for each device and stream."""
    key = s.device, torch._C._cuda_getCurrentRawStream(s.device)
    held = _trusted.get(key)
    if held is None:
        from paper_2606_17421_b200 import bifrost as bf
        with torch.cuda.device(s.device):
            held = _trusted[key] = bf, bf.bf_trusted_create(0, key[1])
    return held


def _cache(bf, s):
    c = s.case
    return bf.bf_kv4_cache.of(s.pool, s.tables, s.lengths, s.refs, head_dim=c["head_dim"], group=c["group"], page_tokens=c["page"])


def _own_linear(s):
    bf, t = _context(s)
    W = bf.bf_q4_matrix.of(s.codes, s.scales, s.offsets, s.case["d_in"], s.case["group"])
    bf.bf_q4_linear(t, W, bf.bf_rows.of(s.x), s.case["n"], bf.bf_rows.of(s.y))
    return {"y": s.y}


def _own_attend(s):
    bf, t = _context(s)
    c = s.case
    starts = s.starts if c["tokens"] > 1 else None          # one token a sequence needs no list of starts
    bf.bf_kv4_attention(t, _cache(bf, s), s.layer, None, starts, c["seqs"], c["tokens"], c["longest"], bf.bf_rows.of(s.q), c["heads"],
                        bf.bf_rows.of(s.out), c["head_dim"] ** -0.5, c["window"], None)
    return {"out": s.out}


def _own_store(s):
    bf, t = _context(s)
    c = s.case
    cache = _cache(bf, s)
    starts = s.starts if c["tokens"] > 1 else None
    bf.bf_kv4_append(t, cache, s.layer, None, starts, c["seqs"], c["tokens"], bf.bf_rows.of(s.k), bf.bf_rows.of(s.v))
    bf.bf_kv4_read(t, cache, s.layer, None, starts, None, c["seqs"], c["tokens"], bf.bf_rows.of(s.k_out), bf.bf_rows.of(s.v_out))
    return {"k": s.k_out, "v": s.v_out}


def _own_fork(s):
    bf, t = _context(s)
    cache = _cache(bf, s)
    bf.bf_kv4_free(t, cache, s.children, s.case["seqs"])
    bf.bf_kv4_fork(t, cache, s.parents, s.children, s.case["seqs"])
    return {"tables": s.tables, "lengths": s.lengths, "refs": s.refs, "pool": s.pool}


def _own_compact(s):
    bf, t = _context(s)
    bf.bf_kv4_compact(t, _cache(bf, s), s.new_tables, s.new_refs, s.n_live)
    return {"tables": s.new_tables, "refs": s.new_refs, "n_live": s.n_live, "pool": s.pool}


# ---------------------------------------------------------------------------------------------- the plain form

def _halves(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _plain_linear(s):
    c = s.case
    code = _halves(s.codes)[:, :c["d_in"]].float()
    scale = s.scales.float().repeat_interleave(c["group"], 1)[:, :c["d_in"]]
    w = (code - 8) * scale
    if s.offsets is not None:
        w = w + s.offsets.float().repeat_interleave(c["group"], 1)[:, :c["d_in"]]
    return {"y": (s.x.float() @ w.t()).to(s.y.dtype)}


def _keys(case, sub):
    """[..., bytes of a sub-block] -> [..., 16, D] keys, and _values the values, in 32 bits."""
    D, G, n = case["head_dim"], case["head_dim"] // case["group"], sub.dim() - 1
    code = _halves(sub[..., :8 * D]).view(*sub.shape[:-1], D // 64, 8, 4, 2, 2, 8).permute(*range(n), n + 4, n + 1, n, n + 3, n + 2, n + 5)
    par = sub[..., 8 * D:8 * D + 64 * G].contiguous().view(torch.float16).view(*sub.shape[:-1], 8, 2, G, 2).transpose(n, n + 1).float()
    par = par.reshape(*sub.shape[:-1], 16, G, 1, 2)
    return (code.reshape(*sub.shape[:-1], 16, G, -1).float() * par[..., 0] + par[..., 1]).flatten(-2)


def _values(case, sub):
    D, G, n = case["head_dim"], case["head_dim"] // case["group"], sub.dim() - 1
    sub = sub[..., 8 * D + 64 * G:]
    code = _halves(sub[..., :8 * D]).view(*sub.shape[:-1], D // 64, 8, 4, 4, 2, 2, 2)
    code = code.permute(*range(n), n + 5, n + 2, n + 4, n, n + 3, n + 6, n + 1)
    par = sub[..., 8 * D:].contiguous().view(torch.float16).view(*sub.shape[:-1], G, 4, 2, 2, 2).permute(*range(n), n + 3, n + 1, n + 4, n, n + 2)
    par = par.float().reshape(*sub.shape[:-1], 16, G, 1, 2)
    return (code.reshape(*sub.shape[:-1], 16, G, -1).float() * par[..., 0] + par[..., 1]).flatten(-2)


def _places(s):
    """Of every row of queries or new tokens: its sequence, its number there, its position."""
    row = torch.arange(s.rows, device="cuda")
    seq = torch.searchsorted(s.starts[1:].long(), row, right=True)
    nth = row - s.starts[seq].long()
    return seq, nth, s.lengths[seq].long() - (s.starts[seq + 1] - s.starts[seq]).long() + nth


def _plain_attend(s):
    c = s.case
    D, page, Hk = c["head_dim"], c["page"], c["kv_heads"]
    seq, nth, pos = _places(s)
    blocks = s.pool[s.layer][s.tables.long().clamp(min=0)].unflatten(-1, (page // 16, -1))       # [seqs, pages, heads, page/16, bytes]
    k, v = (f(c, blocks).permute(0, 2, 1, 3, 4, 5).flatten(2, 4) for f in (_keys, _values))      # [seqs, heads, tokens, D]
    T = k.shape[2]
    q = torch.zeros((c["seqs"], c["tokens"], c["heads"], D), device="cuda")
    q[seq, nth] = s.q.float()
    at = torch.full((c["seqs"], c["tokens"]), -1, dtype=torch.long, device="cuda")
    at[seq, nth] = pos
    q = q.unflatten(2, (Hk, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)                            # [seqs, kv heads, group * tokens, D]
    score = (q @ k.transpose(-1, -2)).unflatten(2, (-1, c["tokens"])) * D ** -0.5
    t = torch.arange(T, device="cuda")
    seen = t <= at[..., None]
    if c["window"]:
        seen = seen & (t > at[..., None] - c["window"])
    score = score.masked_fill(~seen[:, None, None], float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    v = torch.where(t[None, None, :, None] < s.lengths[:, None, None, None], v, 0.0)
    o = (p.flatten(2, 3) @ v).unflatten(2, (-1, c["tokens"])).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return {"out": o[seq, nth].to(s.out.dtype)}


def _plain_store(s):
    c = s.case
    seq, _, pos = _places(s)
    page = s.tables[seq, pos // c["page"]].long()
    held = []
    for x in (s.k, s.v):
        code, scale, low = _groups(x, c["group"])
        # the cache as values: what a page holds of each token, written and then read through the page tables
        store = torch.empty((s.n_pages, c["page"], c["kv_heads"], c["head_dim"]), device="cuda")
        store[page, pos % c["page"]] = (code.unflatten(-1, (-1, c["group"])).float() * scale.float().unsqueeze(-1) + low.float().unsqueeze(-1)).flatten(-2)
        held.append(store[page, pos % c["page"]])
    return {"k": held[0], "v": held[1]}


def _plain_fork(s):
    c = s.case
    page, slot = c["page"], torch.arange(s.max_pages, device="cuda")
    child, parent = s.children.long(), s.parents.long()
    old = s.tables[child]
    gone = slot < -(-s.lengths[child] // page)[:, None]
    s.refs.index_add_(0, torch.where(gone, old, 0).flatten().long(), -gone.flatten().int())
    s.lengths[child] = 0
    lens = s.lengths[parent]
    full, rest = lens // page, lens % page > 0
    whole, table = slot < full[:, None], s.tables[parent]
    s.refs.index_add_(0, torch.where(whole, table, 0).flatten().long(), whole.flatten().int())
    free = torch.argsort((s.refs > 0).int(), stable=True)                                        # the lowest free pages, in order
    new = free[(rest.long().cumsum(0) - 1).clamp(min=0)]
    last = table.gather(1, full[:, None].clamp(max=s.max_pages - 1).long())[:, 0].long()
    # (a sequence that ends with a page copies nothing: its last page onto itself)
    at = torch.where(rest, last, table[:, 0].long())
    s.pool[:, torch.where(rest, new, at)] = s.pool[:, at]
    s.refs.index_add_(0, new, rest.int())
    s.tables[child] = torch.where(whole, table, torch.where(rest[:, None] & (slot == full[:, None]), new[:, None].int(), -1))
    s.lengths[child] = lens
    return {"tables": s.tables, "lengths": s.lengths, "refs": s.refs, "pool": s.pool}


def _plain_compact(s):
    live = s.refs > 0
    n_live = live.sum()
    here = torch.arange(s.n_pages, device="cuda")
    movers, holes = live & (here >= n_live), ~live & (here < n_live)
    # the k-th live page behind the boundary goes to the k-th hole before it
    moving = here < movers.sum()
    src, to = (torch.argsort((~x).int(), stable=True) for x in (movers, holes))
    src, to = (torch.where(moving, x, x[0]) for x in (src, to))                                  # (the rest repeat the first)
    s.pool[:, to] = s.pool[:, src]
    new = here.clone()
    new[src] = to
    refs = torch.where(here < n_live, s.refs, 0)
    refs = refs.index_add(0, to, torch.where(moving, s.refs[src], 0))
    tables = torch.where(s.tables >= 0, new[s.tables.clamp(min=0).long()].int(), -1)
    return {"tables": tables, "refs": refs, "n_live": n_live.int().view(1), "pool": s.pool}


def run(s):
    if own:
        return {"linear": _own_linear, "attend": _own_attend, "store": _own_store, "fork": _own_fork, "compact": _own_compact}[s.case["op"]](s)
    return {"linear": _plain_linear, "attend": _plain_attend, "store": _plain_store, "fork": _plain_fork, "compact": _plain_compact}[s.case["op"]](s)


# ---------------------------------------------------------------------------------------------- work, and 64 bits

def work(case):
    """Bytes: every input once, every output once.  Operations: two per multiply-accumulate of the products."""
    size = {"fp32": 4, "fp16": 2, "bf16": 2}
    if case["op"] == "linear":
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        per_weight = 0.5 + (4 if case["offsets"] else 2) / case["group"]
        return {"bytes": d_in * d_out * per_weight + n * d_in * size[case["x"]] + n * d_out * size[case["y"]], "flops": 2.0 * n * d_in * d_out}
    D, lens, counts = case["head_dim"], _lengths(case), _counts(case)
    token = 2 * case["kv_heads"] * (D / 2 + 4 * D / case["group"])               # bytes of a token in one layer
    if case["op"] == "attend":
        window = case["window"] or case["longest"]
        held = sum(min(l, window + c - 1) for l, c in zip(lens, counts))
        seen = sum(min(l - c + 1 + i, window) for l, c in zip(lens, counts) for i in range(c))
        return {"bytes": held * token + 2 * sum(counts) * case["heads"] * D * 2, "flops": 4.0 * case["heads"] * D * seen}
    if case["op"] == "store":
        # in, into the cache, out of it, and out
        return {"bytes": sum(counts) * (2 * case["kv_heads"] * D * (2 + 4) + 2 * token), "flops": 0.0}
    pages = sum(-(-l // case["page"]) for l in lens)
    if case["op"] == "fork":
        # the last page of every sequence in every layer, read and written; tables and reference counts
        return {"bytes": sum(l % case["page"] > 0 for l in lens) * 2 * case["layers"] * case["page"] * token + 5 * 4 * pages, "flops": 0.0}
    # a third of the live pages lies behind the boundary
    return {"bytes": pages / 3 * 2 * case["layers"] * case["page"] * token + 4 * 4 * pages, "flops": 0.0}


def _held(case, block, keys):
    """[pages, heads, bytes] -> [pages, heads, page, D] in 64 bits: each element by the place of its code in the block."""
    D, G, page = case["head_dim"], case["head_dim"] // case["group"], case["page"]
    t, ch = torch.meshgrid(torch.arange(page, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")
    base, u = t // 16 * (16 * D + 128 * G), t % 16
    if keys:
        nibble = ch % 8 + 8 * (u // 8 + 2 * (ch // 32 % 2 + 2 * (ch // 8 % 4 + 4 * (u % 8 + 8 * (ch // 64)))))
        par = base + 8 * D + 4 * (ch // case["group"] + G * (u // 8 + 2 * (u % 8)))
        scale, low = par, par + 2
    else:
        base = base + 8 * D + 64 * G
        nibble = ch // 8 % 2 + 2 * (u // 8) + 4 * (u % 2) + 8 * (ch // 16 % 4 + 4 * (u // 2 % 4 + 4 * (ch % 8 + 8 * (ch // 64))))
        scale = base + 8 * D + 2 * (u % 2 + 2 * (u // 8) + 8 * (u // 2 % 4 + 4 * (ch // case["group"])))
        low = scale + 8
    half = block.view(torch.float16)
    code = (block[..., base + nibble // 2] >> (4 * (nibble % 2)).to(torch.uint8)) & 15
    return code.double() * half[..., scale // 2].double() + half[..., low // 2].double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        y = torch.empty((case["n"], case["d_out"]), dtype=torch.float64, device="cuda")
        col = torch.arange(case["d_in"], device="cuda")
        for at in range(0, case["d_out"], 8192):
            some = slice(at, at + 8192)
            code = ((s.codes[some][:, col // 2].int() >> (4 * (col % 2))) & 15).double()
            w = s.scales[some][:, col // case["group"]].double() * (code - 8)
            if s.offsets is not None:
                w += s.offsets[some][:, col // case["group"]].double()
            y[:, some] = (w @ s.x.double().t()).t()
        return {"y": y}
    starts, lens = s.starts.tolist() if case["tokens"] else [], _lengths(case)
    if case["op"] == "attend":
        out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
        for i in range(case["seqs"]):
            pages = s.tables[i, :-(-lens[i] // case["page"])].long()
            k, v = (_held(case, s.pool[s.layer][pages], keys).transpose(0, 1).flatten(1, 2)[:, :lens[i]] for keys in (True, False))
            n = starts[i + 1] - starts[i]
            q = s.q[starts[i]:starts[i + 1]].double().view(n, case["kv_heads"], -1, case["head_dim"])
            score = torch.einsum("nhgd,htd->hgnt", q, k) / math.sqrt(case["head_dim"])
            back = (torch.arange(n, device="cuda") + lens[i] - n)[:, None] - torch.arange(lens[i], device="cuda")
            hidden = (back < 0) | (back >= case["window"]) if case["window"] else back < 0
            score[..., hidden] = -math.inf
            out[starts[i]:starts[i + 1]] = torch.einsum("hgnt,htd->nhgd", torch.softmax(score, -1), v).reshape(n, case["heads"], -1)
        return {"out": out}
    if case["op"] == "store":
        held = []
        for x in (s.k, s.v):
            x = x.double().view(s.rows, case["kv_heads"], -1, case["group"])
            low, step = x.amin(-1, keepdim=True).float().half().double(), ((x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)) / 15).float().half().double()
            held.append((low + step * ((x - low) / step).round().clamp(0, 15)).flatten(-2))
        return {"k": held[0], "v": held[1]}
    return None                                             # page tables and bytes: whole numbers, no rounding in them
