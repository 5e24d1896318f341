"""Work of agents that were forked from a common context, as cases that can be timed: block copies in the pool, attention
of a batch over shared prefixes, and the norm and rotation of new query and key rows.

`own` false: the operators in plain torch, in 32 bits (64 for angles); true: the library's entry points.  Lengths and block
tables follow from the case, values from the seed.
"""
import math
import random

import torch

own = False

BLOCK, CHUNK, GROUP = 256, 32, 64

DEFAULTS = {
    "op": "prefix",        # prefix | copy | norm_rope
    "layers": 1, "q_heads": 32, "kv_heads": 8, "d_qk": 128, "d_v": 128, "sb_bf16": False,
    "lens_seed": 0,
    # prefix: groups of agents; a group's agents share a prefix and hold some tokens of their own
    "groups": 1, "agents_lo": 1, "agents_hi": 1, "prefix_lo": 256, "prefix_hi": 256, "own_lo": 1, "own_hi": 1,
    "idle": 0,             # agents of the batch without any token (a padded batch)
    "outliers": False,     # 1 % of the channels carry 8x the values
    # copy: `copies` blocks go to others, lo to hi tokens of each
    "blocks": 8, "copies": 1, "tokens_lo": 256, "tokens_hi": 256,
    # norm_rope: agents with new tokens behind their cached ones
    "agents": 1, "new_lo": 1, "new_hi": 1, "cached_lo": 0, "cached_hi": 0,
    "norm": True, "offset": 0.0, "theta": 10000.0, "rot_begin": 0, "rot_dim": 128, "interleaved": False,
    "strided": True,       # the rows are views of one [tokens][q | k | v] projection (else tensors of their own)
}


def listed():
    return [
        # Two agents forked from a short context, one layer: the smallest step, all launch and host latency.
        dict(name="prefix_tiny", op="prefix", q_heads=8, kv_heads=2, agents_lo=2, agents_hi=2, prefix_lo=300, prefix_hi=300,
             own_lo=10, own_hi=60),
        # Five Llama-3.1-8B-shaped agents on one 4096-token context, four layers of a step.
        dict(name="prefix_agents", op="prefix", layers=4, agents_lo=5, agents_hi=5, prefix_lo=4096, prefix_hi=4096, own_lo=64,
             own_hi=512, lens_seed=1),
        # 32 branches of one 16384-token document.
        dict(name="prefix_fanout", op="prefix", layers=2, agents_lo=32, agents_hi=32, prefix_lo=16384, prefix_hi=16384,
             own_lo=100, own_hi=1000, lens_seed=2, outliers=True),
        # Global layers of a Gemma-3-12B-shaped model, three groups of different sizes and odd prefixes, an idle slot.
        dict(name="prefix_groups_d256", op="prefix", layers=2, q_heads=16, kv_heads=8, d_qk=256, d_v=256, groups=3, agents_lo=2,
             agents_hi=9, prefix_lo=1000, prefix_hi=9000, own_lo=1, own_hi=700, lens_seed=5, idle=1),
        # Per-head MLA shape (192 / 128), bfloat16 scales, ten agents.
        dict(name="prefix_mla_heads", op="prefix", layers=2, q_heads=16, kv_heads=16, d_qk=192, d_v=128, agents_lo=10,
             agents_hi=10, prefix_lo=8191, prefix_hi=8191, own_lo=30, own_hi=400, lens_seed=4, sb_bf16=True),
        # 64 branches of a 32768-token context with up to 2000 tokens each: the largest step.
        dict(name="prefix_large", op="prefix", agents_lo=64, agents_hi=64, prefix_lo=32768, prefix_hi=32768, own_lo=500,
             own_hi=2000, lens_seed=6),
        # One agent forks with 40 tokens in its last block, all layers.
        dict(name="copy_fork", op="copy", layers=32, blocks=8, copies=1, tokens_lo=40, tokens_hi=40),
        # Sixteen forks, ragged last blocks, Gemma-3-12B shape.
        dict(name="copy_forks", op="copy", layers=48, kv_heads=8, q_heads=16, d_qk=256, d_v=256, blocks=40, copies=16,
             tokens_lo=1, tokens_hi=256, lens_seed=7),
        # Compaction of a fragmented pool: whole blocks move, all layers.
        dict(name="copy_compact", op="copy", layers=32, blocks=130, copies=60, lens_seed=8),
        # One decode token of five agents, Llama-3.1-8B shape, rotation alone.
        dict(name="rope_decode", op="norm_rope", agents=5, cached_lo=4096, cached_hi=4096, norm=False, theta=500000.0),
        # A phase of new tokens, Gemma-3-12B shape: norms with the weight's offset of one, and the rotation.
        dict(name="norm_rope_phase", op="norm_rope", q_heads=16, kv_heads=8, d_qk=256, d_v=256, rot_dim=256, agents=8, new_lo=200,
             new_hi=1024, cached_lo=1000, cached_hi=8192, lens_seed=9, offset=1.0, theta=1000000.0),
        # A long prompt of one agent, per-head MLA shape: the last 64 elements turn, adjacent pairs.
        dict(name="norm_rope_prompt", op="norm_rope", q_heads=16, kv_heads=16, d_qk=192, rot_begin=128, rot_dim=64,
             interleaved=True, new_lo=32768, new_hi=32768, cached_lo=98304, cached_hi=98304, norm=False, strided=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prefix", "prefix", "prefix", "copy", "norm_rope"])
    c = {"op": op, "lens_seed": rng.randrange(1 << 20), "sb_bf16": rng.random() < 0.4}
    hq, hkv, d, dv = rng.choice([(8, 2, 128, 128), (32, 8, 128, 128), (64, 8, 128, 128), (16, 16, 128, 128), (16, 8, 256, 256),
                                 (16, 16, 192, 128)])
    c.update(q_heads=hq, kv_heads=hkv, d_qk=d, d_v=dv)
    if op == "prefix":
        top, prefix, mine = _log(rng, 1, 32), _log(rng, 40, 24000), _log(rng, 1, 2000)
        c.update(groups=rng.choice([1, 1, 2, 3]), agents_hi=top, agents_lo=max(1, top // rng.choice([1, 4])), prefix_hi=prefix,
                 prefix_lo=rng.choice([prefix, prefix, max(1, prefix // 10), 0]), own_hi=mine, own_lo=max(0, mine // rng.choice([1, 5, 100])),
                 idle=rng.choice([0, 0, 1, 3]), outliers=d == 128 and rng.random() < 0.4)
        while work(c)["flops"] > 2e10:
            c["agents_hi"] = max(1, c["agents_hi"] // 2)
            c["agents_lo"] = min(c["agents_lo"], c["agents_hi"])
        c["layers"] = max(1, min(_log(rng, 1, 4), int(3e8 / work(c)["bytes"])))
    elif op == "copy":
        n, top = _log(rng, 1, 40), _log(rng, 1, 256)
        c.update(copies=n, blocks=2 * n + rng.randrange(1, 6), tokens_hi=top, tokens_lo=max(1, top // rng.choice([1, 1, 8])))
        c["layers"] = max(1, min(_log(rng, 1, 32), int(1.2e9 / (c["blocks"] * BLOCK * _row_bytes(_full(c))))))
    else:
        top, cached = _log(rng, 1, 4096), _log(rng, 1, 120000)
        c.update(agents=_log(rng, 1, 6), new_hi=top, new_lo=max(1, top // rng.choice([1, 4])), cached_hi=cached,
                 cached_lo=max(0, cached // rng.choice([1, 9])), norm=rng.random() < 0.6, offset=rng.choice([0.0, 1.0]),
                 theta=rng.choice([1e4, 5e5, 1e6]), rot_dim=rng.choice([64, d if d != 192 else 64, 32]),
                 interleaved=rng.random() < 0.4, strided=rng.random() < 0.7)
        c["rot_begin"] = 128 if d == 192 else 0
    return c


# ---- sizes -------------------------------------------------------------------------------------------------------------

def _full(case):
    return dict(DEFAULTS, **case)


def _groups(c):
    """(prefix tokens, own tokens of each agent) of every group; None: an idle agent."""
    r = random.Random(c["lens_seed"])

    def between(lo, hi):
        return min(hi, max(lo, _log(r, max(lo, 1), max(hi, 1)))) if r.random() < 0.95 else lo
    out = []
    for _ in range(c["groups"]):
        prefix, n = between(c["prefix_lo"], c["prefix_hi"]), between(c["agents_lo"], c["agents_hi"])
        out.append((prefix, [between(c["own_lo"], c["own_hi"]) for _ in range(n)]))
    for _ in range(c["idle"]):
        out[r.randrange(len(out))][1].append(None)
    return out


def _copies(c):
    """(source, destination, tokens) of every copy; no block is named twice."""
    r = random.Random(c["lens_seed"])
    ids = r.sample(range(c["blocks"]), 2 * c["copies"])
    return [(ids[2 * i], ids[2 * i + 1], r.randint(c["tokens_lo"], c["tokens_hi"])) for i in range(c["copies"])]


def _new(c):
    """(cached tokens, new tokens) of every agent."""
    r = random.Random(c["lens_seed"])
    return [(r.randint(c["cached_lo"], c["cached_hi"]), r.randint(c["new_lo"], c["new_hi"])) for _ in range(c["agents"])]


def _row_bytes(c):
    """Q4 bytes of one token of one layer, all KV heads."""
    return c["kv_heads"] * (c["d_qk"] // 2 + c["d_qk"] // 16 + c["d_v"] // 2 + c["d_v"] // 16)


def work(case):
    c = _full(case)
    if c["op"] == "copy":
        chunks = sum(-(-n // CHUNK) for _, _, n in _copies(c))
        return {"bytes": 2.0 * c["layers"] * chunks * CHUNK * _row_bytes(c), "flops": 0.0}
    if c["op"] == "norm_rope":
        elements = sum(n for _, n in _new(c)) * (c["q_heads"] + c["kv_heads"]) * c["d_qk"]
        return {"bytes": 4.0 * elements, "flops": 0.0}
    rows = pairs = agents = 0
    for prefix, tails in _groups(c):
        live = [n for n in tails if n is not None]
        rows += (prefix if live else 0) + sum(live)
        pairs += sum(prefix + n for n in live)
        agents += len(tails)
    moved = rows * _row_bytes(c) + agents * c["q_heads"] * 2 * (c["d_qk"] + c["d_v"])
    return {"bytes": float(c["layers"] * moved), "flops": 2.0 * c["layers"] * c["q_heads"] * (c["d_qk"] + c["d_v"]) * pairs}


# ---- inputs ------------------------------------------------------------------------------------------------------------

class State:
    pass


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _quantized(g, c, n_blocks, d):
    """Random rows of one layer's keys or values, quantized: words [block][kv head][256][d / 8] of eight codes, and the
    scales and biases [block][kv head][256][d / 64]."""
    kind = torch.bfloat16 if c["sb_bf16"] else torch.float16
    x = torch.randn((n_blocks, c["kv_heads"], BLOCK, d), generator=g, device="cuda")
    if c["outliers"]:
        hot = torch.rand((c["kv_heads"], d), generator=g, device="cuda") < 0.01
        x *= torch.where(hot, 8.0, 1.0)[None, :, None, :]
    x = x.view(n_blocks, c["kv_heads"], BLOCK, d // GROUP, GROUP)
    bias = x.amin(-1).to(kind)
    scale = ((x.amax(-1) - bias.float()) / 15).to(kind)
    codes = ((x - bias.float()[..., None]) / scale.float()[..., None]).round_().clamp_(0, 15).to(torch.int32)
    codes = codes.view(n_blocks, c["kv_heads"], BLOCK, d // 8, 8)
    words = codes[..., 0].clone()
    for k in range(1, 8):
        words |= codes[..., k] << (4 * k)
    return [words, scale, bias]


def _tables(c):
    """Block tables of a batch whose groups share their prefix's whole blocks, a fork's last partly filled block being each
    agent's own: (rows, number of blocks, [(source, destination, tokens)] of the copied ones, kv lengths)."""
    r = random.Random(c["lens_seed"] + 1)
    rows, copies, lens, n = [], [], [], 0
    for prefix, tails in _groups(c):
        whole, part = prefix // BLOCK, prefix % BLOCK
        shared = list(range(n, n + whole))
        n += whole
        lead = None
        for t in tails:
            if t is None:
                rows.append([])
                lens.append(0)
                continue
            mine = list(range(n, n + -(-(prefix + t) // BLOCK) - whole))
            n += len(mine)
            if part and mine:
                if lead is None:
                    lead = mine[0]
                else:
                    copies.append((lead, mine[0], part))
            rows.append(shared + mine)
            lens.append(prefix + t)
    n += 2
    order = list(range(n))
    r.shuffle(order)
    wide = max(1, max(len(x) for x in rows))
    return ([[order[b] for b in x] + [-1] * (wide - len(x)) for x in rows], n,
            [(order[a], order[b], m) for a, b, m in copies], lens)


def _prefix_inputs(c, seed):
    g = _generator(seed)
    rows, n_blocks, copies, lens = _tables(c)
    layers = []
    for _ in range(c["layers"]):
        parts = _quantized(g, c, n_blocks, c["d_qk"]) + _quantized(g, c, n_blocks, c["d_v"])
        for src, dst, m in copies:
            for t in parts:
                t[dst, :, :m] = t[src, :, :m]
        layers.append(parts)
    q = torch.randn((c["layers"], len(lens), c["q_heads"], c["d_qk"]), generator=g, device="cuda").to(torch.bfloat16)
    return rows, n_blocks, lens, layers, q


def _norm_rope_inputs(c, seed):
    g = _generator(seed)
    total = sum(n for _, n in _new(c))
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["d_qk"]
    x = torch.randn((total, hq + 2 * hkv, d), generator=g, device="cuda")
    x = (x * (0.25 + torch.rand((1, hq + 2 * hkv, 1), generator=g, device="cuda") * 4)).to(torch.bfloat16)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    if not c["strided"]:
        q, k = q.contiguous(), k.contiguous()
    w = (torch.randn((2, d), generator=g, device="cuda") * 0.2 + (1.0 - c["offset"])).to(torch.bfloat16)
    i = torch.arange(c["rot_dim"] // 2, dtype=torch.float64)
    freq = (c["theta"] ** (-2.0 * i / c["rot_dim"])).to(torch.float32).cuda()
    return q, k, w, freq


def _offsets(counts):
    offs = [0]
    for n in counts:
        offs.append(offs[-1] + n)
    return offs


def _copy_pool(c, seed):
    """A pool's bytes as 32-bit words, [layer][block][kv head][chunk of 32 tokens][words]."""
    words = CHUNK * _row_bytes(c) // c["kv_heads"] // 4
    return torch.randint(-2**31, 2**31 - 1, (c["layers"], c["blocks"], c["kv_heads"], BLOCK // CHUNK, words), dtype=torch.int32,
                         generator=_generator(seed), device="cuda")


def prepare(case, seed):
    c = _full(case)
    s = State()
    s.c = c
    if own:
        from paper_2603_04428_b200 import binding as B
        s.B = B
        s.spec = B.Spec.make(c["layers"], c["q_heads"], c["kv_heads"], c["d_qk"], c["d_v"], sb_dtype=1 if c["sb_bf16"] else 0)
        s.flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "copy":
        s.pool = _copy_pool(c, seed)
        copies = _copies(c)
        s.copies = _ints(copies)
        s.by_chunk = []
        for k in range(BLOCK // CHUNK):                 # the copies that reach chunk k of a block
            some = [(a, b) for a, b, n in copies if n > k * CHUNK]
            s.by_chunk.append((_ints([a for a, _ in some]).long(), _ints([b for _, b in some]).long()) if some else None)
        return s
    if c["op"] == "norm_rope":
        s.q, s.k, s.w, s.freq = _norm_rope_inputs(c, seed)
        s.pos, s.offs = _ints([p for p, _ in _new(c)]), _ints(_offsets([n for _, n in _new(c)]))
        s.total, s.eps = s.q.shape[0], 1e-6
        if own:
            s.how = s.B.NormRotation.make(norm_dim=c["d_qk"] if c["norm"] else 0, q_weight=s.w[0] if c["norm"] else None,
                                          k_weight=s.w[1] if c["norm"] else None, eps=s.eps, weight_offset=c["offset"],
                                          rot_begin=c["rot_begin"], rot_dim=c["rot_dim"], interleaved=c["interleaved"],
                                          inv_freq=s.freq)
            s.q_out = torch.empty(s.q.shape, dtype=torch.bfloat16, device="cuda")
            s.k_out = torch.empty(s.k.shape, dtype=torch.bfloat16, device="cuda")
        return s
    s.rows, s.n_blocks, s.lens, s.layers, s.q = _prefix_inputs(c, seed)
    s.groups = _groups(c)
    s.scale = 1.0 / math.sqrt(c["d_qk"])
    if own:
        # the persisted layout, block by block, into the pool
        image = torch.cat([torch.cat([t.contiguous().view(torch.uint8).view(s.n_blocks, -1) for t in parts], 1).flatten()
                           for parts in s.layers])
        s.layers = None
        s.pool = torch.zeros(s.B.q4kv_pool_bytes(s.spec, s.n_blocks), dtype=torch.uint8, device="cuda")
        s.B.q4kv_unpack(s.spec, image, s.n_blocks * BLOCK, s.pool, s.n_blocks, _ints(range(s.n_blocks)), s.flags)
        s.tables, s.kv_lens, s.most = _ints(s.rows), _ints(s.lens), max(s.lens)
        s.batch = s.B.batch(s.tables)
        s.group_offs, s.prefix_lens = _ints(_offsets([len(t) for _, t in s.groups])), _ints([p for p, _ in s.groups])
        s.out = torch.empty((c["layers"], len(s.lens), c["q_heads"], c["d_v"]), dtype=torch.bfloat16, device="cuda")
        s.qs, s.outs = list(s.q), list(s.out)
        s.ws = torch.zeros(s.B.q4kv_workspace_bytes_shared_prefix(s.spec, len(s.lens), s.most, len(s.groups)), dtype=torch.uint8,
                           device="cuda")
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def _values(words, scale, bias, ids):
    """float32 [kv head][256 * blocks][d] of some blocks."""
    w, sc, b = words[ids].transpose(0, 1), scale[ids].transpose(0, 1), bias[ids].transpose(0, 1)
    codes = torch.stack([(w >> (4 * k)) & 15 for k in range(8)], -1).float()
    h, n, d = w.shape[0], w.shape[1] * BLOCK, w.shape[-1] * 8
    x = codes.view(h, n, d // GROUP, GROUP) * sc.reshape(h, n, d // GROUP, 1).float() + b.reshape(h, n, d // GROUP, 1).float()
    return x.view(h, n, d)


def _plain_prefix(s):
    c = s.c
    out = torch.zeros(s.q.shape[:3] + (c["d_v"],), dtype=torch.bfloat16, device="cuda")
    for layer, (kw, ks, kb, vw, vs, vb) in enumerate(s.layers):
        a = 0
        for prefix, tails in s.groups:
            live = [a + i for i, t in enumerate(tails) if t is not None]
            a += len(tails)
            if not live:
                continue
            ids = s.rows[live[0]][:-(-prefix // BLOCK)]
            kp, vp = _values(kw, ks, kb, ids)[:, :prefix], _values(vw, vs, vb, ids)[:, :prefix]
            q = s.q[layer, live].float().view(len(live), c["kv_heads"], -1, c["d_qk"]) * s.scale     # [agent][kv head][rep][d]
            scores = torch.einsum("ahrd,hnd->ahrn", q, kp)
            for i, agent in enumerate(live):
                first = prefix // BLOCK
                ids = s.rows[agent][first:-(-s.lens[agent] // BLOCK)]
                x, v = scores[i], None
                if s.lens[agent] > prefix:
                    part = slice(prefix - first * BLOCK, s.lens[agent] - first * BLOCK)
                    v = _values(vw, vs, vb, ids)[:, part]
                    x = torch.cat([x, q[i] @ _values(kw, ks, kb, ids)[:, part].transpose(1, 2)], -1)
                p = torch.exp(x - x.amax(-1, keepdim=True))
                y = p[..., :prefix] @ vp
                if v is not None:
                    y = y + p[..., prefix:] @ v
                out[layer, agent] = (y / p.sum(-1, keepdim=True)).view(c["q_heads"], c["d_v"]).to(torch.bfloat16)
    return out


def _plain_norm_rope(s):
    c = s.c
    n = s.total
    row = torch.arange(n, device="cuda", dtype=torch.int32)
    agent = torch.searchsorted(s.offs[1:], row, right=True)
    angle = (s.pos[agent] + row - s.offs[agent]).double()[:, None] * s.freq.double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = []
    for x, w in ((s.q, s.w[0]), (s.k, s.w[1])):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps) * (w.float() + c["offset"])
        r = x[..., c["rot_begin"]:c["rot_begin"] + c["rot_dim"]]
        a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else r.chunk(2, -1)
        t, u = a * cos - b * sin, b * cos + a * sin
        a.copy_(t)
        b.copy_(u)
        out.append(x.to(torch.bfloat16))
    return out


def run(s):
    c = s.c
    if c["op"] == "copy":
        if own:
            s.B.q4kv_copy_blocks(s.spec, s.pool, c["blocks"], s.pool, c["blocks"], 0, c["layers"], s.copies, c["copies"], s.flags)
        else:
            for k, pair in enumerate(s.by_chunk):
                if pair is not None:
                    s.pool[:, pair[1], :, k] = s.pool[:, pair[0], :, k]
        return s.pool
    if c["op"] == "norm_rope":
        if not own:
            return _plain_norm_rope(s)
        s.B.q4kv_norm_rope(s.spec, s.how, c["agents"], s.pos, s.offs, s.total, s.q, s.k, s.q_out, s.k_out, s.flags)
        return [s.q_out, s.k_out]
    if not own:
        return _plain_prefix(s)
    for layer in range(c["layers"]):
        s.B.q4kv_shared_prefix_decode_attention(s.spec, s.pool, s.n_blocks, layer, s.batch, s.kv_lens, s.most, s.group_offs,
                                                s.prefix_lens, len(s.groups), s.qs[layer], s.scale, s.outs[layer], s.B.OUT_BF16,
                                                None, s.ws, s.flags)
    return s.out


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    c = _full(case)
    if c["op"] == "copy":
        return None
    if c["op"] == "norm_rope":
        q, k, w, freq = _norm_rope_inputs(c, seed)
        where = torch.cat([torch.arange(p, p + n, dtype=torch.float64, device="cuda") for p, n in _new(c)])
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(where, freq.double()))[:, None, :]
        half, lo = c["rot_dim"] // 2, c["rot_begin"]
        step = torch.arange(half, device="cuda")
        ia, ib = (lo + 2 * step, lo + 2 * step + 1) if c["interleaved"] else (lo + step, lo + step + half)
        both = []
        for x, weight in ((q, w[0]), (k, w[1])):
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for h in range(x.shape[1]):
                z = x[:, h].double()
                if c["norm"]:
                    z = z / ((z * z).sum(-1, keepdim=True) / z.shape[-1] + 1e-6).sqrt() * (weight.double() + c["offset"])
                r = torch.complex(z[:, ia], z[:, ib]) * turn[:, 0]
                z[:, ia], z[:, ib] = r.real, r.imag
                y[:, h] = z
            both.append(y)
        return both
    rows, _, lens, layers, q = _prefix_inputs(c, seed)
    shift = 4 * torch.arange(8, device="cuda", dtype=torch.int32)

    def numbers(parts, ids, h, n):
        words, scale, bias = (t[ids, h].reshape(len(ids) * BLOCK, -1)[:n] for t in parts)
        x = ((words[..., None] >> shift) & 15).double().view(n, -1, GROUP)
        return (x * scale.double()[..., None] + bias.double()[..., None]).view(n, -1)

    rep = c["q_heads"] // c["kv_heads"]
    out = torch.zeros((c["layers"], len(lens), c["q_heads"], c["d_v"]), dtype=torch.float64, device="cuda")
    for layer, parts in enumerate(layers):
        for agent, n in enumerate(lens):
            ids = rows[agent][:-(-n // BLOCK)]
            for h in range(c["kv_heads"] if n else 0):
                heads = slice(h * rep, (h + 1) * rep)
                weights = torch.softmax(q[layer, agent, heads].double() @ numbers(parts[:3], ids, h, n).T / math.sqrt(c["d_qk"]), -1)
                out[layer, agent, heads] = weights @ numbers(parts[3:], ids, h, n)
    return out
