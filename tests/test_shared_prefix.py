"""Attention of agents that share prefixes, against the float64 oracle's decode attention of each agent alone."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import q4kv_oracle as O
from paper_2603_04428_b200 import binding as B, synth

ATOL, RTOL_ROW = 2e-3, 1e-2      # the library's parity bounds for unit-variance caches (binary32 output)


class Forked:
    """Groups [(prefix, [own tokens or None for an idle agent])] as an oracle pool and a device pool, where every slot past a length is
    poison.  wide: entries of a block-table row.  Which way a call takes is chosen by what the host knows, the number of agents and
    groups and the width of the rows: wide rows stand for long contexts, where prefixes are attended once for their group."""

    def __init__(self, shape, groups, seed, sb_dtype=0, layers=1, edit=None, wide=1):
        from paper_2603_04428_b200 import harness as H
        hq, hkv, d, dv = shape
        self.shape, self.groups = shape, groups
        rows, lens, n, lead_of = [], [], 0, []
        g = synth.rng(seed, 1)
        poison, copies = [], []
        for prefix, tails in groups:
            whole, part = divmod(prefix, 256)
            shared = list(range(n, n + whole))
            n += whole
            lead = None
            for t in tails:
                if t is None:
                    rows.append([])
                    lens.append(0)
                    continue
                mine = list(range(n, n + -(-(prefix + t) // 256) - whole))
                n += len(mine)
                first = lead is None
                if part and not first:
                    copies.append((lead[whole], mine[0], part))
                elif first:
                    lead = shared + mine
                if (prefix + t) % 256:
                    poison.append(((shared + mine)[-1], (prefix + t) % 256, 256))
                rows.append(shared + mine)
                lens.append(prefix + t)
        self.n_blocks = n + 2
        order = g.permutation(self.n_blocks)
        real = np.full((len(rows), max([wide] + [len(r) for r in rows])), -1, np.int32)
        for i, a in enumerate(rows):
            real[i, :len(a)] = [order[x] for x in a]
        self.lens, self.tables = lens, real
        self.offs = np.concatenate([[0], np.cumsum([len(t) for _, t in groups])]).astype(np.int32)
        self.prefix = [p for p, _ in groups]
        self.opool = O.Pool(O.Spec(layers, hq, hkv, d, dv, sb_dtype=sb_dtype), self.n_blocks)
        for name, dd in (("K", d), ("V", dv)):
            x = synth.bf16_bits_to_f32(synth.normal_bf16(seed, 2 if name == "K" else 3, (layers, self.n_blocks, hkv, 256, dd)))
            codes, sc, bi = O.quantize_rows(x, sb_dtype)
            getattr(self.opool, name + "c")[:] = O.pack_codes(codes)
            getattr(self.opool, name + "s")[:] = sc
            getattr(self.opool, name + "b")[:] = bi
        if edit:
            edit(self)
        for a, b, m in copies:
            for t in self.opool.tensors():
                t[:, order[b], :, :m] = t[:, order[a], :, :m]
        clean = [t.copy() for t in self.opool.tensors()]
        nan = np.float16(np.nan) if sb_dtype == 0 else np.uint16(0x7FC0)
        for b, lo, hi in poison:
            for name in ("Kc", "Vc"):
                getattr(self.opool, name)[:, order[b], :, lo:hi] = 0xFFFFFFFF
            for name in ("Ks", "Kb", "Vs", "Vb"):
                getattr(self.opool, name)[:, order[b], :, lo:hi] = nan
        image = O.pack(self.opool, np.arange(self.n_blocks), self.n_blocks * 256)
        for t, c in zip(self.opool.tensors(), clean):
            t[:] = c
        self.dc = H.DeviceCache(layers, hq, hkv, d, dv, False, self.n_blocks, real, sb_dtype=sb_dtype)
        B.q4kv_unpack(self.dc.spec, H.dev(image), self.n_blocks * 256, self.dc.pool, self.n_blocks,
                      H.dev(np.arange(self.n_blocks, dtype=np.int32)), self.dc.flags)

    def q(self, stream=7):
        return synth.normal_bf16(5, stream, (len(self.lens), self.shape[0], self.shape[2]))

    def want(self, q, scale, layer=0):
        return O.decode_attention(self.opool, layer, self.tables, self.lens, 0, synth.bf16_bits_to_f32(q), scale)

    def run(self, q, scale, **kw):
        return self.dc.shared_prefix_decode(kw.pop("layer", 0), self.lens, self.offs, self.prefix, q, scale, **kw)


def close(out, lse, want, want_lse, bf16=False):
    out = out.double().cpu().numpy()
    assert np.all(np.isfinite(out))
    err, extra = np.abs(out - want), 2.0 ** -8 * np.abs(want) if bf16 else 0.0
    assert (err - extra).max() <= ATOL, err.max()
    row = (err - extra).reshape(-1, want.shape[-1]).max(1)
    assert np.all(row <= RTOL_ROW * np.abs(want).reshape(-1, want.shape[-1]).max(1) + 1e-30)
    if lse is not None:
        lse = lse.double().cpu().numpy()
        assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
        fin = np.isfinite(want_lse)
        assert np.abs(lse[fin] - want_lse[fin]).max(initial=0.0) <= 2e-3


GROUPS = {
    "one": [(1, [0])],
    "pair": [(300, [17, 1])],
    "edges": [(127, [0, 1, 2]), (128, [0, 1]), (129, [130, 0]), (255, [1, 2]), (256, [0, 300]), (257, [1, 255])],
    "alone": [(0, [5]), (0, [700]), (513, [40])],
    "idle": [(400, [None, 30, None, 0]), (0, [None]), (200, [None, None]), (640, [64])],
    "empty": [(77, []), (500, [9, 200]), (0, []), (0, [1, 2, 3])],
    "many": [(1100, [(7 * i) % 40 for i in range(37)])],
    "long": [(4000, [3, 500]), (129, [900])],
}


WIDE = 2048                      # rows of 524288 tokens


def crowd(groups, n):
    """n more agents with a few tokens of their own in every group that has any."""
    return [(prefix, tails + [i % 3 for i in range(n)] if tails else []) for prefix, tails in groups]


@pytest.mark.gpu
@pytest.mark.parametrize("wide, more", [(1, 0), (WIDE, 0), (WIDE, 4), (WIDE, 13)])
@pytest.mark.parametrize("groups", list(GROUPS))
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (3, 1, 128, 128), (4, 4, 128, 128), (8, 1, 128, 128), (2, 2, 192, 128),
                                   (4, 2, 256, 256), (5, 1, 256, 256)])
def test_against_each_agent_alone(shape, groups, wide, more):
    f = Forked(shape, crowd(GROUPS[groups], more), seed=31, wide=wide)
    q = f.q()
    for sharp in (1.0, 2.5):                             # a scale above 2 / sqrt(d) does not go to tiles rounded to binary16
        scale = sharp / math.sqrt(shape[2])
        out, lse = f.run(q, scale)
        close(out, lse, *f.want(q, scale))
    assert f.dc.read_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("more", [0, 3, 12])
@pytest.mark.parametrize("shape", [(64, 1, 128, 128), (34, 2, 128, 128), (32, 1, 256, 256), (32, 1, 192, 128), (22, 2, 192, 128), (100, 1, 128, 128)])
def test_many_query_heads_to_a_kv_head(shape, more):
    f = Forked(shape, crowd([(333, [1, 50, 0]), (0, [20])], more), seed=32, wide=WIDE)
    q = f.q()
    for sharp in (1.0, 2.5):
        scale = sharp / math.sqrt(shape[2])
        out, lse = f.run(q, scale)
        close(out, lse, *f.want(q, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [[(700, [1, 90, 300]), (40, [5])], [(700, [i % 5 for i in range(8)])], [(700, [i % 5 for i in range(24)])], [(700, [i % 5 for i in range(70)])]])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (2, 2, 192, 128), (4, 2, 256, 256)])
def test_bfloat16_scales_and_bfloat16_output(shape, groups):
    f = Forked(shape, groups, seed=33, sb_dtype=1, layers=2, wide=WIDE)
    q, scale = f.q(), 1.0 / math.sqrt(shape[2])
    for layer in range(2):
        out, lse = f.run(q, scale, layer=layer)
        close(out, lse, *f.want(q, scale, layer))
        half, none = f.run(q, scale, layer=layer, out_dtype=B.OUT_BF16, want_lse=False)
        assert torch.equal(half, out.to(torch.bfloat16)) and none is None
    assert f.dc.read_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(16, 8, 128, 128), (32, 8, 128, 128), (8, 8, 192, 128), (16, 8, 256, 256)])
def test_references_that_have_to_move(shape):
    """Scores that climb by thirty binary orders within 512 keys, again and again, with enough keys for several steps to a CTA: the
    references of the rows' exponentials move, and what was added up before is scaled.  Scores are exact up to binary32 sums (of
    magnitude 30: 16 * 2^-24 * 30 < 1e-4 in an exponent); the probabilities times a value's scale are rounded once to binary16, half a
    step or 2^-11 of p s c, and s c is at most the span of a group, twice the largest value."""
    def climb(f):
        n = f.lens[0]
        pos = np.arange(n)
        blk, slot = f.tables[0][pos // 256], pos % 256
        for h in range(shape[1]):
            at = (0, blk, h, slot)
            x = O.dequantize(O.unpack_codes(f.opool.Kc[at]), f.opool.Ks[at], f.opool.Kb[at]).astype(np.float32)
            x[:, 0] = (pos % 512) * 0.12 * math.sqrt(shape[2] / 128)
            c, s, b = O.quantize_rows(synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x)))
            f.opool.Kc[at], f.opool.Ks[at], f.opool.Kb[at] = O.pack_codes(c), s, b

    f = Forked(shape, [(20000, [40, 0, 200])], seed=34, edit=climb, wide=WIDE)
    qf = synth.bf16_bits_to_f32(f.q())
    qf[..., 0] = 4.0 + np.abs(qf[..., 0])                # every query has a part along the climbing element
    q, scale = synth.f32_to_bf16_bits(qf), 1.0 / math.sqrt(shape[2])
    out, lse = f.run(q, scale)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    qd, rep, most = synth.bf16_bits_to_f32(q).astype(np.float64), shape[0] // shape[1], 0.0
    for a, n in enumerate(f.lens):
        for h in range(shape[1]):
            K, V = O.gather_dequant(f.opool, 0, f.tables[a], 0, n, h)
            s = scale * qd[a, h * rep:(h + 1) * rep] @ K.T
            top = s.max(1, keepdims=True)
            assert top.max() > 15.0
            p = np.exp(s - top)
            want, want_lse = p @ V / p.sum(1, keepdims=True), top[:, 0] + np.log(p.sum(1))
            assert np.abs(out[a, h * rep:(h + 1) * rep] - want).max() <= 2.0 ** -10 * np.abs(V).max() + 1e-3
            assert np.abs(lse[a, h * rep:(h + 1) * rep] - want_lse).max() <= 1e-3


def attended(f, a, h, s):
    """Attention of query rows of KV head h over agent a's first keys, given the rows' scores: output, lse, and what its error is measured
    in: the mean span of the values' groups (15 scales), the mean size of the values, the largest span."""
    n = s.shape[1]
    pos = np.arange(n)
    _, V = O.gather_dequant(f.opool, 0, f.tables[a], 0, n, h)
    span = 15.0 * np.repeat(O.sb_values(f.opool.Vs[0, f.tables[a][pos // 256], h, pos % 256]), 64, axis=-1)
    top = s.max(1, keepdims=True)
    p = np.exp(s - top)
    l = p.sum(1, keepdims=True)
    return p @ V / l, top[:, 0] + np.log(l[:, 0]), p @ span / l, p @ np.abs(V) / l, span.max()


def code_bound(n, span, size, most):
    """What the list may be off by, with one rounding of p s to binary16:
      half a step, 2^-11 of p s, times a code of at most 15                                 -> 2^-11 * sum p span / sum p
      scores of magnitude up to 20 from 16 sums of binary32 numbers, and an exponential     -> 1e-4 * sum p |v| / sum p
      below binary16's range at most half of its smallest step 2^-24, sixteen times that for odd tokens, where the row's sum of p, lifted by
      2^11 over the largest scale, is 2^10 over that scale or more: 15 * 2^-21 / 2^10 scales for a key, doubled -> n * 2^-30 * span."""
    return 2.0 ** -11 * span + 1e-4 * size + n * 2.0 ** -30 * most


N_SINK = 8192


def behind_a_sink(shape, sharp, sigma, at, agents):
    """Agents on one prefix in which key `at` is ten nats above the rest, which still have a good part of the weight together, and
    values of size sigma: each probability by itself is small, and so is a value's scale."""
    pos = np.arange(N_SINK)

    def sink(f):
        for t in (f.opool.Vs, f.opool.Vb):
            t[:] = (t.astype(np.float32) * np.float32(sigma)).astype(np.float16)
        for h in range(shape[1]):
            where = (0, f.tables[0][pos // 256], h, pos % 256)
            x = O.dequantize(O.unpack_codes(f.opool.Kc[where]), f.opool.Ks[where], f.opool.Kb[where]).astype(np.float32)
            x[:, 0] = 0.0
            x[at, 0] = 10.0 * math.sqrt(shape[2]) / (4.0 * sharp)
            c, sc, b = O.quantize_rows(synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x)))
            f.opool.Kc[where], f.opool.Ks[where], f.opool.Kb[where] = O.pack_codes(c), sc, b

    f = Forked(shape, [(N_SINK, [0] * agents)], seed=45, edit=sink, wide=WIDE)
    qf = synth.bf16_bits_to_f32(f.q()) * np.float32(0.5 / sharp)
    qf[..., 0] = 4.0
    return f, synth.f32_to_bf16_bits(qf), sharp / math.sqrt(shape[2])


def close_behind_a_sink(f, q, scale, at, out, lse, codes):
    """codes: the route multiplies the codes; else it expands keys and values into binary16 tiles, which costs every key element a
    rounding of 2^-11 at most, a score d = 2^-11 * scale * sum |q k| at most, a weight 2 d of itself; and 2^-11 each for values and
    probabilities."""
    shape = f.shape
    qd, rep = synth.bf16_bits_to_f32(q).astype(np.float64), shape[0] // shape[1]
    for h in range(shape[1]):
        heads = slice(h * rep, (h + 1) * rep)
        K, V = O.gather_dequant(f.opool, 0, f.tables[0], 0, N_SINK, h)
        rows = qd[:, heads].reshape(-1, shape[2])
        s = scale * rows @ K.T
        want, want_lse, *sizes = attended(f, 0, h, s)
        assert 0.3 < np.exp(s[:, at] - want_lse).mean() < 0.97           # the sink has much of the weight, and so have the others
        err = np.abs(out[:, heads].double().cpu().numpy().reshape(-1, shape[3]) - want)
        off = np.abs(lse[:, heads].double().cpu().numpy().reshape(-1) - want_lse)
        assert np.all(err.max(1) <= RTOL_ROW * np.abs(want).max(1)), (err.max(1) / np.abs(want).max(1)).max()
        d = 2.0 ** -11 * scale * (np.abs(rows) @ np.abs(K).T).max(1)
        if codes:
            assert np.all(err <= code_bound(N_SINK, *sizes)) and off.max() <= 2e-3
        else:
            assert np.all(err <= (2.0 ** -10 + 2.1 * d[:, None]) * np.abs(V).max()) and np.all(off <= d + 1e-3)


@pytest.mark.gpu
@pytest.mark.parametrize("at", [0, 1, 5003])
@pytest.mark.parametrize("sigma", [1.0, 0.1, 0.05, 0.01])
@pytest.mark.parametrize("sharp", [1.0, 2.5])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (8, 2, 192, 128), (4, 2, 256, 256)])
def test_keys_behind_a_sink_keep_their_values(shape, sharp, sigma, at):
    """152 agents, so that a CTA of the list has some 2000 keys.  The larger scale does not go to tiles."""
    f, q, scale = behind_a_sink(shape, sharp, sigma, at, 152)
    out, lse = f.run(q, scale)
    assert f.dc.read_flags() == 0
    close_behind_a_sink(f, q, scale, at, out, lse, codes=sharp > 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("at", [0, 1, 5003])
@pytest.mark.parametrize("sigma", [1.0, 0.1, 0.05, 0.01])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (16, 2, 128, 128), (3, 3, 128, 128), (8, 2, 192, 128), (4, 2, 256, 256)])
def test_agents_by_themselves_keep_values_behind_a_sink(shape, sigma, at):
    """The same keys, attended by every agent alone: in this call and in the decode call."""
    f, q, scale = behind_a_sink(shape, 1.0, sigma, at, 40)
    out, lse = f.dc.shared_prefix_decode(0, f.lens, list(range(41)), [N_SINK] * 40, q, scale)
    close_behind_a_sink(f, q, scale, at, out, lse, codes=True)
    out, lse = f.dc.decode(0, f.lens, 0, q, scale)
    close_behind_a_sink(f, q, scale, at, out, lse, codes=True)
    assert f.dc.read_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("at", [0, 1, 5003])
@pytest.mark.parametrize("sigma", [1.0, 0.1, 0.01])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (3, 3, 128, 128), (4, 2, 256, 256)])
def test_exact_prefill_keeps_values_behind_a_sink(shape, sigma, at):
    """The same keys in the prefill kernel that multiplies codes (its queries being the last token of each agent)."""
    f, q, scale = behind_a_sink(shape, 2.5, sigma, at, 5)
    out, lse = f.dc.prefill(0, f.lens, list(range(6)), 0, q, scale)
    assert f.dc.read_flags() == 0
    close_behind_a_sink(f, q, scale, at, out, lse, codes=True)


@pytest.mark.gpu
@pytest.mark.parametrize("sb_dtype", [0, 1])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (8, 2, 192, 128), (4, 2, 256, 256)])
def test_values_whose_size_changes_along_the_prefix(shape, sb_dtype):
    """Value scales that climb and fall by sixteen binary orders within 1024 keys, and groups that are all one number (scale 0)."""
    n = 8192
    pos = np.arange(n)

    def climb(f):
        for h in range(shape[1]):
            where = (0, f.tables[0][pos // 256], h, pos % 256)
            x = O.dequantize(O.unpack_codes(f.opool.Vc[where]), f.opool.Vs[where], f.opool.Vb[where]).astype(np.float32)
            x *= (2.0 ** (np.abs(pos % 1024 - 512) / 32.0 - 10.0))[:, None].astype(np.float32)
            x[pos % 7 == 3, :64] = 0.375
            x[:200] = 0.375
            c, sc, b = O.quantize_rows(synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x)), sb_dtype)
            f.opool.Vc[where], f.opool.Vs[where], f.opool.Vb[where] = O.pack_codes(c), sc, b

    f = Forked(shape, [(n, [0] * 152)], seed=46, sb_dtype=sb_dtype, edit=climb, wide=WIDE)
    q, scale = f.q(), 2.5 / math.sqrt(shape[2])          # not by tiles
    out, lse = f.run(q, scale)
    assert f.dc.read_flags() == 0
    qd, rep = synth.bf16_bits_to_f32(q).astype(np.float64), shape[0] // shape[1]
    for h in range(shape[1]):
        heads = slice(h * rep, (h + 1) * rep)
        K, _ = O.gather_dequant(f.opool, 0, f.tables[0], 0, n, h)
        want, want_lse, *sizes = attended(f, 0, h, scale * qd[:, heads].reshape(-1, shape[2]) @ K.T)
        err = np.abs(out[:, heads].double().cpu().numpy().reshape(-1, shape[3]) - want)
        assert np.all(err <= code_bound(n, *sizes))
        assert np.abs(lse[:, heads].double().cpu().numpy().reshape(-1) - want_lse).max() <= 2e-3


@pytest.mark.gpu
@pytest.mark.parametrize("shape, agents", [((4, 2, 128, 128), 4), ((4, 4, 192, 128), 8), ((4, 2, 256, 256), 3)])
def test_groups_of_at_most_eight_rows(shape, agents):
    """Half of the softmax warps have no rows then, and may be behind the others in any step: many steps, call after call."""
    f = Forked(shape, [(9000, [i % 3 for i in range(agents)])], seed=44, wide=WIDE)
    q, scale = f.q(), 2.5 / math.sqrt(shape[2])
    out, lse = f.run(q, scale)
    close(out, lse, *f.want(q, scale))
    for _ in range(300):
        again, again_lse = f.run(q, scale)
    assert torch.equal(again, out) and torch.equal(again_lse, lse) and f.dc.read_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("more", [0, 4, 60])
def test_one_agents_bad_query_leaves_the_others_alone(more):
    f = Forked((8, 2, 128, 128), [(600, [20, 30, 1, 0] + [2] * more)], seed=35, wide=WIDE)
    q, scale = f.q(), 1.0 / math.sqrt(128)
    good, _ = f.run(q, scale)
    bad = q.copy()
    bad[1, :4] = 0x7F80                                  # infinities
    bad[1, 4:] = 0x7FC0                                  # NaN
    bad[3] = synth.f32_to_bf16_bits(synth.bf16_bits_to_f32(bad[3]) * np.float32(1e30))
    out, _ = f.run(bad, scale)
    assert torch.equal(out[[0, 2]], good[[0, 2]])
    tiny = q.copy()
    tiny[2] = 0
    out, _ = f.run(tiny, scale)
    assert torch.equal(out[[0, 1, 3]], good[[0, 1, 3]])
    close(out, None, *f.want(tiny, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("wide, more", [(1, 0), (WIDE, 4), (WIDE, 80)])
def test_lengths_that_cannot_be_raise_the_flag_and_give_zeros(wide, more):
    f = Forked((8, 2, 128, 128), [(300, [20, 30, 9]), (40, [100, 3] + [1] * more)], seed=36, wide=wide)
    q, scale = f.q(), 1.0 / math.sqrt(128)
    good, good_lse = f.run(q, scale)
    width, A = f.tables.shape[1] * 256, len(f.lens)

    def call(lens=None, offs=None, prefix=None, **kw):
        f.dc.flags.zero_()
        out, lse = f.dc.shared_prefix_decode(0, f.lens if lens is None else lens, f.offs if offs is None else offs,
                                             f.prefix if prefix is None else prefix, q, scale, **kw)
        return out, lse, f.dc.read_flags()

    def near(x, y, agents):                              # both within ATOL of the truth; the keys may be cut elsewhere
        return torch.allclose(x[agents], y[agents], rtol=0, atol=2 * ATOL)

    for a, n in ((0, 299), (1, -1), (2, width + 1), (2, 2**31 - 1), (4, 39)):
        lens = list(f.lens)
        lens[a] = n
        out, lse, flag = call(lens=lens)
        rest = [i for i in range(A) if i != a]
        assert flag == B.FLAG_BAD_LENGTH and torch.all(out[a] == 0) and torch.all(torch.isneginf(lse[a])) and near(out, good, rest)
    out, lse, flag = call(max_kv_len=325)
    assert flag == B.FLAG_BAD_LENGTH and torch.all(out[1] == 0) and near(out, good, [0] + list(range(2, A)))
    for prefix in ([-1, 40], [width + 1, 40]):
        out, lse, flag = call(prefix=prefix)
        assert flag == B.FLAG_BAD_LENGTH and torch.all(out[:3] == 0) and near(out, good, list(range(3, A)))
    for offs in ([0, 4, 3], [-1, 3, A], [0, 3, A + 1], [0, 3, 2**31 - 1], [A, 3, 0]):
        out, lse, flag = call(offs=offs)
        assert flag == B.FLAG_BAD_LENGTH and torch.all(out == 0) and torch.all(torch.isneginf(lse)), offs
    out, lse, flag = call(offs=[0, 3, 4])                # the agents from 4 on belong to no group
    assert flag == B.FLAG_BAD_LENGTH and torch.all(out[4:] == 0) and near(out, good, [0, 1, 2, 3])
    out, lse, flag = call(offs=[3, 3, A])
    assert flag == B.FLAG_BAD_LENGTH and torch.all(out[:3] == 0)
    out, lse, flag = call()
    assert flag == 0 and torch.equal(out, good) and torch.equal(lse, good_lse)


@pytest.mark.gpu
@pytest.mark.parametrize("sharp", [1.0, 2.5])
@pytest.mark.parametrize("n_groups", [8, 20, 31])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (8, 2, 192, 128), (4, 2, 256, 256)])
def test_groups_that_overlap_stay_inside_the_workspace(shape, n_groups, sharp):
    """Offsets 0, A, 0, A, ...: every second group is in order by itself and names all agents.  Together they have several times the
    score rows that the workspace was sized for, so nothing may be computed for them.  The workspace is as small as the call accepts."""
    from paper_2603_04428_b200 import harness as H
    A, longest = 64, WIDE * 256
    f = Forked(shape, [(1500, [i % 3 for i in range(A)])], seed=43, wide=WIDE)
    dc, scale = f.dc, sharp / math.sqrt(shape[2])
    offs = H.dev(np.array([A * (i % 2) for i in range(n_groups + 1)], np.int32))
    lens, pre, q = H.dev(np.asarray(f.lens, np.int32)), H.dev(np.full(n_groups, 1500, np.int32)), H.bf16_dev(f.q())
    out, lse = torch.empty((A, shape[0], shape[3]), device="cuda"), torch.empty((A, shape[0]), device="cuda")
    most = B.q4kv_workspace_bytes_shared_prefix(dc.spec, A, longest, n_groups)
    room = torch.zeros(most + (64 << 20), dtype=torch.uint8, device="cuda")

    def call(size):
        out.fill_(9.0)
        lse.fill_(9.0)
        dc.flags.zero_()
        room[B.WORKSPACE_HEADER_BYTES:] = 0xA5
        B.q4kv_shared_prefix_decode_attention(dc.spec, dc.pool, f.n_blocks, 0, dc.bt, lens, longest, offs, pre, n_groups, q, scale, out,
                                              B.OUT_F32, lse, room[:size], dc.flags)
        assert torch.all(room[size:] == 0xA5) and int(room[:B.WORKSPACE_HEADER_BYTES].max()) == 0
        assert dc.read_flags() == B.FLAG_BAD_LENGTH and torch.all(out == 0) and torch.all(torch.isneginf(lse))

    low, high = 0, most                                  # the least size that is accepted
    while high - low > 1:
        size = (low + high) // 2
        try:
            call(size)
            high = size
        except B.Q4KVError as e:
            assert e.code == B.EWORKSPACE
            low = size
    call(high)
    call(most)


@pytest.mark.gpu
@pytest.mark.parametrize("wide, more", [(1, 0), (WIDE, 4), (WIDE, 80)])
def test_bad_blocks_spoil_the_agents_that_read_them(wide, more):
    f = Forked((8, 2, 128, 128), [(600, [20, 300, 9] + [1] * more), (40, [100, 3])], seed=37, wide=wide)
    q, scale = f.q(), 1.0 / math.sqrt(128)
    good, _ = f.run(q, scale)
    keep, A, n = f.dc.tables.clone(), len(f.lens), 3 + more
    for bad in (-1, f.n_blocks, 2**31 - 1, -2**31):
        f.dc.tables.copy_(keep)
        f.dc.tables[0, 1] = bad                          # of the prefix, which the whole group reads through this row, or this agent alone
        out, lse = f.run(q, scale)
        k = n if wide == WIDE else 1
        assert f.dc.read_flags() == B.FLAG_BAD_BLOCK and torch.all(out[:k] == 0) and torch.all(torch.isneginf(lse[:k]))
        assert torch.equal(out[k:], good[k:])
        f.dc.flags.zero_()
        f.dc.tables.copy_(keep)
        f.dc.tables[1, 3] = bad
        out, lse = f.run(q, scale)
        rest = [0] + list(range(2, A))
        assert f.dc.read_flags() == B.FLAG_BAD_BLOCK and torch.all(out[1] == 0) and torch.equal(out[rest], good[rest])
        f.dc.flags.zero_()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [-1.0, -0.05, 0.0, 3.0])
@pytest.mark.parametrize("shape, more", [((8, 2, 128, 128), 4), ((2, 2, 192, 128), 4), ((4, 2, 256, 256), 80)])
def test_any_softmax_scale(shape, more, scale):
    f = Forked(shape, [(600, [20, 300] + [1] * more), (300, [9, 0])], seed=41, wide=WIDE)
    q = f.q()
    out, lse = f.run(q, scale)
    close(out, lse, *f.want(q, scale))


@pytest.mark.gpu
@pytest.mark.parametrize("wide, more", [(1, 0), (WIDE, 4), (WIDE, 60)])
@pytest.mark.parametrize("shape", [(8, 2, 128, 128), (2, 2, 192, 128), (4, 2, 256, 256)])
def test_blocks_beyond_four_gigabytes(shape, wide, more):
    """The same blocks, moved to the end of a pool of 9 GB and to its last layer: the same bits."""
    from paper_2603_04428_b200 import harness as H
    f = Forked(shape, [(700, [20, 300] + [1] * more), (300, [9, 0])], seed=40, wide=wide)
    q, scale = f.q(), 1.0 / math.sqrt(shape[2])
    out, lse = f.run(q, scale)
    layers = 6
    spec = B.Spec.make(layers, *shape)
    one = B.q4kv_pool_bytes(spec, 1)
    n = (9 << 30) // one
    first = n - f.n_blocks
    assert B.q4kv_pool_bytes(spec, n) * (layers - 1) // layers > 2 ** 32
    big = H.DeviceCache(layers, *shape, False, n, np.where(f.tables >= 0, f.tables + first, -1).astype(np.int32))
    # the small pool has one layer; it goes to the big one's last through a pool of as many layers
    mid = torch.zeros(B.q4kv_pool_bytes(spec, f.n_blocks), dtype=torch.uint8, device="cuda")
    mid[f.dc.pool.numel() * (layers - 1):] = f.dc.pool
    copies = H.dev(np.array([(i, first + i, 256) for i in range(f.n_blocks)], np.int32))
    B.q4kv_copy_blocks(spec, mid, f.n_blocks, big.pool, n, layers - 1, 1, copies, f.n_blocks, big.flags)
    far, far_lse = big.shared_prefix_decode(layers - 1, f.lens, f.offs, f.prefix, q, scale)
    assert big.read_flags() == 0 and torch.equal(far, out) and torch.equal(far_lse, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(4, 1, 128, 128), (2, 1, 256, 256)])
def test_a_workspace_for_the_largest_call_serves_smaller_ones(shape):
    """Fewer agents can be cut into more parts, which need more room than the largest batch's plan: parts follow the room."""
    from paper_2603_04428_b200 import harness as H
    f = Forked(shape, [(3000, [i % 4 for i in range(65)])], seed=42, wide=WIDE)
    q, scale, dc, most = f.q(), 1.0 / math.sqrt(shape[2]), f.dc, WIDE * 256
    want, want_lse = f.want(q, scale)
    room = B.q4kv_workspace_bytes_shared_prefix(dc.spec, 65, most, 1)
    assert B.q4kv_workspace_bytes_shared_prefix(dc.spec, 64, most, 1) > room          # or nothing is tested here
    ws = torch.zeros(room, dtype=torch.uint8, device="cuda")
    qd, lens, pre = H.bf16_dev(q), H.dev(np.asarray(f.lens, np.int32)), H.dev(np.asarray(f.prefix, np.int32))
    for a, longest in ((65, most), (64, most), (33, most), (64, 100000), (64, 20000), (64, 4096), (5, 4096), (1, 4096)):
        out = torch.full((65, shape[0], shape[3]), 9.0, device="cuda")
        lse = torch.full((65, shape[0]), 9.0, device="cuda")
        offs = H.dev(np.array([0, a], np.int32))
        B.q4kv_shared_prefix_decode_attention(dc.spec, dc.pool, f.n_blocks, 0, B.Batch(a, WIDE, dc.bt.block_tables), lens, longest, offs,
                                              pre, 1, qd, scale, out, B.OUT_F32, lse, ws, dc.flags)
        close(out[:a], lse[:a], want[:a], want_lse[:a])
        assert torch.all(out[a:] == 9.0) and torch.all(lse[a:] == 9.0)                # rows behind the last agent
    assert dc.read_flags() == 0 and int(ws[:B.WORKSPACE_HEADER_BYTES].max()) == 0


@pytest.mark.gpu
def test_the_largest_batch_and_runs_that_repeat():
    """512 agents in uneven groups; the same bits every time, from a workspace that other calls have used, eager and replayed."""
    r = np.random.default_rng(4)
    sizes = [200, 1, 100, 64, 33, 114]
    f = Forked((2, 1, 128, 128), [(int(r.integers(0, 700)), [int(x) for x in r.integers(0, 60, n)]) for n in sizes], seed=38, wide=WIDE)
    q, scale = f.q(), 1.0 / math.sqrt(128)
    out, lse = f.run(q, scale)
    close(out, lse, *f.want(q, scale))
    A, spec, dc = 512, f.dc.spec, f.dc
    most = WIDE * 256
    need = max(B.q4kv_workspace_bytes_shared_prefix(spec, A, most, 6), B.q4kv_workspace_bytes(spec, A, most, 0))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:B.WORKSPACE_HEADER_BYTES] = 0
    from paper_2603_04428_b200 import harness as H
    lens, offs, pre, qd = H.dev(np.asarray(f.lens, np.int32)), H.dev(f.offs), H.dev(np.asarray(f.prefix, np.int32)), H.bf16_dev(q)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)

    def call():
        B.q4kv_shared_prefix_decode_attention(spec, dc.pool, f.n_blocks, 0, dc.bt, lens, most, offs, pre, 6, qd, scale, o2, B.OUT_F32,
                                              l2, ws, dc.flags)
    call()
    assert torch.equal(o2, out) and torch.equal(l2, lse) and int(ws[:B.WORKSPACE_HEADER_BYTES].max()) == 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(3):
            call()
    ws[B.WORKSPACE_HEADER_BYTES:] = 0xFF
    o2.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    gone = torch.arange(A, device="cuda") % 3 == 0       # the replay reads the lengths of the moment
    lens.copy_(torch.where(gone, 0, lens))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.all(o2[gone] == 0) and torch.allclose(o2[~gone], out[~gone], rtol=0, atol=2 * ATOL)
    assert dc.read_flags() == 0


@pytest.mark.gpu
def test_a_decode_step_of_forked_agents():
    """Fork, copy, norm and rotate, append, attend: the step as it is used, against agents that hold everything themselves."""
    from paper_2603_04428_b200 import harness as H
    hq, hkv, d, n_blocks, parent_len, steps = 8, 2, 128, 24, 700, 3
    al = B.Allocator(n_blocks)
    tables = np.full((5, 4), -1, np.int32)
    tables[0] = al.reserve(0, parent_len, 4)
    cache = H.DeviceCache(1, hq, hkv, d, d, False, n_blocks, tables)
    f = torch.from_numpy((10000.0 ** (-2.0 * np.arange(64) / 128)).astype(np.float32)).cuda()
    w = torch.from_numpy(synth.bf16_bits_to_f32(synth.normal_bf16(6, 1, (2, d)))).cuda().to(torch.bfloat16)
    how = B.NormRotation.make(norm_dim=d, q_weight=w[0], k_weight=w[1], weight_offset=1.0, rot_dim=d, inv_freq=f)

    def rows(c, bt, pos, offs, qkv):
        n = qkv.shape[0]
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:].contiguous()
        qo, ko = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda")
        B.q4kv_norm_rope(c.spec, how, len(pos), pos, offs, n, q, k, qo, ko, c.flags)
        B.q4kv_quantize_append(c.spec, c.pool, c.n_blocks, 0, bt, pos, offs, n, ko, v, c.flags)
        return qo

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    prompt = H.bf16_dev(synth.normal_bf16(6, 2, (parent_len, hq + 2 * hkv, d)))
    keep, bt0 = cache.sub_batch(0, 1)
    rows(cache, bt0, ints([0]), ints([0, parent_len]), prompt)
    copies = []
    for child in range(1, 5):
        tables[child], copy = al.fork(0, child, parent_len, 4)
        copies.append(copy)
    B.q4kv_copy_blocks(cache.spec, cache.pool, n_blocks, cache.pool, n_blocks, 0, 1, ints(copies), 4, cache.flags)
    for a in range(5):
        tables[a] = al.reserve(a, parent_len + steps, 4)
    cache.tables.copy_(torch.from_numpy(tables))
    alone = H.DeviceCache(1, hq, hkv, d, d, False, 20, np.arange(20, dtype=np.int32).reshape(5, 4)[:, ::-1].copy())
    rows(alone, alone.bt, ints([0] * 5), ints([parent_len * i for i in range(6)]), prompt.repeat(5, 1, 1))
    for step in range(steps):
        new = H.bf16_dev(synth.normal_bf16(6, 10 + step, (5, hq + 2 * hkv, d)))
        pos, offs = ints([parent_len + step] * 5), ints(range(6))
        q1, q2 = rows(cache, cache.bt, pos, offs, new), rows(alone, alone.bt, pos, offs, new)
        assert torch.equal(q1, q2)
        lens = [parent_len + step + 1] * 5
        out, lse = cache.shared_prefix_decode(0, lens, [0, 5], [parent_len], q1, 1 / math.sqrt(d))
        ref, ref_lse = alone.decode(0, lens, 0, q2, 1 / math.sqrt(d))
        close(out, lse, ref.double().cpu().numpy(), ref_lse.double().cpu().numpy())
    for a in range(5):
        assert torch.equal(cache.pack(a, parent_len + steps), alone.pack(a, parent_len + steps))
    assert cache.read_flags() == alone.read_flags() == 0


def test_refusals():
    if torch.cuda.is_available():
        pytest.skip("placeholder pointers are only handed to the library on a host without a CUDA device")
    lib, p = B.lib(), 0x1000
    spec = B.Spec.make(2, 8, 2, 128, 128)

    def call(sp=spec, agents=2, max_blocks=4, pool=p, n_blocks=4, layer=0, lens=p, max_kv=1024, offs=p, prefix=p, groups=1, q=p,
             scale=0.1, out=p, out_dtype=0, ws=p, size=1 << 40, tables=p):
        bt = B.Batch(agents, max_blocks, tables)
        return lib.q4kv_shared_prefix_decode_attention(ctypes.byref(sp), pool, n_blocks, layer, ctypes.byref(bt), lens, max_kv, offs,
                                                       prefix, groups, q, scale, out, out_dtype, None, ws, size, None, None)

    for bad in (dict(agents=-1), dict(max_blocks=0), dict(pool=None), dict(n_blocks=0), dict(layer=2), dict(layer=-1), dict(lens=None),
                dict(max_kv=-1), dict(offs=None), dict(prefix=None), dict(groups=0), dict(groups=-1), dict(groups=3), dict(q=None),
                dict(out=None), dict(out_dtype=2), dict(ws=None), dict(tables=None), dict(pool=0x1008), dict(q=0x1004), dict(out=0x1001),
                dict(ws=0x1008)):
        assert call(**bad) == B.EINVAL, bad
    make = B.Spec.make
    for bad in (dict(sp=make(2, 8, 2, 64, 64)), dict(sp=make(2, 16, 1, 576, 512, True)), dict(sp=make(2, 8, 2, 128, 128, True)),
                dict(sp=make(2, 8, 2, 192, 192)), dict(sp=make(2, 8, 2, 128, 128, exact_products=True)),
                dict(agents=8193), dict(max_blocks=2**23), dict(agents=512, max_blocks=2**22, max_kv=0, sp=make(2, 64, 64, 128, 128))):
        assert call(**bad) == B.EUNSUPPORTED, bad
    need = B.q4kv_workspace_bytes_shared_prefix(spec, 2, 1024, 1)
    assert need > B.WORKSPACE_HEADER_BYTES and call(size=need - 1) == B.EWORKSPACE
    assert call(agents=0, tables=None) == B.OK
    for args in ((make(2, 8, 2, 64, 64), 2, 1024, 1), (spec, 8193, 1024, 1), (spec, -1, 1024, 1), (spec, 2, -1, 1), (spec, 2, 1024, 3),
                 (spec, 2, 1024, -1)):
        assert B.q4kv_workspace_bytes_shared_prefix(*args) == 0
    assert B.q4kv_workspace_bytes_shared_prefix(spec, 3, 1024, 1) >= need
