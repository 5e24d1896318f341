"""Forked agents: block sharing in the allocator (host only), and the block copies that go with it (GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_04428_b200 import binding as B, synth


# ---- allocator (no GPU) --------------------------------------------------------------------------------------------------

def test_a_fork_shares_whole_blocks_and_copies_the_last():
    al = B.Allocator(10)
    parent = al.reserve(1, 700, 4)
    row, copy = al.fork(1, 2, 600, 4)
    assert row == parent[:2] + [3, -1] and copy == (parent[2], 3, 88)
    assert [al.block_holders(b) for b in range(5)] == [2, 2, 1, 1, 0] and al.free_blocks() == 6
    assert al.table(2, 4) == row and al.table(1, 4) == parent
    row3, copy3 = al.fork(2, 3, 512, 2)                                     # a fork of a fork, at a block's end
    assert row3 == parent[:2] and copy3 is None and al.block_holders(parent[0]) == 3
    row4, copy4 = al.fork(1, 4, 0, 1)
    assert row4 == [-1] and copy4 is None and al.agent_blocks(4) == 0
    grown = al.reserve(2, 800, 4)                                           # growth adds blocks of its own
    assert grown[:3] == row[:3] and al.block_holders(grown[3]) == 1
    al.release(1)
    assert al.free_blocks() == 6 and [al.block_holders(b) for b in parent[:3]] == [2, 2, 0]
    al.release(3)
    al.release(2)
    assert al.free_blocks() == 10 and all(al.block_holders(b) == 0 for b in range(10))


def test_forks_that_cannot_be_leave_everything_as_it_was():
    al = B.Allocator(3)
    al.reserve(1, 600, 3)
    for args in ((9, 2, 10, 3), (1, 1, 10, 3), (1, 2, 769, 3), (1, 2, 600, 2), (1, 2, -1, 3)):
        with pytest.raises(B.Q4KVError) as e:
            al.fork(*args)
        assert e.value.code == B.EINVAL
    with pytest.raises(B.Q4KVError) as e:
        al.fork(1, 2, 300, 3)                                               # no free block for the partly filled one
    assert e.value.code == B.EWORKSPACE and al.agent_blocks(2) == 0 and [al.block_holders(b) for b in range(3)] == [1, 1, 1]
    row, copy = al.fork(1, 2, 512, 3)                                       # whole blocks need none
    assert copy is None and row == [0, 1, -1] and al.pick_victim() == 1
    lib, three, row = B.lib(), (ctypes.c_int32 * 3)(), (ctypes.c_int32 * 3)()
    assert lib.q4kv_allocator_fork(None, 1, 5, 0, row, 3, three) == B.EINVAL
    assert lib.q4kv_allocator_fork(al._h, 1, 5, 0, row, 3, None) == B.EINVAL
    assert al.block_holders(-1) == al.block_holders(3) == -1
    with pytest.raises(B.Q4KVError):
        al.table(7, 3)
    with pytest.raises(B.Q4KVError):
        al.table(1, 2)                                                      # its row does not fit


def test_truncation_gives_blocks_back_and_leaves_shared_ones():
    al = B.Allocator(6)
    parent = al.reserve(1, 1000, 4)
    al.fork(1, 2, 768, 4)
    row, copy = al.truncate(2, 700, 4)                                      # block 2 is shared and will be written by agent 2
    assert copy == (parent[2], 4, 188) and row == parent[:2] + [4, -1] and al.block_holders(parent[2]) == 1
    assert al.table(1, 4) == parent
    row, copy = al.truncate(2, 650, 4)                                      # its own block by now
    assert copy is None and row == parent[:2] + [4, -1]
    row, copy = al.truncate(2, 256, 4)
    assert copy is None and row == [parent[0], -1, -1, -1] and al.free_blocks() == 2
    row, copy = al.truncate(1, 0, 4)
    assert copy is None and row == [-1] * 4 and al.free_blocks() == 5 and al.block_holders(parent[0]) == 1
    with pytest.raises(B.Q4KVError) as e:
        al.truncate(2, 300, 4)
    assert e.value.code == B.EINVAL                                         # it never had that many
    full = B.Allocator(2)
    full.reserve(1, 512, 2)
    full.fork(1, 2, 512, 2)
    with pytest.raises(B.Q4KVError) as e:
        full.truncate(2, 300, 2)
    assert e.value.code == B.EWORKSPACE and full.table(2, 2) == [0, 1] and full.block_holders(1) == 2
    full2 = B.Allocator(3)
    full2.reserve(1, 512, 3)
    full2.fork(1, 2, 512, 3)
    full2.reserve(2, 600, 3)                                                # no block is free, but the truncation frees one
    row, copy = full2.truncate(2, 300, 3)
    assert copy == (1, 2, 44) and row == [0, 2, -1] and full2.free_blocks() == 0


def test_compaction_moves_the_highest_blocks_down_and_the_tables_follow():
    al = B.Allocator(12)
    for agent in range(4):
        al.reserve(agent, 700, 4)
    al.fork(3, 9, 512, 4)
    al.release(0)
    al.release(2)
    before = {a: al.table(a, 4) for a in (1, 3, 9)}
    assert al.compact(0) == []
    moves = al.compact(2)
    assert moves == [(11, 0, 256), (10, 1, 256)]
    moves += al.compact(10)
    to = {a: b for a, b, _ in moves}
    assert set(to).isdisjoint(to.values()) and len(set(to.values())) == len(to)
    for a, row in before.items():
        assert al.table(a, 4) == [to.get(b, b) for b in row]
    held = [b for b in range(12) if al.block_holders(b)]
    assert held == list(range(6)) and al.free_blocks() == 6 and al.compact(10) == []
    assert al.table(9, 4)[:2] == al.table(3, 4)[:2] and al.block_holders(al.table(9, 4)[0]) == 2
    assert al.reserve(50, 1, 1) == [6]                                      # the lowest free block comes first
    with pytest.raises(B.Q4KVError):
        al.compact(-1)


def test_a_schedule_of_forks_truncations_and_releases_keeps_the_counts():
    g = np.random.default_rng(5)
    al, live, nxt = B.Allocator(40), {}, 0                                  # live: agent -> tokens
    for _ in range(600):
        what = g.integers(0, 5)
        agent = int(g.choice(list(live))) if live else None
        try:
            if what == 0 or agent is None:
                n = int(g.integers(0, 1500))
                al.reserve(nxt, n, 8)
                live[nxt] = n
                nxt += 1
            elif what == 1:
                n = int(g.integers(0, live[agent] + 1))
                al.fork(agent, nxt, n, 8)
                live[nxt] = n
                nxt += 1
            elif what == 2:
                n = int(g.integers(0, live[agent] + 1))
                al.truncate(agent, n, 8)
                live[agent] = n
            elif what == 3:
                al.release(agent)
                del live[agent]
            else:
                al.compact(int(g.integers(0, 6)))
        except B.Q4KVError as e:
            assert e.code == B.EWORKSPACE
        rows = {a: [b for b in al.table(a, 8) if b >= 0] for a in live}
        count = np.zeros(40, int)
        for a, row in rows.items():
            assert len(set(row)) == len(row) >= -(-live[a] // 256)
            for b in row:
                count[b] += 1
        assert [al.block_holders(b) for b in range(40)] == count.tolist() and al.free_blocks() == int((count == 0).sum())
        for a, row in rows.items():                                         # a block that is still to be written has one holder
            assert live[a] % 256 == 0 or count[row[live[a] // 256]] == 1


def test_copy_refusals_come_before_the_device():
    if torch.cuda.is_available():
        pytest.skip("placeholder pointers are only handed to the library on a host without a CUDA device")
    lib, spec = B.lib(), B.Spec.make(4, 8, 2, 128, 128)
    p, odd = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)

    def call(sp=spec, src=p, ns=4, dst=p, nd=4, l0=0, nl=4, copies=p, n=1):
        return lib.q4kv_copy_blocks(ctypes.byref(sp), src, ns, dst, nd, l0, nl, copies, n, None, None)

    for bad in (dict(src=None), dict(dst=None), dict(ns=0), dict(nd=-1), dict(l0=-1), dict(l0=1), dict(nl=-1), dict(l0=2**31 - 1),
                dict(copies=None), dict(n=-1), dict(src=odd), dict(dst=odd), dict(nd=5)):
        assert call(**bad) == B.EINVAL, bad
    assert call(sp=B.Spec.make(4, 8, 2, 96, 128)) == B.EUNSUPPORTED
    assert call(n=2**31 - 1) == B.EUNSUPPORTED
    assert call(n=0) == call(nl=0) == B.OK


# ---- copies on the GPU ---------------------------------------------------------------------------------------------------

SHAPES = [(3, 8, 2, 128, 128, False), (2, 16, 8, 256, 256, False), (2, 16, 16, 192, 128, False), (2, 16, 1, 576, 512, True),
          (1, 4, 4, 64, 64, False)]


def _pool(shape, n_blocks, seed):
    spec = B.Spec.make(*shape)
    n = B.q4kv_pool_bytes(spec, n_blocks)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.randint(0, 256, (n,), dtype=torch.uint8, generator=g, device="cuda")
    return spec, pool, pool.view(shape[0], n_blocks, shape[2], 8, -1)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_copies_move_whole_chunks_and_nothing_else(shape):
    spec, src, sv = _pool(shape, 9, 1)
    _, dst, dv = _pool(shape, 13, 2)
    copies = [(0, 12, 256), (8, 0, 1), (3, 5, 32), (3, 6, 33), (4, 7, 0), (7, 8, 255), (1, 1, 100)]
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = dv.clone()
    first, count = (1, shape[0] - 1) if shape[0] > 2 else (0, shape[0])
    for a, b, n in copies:
        c = -(-n // 32)
        want[first:first + count, b, :, :c] = sv[first:first + count, a, :, :c]
    t = torch.tensor(copies, dtype=torch.int32, device="cuda")
    B.q4kv_copy_blocks(spec, src, 9, dst, 13, first, count, t, len(copies), flags)
    assert torch.equal(dv, want) and flags.item() == 0
    # within one pool, a block onto itself among them
    want = sv.clone()
    for a, b, n in [(2, 5, 200), (6, 6, 256), (0, 8, 40)]:
        want[:, b, :, :-(-n // 32)] = sv[:, a, :, :-(-n // 32)]
    t = torch.tensor([(2, 5, 200), (6, 6, 256), (0, 8, 40)], dtype=torch.int32, device="cuda")
    B.q4kv_copy_blocks(spec, src, 9, src, 9, 0, shape[0], t, 3, flags)
    assert torch.equal(sv, want) and flags.item() == 0


@pytest.mark.gpu
def test_bad_copies_raise_their_flags_and_are_skipped():
    spec, pool, v = _pool(SHAPES[0], 6, 3)
    want = v.clone()
    want[:, 4] = v[:, 2]
    for bad, flag in (((-1, 1, 256), B.FLAG_BAD_BLOCK), ((6, 1, 256), B.FLAG_BAD_BLOCK), ((0, -1, 256), B.FLAG_BAD_BLOCK),
                      ((0, 6, 256), B.FLAG_BAD_BLOCK), ((0, 2**31 - 1, 256), B.FLAG_BAD_BLOCK), ((0, 1, 257), B.FLAG_BAD_LENGTH),
                      ((0, 1, -1), B.FLAG_BAD_LENGTH)):
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        t = torch.tensor([bad, (2, 4, 256)], dtype=torch.int32, device="cuda")
        B.q4kv_copy_blocks(spec, pool, 6, pool, 6, 0, 3, t, 2, flags)
        assert flags.item() == flag and torch.equal(v, want), bad
    B.q4kv_copy_blocks(spec, pool, 6, pool, 6, 0, 3, None, 0)                 # nothing to do


@pytest.mark.gpu
def test_a_captured_copy_replays_with_the_list_of_the_moment():
    spec, pool, v = _pool(SHAPES[0], 6, 4)
    t = torch.tensor([(0, 3, 256)], dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        B.q4kv_copy_blocks(spec, pool, 6, pool, 6, 0, 3, t, 1)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        B.q4kv_copy_blocks(spec, pool, 6, pool, 6, 0, 3, t, 1)
    want = v.clone()
    want[:, 5, :, :2] = v[:, 1, :, :2]
    t.copy_(torch.tensor([(1, 5, 64)], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(v, want)


@pytest.mark.gpu
def test_a_list_of_copies_beyond_two_gigaentries():
    """The list's last copies lie past entry 2^31; those before them copy nothing."""
    n = 2 ** 31 // 3 + 20
    spec = B.Spec.make(1, 1, 1, 128, 128)
    pool = torch.randint(0, 256, (B.q4kv_pool_bytes(spec, 40),), dtype=torch.uint8, device="cuda")
    t = torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    t[-20:] = torch.tensor([(i, 20 + i, 256) for i in range(20)], dtype=torch.int32)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = pool.clone().view(40, -1)
    want[20:] = want[:20]
    B.q4kv_copy_blocks(spec, pool, 40, pool, 40, 0, 1, t, n, flags)
    assert torch.equal(pool.view(40, -1), want) and int(flags) == 0


@pytest.mark.gpu
def test_forked_agents_hold_what_they_would_have_built_alone():
    """A parent of 600 tokens, a fork at 550, more tokens for both, then compaction: the packed bytes of both equal those of
    agents that appended the same rows by themselves."""
    from paper_2603_04428_b200 import harness as H
    n_blocks, layers, hkv, d = 12, 2, 2, 128
    al = B.Allocator(n_blocks)
    al.reserve(77, 700, 4)
    rows = np.full((2, 4), -1, np.int32)
    rows[0] = al.reserve(1, 600, 4)
    cache = H.DeviceCache(layers, 8, hkv, d, d, False, n_blocks, rows)
    alone = H.DeviceCache(layers, 8, hkv, d, d, False, n_blocks, np.array([[5, 2, 9, 4], [0, 7, 1, 3]], np.int32))
    kv = [[synth.normal_bf16(11, 10 * l + i, (1000, hkv, d)) for i in range(4)] for l in range(layers)]

    def put(c, agent, layer, at, k, v):
        _, b = c.sub_batch(agent, agent + 1)
        c.append(layer, [at], [0, len(k)], k, v, bt=b)

    for l in range(layers):
        k, v = kv[l][0], kv[l][1]
        put(cache, 0, l, 0, k[:600], v[:600])
        for a in range(2):
            put(alone, a, l, 0, k[:600 if a == 0 else 550], v[:600 if a == 0 else 550])
    rows[1], copy = al.fork(1, 2, 550, 4)
    assert copy[2] == 550 - 512
    B.q4kv_copy_blocks(cache.spec, cache.pool, n_blocks, cache.pool, n_blocks, 0, layers, H.dev(np.array([copy], np.int32)), 1,
                       cache.flags)
    rows[1], rows[0] = al.reserve(2, 950, 4), al.reserve(1, 800, 4)
    cache.tables.copy_(torch.from_numpy(rows))
    for l in range(layers):
        for c in (cache, alone):
            put(c, 0, l, 600, kv[l][0][600:800], kv[l][1][600:800])
            put(c, 1, l, 550, kv[l][2][:400], kv[l][3][:400])
    assert al.release(77) is None
    moves = al.compact(12)
    assert len(moves) == 3
    B.q4kv_copy_blocks(cache.spec, cache.pool, n_blocks, cache.pool, n_blocks, 0, layers, H.dev(np.array(moves, np.int32)), 3,
                       cache.flags)
    cache.tables.copy_(torch.tensor([al.table(1, 4), al.table(2, 4)], dtype=torch.int32))
    for agent, n in ((0, 800), (1, 950)):
        assert torch.equal(cache.pack(agent, n), alone.pack(agent, n))
    assert cache.read_flags() == alone.read_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("between", ["no tokens", "bad blocks", "onto themselves", "rows of no agent", "agents of no group"])
def test_a_call_without_work_does_not_let_its_successor_overtake_its_predecessor(between):
    """Copy, a call that has nothing to do, a copy of what the first one wrote: launches that overlap in a stream have to wait for
    their predecessors also when they do nothing."""
    n = 1500
    spec, a, _ = _pool((2, 32, 8, 128, 128, False), n, 5)
    b, c = torch.zeros_like(a), torch.zeros_like(a)
    every = torch.tensor([(i, i, 256) for i in range(n)], dtype=torch.int32, device="cuda")
    last = torch.tensor([(i, i, 256) for i in range(n - 40, n)], dtype=torch.int32, device="cuda")
    none = {"no tokens": (0, 1, 0), "bad blocks": (-1, 0, 256), "onto themselves": (3, 3, 256)}.get(between)
    x = torch.zeros((4, 32, 128), dtype=torch.bfloat16, device="cuda")
    zeros = torch.zeros(256, dtype=torch.int32, device="cuda")
    if none:
        idle = torch.tensor([none] * 8, dtype=torch.int32, device="cuda")
        call = lambda: B.q4kv_copy_blocks(spec, a, n, a, n, 0, 2, idle, 8)
    elif between == "rows of no agent":
        f = torch.ones(64, device="cuda")
        how = B.NormRotation.make(rot_dim=128, inv_freq=f)
        call = lambda: B.q4kv_norm_rope(spec, how, 2, zeros, zeros, 4, x, None, x, None)
    else:
        q = torch.zeros((200, 32, 128), dtype=torch.bfloat16, device="cuda")
        out = torch.zeros_like(q)
        tables = torch.zeros((200, 64), dtype=torch.int32, device="cuda")
        bt = B.Batch(200, 64, tables.data_ptr())
        ws = torch.zeros(B.q4kv_workspace_bytes_shared_prefix(spec, 200, 64 * 256, 1), dtype=torch.uint8, device="cuda")
        call = lambda: B.q4kv_shared_prefix_decode_attention(spec, a, n, 0, bt, zeros, 64 * 256, zeros, zeros, 1, q, 0.1, out, B.OUT_BF16,
                                                             None, ws)
    for _ in range(10):
        b.zero_()
        c.zero_()
        B.q4kv_copy_blocks(spec, a, n, b, n, 0, 2, every, n)
        call()
        B.q4kv_copy_blocks(spec, b, n, c, n, 0, 2, last, 40)
        got, want = (t.view(2, n, 8, 8, -1)[:, n - 40:] for t in (c, a))
        assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("agents", [1, 3, 40])
@pytest.mark.parametrize("shape, sharp", [((8, 2, 128, 128, False), 1.0), ((8, 2, 256, 256, False), 1.0), ((4, 4, 192, 128, False), 1.0),
                                          ((16, 1, 576, 512, True), 1.0), ((8, 2, 128, 128, False), 2.5), ((8, 2, 256, 256, False), 2.5),
                                          ((4, 2, 64, 64, False), 1.0)])
def test_a_prefill_without_queries_does_not_let_its_successor_overtake_its_predecessor(shape, sharp, agents):
    """As above, for a prefill call in which no agent has a query (a step of a captured schedule with nothing to do)."""
    n = 1500
    spec, a, _ = _pool((2, 32, 8, 128, 128, False), n, 5)
    b, c = torch.zeros_like(a), torch.zeros_like(a)
    every = torch.tensor([(i, i, 256) for i in range(n)], dtype=torch.int32, device="cuda")
    last = torch.tensor([(i, i, 256) for i in range(n - 40, n)], dtype=torch.int32, device="cuda")
    other = B.Spec.make(1, *shape)
    rows, width = 64, 64
    pool = torch.zeros(B.q4kv_pool_bytes(other, 2), dtype=torch.uint8, device="cuda")
    q = torch.zeros((rows, shape[0], shape[2]), dtype=torch.bfloat16, device="cuda")
    out = torch.full((rows, shape[0], shape[3]), 9.0, dtype=torch.bfloat16, device="cuda")
    tables, zeros = torch.zeros((agents, width), dtype=torch.int32, device="cuda"), torch.zeros(256, dtype=torch.int32, device="cuda")
    ws = torch.zeros(B.q4kv_workspace_bytes(other, agents, width * 256, rows), dtype=torch.uint8, device="cuda")
    bt = B.Batch(agents, width, tables.data_ptr())
    for _ in range(10):
        b.zero_()
        c.zero_()
        B.q4kv_copy_blocks(spec, a, n, b, n, 0, 2, every, n)
        B.q4kv_prefill_attention(other, pool, 2, 0, bt, zeros, zeros, rows, rows, width * 256, 0, q, sharp / shape[2] ** 0.5, out,
                                 B.OUT_BF16, None, ws)
        B.q4kv_copy_blocks(spec, b, n, c, n, 0, 2, last, 40)
        got, want = (t.view(2, n, 8, 8, -1)[:, n - 40:] for t in (c, a))
        assert torch.equal(got, want)
