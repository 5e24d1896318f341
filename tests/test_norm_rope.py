"""q4kv_norm_rope against the formula in 64 bits (80 where angles are large), and its refusals."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_04428_b200 import binding as B, synth


def reference(x, weight, norm_dim, eps, offset, rot_begin, rot_dim, interleaved, scale, inv_freq, position):
    """x: float64 [rows][heads][d].  (the result, the magnitude that its errors scale with)"""
    y = x.copy()
    if norm_dim and weight is not None:
        part = x[..., :norm_dim]
        y[..., :norm_dim] = part / np.sqrt((part * part).mean(-1, keepdims=True) + eps) * (weight + offset)
    size = np.abs(y)
    if rot_dim:
        j = np.arange(rot_dim // 2)
        a, b = (rot_begin + 2 * j, rot_begin + 2 * j + 1) if interleaved else (rot_begin + j, rot_begin + j + rot_dim // 2)
        turn = position.astype(np.longdouble)[:, None] * inv_freq.astype(np.longdouble)
        cos, sin = (f(turn).astype(np.float64)[:, None] * scale for f in (np.cos, np.sin))
        ya, yb = y[..., a], y[..., b]
        size[..., a] = size[..., b] = (np.abs(ya) + np.abs(yb)) * abs(scale)
        y[..., a], y[..., b] = ya * cos - yb * sin, yb * cos + ya * sin
    return y, size


def check(got, want, size):
    # one rounding to bfloat16 (half a step: 2^-8 of the value), and binary32 arithmetic: at most 16 roundings of 2^-24 in the
    # norm's sum, root and products, 1.6 * 2^-24 for the reduced angle, 4 for sine or cosine and 3 for the rotation itself, below
    # 32 * 2^-24 of the pair's magnitude
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.all(np.isfinite(got))
    err = np.abs(got - want) - (2.0 ** -8 * (np.abs(want) + 2.0 ** -19 * size) + 2.0 ** -19 * size)
    assert err.max() <= 0, err.max()


def theta(rot_dim, base=10000.0):
    return (base ** (-2.0 * np.arange(rot_dim // 2) / rot_dim)).astype(np.float32) if rot_dim else None


#        Hq  Hkv  d   norm offset rot_begin rot_dim interleaved scale
CASES = [(8, 2, 128, 0, 0.0, 0, 128, False, 1.0),
         (8, 2, 128, 128, 1.0, 0, 128, True, 1.0),
         (5, 5, 64, 64, 0.0, 0, 64, False, 1.25),
         (3, 1, 64, 40, 0.5, 16, 32, False, 1.0),
         (16, 16, 192, 0, 0.0, 128, 64, True, 1.0),
         (7, 7, 192, 192, 0.0, 40, 144, False, 1.0),
         (16, 8, 256, 256, 1.0, 0, 256, False, 1.0),
         (6, 2, 256, 256, 0.0, 64, 48, False, 0.5),
         (2, 1, 320, 320, 0.0, 0, 320, False, 1.0),
         (4, 4, 512, 512, 0.0, 256, 256, True, 1.0),
         (16, 1, 576, 512, 0.0, 512, 64, False, 1.0),
         (2, 2, 1024, 1024, 0.0, 0, 1024, False, 1.0),
         (4, 2, 128, 128, 0.0, 0, 0, False, 1.0),
         (4, 2, 128, 0, 0.0, 0, 0, False, 1.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("news, cached", [([1, 1, 1], [0, 4095, 131071]), ([700], [3]), ([0, 5, 0, 31, 2], [7, 0, 1, 120000, 2**31 - 2])])
def test_against_the_formula(case, news, cached):
    hq, hkv, d, norm, offset, rot_begin, rot_dim, inter, scale = case
    total, eps = sum(news), 1e-6
    f = theta(rot_dim)
    x = synth.bf16_bits_to_f32(synth.normal_bf16(3, 1, (total, hq + 2 * hkv, d))) * 3.0
    if total > 2:
        x[1, 0] = 0.0                                    # a head of zeros
        x[2, 1] *= 1e-4                                  # one whose mean square is no larger than eps
    t = torch.from_numpy(x).cuda().to(torch.bfloat16)
    q, k = t[:, :hq], t[:, hq:hq + hkv]                  # views of one projection
    w = torch.from_numpy(synth.bf16_bits_to_f32(synth.normal_bf16(3, 2, (2, max(norm, 8))))).cuda().to(torch.bfloat16)
    how = B.NormRotation.make(norm_dim=norm, q_weight=w[0] if norm else None, k_weight=w[1] if norm else None, eps=eps,
                              weight_offset=offset, rot_begin=rot_begin, rot_dim=rot_dim, interleaved=inter, rot_scale=scale,
                              inv_freq=None if f is None else torch.from_numpy(f).cuda())
    spec = B.Spec.make(1, hq, hkv, d, min(d, 512))
    pos = torch.tensor(cached, dtype=torch.int32).cuda()
    offs = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
    q_out = torch.full((total + 1, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    k_out = torch.full((total + 1, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.q4kv_norm_rope(spec, how, len(news), pos, offs, total, q, k, q_out[:total], k_out[:total], flags)
    position = np.concatenate([c + np.arange(n, dtype=np.int64) for c, n in zip(cached, news)])
    for got, src, weight in ((q_out, q, w[0]), (k_out, k, w[1])):
        want, size = reference(src.float().cpu().numpy().astype(np.float64), weight.float().cpu().numpy().astype(np.float64)[:norm],
                               norm, eps, offset, rot_begin, rot_dim, inter, scale, f, position)
        check(got[:total], want, size)
        assert torch.all(got[total] == 7.0)
    assert flags.item() == 0
    # contiguous rows, in place: the same bits
    qc, kc = q.contiguous(), k.contiguous()
    B.q4kv_norm_rope(spec, how, len(news), pos, offs, total, qc, kc, qc, kc, flags)
    assert torch.equal(qc, q_out[:total]) and torch.equal(kc, k_out[:total])
    # one side alone
    qa = torch.empty_like(qc)
    B.q4kv_norm_rope(spec, how, len(news), pos, offs, total, q, None, qa, None, flags)
    ka = torch.empty_like(kc)
    B.q4kv_norm_rope(spec, how, len(news), pos, offs, total, None, k, None, ka, flags)
    assert torch.equal(qa, qc) and torch.equal(ka, kc)


@pytest.mark.gpu
def test_many_rows_and_few_give_the_same_bits():
    """The launch shape depends on the number of rows; the values do not."""
    for hq, hkv, d in ((8, 2, 128), (16, 16, 192), (16, 8, 256), (4, 4, 64)):
        n, f = 1500, torch.from_numpy(theta(64)).cuda()
        x = torch.randn((n, hq, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
        w = torch.ones(d, dtype=torch.bfloat16, device="cuda") * 0.75
        how = B.NormRotation.make(norm_dim=d, q_weight=w, rot_dim=64, inv_freq=f)
        spec, out, one = B.Spec.make(1, hq, hkv, d, 64), torch.empty_like(x), torch.empty_like(x)
        z = torch.zeros(1, dtype=torch.int32, device="cuda")
        B.q4kv_norm_rope(spec, how, 1, z, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, x, None, out, None)
        for i in (0, 1, 777, n - 1):
            B.q4kv_norm_rope(spec, how, 1, z + i, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1, x[i:i + 1], None,
                             one[i:i + 1], None)
            assert torch.equal(one[i], out[i])


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_a_warp_that_takes_whole_tokens_gives_the_same_bits(case):
    """Enough rows that a warp has a token's query and key heads, out of place and in place, against calls of few rows."""
    hq, hkv, d, norm, offset, rot_begin, rot_dim, inter, scale = case
    hq, hkv, n = 2 * hkv + 1 if hq > 2 * hkv else hq, hkv, 15001
    if hq % hkv:
        hq = hkv
    f = theta(rot_dim)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((n, hq + hkv, d), device="cuda", generator=g).to(torch.bfloat16)
    w = torch.randn((2, max(norm, 8)), device="cuda", generator=g).to(torch.bfloat16)
    how = B.NormRotation.make(norm_dim=norm, q_weight=w[0] if norm else None, k_weight=w[1] if norm else None, weight_offset=offset,
                              rot_begin=rot_begin, rot_dim=rot_dim, interleaved=inter, rot_scale=scale,
                              inv_freq=None if f is None else torch.from_numpy(f).cuda())
    spec = B.Spec.make(1, hq, hkv, d, min(d, 512))
    q, k = x[:, :hq], x[:, hq:]
    qo, ko, q1, k1 = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hq, hkv))
    dev = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    B.q4kv_norm_rope(spec, how, 2, dev(5, 100), dev(0, 7000, n), n, q, k, qo, ko)
    for lo in range(0, n, 500):
        hi = min(lo + 500, n)
        B.q4kv_norm_rope(spec, how, 2, dev(5 + lo, 100 + max(lo - 7000, 0)), dev(0, min(max(7000 - lo, 0), hi - lo), hi - lo), hi - lo,
                         q[lo:hi], k[lo:hi], q1[lo:hi], k1[lo:hi])
    assert torch.equal(qo, q1) and torch.equal(ko, k1)
    q, k = q.contiguous(), k.contiguous()
    B.q4kv_norm_rope(spec, how, 2, dev(5, 100), dev(0, 7000, n), n, q, k, q, k)
    assert torch.equal(q, q1) and torch.equal(k, k1)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 900])
@pytest.mark.parametrize("d, begin, dim, inter", [(128, 32, 64, False), (128, 32, 64, True), (192, 128, 64, True), (256, 0, 256, False),
                                                  (512, 256, 64, False)])
def test_elements_that_are_not_finite_reach_their_pair_alone(d, begin, dim, inter, rows):
    f = torch.from_numpy(theta(dim)).cuda()
    how = B.NormRotation.make(rot_begin=begin, rot_dim=dim, interleaved=inter, inv_freq=f)
    spec = B.Spec.make(1, 2, 2, d, min(d, 256))
    x = torch.randn((rows, 2, d), device="cuda").to(torch.bfloat16)
    out, again = torch.empty_like(x), torch.empty_like(x)
    offs, pos = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([9], dtype=torch.int32, device="cuda")
    B.q4kv_norm_rope(spec, how, 1, pos, offs, rows, x, None, out, None)
    for at, value in ((begin + 3, float("inf")), (begin + dim - 1, float("nan")), (d - 1, float("inf")), (0, float("nan"))):
        y = x.clone()
        y[1, 1, at] = value
        B.q4kv_norm_rope(spec, how, 1, pos, offs, rows, y, None, again, None)
        j = at - begin
        mates = {at} if not 0 <= j < dim else {at, begin + (j ^ 1 if inter else (j + dim // 2) % dim)}
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[1, 1, list(mates)] = True
        assert not torch.isfinite(again[hit]).any() and torch.equal(again[~hit], out[~hit])


@pytest.mark.gpu
def test_a_weight_for_one_side_leaves_the_other_without_norm():
    hq, hkv, d = 3, 1, 64                                # a warp holds query and key heads
    x = torch.randn((4, hq + hkv, d), device="cuda").to(torch.bfloat16)
    w = torch.full((d,), 2.0, dtype=torch.bfloat16, device="cuda")
    spec, offs = B.Spec.make(1, hq, hkv, d, d), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out, k_out = torch.empty((4, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((4, hkv, d), dtype=torch.bfloat16, device="cuda")
    how = B.NormRotation.make(norm_dim=d, k_weight=w)
    B.q4kv_norm_rope(spec, how, 1, pos, offs, 4, x[:, :hq], x[:, hq:], q_out, k_out)
    assert torch.equal(q_out, x[:, :hq])
    want, size = reference(x[:, hq:].float().cpu().numpy().astype(np.float64), 2.0, d, 1e-6, 0.0, 0, 0, False, 1.0, None, None)
    check(k_out, want, size)


@pytest.mark.gpu
def test_bad_positions_and_rows_of_no_agent():
    spec, f = B.Spec.make(1, 2, 2, 64, 64), torch.from_numpy(theta(64)).cuda()
    how = B.NormRotation.make(rot_dim=64, inv_freq=f)
    x = torch.randn((8, 2, 64), device="cuda").to(torch.bfloat16)
    out, flags = torch.full_like(x, 5.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, -1, 0], dtype=torch.int32, device="cuda")
    offs = torch.tensor([1, 3, 5, 7], dtype=torch.int32, device="cuda")
    B.q4kv_norm_rope(spec, how, 3, pos, offs, 8, x, None, out, None, flags)
    assert flags.item() == B.FLAG_BAD_LENGTH
    assert torch.all(out[0] == 5.0) and torch.all(out[7] == 5.0) and torch.all(out[3:5] == 0.0)
    assert torch.equal(out[1], x[1]) and torch.equal(out[5], x[5])               # position 0
    assert not torch.equal(out[2], x[2])


def test_refusals():
    if torch.cuda.is_available():
        pytest.skip("placeholder pointers are only handed to the library on a host without a CUDA device")
    lib = B.lib()
    spec = B.Spec.make(1, 8, 2, 128, 128)

    def call(sp=spec, agents=1, pos=0x1000, offs=0x1000, total=4, q=0x100000, qs=1024, k=0x200000, ks=256, qo=0x300000, ko=0x400000,
             drop=(), **how):
        h = B.NormRotation(0, 0, 128, 0, 1e-6, 0.0, 1.0, 0, None, None, 0x1000)
        for name, value in how.items():
            setattr(h, name, value)
        return lib.q4kv_norm_rope(ctypes.byref(sp), ctypes.byref(h), agents, pos, offs, total, q, qs, k, ks, qo, ko, None, None)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(agents=-1), dict(total=-1), dict(norm_dim=-8), dict(norm_dim=136), dict(rot_dim=136), dict(rot_dim=-16),
                dict(rot_begin=8), dict(rot_begin=-8), dict(interleaved=2), dict(reserved=1), dict(inv_freq=None),
                dict(rot_scale=nan), dict(rot_scale=inf), dict(q_weight=0x1000), dict(norm_dim=128, eps=0.0),
                dict(norm_dim=128, eps=nan), dict(norm_dim=128, eps=inf), dict(norm_dim=128, weight_offset=nan),
                dict(norm_dim=128, q_weight=0x1008), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None),
                dict(offs=None), dict(q=0x100008), dict(ko=0x400004), dict(qs=1016), dict(qs=1028), dict(ks=248), dict(qs=2**62),
                dict(qo=0x100000, qs=1032), dict(qo=0x100010), dict(qo=0x200000), dict(ko=0x300000), dict(ko=0x101000),
                dict(ko=0x200000, ks=264)):
        assert call(**bad) == B.EINVAL, bad
    for bad in (dict(norm_dim=12), dict(rot_dim=24), dict(rot_begin=4, rot_dim=64), dict(rot_dim=12, interleaved=1),
                dict(sp=B.Spec.make(1, 8, 2, 96, 128)), dict(sp=B.Spec.make(1, 65535, 1, 128, 128))):
        assert call(**bad) == B.EUNSUPPORTED, bad
    assert call(total=0) == call(agents=0) == call(q=None, qo=None, k=None, ko=None) == B.OK


class _Fake:
    """Looks like a CUDA tensor on another device."""
    is_cuda, nbytes = True, 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000

    def get_device(self):
        return 1

    def stride(self):
        return (1024, 128, 1)

    def element_size(self):
        return 2

    def __len__(self):
        return 4


def test_tensors_of_another_device_are_refused():
    if torch.cuda.is_available():
        pytest.skip("placeholder pointers are only handed to the library on a host without a CUDA device")
    call, spec, how, t = B._native(), B.Spec.make(1, 8, 2, 128, 128), B.NormRotation(), _Fake()
    with pytest.raises(AssertionError, match="another device"):
        call.norm_rope(spec, how, 1, 0x1000, 0x1000, 0, t, None, 0x2000, None, None, None, 0)
    with pytest.raises(AssertionError, match="another device"):
        call.copy_blocks(spec, t, 4, t, 4, 0, 1, t, 0, None, None, 0)
    assert call.norm_rope(spec, how, 1, 0x1000, 0x1000, 0, t, None, 0x2000, None, None, None, 1) == B.OK
    with pytest.raises(AssertionError, match="rows are"):
        call.norm_rope(spec, how, 1, 0x1000, 0x1000, 5, t, None, 0x2000, None, None, None, 1)
    how.device = 1                                       # of its weights and frequencies
    with pytest.raises(AssertionError, match="another device"):
        _call_on(0, spec, how)


def _call_on(device, spec, how):
    keep, B._device = B._device, lambda: device
    try:
        B.q4kv_norm_rope(spec, how, 1, 0x1000, 0x1000, 0, None, None, None, None)
    finally:
        B._device = keep


class _Rows:
    """Looks like a CUDA tensor [tokens][heads][d] on device 0."""
    is_cuda = True

    def __init__(self, shape, dtype=torch.bfloat16, stride=None):
        self.shape, self.dtype, self._t = torch.Size(shape), dtype, torch.empty(shape, dtype=dtype, device="meta")
        self.nbytes, self._stride = self._t.nbytes, stride or self._t.stride()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return id(self) & ~0xFFFF

    def get_device(self):
        return 0

    def stride(self):
        return self._stride

    def element_size(self):
        return self._t.element_size()

    def __len__(self):
        return self.shape[0]


def test_tensors_of_other_sizes_and_types_are_refused():
    if torch.cuda.is_available():
        pytest.skip("placeholder pointers are only handed to the library on a host without a CUDA device")
    call, spec, how = B._native(), B.Spec.make(1, 8, 2, 128, 128), B.NormRotation()

    def norm_rope(q=None, k=None, q_out=None, k_out=None, total=4):
        q, k = q or _Rows((4, 8, 128)), k or _Rows((4, 2, 128))
        q_out, k_out = q_out or _Rows((4, 8, 128)), k_out or _Rows((4, 2, 128))
        return call.norm_rope(spec, how, 0, 0x1000, 0x1000, total, q, k, q_out, k_out, None, None, 0)     # no agents: nothing is launched

    assert norm_rope() == norm_rope(q=_Rows((4, 8, 128), stride=(1536, 128, 1))) == norm_rope(q_out=_Rows((4, 1024, 1))) == B.OK
    assert norm_rope(total=3) == norm_rope(q=_Rows((9, 8, 128)), k_out=_Rows((5, 2, 128))) == B.OK
    for bad in (dict(q=_Rows((4, 8, 128), torch.float16)), dict(q=_Rows((4, 8, 128), torch.float32)), dict(k=_Rows((4, 2, 128), torch.int16)),
                dict(q=_Rows((4, 2, 128))), dict(k=_Rows((4, 1, 128))), dict(q=_Rows((4, 9, 128))), dict(q=_Rows((4, 8, 64), stride=(1024, 128, 1))),
                dict(q=_Rows((3, 8, 128))), dict(k=_Rows((4, 2, 128), stride=(512, 256, 1)))):
        with pytest.raises(AssertionError, match="rows are"):
            norm_rope(**bad)
    for bad in (dict(q_out=_Rows((3, 8, 128))), dict(k_out=_Rows((4, 2, 64))), dict(q_out=_Rows((4, 2, 128))),
                dict(q_out=_Rows((4, 8, 128), torch.float16)), dict(k_out=_Rows((4, 2, 128), torch.float32))):
        with pytest.raises(AssertionError, match="an output is"):
            norm_rope(**bad)


@pytest.mark.gpu
def test_rows_of_other_heads_and_types_are_refused_on_the_device():
    f = torch.from_numpy(theta(128)).cuda()
    spec, how = B.Spec.make(1, 8, 2, 128, 128), B.NormRotation.make(rot_dim=128, inv_freq=f)
    x = torch.zeros((4, 12, 128), dtype=torch.bfloat16, device="cuda")
    pos, offs = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    out = torch.empty((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    B.q4kv_norm_rope(spec, how, 1, pos, offs, 4, x[:, :8], None, out, None)
    for q, o in ((x[:, 8:10], out), (x[:, :8].half(), out), (x[:, :8, :64], out), (x[:, :8], out[:3]), (x[:, :8], out.float())):
        with pytest.raises(AssertionError):
            B.q4kv_norm_rope(spec, how, 1, pos, offs, 4, q, None, o, None)
