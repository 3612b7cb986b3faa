"""GPU parity of the rotary positions, the 8-bit KV cache and attention over it against the CPU oracle in 64 bits.

Tolerances count roundings.  eps/2 of a type is its half step relative to the value: fp32 2^-24, bf16 2^-8 at most, e4m3 2^-4 (and
2^-10 of the scale below the normal values)."""
import math

import numpy as np
import pytest
import torch

from oracle import forward as ofwd, kv8, rotary
import paper_2510_26527_amd as psd
from paper_2510_26527_amd import runtime, synth

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SCALED = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=2.0),
          "parts": dict(factor=8.0, low=1.0, high=4.0, original_len=8192)}


def _randn(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float32) * std


def _rope(d, rot, layout, scaling, theta=5e5, magnitude=1.0):
    """The handle, and the oracle's turn(x, positions)."""
    r = runtime.Rope(d, rot_dim=rot, layout=layout, theta=theta, scaling=scaling, magnitude=magnitude, **SCALED[scaling])
    f = rotary.frequencies(rot, theta, scaling, **SCALED[scaling])
    return r, lambda x, pos: rotary.turn(x, pos, f, layout == "interleaved", magnitude)


def _turn_error(x, pos, rot, layout, magnitude=1.0):
    """What fp32 may be off by in a rotated entry: (|x1| + |x2|) times six half steps (cos and sin two and a half, products, their
    sum, the magnitude) and the rounding of position * frequency in fp64 on both sides, 2^-51 of the position in radians at most."""
    a = np.abs(x)
    other = a.copy()
    if layout == "interleaved":
        other[..., 0:rot:2], other[..., 1:rot:2] = a[..., 1:rot:2], a[..., 0:rot:2]
    else:
        other[..., :rot // 2], other[..., rot // 2:rot] = a[..., rot // 2:rot], a[..., :rot // 2]
    tol = (a + other) * magnitude * (6 * 2.0 ** -24 + np.abs(np.asarray(pos, np.float64))[:, None, None] * 2.0 ** -51)
    tol[..., rot:] = 0
    return tol


# ---------------------------------------------------------------------------------------------------- rotary positions
ROPE_CASES = [  # rows, heads, d, rot, layout, scaling, type, elements between rows beyond the heads, offset into the buffer
    (1, 1, 2, 2, "half", "none", F32, 0, 0), (1, 1, 128, 128, "half", "none", BF16, 0, 0), (9, 40, 128, 128, "half", "parts", BF16, 0, 0),
    (9, 40, 128, 128, "interleaved", "parts", BF16, 128, 0), (257, 3, 64, 32, "half", "linear", F32, 0, 0),
    (1023, 5, 64, 16, "interleaved", "base", BF16, 64, 0), (33, 7, 80, 80, "half", "none", BF16, 0, 0), (33, 7, 80, 20, "half", "base", F32, 0, 0),
    (65, 2, 256, 256, "half", "parts", F32, 0, 0), (300, 17, 256, 64, "interleaved", "none", BF16, 8, 8), (64, 9, 96, 24, "half", "none", BF16, 3, 1),
    (50, 3, 6, 4, "interleaved", "linear", BF16, 0, 1), (50, 3, 10, 6, "half", "none", F32, 1, 3), (2100, 64, 128, 96, "half", "parts", BF16, 0, 0),
    (3, 300, 256, 256, "interleaved", "none", F32, 0, 0),
    # more than two million items: two a thread
    (8200, 33, 128, 128, "half", "parts", BF16, 0, 0), (5000, 4, 256, 222, "interleaved", "none", F32, 2, 1), (9001, 31, 64, 32, "half", "base", F32, 0, 0)]


@pytest.mark.parametrize("case", ROPE_CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}-{c[3]}-{c[4]}-{c[5]}" for c in ROPE_CASES])
@pytest.mark.parametrize("in_place", [False, True])
def test_rotation(case, in_place):
    rows, heads, d, rot, layout, scaling, dtype, gap, offset = case
    r, turn = _rope(d, rot, layout, scaling, magnitude=1.25)
    stride = heads * d + gap
    buf = torch.full((offset + rows * stride + 5,), 7.5, dtype=dtype, device="cuda")
    x = buf[offset:offset + rows * stride].as_strided((rows, heads, d), (stride, d, 1), offset)
    data = _randn(rows + d, rows, heads, d).to(dtype)
    x.copy_(data)
    before = buf.clone()
    pos = torch.randint(0, 200000, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    pos[0] = 0
    y = r.rotate(x, pos.cuda(), out=x if in_place else None)
    ref, tol = turn(data.double().numpy(), pos.numpy()), _turn_error(data.double().numpy(), pos.numpy(), rot, layout, 1.25)
    if dtype == BF16:
        tol = tol + np.abs(ref) * 2.0 ** -8
    got = y.double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) / np.maximum(tol, 1e-30))
    if in_place:                                             # nothing between or behind the rows
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[offset:offset + rows * stride].as_strided((rows, heads, d), (stride, d, 1), offset).fill_(False)
        assert torch.equal(buf[keep], before[keep])
    else:
        assert torch.equal(buf, before)
    r.close()


def test_rotation_at_far_and_negative_positions():
    r, turn = _rope(128, 128, "half", "none")
    pos = torch.tensor([0, 1, 65535, 1 << 20, (1 << 30) + 7, (1 << 31) - 1, -1, -(1 << 20)], dtype=torch.int32)
    x = _randn(5, 8, 3, 128)
    got = r.rotate(x.cuda(), pos.cuda()).double().cpu().numpy()
    ref, tol = turn(x.double().numpy(), pos.numpy()), _turn_error(x.double().numpy(), pos.numpy(), 128, "half")
    assert np.all(np.abs(got - ref) <= tol), np.max(np.abs(got - ref) / tol)
    # rows of a batch, and none at all
    again = r.rotate(x.cuda().view(2, 4, 3, 128), pos.cuda().view(2, 4))
    assert np.array_equal(again.view(8, 3, 128).double().cpu().numpy(), got)
    assert r.rotate(x.cuda()[:0], pos.cuda()[:0]).shape == (0, 3, 128)


# ---------------------------------------------------------------------------------------------------- the cache
class Cache:
    """One layer on the GPU and plane by plane in the oracle, filled alike up to `lens` and with garbage behind."""

    def __init__(self, B, h, d, max_len, lens, seed=0, spread=1.0):
        self.B, self.h, self.d, self.max_len, self.start = B, h, d, max_len, list(lens)
        rng = np.random.default_rng(seed)
        self.k = [[kv8.Plane(max_len, d) for _ in range(h)] for _ in range(B)]
        self.v = [[kv8.Plane(max_len, d) for _ in range(h)] for _ in range(B)]
        for planes in (self.k, self.v):
            for b in range(B):
                for p in planes[b]:
                    if lens[b]:
                        size = 2.0 ** rng.uniform(-spread, spread, (lens[b] + 63) // 64)
                        p.append(0, rng.normal(size=(lens[b], d)) * np.repeat(size, 64)[:lens[b], None])
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.layer = runtime.KV8Layer(*self.tensors(), self.lens)

    def tensors(self):
        k = np.stack([[p.codes for p in row] for row in self.k])
        v = np.stack([[p.codes.reshape(-1, 64, self.d).transpose(0, 2, 1) for p in row] for row in self.v])
        ks, vs = (np.stack([[p.scale for p in row] for row in planes]).astype(np.float32) for planes in (self.k, self.v))
        return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (k, v, ks, vs)]

    def state(self):
        return [self.layer.k, self.layer.v, self.layer.k_scale, self.layer.v_scale]

    def append_oracle(self, k, v):
        """k, v [B, R, h, d] as the oracle has them."""
        for b in range(self.B):
            for h in range(self.h):
                self.k[b][h].append(self.start[b], k[b, :, h])
                self.v[b][h].append(self.start[b], v[b, :, h])


def _same_bits(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def _same_number(a, b):
    return np.array_equal(kv8.decode(a), kv8.decode(b), equal_nan=True)


APPEND_CASES = [  # B, R, h_q, h_kv, d, max_len, lens, rot, layout, scaling, type
    (1, 1, 4, 2, 64, 64, [0], 64, "half", "none", F32), (1, 1, 8, 2, 128, 128, [63], 128, "half", "parts", BF16),
    (1, 1, 8, 2, 128, 128, [64], 128, "interleaved", "none", BF16), (3, 9, 6, 3, 128, 192, [0, 60, 119], 128, "half", "none", F32),
    (2, 64, 4, 4, 128, 256, [0, 64], 64, "half", "linear", BF16), (2, 65, 2, 1, 64, 256, [63, 1], 32, "interleaved", "base", BF16),
    (1, 200, 7, 1, 128, 256, [37], 128, "half", "none", F32), (1, 333, 4, 2, 64, 448, [100], 64, "interleaved", "parts", BF16),
    (2, 5, 4, 2, 128, 128, [50, 62], 20, "half", "none", F32), (2, 70, 4, 2, 64, 192, [50, 62], 6, "interleaved", "base", BF16),
    (5, 1, 28, 4, 128, 128, [0, 15, 16, 17, 127], 128, "half", "none", BF16)]


@pytest.mark.parametrize("case", APPEND_CASES, ids=[f"{c[0]}x{c[1]}-{c[2]}/{c[3]}x{c[4]}-rot{c[7]}" for c in APPEND_CASES])
def test_append(case):
    B, R, h_q, h_kv, d, max_len, lens, rot, layout, scaling, dtype = case
    c = Cache(B, h_kv, d, max_len, lens, seed=R)
    r, turn = _rope(d, rot, layout, scaling)
    # one buffer of projections; the new rows outgrow some of the older blocks
    qkv = (_randn(R + d, B, R, h_q + 2 * h_kv, d) * 2.0 ** _randn(1, B, R, 1, 1, std=2.0)).to(dtype)
    q, k, v = qkv.cuda().split((h_q, h_kv, h_kv), dim=2)
    before = [t.clone() for t in c.state()]
    q_out = c.layer.append(q, k, v, r, len_upper_bound=max(lens) + R)
    pos = np.concatenate([np.arange(n, n + R) for n in lens])
    flat = qkv.double().numpy().reshape(B * R, -1, d)
    turned, off = turn(flat[:, :h_q + h_kv], pos), _turn_error(flat[:, :h_q + h_kv], pos, rot, layout)
    tol = off[:, :h_q] + (np.abs(turned[:, :h_q]) * 2.0 ** -8 if dtype == BF16 else 0)
    assert np.all(np.abs(q_out.double().cpu().numpy().reshape(B * R, h_q, d) - turned[:, :h_q]) <= tol)

    ok = turned[:, h_q:].reshape(B, R, h_kv, d)
    c.append_oracle(ok, flat[:, h_q + h_kv:].reshape(B, R, h_kv, d))
    gk, gv, gks, gvs = (t.cpu().numpy() for t in c.state())
    for b in range(B):
        n, end = lens[b], lens[b] + R
        blocks = slice(n // 64, (end - 1) // 64 + 1)
        for h in range(h_kv):
            # values are quantised as they come: the same codes and scales, older tokens' included
            pv, pk = c.v[b][h], c.k[b][h]
            assert np.array_equal(gvs[b, h, blocks], pv.scale[blocks]) and np.array_equal(gks[b, h, blocks], pk.scale[blocks])
            assert _same_number(gv[b, h].transpose(0, 2, 1).reshape(max_len, d)[:end], pv.codes[:end])
            assert _same_number(gk[b, h, :n], pk.codes[:n])
            # keys within half a step of what fp32 makes of them
            scale = np.repeat(pk.scale, 64)[n:end, None]
            err = np.abs(kv8.decode(gk[b, h, n:end]) * scale - ok[b, :, h])
            room = np.maximum(np.abs(ok[b, :, h]) * 2.0 ** -4, scale * 2.0 ** -10) + 2 * off[b * R:(b + 1) * R, h_q + h]
            assert np.all(err <= room)
            # and nothing else: tokens behind the new ones, blocks before and behind
            assert np.array_equal(gk[b, h, end:], before[0][b, h, end:].cpu().numpy())
            assert np.array_equal(gv[b, h].transpose(0, 2, 1).reshape(max_len, d)[end:],
                                  before[1][b, h].cpu().numpy().transpose(0, 2, 1).reshape(max_len, d)[end:])
            rest = np.ones(max_len // 64, bool)
            rest[blocks] = False
            for g, was in ((gks, before[2]), (gvs, before[3])):
                assert np.array_equal(g[b, h, rest], was[b, h].cpu().numpy()[rest], equal_nan=True)
    assert c.lens.tolist() == list(lens)
    # the same rows again: the same cache
    state = [t.clone() for t in c.state()]
    c.layer.append(q, k, v, r, len_upper_bound=max(lens) + R, q_out=torch.empty_like(q_out))
    assert _same_bits(state, c.state())
    # in place, in the buffer of projections
    again = c.layer.append(q, k, v, r, len_upper_bound=max(lens) + R, q_out=q)
    assert again.data_ptr() == q.data_ptr() and torch.equal(q, q_out) and _same_bits(state, c.state())
    r.close()


def test_append_of_what_is_no_number_and_of_the_largest_and_smallest():
    c = Cache(1, 1, 64, 64, [0])
    x = _randn(2, 1, 8, 1, 64)
    x[0, 0, 0, :3] = torch.tensor([math.inf, -math.inf, math.nan])
    x[0, 1] = 0
    x[0, 2, 0, 0] = 1e-30
    c.layer.append(None, x.cuda(), (x * 1e20).cuda(), None, len_upper_bound=8)
    c.append_oracle(x.double().numpy(), (x * 1e20).double().numpy())
    gk, gv, gks, gvs = (t.cpu().numpy() for t in c.state())
    assert gks[0, 0, 0] == c.k[0][0].scale[0] and gvs[0, 0, 0] == 2.0 ** 40
    assert _same_number(gk[0, 0, :8], c.k[0][0].codes[:8])
    assert _same_number(gv[0, 0, 0].T[:8], c.v[0][0].codes[:8])
    assert np.nanmax(np.abs(kv8.decode(gv[0, 0, 0].T[:8]))) == 448
    zero = Cache(1, 1, 64, 64, [0])
    zero.layer.append(None, torch.zeros(1, 3, 1, 64, device="cuda"), torch.zeros(1, 3, 1, 64, device="cuda"), None, len_upper_bound=3)
    assert zero.layer.k_scale[0, 0, 0].item() == 2.0 ** -40 and not zero.layer.k[0, 0, :3].any()


def test_append_never_writes_behind_the_cache():
    """Lengths beyond what the bound says (a caller's mistake): rows past max_len are dropped, guards on both sides stay."""
    B, h, d, n = 2, 2, 64, 128
    guard = 4096
    size, blocks = B * h * n * d, B * h * n // 64
    codes = torch.full((2, guard + size + guard), 171, dtype=torch.uint8, device="cuda")
    scales = torch.full((2, guard + blocks + guard), 3.0, device="cuda")
    k, v = (codes[i, guard:guard + size] for i in range(2))
    ks, vs = (scales[i, guard:guard + blocks].view(B, h, n // 64) for i in range(2))
    layer = runtime.KV8Layer(k.view(B, h, n, d), v.view(B, h, n // 64, d, 64), ks, vs, torch.tensor([120, 1000], dtype=torch.int32, device="cuda"))
    x = _randn(3, B, 20, h, d).cuda()
    layer.append(None, x, x, None, len_upper_bound=n)
    for t in (codes, scales):
        assert torch.all(t[:, :guard] == t[0, 0]) and torch.all(t[:, -guard:] == t[0, 0])
    assert torch.all(k.view(B, h, n, d)[0, :, :120] == 171)
    assert torch.all(k.view(B, h, n, d)[1] == 171) and torch.all(ks[1] == 3.0)


# ---------------------------------------------------------------------------------------------------- attention
def _attention_oracle(c, q, lens, R, scale):
    """q [B, R, h_q, d] fp64 -> the result and the weighted sum of |v|, in it 2^-18 of the plain sum (see _room)."""
    B, _, h_q, d = q.shape
    out, room = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        end = lens[b] + R
        for h in range(h_q):
            k, v = c.k[b][h // (h_q // c.h)].numbers(end), c.v[b][h // (h_q // c.h)].numbers(end)
            for r in range(R):
                n = lens[b] + r + 1
                s = k[:n] @ q[b, r, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[b, r, h], room[b, r, h] = w @ v[:n], w @ np.abs(v[:n]) + 2.0 ** -18 * np.abs(v[:n]).sum(0)
    return out, room


def _room(ref, weighted):
    """bf16's half step of the result; each weight rounded to fp16, 2^-11 of it; and for scores, references and sums in fp32 a quarter of
    that again.  A weight below fp16's normal range is off by half of its smallest step, 2^-25, instead: weights are held times 2^7 against a
    reference whose own weight is one of them, and times V's scale over the outputs' unit, 2^-3 at least, so that is 2^-25 / 2^7 * 2^3 = 2^-29
    of |v| for a sum of weights of at least one, wherever the heavy keys' entries are zero: 2^-11 times the 2^-18 that `weighted` holds."""
    return np.abs(ref) * 2.0 ** -8 + weighted * (2.0 ** -11 + 2.0 ** -13)


ATTN_CASES = [  # B, R, h_q, h_kv, d, lens (before the rows)
    (1, 1, 1, 1, 64, [0]), (1, 1, 8, 2, 128, [0]), (2, 1, 8, 2, 128, [63, 64]), (1, 9, 4, 4, 128, [1024]), (3, 5, 8, 2, 64, [0, 1, 700]),
    (2, 16, 7, 1, 128, [130, 5]), (1, 33, 4, 1, 128, [95]), (1, 200, 2, 2, 64, [0]), (1, 130, 4, 2, 128, [61]), (4, 3, 28, 4, 128, [0, 63, 65, 3000]),
    (1, 1, 32, 8, 128, [5000]), (2, 70, 14, 2, 128, [0, 260]), (1, 1, 4, 1, 64, [9000]),
    # many rows or many keys for them: blocks of 128 rows without and with splits of the keys, of 64 rows likewise
    (3, 250, 12, 6, 64, [0, 100, 37]), (2, 170, 32, 16, 128, [70, 3]), (1, 100, 16, 4, 128, [4000]), (9, 12, 32, 8, 128, [2000 - 61 * i for i in range(9)]),
    (17, 20, 16, 16, 128, [3 * i for i in range(17)]), (6, 40, 32, 32, 64, [1200, 0, 64, 63, 1199, 500]), (1, 300, 3, 1, 128, [0]), (1, 2, 16, 1, 64, [129]), (9, 17, 2, 1, 64, [7 * i for i in range(9)]),
    (1, 100, 32, 8, 128, [4000]), (9, 12, 32, 8, 128, [4000 - 61 * i for i in range(9)]), (1, 11, 16, 4, 128, [8100]), (1, 1, 8, 2, 128, [17000]),
    (5, 5, 16, 8, 64, [0, 900, 777, 1000, 63]), (3, 130, 64, 64, 64, [0, 73, 5]), (5, 70, 64, 64, 128, [90, 0, 1, 63, 64])]


@pytest.mark.parametrize("case", ATTN_CASES, ids=[f"{c[0]}x{c[1]}-{c[2]}/{c[3]}x{c[4]}-{max(c[5])}" for c in ATTN_CASES])
def test_attention(case):
    B, R, h_q, h_kv, d, lens = case
    max_len = (max(lens) + R + 63) // 64 * 64 + 64
    c = Cache(B, h_kv, d, max_len, [n + R for n in lens], seed=B * R, spread=3.0)
    c.lens.copy_(torch.tensor(lens))
    q = _randn(7, B, R, h_q, d, std=2.0).to(BF16)
    wide = torch.full((B, R, h_q * d + 24), 5.0, dtype=BF16, device="cuda")       # rows of a wider buffer
    out = wide[..., 8:8 + h_q * d].unflatten(-1, (h_q, d))
    got = runtime.KV8Attention()(c.layer, q.cuda(), len_upper_bound=max(lens) + R, out=out)
    ref, weighted = _attention_oracle(c, q.double().numpy(), lens, R, 1 / math.sqrt(d))
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= _room(ref, weighted)), np.nanmax(err / _room(ref, weighted))
    assert torch.all(wide[..., :8] == 5) and torch.all(wide[..., 8 + h_q * d:] == 5)
    # without a bound of its own: more splits of the keys, some of them empty
    free = runtime.KV8Attention()(c.layer, q.cuda())
    assert np.all(np.abs(free.double().cpu().numpy() - ref) <= _room(ref, weighted))
    assert torch.equal(free, runtime.KV8Attention()(c.layer, q.cuda()))


@pytest.mark.parametrize("R,h_kv,group,d", [(1, 1, 4, 128), (5, 1, 4, 128), (40, 1, 4, 128), (150, 1, 4, 64),
                                            (150, 8, 4, 128), (20, 130, 1, 64), (20, 130, 1, 128), (150, 90, 1, 64), (150, 90, 1, 128)])        # the last five: blocks of 64 and of 128 rows
def test_what_a_row_does_not_see_has_no_part_in_it(R, h_kv, group, d):
    """Later rows of the step, and everything behind it, may hold NaN; a row that sees one gets NaN in V's entries, or all over for K."""
    lens, B = [70, 200], 2
    c = Cache(B, h_kv, d, 448, [n + R for n in lens], seed=R)
    c.lens.copy_(torch.tensor(lens))
    q = _randn(9, B, R, group * h_kv, d).to(BF16).cuda()
    attend = runtime.KV8Attention()
    clean = attend(c.layer, q, len_upper_bound=448)
    first = R // 2                                           # sequence 0: row `first` on sees a NaN value in entry 3
    c.layer.v[0, 0, (70 + first) // 64, 3, (70 + first) % 64] = 127
    got = attend(c.layer, q, len_upper_bound=448)
    assert torch.equal(got[1], clean[1]) and torch.equal(got[0, :first], clean[0, :first])
    assert torch.isnan(got[0, first:, :group, 3]).all() and torch.isnan(got).sum().item() == (R - first) * group
    rest = [e for e in range(d) if e != 3]
    assert torch.equal(got[0][:, :, rest], clean[0][:, :, rest]) and torch.equal(got[0][:, group:], clean[0][:, group:])
    c.layer.k[1, 0, 200 + R - 1, 5] = 255                    # sequence 1: the last row sees a NaN key
    got = attend(c.layer, q, len_upper_bound=448)
    assert torch.equal(got[1, :R - 1], clean[1, :R - 1]) and torch.isnan(got[1, R - 1, :group]).all()
    assert torch.equal(got[1, :, group:], clean[1, :, group:])


def test_attention_scores_far_apart_and_scales_far_apart():
    """One key takes all weight from 2^20 others or shares it with them; blocks whose scales lie 2^60 apart."""
    d, n = 64, 4096
    c = Cache(1, 1, d, n, [0])
    for b in range(n // 64):
        c.k[0][0].append(64 * b, np.ones((64, d)) * (1.0 if b else -1.0))
        c.v[0][0].append(64 * b, np.ones((64, d)) * 2.0 ** (-30 if b % 2 else 30))
    c.layer = runtime.KV8Layer(*c.tensors(), c.lens)
    c.lens.fill_(n - 1)
    for size in (0.0, 0.01, 1.0, 30.0, -30.0, 1e30):
        q = torch.full((1, 1, 1, d), size).to(BF16)
        got = runtime.KV8Attention()(c.layer, q.cuda(), len_upper_bound=n)
        ref, weighted = _attention_oracle(c, q.double().numpy(), [n - 1], 1, 1 / 8)
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= _room(ref, weighted)), size
    # a softmax scale of the caller's, a negative one too
    q = _randn(4, 1, 1, 1, d).to(BF16)
    for scale in (0.5, -0.25):
        got = runtime.KV8Attention()(c.layer, q.cuda(), scale=scale, len_upper_bound=n)
        ref, weighted = _attention_oracle(c, q.double().numpy(), [n - 1], 1, scale)
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= _room(ref, weighted))


@pytest.mark.parametrize("heads,R", [(1, 3), (2, 40), (5, 60), (64, 140), (256, 140)])            # the last two: blocks of 64 and of 128 rows
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_large_scores(heads, R, d):
    """Scores of 2^20 and 2^100, all equal or far apart: weights of 1 and 0."""
    n = 64 * 5
    c = Cache(1, 1, d, n, [0])
    c.k[0][0].append(0, np.ones((n, d)))
    c.v[0][0].append(0, np.random.default_rng(R).normal(size=(n, d)))
    c.k[0][0].append(70, np.full((1, d), 2.0))
    c.layer = runtime.KV8Layer(*c.tensors(), c.lens)
    c.lens.fill_(n - R)
    for size in (2.0 ** 18, 2.0 ** 100, -(2.0 ** 100)):
        q = (torch.ones(1, R, heads, d) * size * (1 + torch.arange(R).view(1, R, 1, 1) / 128)).to(BF16)
        got = runtime.KV8Attention()(c.layer, q.cuda(), len_upper_bound=n)
        ref, weighted = _attention_oracle(c, q.double().numpy(), [n - R], R, 1 / math.sqrt(d))
        assert np.all(np.abs(got.double().cpu().numpy() - ref) <= _room(ref, weighted)), size


def test_attention_over_more_than_four_gigabytes_of_codes():
    """Zero codes but for two far tokens of the last head: byte offsets beyond 2^32."""
    h, d, n = 9, 128, 1 << 22
    k = torch.zeros((1, h, n, d), dtype=torch.uint8, device="cuda")
    v = torch.zeros((1, h, n // 64, d, 64), dtype=torch.uint8, device="cuda")
    one = torch.ones((1, h, n // 64), device="cuda")
    layer = runtime.KV8Layer(k, v, one, one, torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
    k[0, h - 1, n - 1, :] = 0x40                             # 2.0
    v[0, h - 1, n // 64 - 1, :, 63] = 0x48                   # 4.0
    k[0, h - 1, n - 100, :] = 0x40
    v[0, h - 1, (n - 100) // 64, :, (n - 100) % 64] = 0x38   # 1.0
    q = torch.ones((1, 1, h, d), dtype=BF16, device="cuda")
    got = runtime.KV8Attention()(layer, q).float().cpu()
    w = math.exp(2 * d / math.sqrt(d))                       # against n - 2 others of weight 1
    assert torch.equal(got[0, 0, :h - 1], torch.zeros(h - 1, d))
    assert torch.allclose(got[0, 0, h - 1], torch.full((d,), 5 * w / (2 * w + n - 2)), rtol=2.0 ** -8 + 2.0 ** -10)
    # appending there
    x = torch.full((1, 1, h, d), 448.0, device="cuda")
    layer.append(None, x, x, None)
    assert torch.all(k[0, :, n - 1] == 0x7e) and torch.all(v[0, :, -1, :, 63] == 0x7e) and int(k[0, h - 1, n - 2].max()) == 0


# ---------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("stream", [False, True])
def test_append_and_attention_captured_and_replayed(stream):
    """One graph of rotation, append and attention on a decoding loop's buffers, replayed between eager work, against eager calls."""
    B, R, h_q, h_kv, d, max_len = 2, 3, 8, 2, 128, 1088
    rope, _ = _rope(d, d, "half", "parts")
    side = torch.cuda.Stream() if stream else torch.cuda.current_stream()
    lens = [60, 900]
    a, b = Cache(B, h_kv, d, max_len, lens, seed=1), Cache(B, h_kv, d, max_len, lens, seed=1)
    qkv = torch.zeros((B, R, h_q + 2 * h_kv, d), dtype=BF16, device="cuda")
    out = torch.zeros((B, R, h_q, d), dtype=BF16, device="cuda")
    attend, eager = runtime.KV8Attention(), runtime.KV8Attention()
    turned = torch.empty((B, R, h_q, d), dtype=BF16, device="cuda")
    pos = torch.zeros((B, R), dtype=torch.int32, device="cuda")
    probe = torch.zeros((B, R, h_q, d), dtype=BF16, device="cuda")

    def step(layer, attend, qkv, out):
        q, k, v = qkv.split((h_q, h_kv, h_kv), dim=2)
        rope.rotate(q, pos, out=probe)
        layer.append(q, k, v, rope, q_out=turned)
        attend(layer, turned, out=out)

    attend(a.layer, turned, out=out)                         # sizes the workspace before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side if stream else None):
        step(a.layer, attend, qkv, out)
    for turn in range(4):
        new = _randn(20 + turn, B, R, h_q + 2 * h_kv, d, std=1.0 + turn).to(BF16).cuda()
        qkv.copy_(new)
        pos.copy_(a.lens[:, None] + torch.arange(R, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(probe, turned)
        want = torch.empty_like(out)
        step(b.layer, eager, new, want)
        assert torch.equal(out, want)
        assert _same_bits(a.state(), b.state())
        a.lens += R - turn % 2                               # a rejected row now and then
        b.lens += R - turn % 2
        torch.cuda.synchronize()
        if turn == 1:                                        # the workspace is outgrown: the graph's stays its own
            wide = Cache(2, 8, d, 1984, [1900, 1900], seed=3)
            attend(wide.layer, torch.zeros((2, 4, 32, d), dtype=BF16, device="cuda"))
            assert attend._outgrown
            torch.full((1 << 24,), float("nan"), device="cuda")


SMALL = synth.Shape(2, 256, 4, 2, 64, 512, 1024, 1.0e4)
GROUPED = synth.Shape(2, 512, 8, 2, 128, 768, 640, 5.0e5)


def _logits_close(gpu, ref, what=""):
    rel = np.abs(gpu.double().cpu().numpy() - ref).max(-1) / np.abs(ref).max(-1)
    assert rel.max() <= 2e-2, f"{what}: {rel.max():.3e}"


class Following(kv8.KVCache8):
    """The oracle's cache for a forward that has run on the GPU: each appended entry has to be a right rounding of the oracle's, and what
    the GPU made of it is what the oracle then reads.  Without that the two would attend to different caches: the forward's keys
    are off by up to its own error, 2e-2 of the largest, and where that straddles the middle of two codes they take different ones,
    2^-3 of the entry apart, which later rows see in full; nothing bounds such a logit by 2e-2."""

    def __init__(self, cfg, batch, max_len, kv):
        ofwd.KVCache.__init__(self, cfg, batch, max_len)     # (the codes are the GPU's)
        self.kv = kv

    def append(self, l, b, s0, k, v):
        end, first = s0 + k.shape[0], s0 // 64 * 64
        if not k.shape[0]:
            return
        for x, codes, scales, mine in ((k, self.kv.k[l, b], self.kv.k_scale[l, b], self.k[l][b]),
                                       (v, self.kv.v[l, b].transpose(-1, -2).flatten(1, 2), self.kv.v_scale[l, b], self.v[l][b])):
            scale = scales.double().cpu().numpy().repeat(64, axis=1)[:, first:end, None]
            mine[:, first:end] = kv8.decode(codes[:, first:end].cpu().numpy()) * scale
            x = np.asarray(x).transpose(1, 0, 2)
            err, scale = np.abs(mine[:, s0:end] - x), scale[:, s0 - first:]
            assert np.all(err <= np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -10) + 2e-2 * np.abs(x).max(-1, keepdims=True))


@pytest.mark.parametrize("shape,pack,w4", [(SMALL, False, False), (SMALL, True, False), (GROUPED, True, False), (GROUPED, True, True)],
                         ids=["rows", "packed", "grouped", "w4"])
def test_forwards_on_an_8_bit_cache(shape, pack, w4):
    """Prompt, verify-shaped steps, single tokens and rollbacks of a ragged batch, in lockstep with the oracle's 8-bit cache."""
    B, max_len = 2, 320
    w = synth.make_weights(shape, 4, BF16, std=0.05)
    if w4:
        from oracle import quant as oquant
        codes, quant = synth.quantize_w4(w)
        model = runtime.Model(shape, codes, quant=quant)
        w = {k: (torch.from_numpy(oquant.dequantize(codes[k].numpy(), quant[k][0].float().numpy(), quant[k][1].numpy())) if k in quant else v)
             for k, v in w.items()}
    else:
        model = runtime.Model(shape, w)
    if pack:
        model.pack()
    kv = runtime.KVCache8(model, B, max_len, fill_garbage=True)
    cfg = ofwd.ModelConfig(**shape.asdict())
    okv = Following(cfg, B, max_len, kv)
    ks, vs = synth.make_kv_fill(shape, B, 100, 6, BF16)
    kv.load(ks, vs, [100, 37])
    for l in range(shape.n_layers):
        for b in range(B):
            okv.append(l, b, 0, ofwd.widen(ks[l][b]).transpose(1, 0, 2), ofwd.widen(vs[l][b]).transpose(1, 0, 2))
    okv.lens[:] = [100, 37]
    toks = synth.make_tokens(shape.vocab, (B, 160), 9)
    at = 0
    for n in (40, 1, 8, 5, 1, 17, 1, 33):
        t = toks[:, at:at + n]
        at += n
        got = runtime.forward(model, kv, torch.from_numpy(t).cuda())
        ref = ofwd.forward(cfg, w, t, okv)
        _logits_close(got, ref, f"{n} rows")
        if n > 4:                                            # some rows are rejected, sequence by sequence
            base = torch.tensor(okv.lens - n, dtype=torch.int32, device="cuda")
            keep = torch.tensor([n - 1, n // 2], dtype=torch.int32, device="cuda")
            psd.psd_kv_truncate(kv.handle, base, keep, 0)
            okv.truncate(okv.lens - n + np.array([n - 1, n // 2]))
            assert kv.lens.tolist() == okv.lens.tolist()
    kv.close()
    model.close()


@pytest.mark.parametrize("h_q,h_kv,R", [(8, 4, 620), (32, 32, 560)])
def test_a_long_prompt_on_an_8_bit_cache(h_q, h_kv, R):
    """More rows than the direct kernel takes: the wide kernel's fp16 output, for the tiled projections, from blocks of 64 and of 128 rows."""
    shape, B = synth.Shape(1, 256, h_q, h_kv, 64, 256, 128, 1.0e4), 2
    model = runtime.Model(shape, synth.make_weights(shape, 2, BF16, std=0.05)).pack()
    w, cfg = {k: v.cpu() for k, v in model.weights.items()}, ofwd.ModelConfig(**shape.asdict())
    kv = runtime.KVCache8(model, B, 704, fill_garbage=True)
    okv = Following(cfg, B, 704, kv)
    toks = synth.make_tokens(shape.vocab, (B, 660), 4)
    for n in (R, 40):
        t = toks[:, int(okv.lens[0]):int(okv.lens[0]) + n]
        got = runtime.forward(model, kv, torch.from_numpy(t).cuda())
        _logits_close(got, ofwd.forward(cfg, w, t, okv), f"{n} rows")
    kv.close()
    model.close()


@pytest.mark.parametrize("ctx", [17000, 25000])
@pytest.mark.parametrize("pack", [False, True])
def test_a_verify_step_on_a_long_8_bit_cache(pack, ctx):
    """36 query rows a KV head: the direct kernel's and, on 25 000 keys, the wide kernel's splits and outputs for steps of up to 16 rows."""
    shape = synth.Shape(1, 512, 32, 8, 128, 256, 320, 5.0e5)
    model = runtime.Model(shape, synth.make_weights(shape, 2, BF16, std=0.05))
    if pack:
        model.pack()
    w, cfg = {k: v.cpu() for k, v in model.weights.items()}, ofwd.ModelConfig(**shape.asdict())
    kv = runtime.KVCache8(model, 1, ctx // 64 * 64 + 128)
    okv = Following(cfg, 1, ctx // 64 * 64 + 128, kv)
    ks, vs = synth.make_kv_fill(shape, 1, ctx, 6, BF16)
    kv.load(ks, vs, ctx)
    okv.append(0, 0, 0, ofwd.widen(ks[0][0]).transpose(1, 0, 2), ofwd.widen(vs[0][0]).transpose(1, 0, 2))
    okv.lens[:] = ctx
    toks = synth.make_tokens(shape.vocab, (1, 10), 9)
    for n in (9, 1):
        got = runtime.forward(model, kv, torch.from_numpy(toks[:, :n]).cuda())
        _logits_close(got, ofwd.forward(cfg, w, toks[:, :n], okv), f"{n} rows")
    kv.close()
    model.close()


@pytest.mark.parametrize("pack", [False, True])
def test_a_small_step_of_many_heads_on_an_8_bit_cache(pack):
    """52 KV heads of eight query heads, five sequences of three rows: the wide kernel without splits in a step of up to 16 rows."""
    shape = synth.Shape(1, 256, 416, 52, 64, 256, 320, 1.0e4)
    model = runtime.Model(shape, synth.make_weights(shape, 2, BF16, std=0.05))
    if pack:
        model.pack()
    w, cfg = {k: v.cpu() for k, v in model.weights.items()}, ofwd.ModelConfig(**shape.asdict())
    kv = runtime.KVCache8(model, 5, 128, fill_garbage=True)
    okv = Following(cfg, 5, 128, kv)
    toks = synth.make_tokens(shape.vocab, (5, 68), 9)
    for at, n in ((0, 62), (62, 3), (65, 3)):
        got = runtime.forward(model, kv, torch.from_numpy(toks[:, at:at + n]).cuda())
        _logits_close(got, ofwd.forward(cfg, w, toks[:, at:at + n], okv), f"{n} rows")
    kv.close()
    model.close()


@pytest.mark.parametrize("layout,rot,scaling", [("half", 64, "parts"), ("interleaved", 64, "none"), ("half", 32, "linear"), ("interleaved", 20, "base")])
@pytest.mark.parametrize("cache", ["f32", "bf16", "bf16 packed", "e4m3", "e4m3 packed"])
def test_forwards_with_rotary_positions_of_the_models_own(layout, rot, scaling, cache):
    dtype = F32 if cache == "f32" else BF16
    w = synth.make_weights(SMALL, 8, dtype, std=0.05)
    model = runtime.Model(SMALL, w)
    rope, turn = _rope(64, rot, layout, scaling, theta=1e4, magnitude=1.1)
    model.set_rope(rope)
    if "packed" in cache:
        model.pack()
    cfg = ofwd.ModelConfig(**SMALL.asdict())
    kv = (runtime.KVCache8 if "e4m3" in cache else runtime.KVCache)(model, 2, 256)
    okv = Following(cfg, 2, 256, kv) if "e4m3" in cache else ofwd.KVCache(cfg, 2, 256)
    toks = synth.make_tokens(SMALL.vocab, (2, 90), 2)
    at = 0
    for n in (50, 3, 9, 1, 20):
        got = runtime.forward(model, kv, torch.from_numpy(toks[:, at:at + n]).cuda())
        ref = ofwd.forward(cfg, w, toks[:, at:at + n], okv, turn)
        at += n
        if cache == "f32":
            assert np.abs(got.double().cpu().numpy() - ref).max() <= 1e-4
        else:
            _logits_close(got, ref, f"{n} rows")
    # trees: the half pairing of the whole head at other frequencies works, other pairings are refused
    if cache == "bf16":
        args = (model, kv, torch.from_numpy(toks[:, at:at + 3]).cuda(), [-1, 0, 0])
        if rot == 64 and layout == "half":
            got = runtime.forward_tree(*args)
            want = [ofwd.forward(cfg, w, toks[:, [at, at + c]], okv, turn)[:, -1:] for c in (1,)]
            _logits_close(got[:, 1:2], want[0])
        else:
            with pytest.raises(psd.PsdError) as e:
                runtime.forward_tree(*args)
            assert e.value.status == psd.PSD_ERR_UNIMPLEMENTED
    model.set_rope(None)                                     # back to the descriptor's
    fresh, ofresh = runtime.KVCache(model, 2, 256), ofwd.KVCache(cfg, 2, 256)
    got = runtime.forward(model, fresh, torch.from_numpy(toks[:, :9]).cuda())
    ref = ofwd.forward(cfg, w, toks[:, :9], ofresh)
    if cache == "f32":
        assert np.abs(got.double().cpu().numpy() - ref).max() <= 1e-4
    else:
        _logits_close(got, ref)
    model.close()
    rope.close()


def test_a_chain_whose_target_keeps_its_cache_in_8_bits():
    """Algorithm 1 with a target on an 8-bit cache and a bf16 draft: every forward of the target, rollbacks and all, against the oracle
    on the same cache."""
    from paper_2510_26527_amd import chain
    target = runtime.Model(SMALL, synth.make_weights(SMALL, 4, BF16, std=0.05)).pack()
    draft_shape = synth.Shape(1, 128, 2, 2, 64, 256, 1024, 1.0e4)
    draft = runtime.Model(draft_shape, synth.make_weights(draft_shape, 5, BF16, std=0.05)).pack()
    levels = [chain.Level(target, 256, 16, kv_bits=8), chain.Level(draft, 256, 16)]
    assert isinstance(levels[0].kv, runtime.KVCache8) and isinstance(levels[1].kv, runtime.KVCache)
    rng = np.random.default_rng(3)
    cfg = ofwd.ModelConfig(**SMALL.asdict())
    okv = Following(cfg, 1, 256, levels[0].kv)
    w = {k: v.cpu() for k, v in target.weights.items()}
    prompt = synth.make_tokens(1024, (30,), 1)
    seen = 0

    def follow(e):                                           # called at once, while the cache is as the forward left it
        nonlocal seen
        if e[0] != "forward" or e[1] != 0:
            return
        _, _, start, toks, rows = e
        if not seen:
            ofwd.forward(cfg, w, prompt[None, :-1], okv)
        okv.truncate([min(start, int(okv.lens[0]))])
        assert int(okv.lens[0]) == start
        ref = ofwd.forward(cfg, w, np.array([toks]), okv)[0]
        if rows is not None:
            _logits_close(rows, ref[-rows.shape[0]:], f"{len(toks)} rows at {start}")
        seen += 1

    c = chain.Chain(levels, [0, 5], [rng.random((60, 6), np.float32), rng.random(400, np.float32)], max_len=256, trace=True, sink=follow)
    assert len(c.generate(prompt, 40)) == 40
    assert seen >= 5
    for lvl in levels:
        lvl.close()


def test_tensors_that_do_not_fit_are_refused_before_a_launch():
    c = Cache(2, 2, 64, 128, [5, 9])
    x = torch.zeros((2, 3, 2, 64), dtype=BF16, device="cuda")
    for q, k, v in ((None, x[:1], x[:1]), (None, x, x.float()), (x.float(), x, x), (None, x.transpose(1, 2), x), (x[:, :2], x, x)):
        with pytest.raises(ValueError):
            c.layer.append(q, k, v)
    for q in (x.float(), x[:1], x.transpose(2, 3)):
        with pytest.raises(ValueError):
            runtime.KV8Attention()(c.layer, q)
    with pytest.raises(ValueError):
        runtime.KV8Attention()(c.layer, x.cpu())
    with pytest.raises(psd.PsdError):
        runtime.KV8Attention()(c.layer, x[:, :, :1])         # fewer query heads than KV heads
    r = runtime.Rope(64)
    for args in ((x, torch.zeros(2, 2, dtype=torch.int32, device="cuda")), (x, torch.zeros(2, 3, device="cuda")), (x[..., :32], torch.zeros(2, 3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            r.rotate(*args)
    with pytest.raises(ValueError):
        runtime.KV8Layer(c.layer.k, c.layer.v.float(), c.layer.k_scale, c.layer.v_scale, c.lens)
    for dtype in (torch.float16, torch.float64):
        with pytest.raises(ValueError):
            r.rotate(x.to(dtype), torch.zeros(2, 3, dtype=torch.int32, device="cuda"))
        with pytest.raises(ValueError):
            c.layer.append(None, x.to(dtype), x.to(dtype))


@pytest.mark.parametrize("as_number", [False, True])
def test_results_made_for_another_stream_take_no_memory_that_this_one_still_reads(as_number):
    """Memory given back while the current stream has work on it pending is free for that stream alone."""
    side = torch.cuda.Stream()
    stream = side.cuda_stream if as_number else side
    B, R, h_q, h_kv, d = 1, 64, 32, 8, 128
    c = Cache(B, h_kv, d, 2048, [1900], seed=2)
    rope, _ = _rope(d, d, "half", "none")
    q, k, v = (_randn(3 + i, B, R, h, d).to(BF16).cuda() for i, h in enumerate((h_q, h_kv, h_kv)))
    pos = torch.arange(R, dtype=torch.int32, device="cuda")[None]
    attend = runtime.KV8Attention()
    torch.cuda.synchronize()
    for make in (lambda: rope.rotate(q, pos, stream=stream), lambda: c.layer.append(q, k, v, rope, stream=stream),
                 lambda: attend(c.layer, q, stream=stream)):
        held = torch.full_like(q, 3.0)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        copy = held.clone()                                  # waits behind the sleep
        del held
        got = make()
        torch.cuda.synchronize()
        assert bool((copy == 3.0).all())
        assert not bool((got == 3.0).all())


def test_a_forward_on_an_8_bit_cache_captured_and_replayed():
    """One graph of a step, replayed as the cache grows to twice the length it was planned for, against eager steps on a twin."""
    model = runtime.Model(GROUPED, synth.make_weights(GROUPED, 6, BF16, std=0.05)).pack()
    a, b = (runtime.KVCache8(model, 2, 512) for _ in range(2))
    prompt = torch.from_numpy(synth.make_tokens(GROUPED.vocab, (2, 70), 1)).cuda()
    logits = torch.zeros((2, 9, GROUPED.vocab), dtype=F32, device="cuda")
    toks = torch.zeros((2, 9), dtype=torch.int32, device="cuda")
    model.workspace_upto(2, 70, 512)
    for kv in (a, b):
        runtime.forward(model, kv, prompt, 0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        runtime.forward(model, a, toks, logits_out=logits)
    for turn in range(8):
        toks.copy_(torch.from_numpy(synth.make_tokens(GROUPED.vocab, (2, 9), 30 + turn)))
        graph.replay()
        torch.cuda.synchronize()
        want = runtime.forward(model, b, toks)
        assert torch.equal(a.lens, b.lens) and torch.equal(logits, want)
        torch.cuda.synchronize()
    model.close()
