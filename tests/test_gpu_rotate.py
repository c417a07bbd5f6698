"""Norms and rotation of queries and keys, alone and into the bf16 pages, against 64 bits."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2602_20732_amd as pk
from paper_2602_20732_amd import binding
import step_reference as ref

pytestmark = pytest.mark.gpu
SUMMARY_DTYPE_SWEEP = False
D = 128


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, seed, rows, Hq, H, turned=128, interleaved=False, axes=1, norms="all", eps=1e-6, scale=1.0, far=False):
        rng = np.random.default_rng(seed)
        self.wide = bf16(rng.normal(0, 1, (rows, Hq + 2 * H, D)) * rng.choice([0.1, 1, 30], (rows, Hq + 2 * H, 1)))
        self.q, self.k, self.v = self.wide[:, :Hq], self.wide[:, Hq:Hq + H], self.wide[:, Hq + H:]
        self.positions = rng.integers(0, 2 ** 31 if far else 200000, (axes, rows)).astype(np.int32)
        pairs = turned // 2
        self.inv_freq = (1e4 ** (-np.arange(pairs) / pairs)).astype(np.float32)
        self.axis = [(i * 7) % axes for i in range(pairs)]
        shape = {"all": lambda h: (D,), "head": lambda h: (h, D)}.get(norms)
        self.norm = [None if shape is None else rng.normal(1, 0.3, shape(h)).astype(np.float32) for h in (Hq, H)]
        self.interleaved, self.eps, self.scale = interleaved, eps, scale
        dev = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
        self.rotary = pk.Rotary(dev(self.inv_freq), self.axis, interleaved, dev(self.norm[0]), dev(self.norm[1]), eps, scale)

    def exact(self, which):
        x = (self.q, self.k)[which].double().numpy()
        y, x = ref.rotated(x, self.positions, self.inv_freq, self.axis, self.interleaved, self.norm[which], self.eps, self.scale)
        return y, ref.rotation_error(y, x, self.inv_freq, self.interleaved, self.scale)

    def cuda(self):
        wide = self.wide.cuda()
        Hq, H = self.q.shape[1], self.k.shape[1]
        return wide[:, :Hq], wide[:, Hq:Hq + H], wide[:, Hq + H:], torch.from_numpy(self.positions).cuda()


def near(got, exact):
    y, off = exact
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - y) <= off)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], y[bad][:5], off[bad][:5])


SHAPES = [dict(), dict(turned=64), dict(turned=96, axes=3), dict(turned=16, norms=None), dict(interleaved=True), dict(interleaved=True, turned=48, axes=4, norms="head"),
          dict(norms="head", axes=2), dict(norms=None, scale=1.25), dict(far=True), dict(far=True, interleaved=True, turned=112)]


@pytest.mark.parametrize("rows", [1, 17, 150])
@pytest.mark.parametrize("heads", [(8, 2), (7, 1), (37, 37)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(f"{k}{v}" for k, v in s.items()) or "plain")
def test_rotate(shape, heads, rows):
    c = Case(rows, rows, *heads, **shape)
    q, k, _, positions = c.cuda()
    lib = pk.Chess(pk.Config(*heads, 16, 1, 4, 4))
    q_out, k_out = torch.full((rows + 1, heads[0], D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows + 1, heads[1], D), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.rotate(c.rotary, q, k, positions, q_out[:rows], k_out[:rows])
    torch.cuda.synchronize()
    near(q_out[:rows], c.exact(0))
    near(k_out[:rows], c.exact(1))
    assert (q_out[rows:] == 7).all() and (k_out[rows:] == 7).all()


def test_one_of_the_two_and_rows_behind_the_last():
    c = Case(3, 40, 8, 2)
    q, k, _, positions = c.cuda()
    lib = pk.Chess(pk.Config(8, 2, 16, 1, 4, 4))
    q_out, k_out = (torch.full((40, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in (8, 2))
    lib.rotate(c.rotary, q, None, positions, q_out, None, counts=ints([21]))
    lib.rotate(c.rotary, None, k, positions, None, k_out, counts=ints([0]))
    torch.cuda.synchronize()
    y, off = c.exact(0)
    near(q_out[:21], (y[:21], off[:21]))
    assert (q_out[21:] == 7).all() and (k_out == 7).all()
    lib.rotate(c.rotary, None, k, positions, None, k_out, counts=ints([10 ** 9]))
    near(k_out, c.exact(1))


@pytest.mark.parametrize("rows", [5, 700])
def test_in_place(rows):
    c = Case(rows, rows, 9, 3, axes=2)
    q, k, _, positions = c.cuda()
    q, k = q.contiguous(), k.contiguous()
    lib = pk.Chess(pk.Config(9, 3, 16, 1, 4, 4))
    lib.rotate(c.rotary, q, k, positions, q, k)
    torch.cuda.synchronize()
    near(q, c.exact(0))
    near(k, c.exact(1))


def entries_of(rng, B, n_pages, spans):
    """Write list of (tokens held, tokens new) spans on pages of their own, shuffled."""
    free, out, row = list(rng.permutation(n_pages)), [], 0
    for held, new in spans:
        at = held
        while at < held + new:
            take = min(held + new, (at // B + 1) * B) - at
            out.append([int(free.pop()), row, at % B, take])
            at, row = at + take, row + take
    return out, row


SPANS = [[(0, 1)], [(15, 1), (16, 1), (31, 2), (4, 5)], [(0, 16), (0, 32), (3, 61), (40, 8)], [(0, 900), (17, 333), (0, 7)]]


@pytest.mark.parametrize("spans", SPANS, ids=len)
@pytest.mark.parametrize("heads", [(8, 2), (5, 5), (32, 8)])
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("shape", [dict(), dict(interleaved=True, turned=64, axes=3), dict(norms=None, turned=32)], ids=["plain", "axes", "unnormed"])
def test_store(shape, B, heads, spans):
    rng = np.random.default_rng(B + heads[0])
    n_pages, H = 130, heads[1]
    writes, n = entries_of(rng, B, n_pages, spans)
    c = Case(n, n, *heads, **shape)
    q, k, v, positions = c.cuda()
    lib = pk.Chess(pk.Config(*heads, B, 8, 64, 64))
    before = bf16(rng.normal(0, 1, (2, n_pages, H, B, D)))
    k_pool, v_pool = before[0].cuda(), before[1].transpose(2, 3).contiguous().cuda()
    q_out = torch.zeros((n, heads[0], D), dtype=torch.bfloat16, device="cuda")
    room = torch.full((len(writes) + 3, 4), 2 ** 30, dtype=torch.int32, device="cuda")
    room[: len(writes)] = ints(writes)
    lib.rotate_store(c.rotary, q, k, v, positions, room, ints([n, len(writes), 0, 0]), q_out, k_pool, v_pool)
    torch.cuda.synchronize()
    near(q_out, c.exact(0))
    y, off = c.exact(1)
    k_want, k_off, v_want = before[0].double().numpy(), np.zeros((n_pages, H, B, D)), before[1].clone()
    for page, row, first, count in writes:
        k_want[page][:, first:first + count] = y[row:row + count].transpose(1, 0, 2)
        k_off[page][:, first:first + count] = off[row:row + count].transpose(1, 0, 2)
        v_want[page][:, first:first + count] = c.v[row:row + count].transpose(0, 1)
    near(k_pool, (k_want, k_off))
    assert torch.equal(v_pool.cpu().view(torch.int16), v_want.transpose(2, 3).contiguous().view(torch.int16))


@pytest.mark.parametrize("B", [16, 32])
def test_entries_that_name_what_is_not_there(B):
    """They do nothing; a larger allocation lies on both sides of the tensors."""
    rng = np.random.default_rng(B)
    n, n_pages, m, top = 40, 9, 2, 2 ** 31 - 1
    c = Case(B, n + 2 * B, 4, 2)
    wide = c.wide.cuda()
    inside = [[0, 0, 0, B], [1, n - 1, 3, 1], [n_pages - 1, n - B, 0, B]]
    outside = [[3, n, 0, 1], [4, n - 1, 2, 2], [5, n - B + 1, 0, B], [6, -1, 0, 4], [7, -top - 1, 0, 4], [2, top, 0, 4], [2, top - 3, 0, B], [n_pages, 0, 0, 4],
               [-1, 0, 0, 4], [top, 0, 0, 4], [-top - 1, 0, 0, 4], [2, 0, 0, 0], [2, 0, 0, -5]]
    writes = [e for pair in zip(outside, inside + [[2, 1, 0, 0]] * 10) for e in pair]
    pools = torch.full((2, n_pages + 2 * m, 2, B, D), 3.0, dtype=torch.bfloat16, device="cuda")
    mid = slice(m, m + n_pages)
    q_out = torch.full((n + 2 * B, 4, D), 3.0, dtype=torch.bfloat16, device="cuda")
    positions = torch.from_numpy(c.positions[:, B:B + n].copy()).cuda()
    lib = pk.Chess(pk.Config(4, 2, B, 1, 4, 4))
    lib.rotate_store(c.rotary, wide[B:B + n, :4], wide[B:B + n, 4:6], wide[B:B + n, 6:], positions, ints(writes), ints([0, len(writes), 0, 0]), q_out[B:B + n],
                     pools[0][mid], pools[1][mid].view(n_pages, 2, D, B))
    torch.cuda.synchronize()
    named = sorted({r for _, r0, _, k in inside for r in range(r0, r0 + k)})
    y, off = c.exact(0)
    want, allowed = np.full(q_out.shape, 3.0), np.zeros(q_out.shape)
    for r in named:
        want[B + r], allowed[B + r] = y[B + r], off[B + r]
    near(q_out, (want, allowed))
    stored = (pools[0] != 3).any(-1).any(1)
    expect = torch.zeros_like(stored)
    for page, _, first, count in inside:
        expect[m + page, first:first + count] = True
    assert torch.equal(stored, expect)
    v = pools[1].view(-1, 2, D, B)
    assert torch.equal((v != 3).any(2).any(1), expect)


def test_values_that_are_not_finite():
    """A pair with an infinity or NaN is what the formula says; other pairs of an unnormed head, and values, keep theirs."""
    c = Case(1, 4, 4, 1, turned=64, norms=None)
    c.wide[0, 0, 5], c.wide[1, 0, 40], c.wide[2, 0, 100], c.wide[3, 5, 9] = float("inf"), float("nan"), float("nan"), float("-inf")
    q, k, v, positions = c.cuda()
    lib = pk.Chess(pk.Config(4, 1, 16, 1, 4, 4))
    q_out, pools = torch.zeros((4, 4, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 2, 1, 16, D), dtype=torch.bfloat16, device="cuda")
    lib.rotate_store(c.rotary, q, k, v, positions, ints([[1, 0, 2, 4]]), ints([4, 1, 0, 0]), q_out, pools[0], pools[1].view(2, 1, D, 16))
    torch.cuda.synchronize()
    y, off = c.exact(0)
    got, odd = q_out.double().cpu().numpy(), np.zeros(y.shape, bool)
    odd[0, 0, [5, 37]] = odd[1, 0, [8, 40]] = odd[2, 0, 100] = True
    assert (~np.isfinite(got) == odd).all() and (np.isinf(got) == np.isinf(y)).all()
    assert (np.abs(got - y) <= off)[~odd].all()
    assert pools[1].view(2, 1, D, 16)[1, 0, 9, 5] == float("-inf")


def test_refusals():
    c = Case(1, 6, 4, 2)
    q, k, v, positions = c.cuda()
    lib = pk.Chess(pk.Config(4, 2, 16, 1, 4, 4))
    out = [torch.zeros((6, h, D), dtype=torch.bfloat16, device="cuda") for h in (4, 2)]
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def call(rot=None, q_stride=8 * D, n=6, q_ptr=q.data_ptr(), q_out=out[0].data_ptr(), **change):
        r = binding._CRotary.from_buffer_copy(c.rotary._c)
        for name, value in change.items():
            if name == "axis":
                r.axis[0] = value
            else:
                setattr(r, name, value)
        return lib.lib.chess_rotate(lib._h, ctypes.byref(r), q_ptr, q_stride, k.data_ptr(), 8 * D, positions.data_ptr(), n, None, q_out, out[1].data_ptr(), stream)

    assert call() == 0
    for bad in (dict(rotary_dim=8), dict(rotary_dim=24), dict(rotary_dim=144), dict(n_axes=0), dict(n_axes=5), dict(axis=1), dict(eps=-1.0), dict(eps=float("nan")),
                dict(scale=float("inf")), dict(inv_freq=None), dict(q_stride=4 * D - 8), dict(q_stride=8 * D + 4), dict(n=0), dict(q_ptr=q.data_ptr() + 2),
                dict(q_out=None), dict(q_ptr=None)):
        assert call(**bad) == -1, bad
    with pytest.raises(pk.ChessError):
        lib.rotate(c.rotary, q.float(), k, positions, *out)
    with pytest.raises(pk.ChessError):
        lib.rotate(c.rotary, q, k, positions[:, :5].contiguous(), *out)
    with pytest.raises(pk.ChessError):
        lib.rotate(c.rotary, q, k, positions, out[0][:5], out[1])
    with pytest.raises(pk.ChessError):
        lib.rotate(c.rotary, None, None, positions)
    torch.cuda.synchronize()


def test_on_a_stream_of_its_own_and_replayed():
    c = Case(2, 33, 8, 2)
    q, k, v, positions = c.cuda()
    lib = pk.Chess(pk.Config(8, 2, 16, 2, 8, 8))
    writes, _ = entries_of(np.random.default_rng(0), 16, 8, [(3, 20), (0, 13)])
    writes, counts = ints(writes), ints([33, len(writes), 0, 0])
    q_out, kp, vp = torch.zeros((33, 8, D), dtype=torch.bfloat16, device="cuda"), *torch.zeros((2, 8, 2, 16, D), dtype=torch.bfloat16, device="cuda")
    want = [torch.zeros_like(x) for x in (q_out, kp, vp)]
    lib.rotate_store(c.rotary, q, k, v, positions, writes, counts, want[0], want[1], want[2].view(8, 2, D, 16))
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        lib.rotate_store(c.rotary, q, k, v, positions, writes, counts, q_out, kp, vp.view(8, 2, D, 16))
    for _ in range(3):
        for x in (q_out, kp, vp):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (q_out, kp, vp)))


shape_name = lambda s: "-".join(f"{k}{v}" for k, v in s.items()) or "plain"  # noqa: E731
MANY = [dict(), dict(interleaved=True, turned=48, axes=4, norms="head"), dict(norms="head", axes=2), dict(norms=None, scale=1.25, turned=96), dict(interleaved=True, turned=64)]


def many_rows():
    """Enough for the kernel of prompts, which turns all heads of a token in one workgroup (16 rows are one, 2 a compute unit are many); the last has 9."""
    return 32 * torch.cuda.get_device_properties(0).multi_processor_count + 9


@pytest.mark.parametrize("heads", [(20, 5), (7, 1), (16, 16)], ids=str)
@pytest.mark.parametrize("shape", MANY, ids=shape_name)
def test_rotate_many_rows(shape, heads):
    n = many_rows()
    c = Case(n, n, *heads, **shape)
    q, k, _, positions = c.cuda()
    lib = pk.Chess(pk.Config(*heads, 16, 1, 4, 4))
    q_out, k_out = (torch.full((n + 1, h, D), 7.0, dtype=torch.bfloat16, device="cuda") for h in heads)
    lib.rotate(c.rotary, q, k, positions, q_out[:n], k_out[:n])
    torch.cuda.synchronize()
    q_exact, k_exact = c.exact(0), c.exact(1)
    near(q_out[:n], q_exact)
    near(k_out[:n], k_exact)
    assert (q_out[n:] == 7).all() and (k_out[n:] == 7).all()
    # one of the two, fewer rows than there is room for, and in place
    some, alone = n - 20, torch.full((n, heads[0], D), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.rotate(c.rotary, q, None, positions, alone, None, counts=ints([some]))
    assert torch.equal(alone[:some], q_out[:some]) and (alone[some:] == 7).all()
    own = k.contiguous()
    lib.rotate(c.rotary, None, own, positions, None, own)
    assert torch.equal(own, k_out[:n])
    both = [q.contiguous(), k.contiguous()]
    lib.rotate(c.rotary, *both, positions, *both)
    assert torch.equal(both[0], q_out[:n]) and torch.equal(both[1], k_out[:n])


@pytest.mark.parametrize("queries", [True, False], ids=["both", "keys"])
@pytest.mark.parametrize("heads", [(20, 5), (8, 2)], ids=str)
@pytest.mark.parametrize("B", [16, 32])
@pytest.mark.parametrize("shape", MANY, ids=shape_name)
def test_store_with_room_for_many_entries(shape, B, heads, queries):
    """The room of the write list chooses the kernel; entries behind counts[1] are anything."""
    rng = np.random.default_rng(B + heads[0])
    n_pages, H = 130, heads[1]
    writes, n = entries_of(rng, B, n_pages, SPANS[3])
    c = Case(n, n, *heads, **shape)
    q, k, v, positions = c.cuda()
    lib = pk.Chess(pk.Config(*heads, B, 8, 64, 64))
    before = bf16(rng.normal(0, 1, (2, n_pages, H, B, D)))
    k_pool, v_pool = before[0].cuda(), before[1].transpose(2, 3).contiguous().cuda()
    q_out = torch.zeros((n, heads[0], D), dtype=torch.bfloat16, device="cuda")
    room = torch.zeros((many_rows() // 16 + 3, 4), dtype=torch.int32, device="cuda")
    room[:, 1] = n - 1
    room[:, 3] = 1
    room[: len(writes)] = ints(writes)
    lib.rotate_store(c.rotary, q if queries else None, k, v, positions, room, ints([n, len(writes), 0, 0]), q_out if queries else None, k_pool, v_pool)
    torch.cuda.synchronize()
    if queries:
        near(q_out, c.exact(0))
    y, off = c.exact(1)
    k_want, k_off, v_want = before[0].double().numpy(), np.zeros((n_pages, H, B, D)), before[1].clone()
    for page, row, first, count in writes:
        k_want[page][:, first:first + count] = y[row:row + count].transpose(1, 0, 2)
        k_off[page][:, first:first + count] = off[row:row + count].transpose(1, 0, 2)
        v_want[page][:, first:first + count] = c.v[row:row + count].transpose(0, 1)
    near(k_pool, (k_want, k_off))
    assert torch.equal(v_pool.cpu().view(torch.int16), v_want.transpose(2, 3).contiguous().view(torch.int16))
