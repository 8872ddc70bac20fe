"""GPU parity of the head operators (alora_heads.h) and of what moves the cache (alora_cache.h) against oracle/heads.py in 64 bits.

Tolerances are per element, from the roundings made: half a step of the stored type relative to the value, and fp32 steps
(u = 2^-24) relative to the size of what was added up (the oracle's second result).  Forward: a mean square of up to 256 terms is 16 additions in
a lane and 6 across lanes, halved by the root, with the root, three products and the turn 20 u at most: 32.  Backward: r^3 carries
three times the root's 16 u, the mean of u x another 25: 96.  The weights' sums: the additions of a lane, of the workgroup and
of the workgroups' parts, with the terms' own error: 256 at these sizes."""
import numpy as np
import pytest
import torch

from oracle import heads as oh
from paper_2512_17910_amd import binding as ab
from gpu_util import raw_bits, to_f64
from test_operators_abi import LAYOUTS, UNITS, heads_of_a_layout

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def values(rng, shape, dt, std=1.0, mean=0.0):
    return dev((rng.standard_normal(shape) * std + mean).astype(np.float32)).to(dt)


def close(got, want, size, dt, k, what):
    got = got if isinstance(got, np.ndarray) else to_f64(got)
    d = k * U32 * size
    over = np.abs(got - want) - (HALF[dt] * (np.abs(want) + d) + d)
    assert np.all(over <= 0), (what, float(over.max()), np.unravel_index(int(np.argmax(over)), over.shape))


def rope_of(rng, n, rot):
    if not rot:
        return None
    a = rng.uniform(-4, 4, (n, rot // 2))
    return dev(np.cos(a).astype(np.float32)), dev(np.sin(a).astype(np.float32))


def angles(rope, pos):
    return (None, None) if rope is None else tuple(to_f64(x)[np.clip(pos, 0, x.shape[0] - 1)] for x in rope)


class Heads:
    """A call's tensors: views of a fused buffer (k, v given) or keys that lie in the cache; strides beyond the rows where pad is given."""

    def __init__(self, dtype, T, hq, hkv, d, rot, il=False, norm=True, cache=False, pad=0, seed=0, eps=1e-5):
        rng = self.rng = np.random.default_rng(seed)
        dt = self.dt = DT[dtype]
        self.T, self.hq, self.hkv, self.d, self.il, self.eps = T, hq, hkv, d, il, eps
        self.rope = rope_of(rng, 50, rot)
        self.pos = rng.integers(0, 50, T).astype(np.int32)
        self.n_slots = 16 * (T // 8 + 2)
        self.slot = rng.permutation(self.n_slots)[:T].astype(np.int64)
        self.slot[rng.random(T) < 0.1] = -1
        y = values(rng, (T, (hq + 2 * hkv) * d + pad), dt)
        self.q, self.k, self.v = y[:, : hq * d], y[:, hq * d: (hq + hkv) * d], y[:, (hq + hkv) * d: (hq + 2 * hkv) * d]
        self.wq, self.wk = (values(rng, (d,), dt, 0.3, 1.0) for _ in range(2)) if norm else (None, None)
        self.kc, self.vc = (values(rng, (self.n_slots, hkv * d + pad), dt)[:, : hkv * d] for _ in range(2))
        if cache:
            self.k = self.v = None
            self.q_out = self.q = values(rng, (T, hq * d), dt)
        else:
            self.q_out = torch.full((T, hq * d), float("nan"), dtype=dt, device="cuda")
        self.dims = ab.make_heads_dims(self.q, self.q_out, self.k, self.kc, hq, hkv, d, rope=self.rope, interleaved=il, norm=norm, eps=eps,
                                       v=self.v, v_out=None if self.v is None else self.vc)
        assert ab.alora_qk_norm_rope_validate(dev(self.pos), dev(self.slot), self.dims) == ab.ALORA_OK
        f = lambda t, w: to_f64(t).reshape(T, -1, d)
        w = lambda t: None if t is None else to_f64(t)
        c, s = angles(self.rope, self.pos)
        self.want_q = [x.reshape(T, -1) for x in oh.heads(f(self.q, 0), w(self.wq), eps, c, s, il)]
        kept = np.flatnonzero(self.slot >= 0)
        k_in = to_f64(self.kc)[self.slot[kept]] if cache else to_f64(self.k)[kept]
        cs = (None, None) if c is None else (c[kept], s[kept])
        self.want_k = [x.reshape(len(kept), hkv * d) for x in oh.heads(k_in.reshape(len(kept), hkv, d), w(self.wk), eps, *cs, il)]
        self.kept, self.k0, self.v0 = kept, raw_bits(self.kc).copy(), raw_bits(self.vc).copy()

    def run(self, stream=None):
        ab.alora_qk_norm_rope(self.q, self.q_out, self.k, self.kc, self.v, None if self.v is None else self.vc, self.wq, self.wk, self.rope,
                              dev(self.pos), dev(self.slot), self.dims, stream=stream)
        torch.cuda.synchronize()

    def check(self):
        close(self.q_out, *self.want_q, self.dt, 32, "q")
        wr = self.slot[self.kept]
        close(to_f64(self.kc)[wr], *self.want_k, self.dt, 32, "k")
        other = np.setdiff1d(np.arange(self.n_slots), wr)
        assert np.array_equal(raw_bits(self.kc)[other], self.k0[other]), "a slot that no row names changed"
        v = raw_bits(self.vc)
        if self.v is None:
            assert np.array_equal(v, self.v0)
        else:
            assert np.array_equal(v[wr], raw_bits(self.v)[self.kept]) and np.array_equal(v[other], self.v0[other])


# every chunk width and lane count: (d, rot) with halves at multiples of 8, 4 and 2 elements; part of a head, none of it
SHAPES = [(128, 128), (128, 64), (128, 0), (64, 64), (64, 8), (32, 32), (32, 8), (80, 80), (80, 20), (80, 40), (96, 24), (96, 96), (112, 28), (112, 56),
          (192, 48), (192, 96), (256, 256), (256, 28), (256, 4), (8, 8), (8, 4), (16, 12)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("il", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("d,rot", SHAPES)
def test_heads(dtype, il, d, rot):
    for T, hq, hkv, norm, cache, pad in ((5, 4, 2, True, False, 8), (3, 7, 1, True, True, 0), (2, 3, 3, False, False, 0), (1, 16, 2, False, True, 16)):
        print(f"[case] {dtype} d={d} rot={rot} il={il} T={T} {hq}/{hkv} norm={norm} cache={cache} pad={pad}", flush=True)
        h = Heads(dtype, T, hq, hkv, d, rot, il, norm, cache, pad, seed=d + rot + T)
        h.run()
        h.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,hq,hkv,d,rot,cache", [(1, 32, 8, 128, 128, True), (300, 28, 4, 112, 28, True), (1100, 64, 8, 128, 64, False), (2049, 5, 5, 64, 64, False),
                                                  (700, 40, 40, 256, 28, False), (9001, 1, 1, 32, 32, True), (16, 71, 1, 64, 32, False),
                                                  (3001, 4, 1, 64, 64, False), (777, 4, 2, 80, 20, False), (300, 3, 1, 80, 20, True),
                                                  (111, 2, 2, 112, 28, True)])
def test_heads_of_larger_calls(dtype, T, hq, hkv, d, rot, cache):
    """Calls whose wavefronts take several units of heads, shapes of one K/V head, more units than wavefronts."""
    for il in (False, True):
        print(f"[case] {dtype} T={T} {hq}/{hkv} d={d} rot={rot} cache={cache} il={il}", flush=True)
        h = Heads(dtype, T, hq, hkv, d, rot, il, cache=cache, seed=T)
        h.run()
        h.check()


@pytest.mark.parametrize("il", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("dtype,d,rot", [("f32", 4, 4), ("f32", 12, 4), ("f32", 20, 20), ("f32", 36, 12), ("f32", 252, 248), ("f32", 252, 200), ("bf16", 24, 24),
                                         ("bf16", 40, 36), ("bf16", 248, 124), ("bf16", 248, 244)])
def test_heads_of_odd_sizes(dtype, d, rot, il):
    for T, hq, hkv, norm, cache, inplace in ((6, 3, 2, True, False, False), (5, 9, 1, True, True, True), (40, 1, 1, False, False, True), (7, 2, 2, True, True, False)):
        print(f"[case] {dtype} d={d} rot={rot} il={il} T={T} {hq}/{hkv} norm={norm} cache={cache}", flush=True)
        h = Heads(dtype, T, hq, hkv, d, rot, il, norm, cache, seed=d + T)
        h.run()
        h.check()
        b = Back(dtype, T, hq, hkv, d, rot, il, norm, seed=d + T, inplace=inplace)
        b.call()
        b.check()


def test_values_stored_beside_keys_that_lie_in_the_cache():
    h = Heads("bf16", 20, 8, 2, 64, 64, cache=True, seed=4)
    v = values(h.rng, (20, 128), h.dt)
    h.v = v
    h.dims = ab.make_heads_dims(h.q, h.q_out, None, h.kc, 8, 2, 64, rope=h.rope, eps=h.eps, v=v, v_out=h.vc)
    h.run()
    h.check()


def test_rows_that_are_left_alone_and_positions_outside():
    h = Heads("bf16", 12, 4, 2, 64, 64, seed=3)
    h.pos[:] = [-1, 50, 1 << 30, -(1 << 31), 0, 49, 7, 8, 9, 10, 11, 12]
    h.slot[:] = [h.n_slots, -2, -(1 << 62), 1 << 62, 5, 6, 7, -1, 9, 10, 11, 12]
    q, k, v = to_f64(h.q), to_f64(h.k), raw_bits(h.v)
    assert ab.alora_qk_norm_rope_validate(dev(h.pos), dev(h.slot), h.dims) == ab.ALORA_EDATA
    h.run()
    c, s = angles(h.rope, h.pos)
    close(h.q_out, *[x.reshape(12, -1) for x in oh.heads(q.reshape(12, 4, 64), to_f64(h.wq), h.eps, c, s, False)], h.dt, 32, "q")
    kept = np.array([4, 5, 6, 8, 9, 10, 11])
    close(to_f64(h.kc)[h.slot[kept]], *[x.reshape(7, -1) for x in oh.heads(k[kept].reshape(7, 2, 64), to_f64(h.wk), h.eps, c[kept], s[kept], False)],
          h.dt, 32, "k")
    other = np.setdiff1d(np.arange(h.n_slots), h.slot[kept])
    assert np.array_equal(raw_bits(h.kc)[other], h.k0[other]) and np.array_equal(raw_bits(h.vc)[h.slot[kept]], v[kept])


def test_infinities_and_nan_stay_in_their_heads():
    """A head of a NaN is NaN, its neighbours are not; without norm an infinity stays in its pair, also beside features that are not turned."""
    for dtype, d, rot, il in (("bf16", 128, 64, False), ("bf16", 64, 24, True), ("f32", 80, 20, True), ("f32", 32, 32, False)):
        h = Heads(dtype, 3, 6, 2, d, rot, il, norm=True, seed=9)
        h.q[1, 2 * d + 1] = float("nan")
        h.run()
        got = to_f64(h.q_out).reshape(3, 6, d)
        assert np.isnan(got[1, 2]).all()
        got[1, 2] = 0
        assert np.isfinite(got).all()
        h = Heads(dtype, 2, 6, 2, d, rot, il, norm=False, seed=10)
        h.q[0, 3 * d + d - 1] = float("inf")
        h.run()
        bad = np.argwhere(~np.isfinite(to_f64(h.q_out).reshape(2, 6, d)))
        assert len(bad) and (bad[:, :2] == [0, 3]).all() and len(bad) <= 2 and bad[-1, 2] == d - 1, bad
    h = Heads("f32", 2, 2, 2, 32, 32, norm=True, seed=11, eps=0.0)     # a head of zeros: zeros over sqrt(eps)
    h = Heads("f32", 2, 2, 2, 32, 32, norm=True, seed=11, eps=1e-6)
    h.q[0, :32] = 0
    h.run()
    assert (to_f64(h.q_out)[0, :32] == 0).all() and np.isfinite(to_f64(h.q_out)).all()


@pytest.mark.parametrize("hq", [1, 33])
def test_many_rows(hq):
    """More rows than one dimension of a grid takes; rows of few heads share wavefronts."""
    T = (1 << 20) + 777
    q = torch.randn((T, 8 * hq), device="cuda").to(torch.bfloat16)
    kc = torch.randn((T, 8), device="cuda").to(torch.bfloat16)
    rope = rope_of(np.random.default_rng(0), 64, 8)
    pos = (torch.arange(T, device="cuda") % 64).int()
    slot = torch.arange(T, device="cuda").flip(0).contiguous()
    at = torch.cat((torch.arange(5), torch.arange((1 << 20) - 3, (1 << 20) + 3), torch.arange(T - 5, T))).cuda()
    q0, k0 = to_f64(q[at]), to_f64(kc[slot[at]])
    dims = ab.make_heads_dims(q, q, None, kc, hq, 1, 8, rope=rope, norm=False)
    ab.alora_qk_norm_rope(q, q, None, kc, None, None, None, None, rope, pos, slot, dims)
    c, s = angles(rope, pos[at].cpu().numpy())
    for got, x in ((q[at], q0), (kc[slot[at]], k0)):
        want, size = oh.heads(x.reshape(len(at), -1, 8), None, 0, c, s, False)
        close(got, want.reshape(len(at), -1), size.reshape(len(at), -1), torch.bfloat16, 32, "rows")


def test_slots_behind_four_gibibytes():
    n = (5 << 30) // 2048
    kc = torch.zeros((n, 1024), dtype=torch.bfloat16, device="cuda")
    h = Heads("bf16", 4, 32, 8, 128, 128, seed=5)
    slot = np.array([n - 1, 0, (1 << 32) // 2048, -1], np.int64)
    dims = ab.make_heads_dims(h.q, h.q_out, h.k, kc, 32, 8, 128, rope=h.rope, norm=True, eps=h.eps, v=h.v, v_out=kc)
    vc = torch.zeros_like(kc)
    ab.alora_qk_norm_rope(h.q, h.q_out, h.k, kc, h.v, vc, h.wq, h.wk, h.rope, dev(h.pos), dev(slot), dims)
    c, s = angles(h.rope, h.pos)
    want, size = oh.heads(to_f64(h.k).reshape(4, 8, 128), to_f64(h.wk), h.eps, c, s, False)
    at = dev(slot[:3])
    close(kc[at], want[:3].reshape(3, -1), size[:3].reshape(3, -1), h.dt, 32, "k")
    assert torch.equal(vc[at], h.v[:3]) and int((kc != 0).any(1).sum()) == 3


def test_calls_on_another_stream_and_in_a_graph():
    h = Heads("bf16", 40, 8, 2, 128, 64, seed=6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h.run(stream=side)
    h.check()
    # recorded, then replayed over other contents, with eager work between the replays
    b = Back("f32", 33, 4, 2, 64, 32, False, True, seed=6)
    pos, slot = dev(h.pos), dev(h.slot)
    call = lambda: (ab.alora_qk_norm_rope(h.q, h.q_out, h.k, h.kc, h.v, h.vc, h.wq, h.wk, h.rope, pos, slot, h.dims), b.call())
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        h.q.normal_()
        h.k.normal_()
        b.gq.normal_()
        g.replay()
        torch.cuda.synchronize()
        outs = (h.q_out, h.kc, h.vc, b.dq, b.dk, b.dwq, b.dwk)
        mine = [x.clone() for x in outs]
        for x in outs:
            x.zero_()
        call()
        torch.cuda.synchronize()
        wr = dev(h.slot[h.kept])
        for i, (x, m) in enumerate(zip(outs, mine)):
            assert torch.equal(x[wr], m[wr]) if i in (1, 2) else torch.equal(x, m), i
        h.kc.normal_()


class Back:
    def __init__(self, dtype, T, hq, hkv, d, rot, il, norm, pad=0, seed=0, inplace=False, eps=1e-5, std=2.0):
        rng = np.random.default_rng(seed)
        dt = self.dt = DT[dtype]
        self.T, self.hq, self.hkv, self.d, self.il, self.norm = T, hq, hkv, d, il, norm
        self.rope = rope_of(rng, 50, rot)
        self.pos_host = rng.integers(-2, 53, T).astype(np.int32)
        self.pos = dev(self.pos_host)
        y = values(rng, (T, (hq + 2 * hkv) * d + pad), dt, std)
        self.q, self.k = y[:, : hq * d], y[:, hq * d: (hq + hkv) * d]
        self.gq, self.gk = values(rng, (T, hq * d), dt), values(rng, (T, hkv * d), dt)
        self.wq, self.wk = (values(rng, (d,), dt, 0.3, 1.0) for _ in range(2)) if norm else (None, None)
        gq, gk = self.gq, self.gk
        if inplace:
            self.dq, self.dk = gq, gk
        else:
            dy = torch.full((T, (hq + hkv) * d + pad), float("nan"), dtype=dt, device="cuda")
            self.dq, self.dk = dy[:, : hq * d], dy[:, hq * d: (hq + hkv) * d]
        self.dwq, self.dwk = (torch.full((d,), float("nan"), device="cuda") for _ in range(2)) if norm else (None, None)
        self.dims = ab.make_heads_dims(self.q, gq, self.k, gk, hq, hkv, d, rope=self.rope, interleaved=il, norm=norm, eps=eps, dq=self.dq, dk=self.dk)
        self.ws = torch.full((max(16, ab.alora_qk_norm_rope_workspace_bytes(self.dims)),), 0xff, dtype=torch.uint8, device="cuda")
        c, s = angles(self.rope, self.pos_host)
        f = lambda t: to_f64(t).reshape(T, -1, d)
        w = lambda t: None if t is None else to_f64(t)
        self.want = [oh.heads_back(f(x), f(g), w(ww), eps, c, s, il) for x, g, ww in ((self.q, gq, self.wq), (self.k, gk, self.wk))]

    def call(self):
        ab.alora_qk_norm_rope_backward(self.q, self.gq, self.dq, self.k, self.gk, self.dk, self.wq, self.wk, self.dwq, self.dwk, self.rope, self.pos,
                                       self.dims, self.ws)

    def check(self):
        for (dx, dxs, dw, dws), got, gw, name in zip(self.want, (self.dq, self.dk), (self.dwq, self.dwk), "qk"):
            close(got, dx.reshape(self.T, -1), dxs.reshape(self.T, -1), self.dt, 96, "d" + name)
            if self.norm:
                close(gw, dw, dws, torch.float32, 256, "dw" + name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("il", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("d,rot", SHAPES)
def test_gradients(dtype, il, d, rot):
    for T, hq, hkv, norm, pad, inplace in ((5, 4, 2, True, 8, False), (3, 7, 1, True, 0, True), (2, 3, 3, False, 0, False), (1, 16, 2, True, 16, False)):
        print(f"[case] {dtype} d={d} rot={rot} il={il} T={T} {hq}/{hkv} norm={norm} pad={pad}", flush=True)
        b = Back(dtype, T, hq, hkv, d, rot, il, norm, pad, seed=d + rot + T, inplace=inplace)
        b.call()
        b.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,hq,hkv,d,rot", [(1100, 32, 8, 128, 128), (2500, 4, 2, 64, 64), (1025, 71, 1, 64, 32), (600, 40, 40, 256, 28),
                                            (1533, 8, 1, 32, 32), (300, 4, 2, 80, 20), (30, 1, 1, 8, 8)])
def test_gradients_of_larger_calls(dtype, T, hq, hkv, d, rot):
    b = Back(dtype, T, hq, hkv, d, rot, False, True, seed=T)
    b.call()
    b.check()
    first = [x.clone() for x in (b.dq, b.dk, b.dwq, b.dwk)]
    b.call()
    assert all(torch.equal(x, y) for x, y in zip(first, (b.dq, b.dk, b.dwq, b.dwk))), "equal calls give equal bits"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("std", [1.0, 1e-15])
def test_gradients_without_eps(dtype, std):
    """eps = 0: lanes without a head, of which there are some here, divide by zero; so may heads as small as 1e-15, whose r^3 no fp32 holds."""
    for T, hq, hkv, d, rot in ((3, 5, 3, 128, 64), (2, 1, 1, 80, 20), (70, 3, 1, 96, 96)):
        b = Back(dtype, T, hq, hkv, d, rot, False, True, seed=T, eps=0.0, std=std)
        b.call()
        b.check()


def test_gradients_of_no_rows():
    b = Back("bf16", 1, 4, 2, 64, 64, False, True)
    e = lambda t: t[:0]
    dims = ab.make_heads_dims(e(b.q), e(b.gq), e(b.k), e(b.gk), 4, 2, 64, rope=b.rope, dq=e(b.dq), dk=e(b.dk))
    ab.alora_qk_norm_rope_backward(e(b.q), e(b.gq), e(b.dq), e(b.k), e(b.gk), e(b.dk), b.wq, b.wk, b.dwq, b.dwk, b.rope, e(b.pos), dims, None)
    assert (b.dwq == 0).all() and (b.dwk == 0).all()


def test_gradient_against_differences_of_the_forward_call():
    """The loss sum(q_out * gq), through the library's own forward call in fp32: central differences with h = 2^-6 leave h^2 / 6 of the third
    derivative (below 2^-10 here: features are N(0, 2), a weight's loss is linear) and the outputs' rounding, 16 u of the size of
    the changed outputs' sum / h."""
    b = Back("f32", 3, 2, 1, 32, 16, True, True, seed=8)
    b.call()
    h = 2.0 ** -6
    kc = torch.zeros((16, 32), device="cuda")
    q_out, slot = torch.empty((3, 64), device="cuda"), torch.full((3,), -1, dtype=torch.int64, device="cuda")

    def loss(q, wq):
        q = q.contiguous()
        dims = ab.make_heads_dims(q, q_out, None, kc, 2, 1, 32, rope=b.rope, interleaved=True, eps=1e-5)
        ab.alora_qk_norm_rope(q, q_out, None, kc, None, None, wq, b.wk, b.rope, b.pos, slot, dims)
        return float((q_out.double() * b.gq.double()).sum())
    sizes = (b.gq.abs() * 4).view(3, 2, 32).sum(-1)          # outputs of a normalised head: below 4
    bound = lambda size: 2 * float(size) * U32 * 16 / h + 2.0 ** -10
    for r, c in ((0, 0), (1, 17), (2, 40), (2, 63)):
        e = torch.zeros_like(b.q)
        e[r, c] = h
        assert abs((loss(b.q + e, b.wq) - loss(b.q - e, b.wq)) / (2 * h) - float(b.dq[r, c])) <= bound(sizes[r, c // 32])
    for c in (0, 9, 31):
        e = torch.zeros_like(b.wq)
        e[c] = h
        assert abs((loss(b.q, b.wq + e) - loss(b.q, b.wq - e)) / (2 * h) - float(b.dwq[c])) <= bound(sizes.sum())


@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_heads_of_every_instantiation(layout, norm):
    """One, two and three units of a wavefront, and rows that share wavefronts; test_operators_abi.py finds the kernels that these sizes take."""
    dtype, d, rot, il = layout
    cases = [(T, *heads_of_a_layout(dtype, d, rot, il, uq, uk)) for T, uq, uk in UNITS.values()] + [(333, 2, 1)]
    for i, (T, hq, hkv) in enumerate(cases):
        print(f"[case] {dtype} T={T} {hq}/{hkv} d={d} rot={rot} il={il} norm={norm}", flush=True)
        h = Heads(dtype, T, hq, hkv, d, rot, il, norm, cache=bool(i % 2), seed=T + d)
        h.run()
        h.check()


@pytest.mark.parametrize("norm", [True, False], ids=["norm", "plain"])
@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_gradients_of_every_instantiation(layout, norm):
    dtype, d, rot, il = layout
    for T, (hq, hkv) in ((333, heads_of_a_layout(dtype, d, rot, il, 4, 2)), (1111, (2, 1))):
        print(f"[case] {dtype} T={T} {hq}/{hkv} d={d} rot={rot} il={il} norm={norm}", flush=True)
        b = Back(dtype, T, hq, hkv, d, rot, il, norm, seed=T + d)
        b.call()
        b.check()


def test_a_head_of_zeros_without_eps():
    """0 / 0: the head is NaN, and so is its gradient; its neighbours are what they would be."""
    for dtype, d, rot, il in (("f32", 32, 32, False), ("bf16", 128, 64, True), ("f32", 80, 20, False), ("bf16", 256, 28, False)):
        h = Heads(dtype, 3, 5, 2, d, rot, il, seed=11, eps=0.0)
        h.q[1, 2 * d: 3 * d] = 0
        h.run()
        got, (want, size) = to_f64(h.q_out).reshape(3, 5, d), (x.reshape(3, 5, d) for x in h.want_q)
        assert np.isnan(got[1, 2]).all()
        got[1, 2] = want[1, 2]
        close(got, want, size, h.dt, 32, "q")
        close(to_f64(h.kc)[h.slot[h.kept]], *h.want_k, h.dt, 32, "k")
        b = Back(dtype, 3, 5, 2, d, rot, il, True, seed=11, eps=0.0)
        b.q[1, 2 * d: 3 * d] = 0
        b.call()
        got, (want, size) = to_f64(b.dq).reshape(3, 5, d), (x for x in b.want[0][:2])
        assert np.isnan(got[1, 2]).all()
        got[1, 2] = want[1, 2]
        close(got, want, size, b.dt, 96, "dq")
        close(b.dk, *[x.reshape(3, -1) for x in b.want[1][:2]], b.dt, 96, "dk")
        close(b.dwk, *b.want[1][2:], torch.float32, 256, "dwk")


def test_gradients_of_infinities_and_nan_stay_in_their_heads():
    """A NaN among a head's features makes its gradient NaN, an infinite gradient of an output makes its head's not finite (without norm: its pair's); other
    heads' gradients, and the other norm's weights', are what they would be."""
    for dtype, d, rot, il in (("bf16", 128, 64, False), ("bf16", 64, 24, True), ("f32", 80, 20, True), ("f32", 32, 32, False), ("f32", 80, 20, False)):
        for norm in (True, False):
            for where, value in (("x", float("nan")), ("x", float("inf")), ("g", float("inf")), ("g", float("nan"))):
                if where == "x" and not norm:
                    continue              # (features are not looked at)
                b = Back(dtype, 70, 6, 2, d, rot, il, norm, seed=9)
                (b.q if where == "x" else b.gq)[41, 2 * d + d - 1] = value
                b.call()
                got, (want, size) = to_f64(b.dq).reshape(70, 6, d), b.want[0][:2]
                bad = np.argwhere(~np.isfinite(got))
                assert len(bad) and (bad[:, :2] == [41, 2]).all(), (dtype, d, norm, where, bad[:4])
                assert len(bad) == d if norm else len(bad) <= 2 and bad[-1, 2] == d - 1, (dtype, d, norm, where, bad)
                keep = np.isfinite(got)
                got[~keep] = want[~keep]
                close(got, want, size, b.dt, 96, "dq")
                close(b.dk, *[x.reshape(70, -1) for x in b.want[1][:2]], b.dt, 96, "dk")
                if norm:
                    close(b.dwk, *b.want[1][2:], torch.float32, 256, "dwk")
                    assert not np.isfinite(to_f64(b.dwq)).all()


@pytest.mark.parametrize("rot,base,first,rows,kw", [
    (128, 1e4, 0, 4097, {}), (64, 1e6, 1000, 777, dict(scaling="linear", factor=4.0)), (20, 5e5, 0, 1, {}), (2, 1e4, 3, 1000, {}), (512, 1e4, 0, 300, {}),
    (256, 1e4, 100, 9, {}), (258, 1e4, 1, 33, {}),
    (128, 5e5, 900000, 100003, dict(scaling="by_parts", factor=16.0, original=8192, low=1, high=32, magnitude=1.27)),
    (96, 1e4, (1 << 24) - 600, 600, dict(scaling="by_parts", factor=40.0, original=4096, low=1, high=4)), (6, 1.0, 0, 50, {}), (8, 0.5, 0, 100, {})])
def test_tables(rot, base, first, rows, kw):
    """Half a step of the result, and what 64-bit angles lose: 2^-50 of the position."""
    wide = torch.full((2, rows * (rot // 2) + 64), 7.0, device="cuda")
    cos, sin = (w[: rows * (rot // 2)].view(rows, rot // 2) for w in wide)
    if cos.data_ptr() % 16 or sin.data_ptr() % 16:
        sin = torch.empty_like(cos)
    ab.alora_rope_tables(cos, sin, ab.make_rope_spec(rot, base, **kw), first)
    c, s = oh.tables(rot, base, first, rows, **kw)
    theta = 1.0 if base >= 1 else base ** -1.0
    slack = kw.get("magnitude", 1.0) * (2.0 ** -40 + theta * (first + rows) * 2.0 ** -50)
    for got, want in ((cos, c), (sin, s)):
        err = np.abs(got.cpu().numpy().astype(np.longdouble) - want)
        step = np.spacing(np.abs(want).astype(np.float32)).astype(np.longdouble)
        assert (err <= step / 2 * (1 + 2.0 ** -20) + slack).all(), float((err - step / 2).max())
    assert (wide[:, rows * (rot // 2):] == 7.0).all(), "written behind the tables"


@pytest.mark.parametrize("rot,base,first,rows,kw", [
    (128, 1e4, 0, 4097, {}), (512, 1e4, 0, 40000, {}), (2, 1e4, 3, 200000, {}), (64, 1e30, 0, 5000, {}), (6, 1.0, 0, 50, {}), (8, 0.5, 0, 100, {}),
    (8, 0.001, 0, 3000, {}), (64, 1e-10, 0, 5000, {}), (64, 1e4, 0, 5000, dict(scaling="linear", factor=0.01)),
    (64, 1e-10, 70000, 500, dict(scaling="linear", factor=1e-3)), (128, 5e5, 0, 70001, dict(scaling="by_parts", factor=16.0, original=8192, low=1, high=32, magnitude=1.27)),
    (96, 1e4, 0, 60000, dict(scaling="by_parts", factor=0.02, original=4096, low=1, high=4, magnitude=0.5)),
    (96, 1e4, 5, 600, dict(scaling="by_parts", factor=40.0, original=4096, low=1, high=1.0001))])
def test_tables_within_the_bound_of_each_position(rot, base, first, rows, kw):
    """Half a step of the result, and of each row's own position what the header states: 2^-49 of it, more where angles of a position are large."""
    cos, sin = (torch.empty((rows, rot // 2), device="cuda") for _ in range(2))
    ab.alora_rope_tables(cos, sin, ab.make_rope_spec(rot, base, **kw), first)
    c, s = oh.tables(rot, base, first, rows, **kw)
    largest = max(1.0, base ** (2 / rot - 1))            # of a position, before scaling
    factor, t = kw.get("factor", 1.0), 1.0
    if base < 1 or factor < 1:
        t = max(1.0, largest * max(1.0, 1 / factor)) * (1 + max(0.0, -np.log2(base)) / 4)
    if kw.get("scaling") == "by_parts":
        t *= 1 + kw["high"] / (kw["high"] - kw["low"])
    slack = kw.get("magnitude", 1.0) * t * 2.0 ** -49 * np.arange(first, first + rows)[:, None].astype(np.longdouble)
    for got, want in ((cos, c), (sin, s)):
        err = np.abs(got.cpu().numpy().astype(np.longdouble) - want)
        step = np.spacing(np.abs(want).astype(np.float32)).astype(np.longdouble)
        over = err - (step / 2 * (1 + 2.0 ** -20) + slack)
        assert (over <= 0).all(), (float(over.max()), np.unravel_index(int(np.argmax(over)), over.shape))


# ---- the cache ----------------------------------------------------------------------------------
class Cache:
    def __init__(self, dtype, layers, blocks, hkv, d, bs, seed=0):
        self.rng = np.random.default_rng(seed)
        self.dt, self.blocks, self.bs, self.hkv, self.d, self.layers = DT[dtype], blocks, bs, hkv, d, layers
        self.k, self.v = ([values(self.rng, (blocks * bs, hkv * d), self.dt) for _ in range(layers)] for _ in range(2))
        self.before = [raw_bits(t).copy() for t in (*self.k, *self.v)]
        self.dims = ab.make_cache_dims(self.k, self.v, hkv, d, bs)

    def after(self):
        return [raw_bits(t) for t in (*self.k, *self.v)]


@pytest.mark.parametrize("dtype,layers,blocks,hkv,d,bs,pairs,clears", [
    ("bf16", 3, 20, 2, 64, 16, 1, 0), ("bf16", 2, 20, 1, 8, 1, 9, 2), ("f32", 1, 9, 1, 4, 3, 4, 4), ("bf16", 5, 70, 8, 128, 16, 33, 3), ("f32", 2, 40, 3, 80, 5, 17, 0),
    ("bf16", 1, 1900, 2, 32, 8, 900, 90), ("bf16", 66, 12, 1, 64, 16, 5, 1), ("f32", 130, 60, 1, 16, 4, 20, 2), ("bf16", 2, 12, 16, 128, 33, 6, 1), ("bf16", 1, 4, 8, 256, 64, 2, 1),
    ("bf16", 2, 300, 8, 128, 16, 140, 7), ("bf16", 2, 300, 9, 128, 16, 140, 3)])
def test_blocks(dtype, layers, blocks, hkv, d, bs, pairs, clears):
    c = Cache(dtype, layers, blocks, hkv, d, bs, seed=blocks)
    perm = c.rng.permutation(blocks).astype(np.int32)
    src, dst = perm[:pairs].copy(), perm[pairs: 2 * pairs].copy()
    src[pairs - clears:] = -1
    ab.alora_cache_copy_blocks(src, dst, c.dims)
    src_then, dst_then = src.copy(), dst.copy()
    src[:], dst[:] = 0, 0                     # (the lists are read before the call returns)
    for got, b in zip(c.after(), c.before):
        want = b.reshape(blocks, -1).copy()
        for s, t in zip(src_then, dst_then):
            want[t] = b.reshape(blocks, -1)[s] if s >= 0 else 0
        assert np.array_equal(got.reshape(blocks, -1), want)


def test_blocks_of_a_source_named_often_and_behind_four_gibibytes():
    n = (5 << 30) // 32768
    k = torch.zeros((n * 16, 1024), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[-16:] = 3.0
    v[:16] = 5.0
    dims = ab.make_cache_dims([k], [v], 8, 128, 16)
    ab.alora_cache_copy_blocks(np.array([n - 1, n - 1, 0], np.int32), np.array([1, n - 2, n - 3], np.int32), dims)
    for b, kk, vv in ((1, 3, 0), (n - 2, 3, 0), (n - 3, 0, 5), (n - 1, 3, 0), (0, 0, 5), (2, 0, 0)):
        assert (k[b * 16: b * 16 + 16] == kk).all() and (v[b * 16: b * 16 + 16] == vv).all(), b
    ab.alora_cache_move_rows(dev(np.array([16 * n - 1, 3], np.int64)), dev(np.array([40, 16 * n - 20], np.int64)), None, None, dims)
    assert (k[40] == 3).all() and (v[16 * n - 20] == 5).all() and (k[41] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("il", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("d,rot", SHAPES)
def test_rows(dtype, il, d, rot):
    """Moves by positive and negative shifts, some of none and beyond the tables; rows turned where they lie; indexes outside the cache."""
    for layers, hkv, n in ((1, 2, 7), (3, 1, 40), (9, 5, 3)):
        print(f"[case] {dtype} d={d} rot={rot} il={il} layers={layers} hkv={hkv} n={n}", flush=True)
        c = Cache(dtype, layers, 2 * n // 4 + 4, hkv, d, 4, seed=d + rot + n)
        n_slots = c.blocks * 4
        perm = c.rng.permutation(n_slots)
        src, dst = perm[:n].copy(), perm[n: 2 * n].copy()
        dst[0] = src[0]
        shift = c.rng.integers(-30, 31, n).astype(np.int32)
        shift[1], shift[2] = 0, -(1 << 31)
        rope = rope_of(c.rng, 25, rot)
        bad = n - 1
        assert ab.alora_cache_move_rows_validate(dev(src), dev(dst), dev(np.clip(shift, -24, 24)) if rot else None, rope, c.dims) == ab.ALORA_OK
        src[bad] = (n_slots, -1, -(1 << 60))[layers % 3]
        assert ab.alora_cache_move_rows_validate(dev(src), dev(dst), None, rope, c.dims) == ab.ALORA_EDATA
        if rot and bad > 2:
            assert ab.alora_cache_move_rows_validate(dev(src[:bad]), dev(dst[:bad]), dev(shift[:bad]), rope, c.dims) == ab.ALORA_EDATA
        ab.alora_cache_move_rows(dev(src), dev(dst), dev(shift) if rot else None, rope, c.dims, interleaved=il)
        for i, (got, b) in enumerate(zip(c.after(), c.before)):
            other = np.setdiff1d(np.arange(n_slots), dst[:bad])
            assert np.array_equal(got[other], b[other])
            plain = np.arange(bad) if i >= layers or not rot else np.flatnonzero(shift[:bad] == 0)
            assert np.array_equal(got[dst[plain]], b[src[plain]])
        if rot:
            far = np.minimum(np.abs(shift[:bad].astype(np.int64)), 24)
            cs, sn = to_f64(rope[0])[far], to_f64(rope[1])[far] * np.sign(shift[:bad])[:, None]
            turned = np.flatnonzero(shift[:bad])
            for t, b in zip(c.k, c.before):
                x = torch.from_numpy(b.view(np.int16 if dtype == "bf16" else np.int32)).view(c.dt)
                x = to_f64(x)[src[turned]].reshape(len(turned), hkv, d)
                want, size = oh.heads(x, None, 0, cs[turned], sn[turned], il)
                close(to_f64(t)[dst[turned]], want.reshape(len(turned), -1), size.reshape(len(turned), -1), c.dt, 32, "k")


@pytest.mark.parametrize("dtype,layers,hkv,d,n", [("bf16", 70, 2, 64, 50), ("bf16", 16, 8, 128, 3000), ("f32", 5, 40, 256, 9), ("bf16", 2, 1, 128, 9001)])
def test_rows_of_larger_calls(dtype, layers, hkv, d, n):
    c = Cache(dtype, layers, 2 * n // 16 + 4, hkv, d, 16, seed=n)
    perm = c.rng.permutation(c.blocks * 16)
    src, dst = perm[:n], perm[n: 2 * n]
    shift = c.rng.integers(-20, 20, n).astype(np.int32)
    shift[shift == 0] = 7
    rope = rope_of(c.rng, 25, d)
    k0 = [t.clone() for t in c.k]
    ab.alora_cache_move_rows(dev(src), dev(dst), dev(shift), rope, c.dims)
    far = np.abs(shift)
    cs, sn = to_f64(rope[0])[far], to_f64(rope[1])[far] * np.sign(shift)[:, None]
    at = c.rng.permutation(n)[:64]
    for l in range(layers):
        want, size = oh.heads(to_f64(k0[l][dev(src[at])]).reshape(len(at), hkv, d), None, 0, cs[at], sn[at], False)
        close(c.k[l][dev(dst[at])], want.reshape(len(at), -1), size.reshape(len(at), -1), c.dt, 32, f"layer {l}")
        assert np.array_equal(raw_bits(c.v[l])[dst], c.before[layers + l][src])
        other = np.setdiff1d(np.arange(c.blocks * 16), dst)
        assert np.array_equal(raw_bits(c.k[l])[other], c.before[l][other])


def test_copies_and_moves_in_a_graph():
    c = Cache("bf16", 3, 60, 2, 64, 16, seed=2)
    src, dst = np.arange(20, dtype=np.int32), np.arange(20, 40, dtype=np.int32)
    rows, to = dev(np.arange(640, 700)), dev(np.arange(720, 780))
    shift, rope = dev(np.full(60, -3, np.int32)), rope_of(c.rng, 9, 64)
    call = lambda: (ab.alora_cache_copy_blocks(src, dst, c.dims), ab.alora_cache_move_rows(rows, to, shift, rope, c.dims))
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    src[:] = 0                                  # (the graph holds the lists it was captured with)
    src_then = np.arange(20, dtype=np.int32)
    for _ in range(3):
        for t in (*c.k, *c.v):
            t.normal_()
        before = [t.clone() for t in (*c.k, *c.v)]
        g.replay()
        torch.cuda.synchronize()
        mine = [t.clone() for t in (*c.k, *c.v)]
        for t, b in zip((*c.k, *c.v), before):
            t.copy_(b)
        ab.alora_cache_copy_blocks(src_then, dst, c.dims)
        ab.alora_cache_move_rows(rows, to, shift, rope, c.dims)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(mine, (*c.k, *c.v)))
