"""Norm, rotation and matrix of queries and keys (flatquant_head_rope) against fp64."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2410_09426_amd import binding as fq
from gpu_util import dev, host_f16

pytestmark = pytest.mark.gpu
D = 128


class Rows:
    def __init__(self, seed, T, Hq, H, rotary=128, interleaved=False, norm=False, P=0, pad=0, q_pad=0, k_pad=0, fused=False, far=5000, gain=1.0, base=10000.0, keys_P=False,
                 eps=1e-6):
        r = np.random.Generator(np.random.PCG64(seed))
        self.T, self.heads, self.rotary, self.interleaved, self.eps = T, (Hq, H), rotary, interleaved, eps
        self.pos = r.integers(0, far, T).astype(np.int32)
        if T:
            self.pos[0], self.pos[T // 2] = 0, far - 1
        if pad:
            self.pos[T - pad:] = -1
        self.f = np.array([base ** (-2 * i / max(rotary, 1)) for i in range(rotary // 2)])
        self.strides = [Hq * D + q_pad, H * D + k_pad]
        self.x = [(r.standard_normal((T, h, D)) * gain).astype(np.float16) for h in (Hq, H)]
        self.fused = fused
        self.w = [(1 + 0.3 * r.standard_normal(D)).astype(np.float16) if norm else None for _ in range(2)]
        self.P = [None, None]
        for x in range(2):
            if P and (x == 0 or keys_P):
                self.P[x] = (np.eye(D) + 0.05 * r.standard_normal((self.heads[x] if P == 2 else 1, D, D))).astype(np.float16)
        self.per_head = P == 2

    def run(self, sides="qk", out_pad=8, stream=None):
        Hq, H = self.heads
        if self.fused:                                           # queries, keys and values of a token in one row
            rows = np.zeros((self.T, Hq + 2 * H, D), dtype=np.float16)
            rows[:, :Hq], rows[:, Hq:Hq + H] = self.x
            d = dev(rows)
            x, strides = [d[:, :Hq], d[:, Hq:Hq + H]], [(Hq + 2 * H) * D] * 2
        else:
            x, strides = [], self.strides
            for a, s in zip(self.x, strides):
                full = np.full((self.T, s), np.nan, dtype=np.float16)
                full[:, :a.shape[1] * D] = a.reshape(self.T, -1)
                x.append(dev(full))
        out = [torch.full((self.T + 1, h * D + out_pad), -7.25, dtype=torch.float16, device="cuda") for h in self.heads]
        turns = torch.from_numpy(fq.fq_rope_turns(self.f).view(np.int64)).cuda() if self.rotary else None
        w, P = ([None if a is None else dev(a) for a in y] for y in (self.w, self.P))
        self.kept = (x, out, turns, w, P, dev(self.pos))
        q, k = "q" in sides, "k" in sides
        fq.flatquant_head_rope(x[0] if q else None, strides[0], Hq, x[1] if k else None, strides[1], H, self.T, self.kept[-1], turns, self.rotary, self.interleaved,
                               w[0], w[1], self.eps, P[0], P[1], self.per_head, out[0] if q else None, Hq * D + out_pad, out[1] if k else None, H * D + out_pad,
                               stream=stream or torch.cuda.current_stream())
        torch.cuda.synchronize()
        got = []
        for a, h, there in zip(out, self.heads, (q, k)):
            g = host_f16(a).reshape(self.T + 1, -1)
            untouched = np.concatenate([g[:, h * D:].ravel(), g[self.T:].ravel(), g[:self.T][self.pos < 0].ravel()])
            assert np.all(untouched == np.float16(-7.25)) and (there or np.all(g == np.float16(-7.25))), "written beside the rows"
            got.append(g[:self.T, :h * D].reshape(self.T, h, D))
        return got

    def check(self, sides="qk", rows=None, **how):
        got = self.run(sides, **how)
        pick = np.arange(self.T) if rows is None else np.asarray(rows)
        pick = pick[self.pos[pick] >= 0]
        for x, side in enumerate("qk"):
            if side not in sides:
                continue
            want, tol = so.rope64(self.x[x][pick], self.w[x], self.eps, self.pos[pick], self.f, self.interleaved, self.P[x])
            err = np.abs(got[x][pick].astype(np.float64) - want)
            worst = float((err / tol).max()) if err.size else 0.0
            print(f"[case] {side}: worst error {worst:.3f} of the bound", flush=True)
            assert np.all(np.isfinite(got[x][pick])) and worst <= 1.0, np.unravel_index(int((err / tol).argmax()), err.shape)
        return got


@pytest.mark.parametrize("rotary", [0, 32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotations_without_a_matrix(rotary, interleaved, norm):
    print(f"[case] rotary={rotary} interleaved={interleaved} norm={norm}", flush=True)
    Rows(rotary + interleaved, 37, 5, 2, rotary, interleaved, norm, pad=3, q_pad=8, k_pad=24).check()


@pytest.mark.parametrize("P", [1, 2])
@pytest.mark.parametrize("rotary", [0, 32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations_with_a_matrix(rotary, interleaved, P):
    print(f"[case] rotary={rotary} interleaved={interleaved} P={P}", flush=True)
    Rows(rotary + interleaved, 37, 5, 2, rotary, interleaved, norm=rotary != 64, P=P, pad=3, q_pad=8, keys_P=interleaved).check()


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 31, 32, 33, 64, 127, 300])
@pytest.mark.parametrize("Hq,H", [(1, 1), (32, 8), (28, 4), (3, 3)])
@pytest.mark.parametrize("P", [0, 1])
def test_row_and_head_counts(T, Hq, H, P):
    print(f"[case] T={T} heads={Hq},{H} P={P}", flush=True)
    Rows(T, T, Hq, H, norm=True, P=P, fused=T % 2 == 0).check(rows=range(0, T, max(1, T // 40)))


@pytest.mark.parametrize("P,keys_P", [(0, False), (1, False), (1, True), (2, True)])
def test_long_launches(P, keys_P):
    """Several heads a wave, several blocks a workgroup."""
    print(f"[case] long P={P}", flush=True)
    T = 4999
    c = Rows(5, T, 32, 8, norm=True, P=P, fused=True, keys_P=keys_P, pad=2)
    c.check(rows=np.unique(np.concatenate([np.arange(8), np.arange(T - 40, T), np.random.default_rng(1).integers(0, T, 60)])))


@pytest.mark.parametrize("sides", ["q", "k"])
@pytest.mark.parametrize("P", [0, 1, 2])
def test_one_side_alone(sides, P):
    print(f"[case] {sides} alone P={P}", flush=True)
    Rows(6, 70, 8, 4, norm=True, P=P, keys_P=True).check(sides)


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 24 + 3, 2 ** 31 - 1])
@pytest.mark.parametrize("base", [100.0, 500000.0])
def test_far_positions(far, base):
    """The angle is exact modulo a turn; fp64 of the oracle is off by 2^-53 of it, 2^31 radians: 2^-22, which is added."""
    print(f"[case] far={far} base={base}", flush=True)
    c = Rows(7, 200, 2, 1, far=far, base=base)
    got = c.run()
    for x in range(2):
        want, size = so.turned64(c.x[x], None, 0.0, c.pos, c.f, False)
        tol = so.half_bound(want, so.turned_bound(size) + size * (far * 2.0 ** -53 + far * 2.0 ** -65))
        assert np.all(np.abs(got[x] - want) <= tol)


def test_values_of_all_sizes():
    """Subnormal rows, the largest ones, zeros; with a norm a row of zeros stays one."""
    print("[case] sizes", flush=True)
    c = Rows(8, 64, 2, 1)
    c.x[0] *= (2.0 ** np.random.default_rng(2).integers(-24, 13, (64, 1, 1))).astype(np.float16)
    c.x[0][5] = 0
    c.check()
    for eps in (1e-5, 1.2e-38):
        c = Rows(9, 64, 2, 1, norm=True, eps=eps)
        c.x[0][5], c.x[0][6] = 0, 60000.0
        got = c.check()
        assert not got[0][5].any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_infinities_stay_in_their_pair(interleaved):
    print(f"[case] infinities interleaved={interleaved}", flush=True)
    for bad in (np.inf, -np.inf, np.nan):
        c = Rows(10, 9, 3, 1, rotary=64, interleaved=interleaved)
        c.x[0][2, 1, 100], c.x[0][4, 0, 3], c.x[1][7, 0, 40] = bad, bad, bad
        clean = Rows(10, 9, 3, 1, rotary=64, interleaved=interleaved).run()
        got = c.run()
        places = [(0, 2, 1, 100), (0, 4, 0, 3), (0, 4, 0, 2 if interleaved else 35), (1, 7, 0, 40), (1, 7, 0, 41 if interleaved else 8)]
        for x in range(2):
            same = got[x] == clean[x]
            assert not any(same[p[1:]] for p in places if p[0] == x) and (~same).sum() == sum(p[0] == x for p in places)
        assert got[0][2, 1, 100] == bad or np.isnan(bad)                       # not turned


def test_a_norm_of_a_row_that_is_no_number_stays_in_its_head():
    print("[case] norm of a NaN", flush=True)
    c = Rows(11, 9, 3, 1, norm=True)
    clean = c.run()
    c.x[0][2, 1, 100] = np.nan
    got = c.run()
    assert np.isnan(got[0][2, 1]).all()
    got[0][2, 1] = clean[0][2, 1]
    assert all(np.array_equal(g, k) for g, k in zip(got, clean))


def test_launch_forms_give_the_same_rows():
    """A row's result does not depend on how many rows there are, but for the matrix kernels' one and the same arithmetic in both."""
    print("[case] forms", flush=True)
    for P in (0, 1, 2):
        c = Rows(12, 3000, 32, 8, norm=True, P=P, keys_P=True, fused=True)
        whole = c.run()
        few = Rows(12, 3000, 32, 8, norm=True, P=P, keys_P=True, fused=True)
        few.T, few.pos, few.x = 21, few.pos[:21], [x[:21] for x in few.x]
        part = few.run()
        assert all(np.array_equal(a[:21], b) for a, b in zip(whole, part)), P


def test_more_rows_than_a_grid_has():
    """2^22 rows and more: workgroups take several blocks; the last rows and some others against those of a short call."""
    print("[case] 2^22 + 77 rows", flush=True)
    T = 2 ** 22 + 77
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn((T, D), generator=gen, device="cuda", dtype=torch.float16)
    pos = torch.randint(0, 2 ** 20, (T,), generator=gen, device="cuda", dtype=torch.int32)
    turns = torch.from_numpy(fq.fq_rope_turns([10000.0 ** (-2 * i / D) for i in range(D // 2)]).view(np.int64)).cuda()
    out = torch.full((T, D), -7.25, dtype=torch.float16, device="cuda")
    call = lambda x, pos, out: fq.flatquant_head_rope(x, D, 1, None, 0, 0, len(x), pos, turns, D, 0, None, None, 0.0, None, None, 0, out, D, None, 0,      # noqa: E731
                                                      stream=torch.cuda.current_stream())
    call(x, pos, out)
    for rows in (slice(0, 500), slice(2 ** 22 - 250, 2 ** 22 + 77), slice(2 ** 21, 2 ** 21 + 100)):
        part = torch.empty_like(out[rows])
        call(x[rows].contiguous(), pos[rows].contiguous(), part)
        assert torch.equal(part, out[rows])


@pytest.mark.parametrize("P", [0, 1, 2])
def test_rows_far_apart(P):
    """Rows 2^31 halves apart: offsets beyond 2^32 bytes, into and out of the call."""
    print(f"[case] far rows P={P}", flush=True)
    stride, T, H = 2 ** 31, 3, 2
    c = Rows(14, T, H, 1, norm=True, P=P)
    near = c.run("q", out_pad=0)[0]
    x, w, P_dev = torch.empty(2 * stride + H * D, dtype=torch.float16, device="cuda"), c.kept[3][0], c.kept[4][0]
    out = torch.empty_like(x)
    for t in range(T):
        x[t * stride:t * stride + H * D] = c.kept[0][0][t, :H * D]
    fq.flatquant_head_rope(x, stride, H, None, 0, 0, T, c.kept[5], c.kept[2], D, 0, w, None, c.eps, P_dev, None, c.per_head, out, stride, None, 0,
                           stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for t in range(T):
        assert np.array_equal(host_f16(out[t * stride:t * stride + H * D]).reshape(H, D), near[t])


def test_the_matrix_is_that_of_the_head_transform():
    """Without norm and rotation: the bits of flatquant_head_transform."""
    print("[case] head transform", flush=True)
    for T, P in ((50, 1), (50, 2), (3000, 1), (3000, 2)):
        c = Rows(13, T, 8, 4, rotary=0, P=P)
        got = c.run("q")[0]
        out = torch.empty((T, 8, D), dtype=torch.float16, device="cuda")
        fq.flatquant_head_transform(dev(c.x[0]), c.kept[4][0], 8 if P == 2 else 1, T, 8, D, out, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert np.array_equal(got, host_f16(out).reshape(got.shape)), (T, P)
