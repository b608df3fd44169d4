"""GPU parity of the paged key-value cache (append, attention of one new token, eviction by accumulated weight) against the fp64
oracle, through the C ABI.

Bounds.  eps = 2^-24 is half a step of fp32.  A logit is a sum of d products of fp32 values: d + 16 roundings of at most
L = sum_c (|q_c| + |q_pair(c)|) |k_c| / sqrt(d) (a rotated channel is at most that), cos and sin off by at most 2^-22 each (twice
that together), and the exponential's argument and result 2^-22 of the largest logit:
    delta = ((d + 16) eps + 2^-21) L + 2^-22 max|x|
A weight p is off by at most p (2 delta + (64 + n / 32) eps) (its own error and the normaliser's, whose n terms are added in
runs of n / 32 at most and joined).  A weight goes to the bf16 matrix cores as a head and a remainder, 2^-14 of it at most lost.
The output adds the error of its own sum, (64 + n / 32) eps of sum p |v|, and one rounding to the storage type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from oracle import paged_oracle as po  # noqa: E402
from paper_2510_24273_amd import binding  # noqa: E402

DEV = "cuda:0"
EPS = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy() if t.is_floating_point() else t.detach().cpu().numpy()


class Cache:
    """A random cache on the device with what lies outside it filled with NaN, and its host copies."""

    def __init__(self, lens, H=8, H_kv=2, d=128, P=16, dtype="bf16", lists=0, mp=None, seed=0, style=0, theta=10000.0, joined=False, holes=(),
                 spread=1.0, spare=5):
        print(f"[case] lens={lens} H={H}/{H_kv} d={d} P={P} {dtype} lists={lists} mp={mp} style={style} joined={joined} holes={holes}", flush=True)
        g = torch.Generator().manual_seed(seed)
        self.lens, self.B, self.H, self.H_kv, self.d, self.P, self.dtype, self.lists = list(lens), len(lens), H, H_kv, d, P, dtype, lists
        self.style, self.theta = style, theta
        self.mp = mp or max(1, -(-max(lens) // P))
        self.cap, self.n_pages = self.mp * P, self.B * self.mp + spare
        B, n_pages, cap = self.B, self.n_pages, self.cap
        perm = torch.randperm(n_pages, generator=g)[: B * self.mp].view(B, self.mp).to(torch.int32)
        for b, pg, to in holes:
            perm[b, pg] = to
        self.table_h = perm.numpy()
        pools = []
        for _ in range(2):
            x = torch.full((n_pages, P, H_kv, d), float("nan"))
            for b, n in enumerate(lens):
                page, row, there = po.slots(self.table_h[b], P, min(n, cap), n_pages)
                vals = torch.randn(int(there.sum()), H_kv, d, generator=g)
                x[torch.from_numpy(page[there]).long(), torch.from_numpy(row[there]).long()] = vals
            pools.append(x.to(DT[dtype]))
        if joined:
            both = torch.stack(pools, dim=1).to(DEV)
            self.Kp, self.Vp = both[:, 0], both[:, 1]
        else:
            self.Kp, self.Vp = (x.to(DEV) for x in pools)
        self.q = (spread * torch.randn(B, H, d, generator=g)).to(DT[dtype]).to(DEV)
        self.q_pos = torch.tensor([n + 3 * b for b, n in enumerate(lens)], dtype=torch.int32, device=DEV)
        self.table = perm.to(DEV)
        self.seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.out = torch.full((B, H, d), float("nan"), dtype=DT[dtype], device=DEV)
        self.weights = self.pos = None
        if lists:
            self.weights = (torch.rand(B, lists, cap, generator=g) * 3).to(DEV)
            self.pos = torch.randint(0, 1 << 20, (B, lists, cap), generator=g, dtype=torch.int32).to(DEV)
        desc = binding.make_paged_desc(B, H, H_kv, d, P, self.mp, n_pages, dtype, weight_heads=lists, page_stride=self.Kp.stride(0),
                                       rope_theta=theta, rope_style=style)
        self.ctx = binding.Paged(desc, DEV)

    def attend(self, weights=True):
        self.ctx.attend(self.q, self.q_pos, self.table, self.Kp, self.Vp, self.seq_len, self.out, weights=self.weights if weights else None)

    def rows(self, pool, b, n):
        """[n, H_kv, d] fp64 of the first n slots (zero where the page is not there), and which are there."""
        page, row, there = po.slots(self.table_h[b], self.P, n, self.n_pages)
        x = np.zeros((n, self.H_kv, self.d))
        if n and there.any():
            t = pool[torch.from_numpy(page[there]).long().to(DEV), torch.from_numpy(row[there]).long().to(DEV)]
            x[there] = _np(t)
        return x, there

    def check_attend(self, before=None):
        worst = 0.0
        for b, n in enumerate(self.lens):
            n = max(0, min(n, self.cap))
            K, there = self.rows(self.Kp, b, n)
            V, _ = self.rows(self.Vp, b, n)
            q, pos = _np(self.q[b]), int(self.q_pos[b])
            want, p = po.attend(q, pos, K, V, there, self.theta, self.style)
            got = _np(self.out[b])
            assert np.isfinite(got).all(), f"b={b}: not finite"
            if not there.any():
                assert not got.any(), f"b={b}: nothing attended, not zero"
            else:
                group = self.H // self.H_kv
                pair = np.roll(np.abs(q), self.d // 2, axis=-1) if not self.style else np.abs(q).reshape(self.H, -1, 2)[..., ::-1].reshape(self.H, -1)
                big = np.abs(q) + pair
                Kh, Vh = np.repeat(np.abs(K), group, axis=1), np.repeat(np.abs(V), group, axis=1)     # [n, H, d]
                L = np.einsum("hc,nhc->hn", big, Kh).max(axis=1) / np.sqrt(self.d)                    # [H]
                delta = ((self.d + 16) * EPS + 2.0 ** -21 + 2.0 ** -22) * L
                run = (64 + n / 32) * EPS
                rel = 2 * delta + run + (2.0 ** -14 if self.dtype == "bf16" else 0.0)
                bound = HALF[self.dtype] * np.abs(want) * (1 + 2.0 ** -6) + (rel + run)[:, None] * np.einsum("hn,nhc->hc", p, Vh) * 1.01 + 1e-30
                err = np.abs(got - want)
                worst = max(worst, float((err / bound).max()))
                assert (err <= bound).all(), f"b={b}: {float((err / bound).max()):.3g} of the bound, at {np.unravel_index((err / bound).argmax(), err.shape)}"
            if before is not None:
                w = po.list_weights(p, self.lists)
                if there.any():
                    wb = po.list_weights(p * (2 * delta + run)[:, None], self.lists)
                else:
                    wb = np.zeros_like(w)
                ref = before[b].cpu().double().numpy()
                ref[:, :n] += w
                got_w = _np(self.weights[b])
                werr = np.abs(got_w - ref)
                wbound = (self.H + 2) * EPS * np.abs(ref)
                wbound[:, :n] += wb * 1.01
                assert (werr <= wbound).all(), f"b={b}: weights {werr.max():.3g}"
                assert np.array_equal(got_w[:, n:], ref[:, n:]), f"b={b}: weights past the length changed"
        print(f"    worst error {worst:.3f} of the bound", flush=True)


# ---- attention ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_from_none_to_long(dtype, d):
    c = Cache([0, 1, 2, 15, 16, 17, 31, 33, 64, 127, 129, 1000, 3333], d=d, dtype=dtype, lists=2)
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)


@pytest.mark.parametrize("H,H_kv", [(1, 1), (4, 4), (8, 2), (8, 1), (32, 8), (12, 4), (20, 1), (15, 5), (64, 8), (40, 2), (34, 2), (96, 32),
                                    (300, 300), (512, 256), (1024, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_layouts(H, H_kv, dtype):
    for lists in ((1, H_kv) if H_kv > 1 else (1,)):
        c = Cache([300, 77, 1024], H=H, H_kv=H_kv, dtype=dtype, lists=lists)
        before = c.weights.clone()
        c.attend()
        torch.cuda.synchronize()
        c.check_attend(before)


@pytest.mark.parametrize("P", [1, 2, 3, 4, 7, 8, 12, 24, 32, 64, 100, 128, 2048])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
def test_page_sizes(P, dtype, d):
    c = Cache([1, 259, 1030], P=P, dtype=dtype, d=d, joined=True, lists=1, mp=-(-1200 // P))
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("style", [0, 1])
def test_pairings_and_far_positions(dtype, style):
    c = Cache([50, 50, 50, 50], style=style, dtype=dtype, theta=500000.0)
    c.q_pos.copy_(torch.tensor([0, 131071, 2 ** 30 + 7, -5], dtype=torch.int32))
    c.attend()
    torch.cuda.synchronize()
    c.check_attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_are_not_there(dtype):
    """-1, n_pages and other numbers outside the pool: no weight; with all pages of a sequence gone, zero."""
    c = Cache([100, 100, 100, 160], P=16, dtype=dtype, lists=2,
              holes=[(0, 0, -1), (0, 3, 2 ** 31 - 1), (0, 6, -2 ** 31), (1, 1, 4 * 10 + 5)] + [(2, k, -1) for k in range(7)] + [(3, 9, -7)])
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_outside_the_cache_are_clamped(dtype):
    c = Cache([64, 64, 64], dtype=dtype, mp=4)
    c.seq_len.copy_(torch.tensor([-3, 10 ** 9, 64], dtype=torch.int32))
    c.lens = [0, 64, 64]
    c.attend()
    torch.cuda.synchronize()
    c.check_attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_logits_and_an_infinite_value(dtype):
    c = Cache([700, 700], dtype=dtype, spread=12.0, lists=2)
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)
    # an infinity in a value row stays one, in its channel only
    c = Cache([40, 333], dtype=dtype)
    pg, row = int(c.table_h[1, 5]), 3
    c.Vp[pg, row, 1, 17] = float("inf")
    c.attend()
    torch.cuda.synchronize()
    out = _np(c.out)
    assert np.isposinf(out[1, 4:, 17]).all()
    out[1, 4:, 17] = 0
    assert np.isfinite(out).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40, 3000])
def test_a_nan_in_a_key_reaches_its_heads_only(dtype, n):
    c = Cache([n, 333], dtype=dtype)
    c.Kp[int(c.table_h[0, 0]), 0, 1, 5] = float("nan")
    c.attend()
    torch.cuda.synchronize()
    out = _np(c.out)
    assert np.isnan(out[0, 4:]).all() and np.isfinite(out[0, :4]).all() and np.isfinite(out[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_keys_give_the_mean(dtype):
    """Logits that are all the same, however large: the plain mean of the values."""
    c = Cache([513], dtype=dtype, H=4, H_kv=1)
    c.q.fill_(64.0)
    c.q_pos.zero_()
    c.Kp.fill_(1.0)
    c.Vp.copy_(torch.where(torch.isnan(c.Vp), torch.zeros_like(c.Vp), torch.full_like(c.Vp, 3.0)))
    c.attend()
    torch.cuda.synchronize()
    assert (np.abs(_np(c.out) - 3.0) <= 3.0 * (HALF[dtype] + 2.0 ** -13)).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("H,H_kv,P,lens", [(32, 32, 16, [1500, 2600, 0, 3333, 1]), (24, 8, 24, [9000, 7, 8500, 0, 300]), (20, 2, 64, [66000, 300]), (6, 6, 7, [12001, 12000]),
                                           (7, 7, 16, [9000, 9000])])
def test_long_batches(H, H_kv, P, lens, dtype, d):
    """Work for two KV heads in a workgroup (and an odd number of them)."""
    c = Cache(lens, H=H, H_kv=H_kv, P=P, d=d, dtype=dtype, lists=1, holes=[(0, 5, -1)])
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)
    first = c.out.clone()
    c.attend(weights=False)
    torch.cuda.synchronize()
    assert torch.equal(first, c.out)


def test_many_ragged_sequences():
    rng = np.random.default_rng(3)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(2500), 70))]
    c = Cache(lens, H=8, H_kv=2, P=32, lists=2)
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)


def test_more_sequences_than_a_workgroup_has_threads():
    lens = [(37 * b) % 150 for b in range(1024)]
    c = Cache(lens, H=2, H_kv=1, d=64, P=8)
    c.attend()
    torch.cuda.synchronize()
    c.check_attend()


def test_results_repeat_bit_for_bit_and_without_weights_too():
    c = Cache([2500, 33, 900, 4100], H=32, H_kv=8, lists=8)
    w0 = c.weights.clone()
    runs = []
    for _ in range(4):
        c.weights.copy_(w0)
        c.out.fill_(float("nan"))
        c.attend()
        runs.append((c.out.clone(), c.weights.clone()))
    c.out.fill_(float("nan"))
    c.attend(weights=False)
    torch.cuda.synchronize()
    for o, w in runs:
        assert torch.equal(o.view(torch.int16), runs[0][0].view(torch.int16)) and torch.equal(w, runs[0][1])
    assert torch.equal(c.out.view(torch.int16), runs[0][0].view(torch.int16))
    assert torch.equal(c.weights, runs[0][1])


def test_contexts_of_different_groups_side_by_side():
    """What one context needs of a kernel is not taken away by another one's set-up."""
    big, small = Cache([300, 40], H=32, H_kv=2, P=16), Cache([300, 40], H=2, H_kv=2, P=16, seed=1)
    for c in (big, small, big):
        c.out.fill_(float("nan"))
        c.attend()
        torch.cuda.synchronize()
        c.check_attend()


def test_one_context_for_two_caches_and_changing_lengths():
    """Nothing of a call stays in the workspace: other caches, lengths, one KV head or two in a workgroup, on one context."""
    c = Cache([9000, 8000, 3], H=16, H_kv=8, P=16, lists=8)
    full = [t.clone() for t in (c.Kp, c.Vp)]
    for lens in ([9000, 8000, 3], [1, 0, 0], [700, 33, 3], [9000, 8000, 0], [5, 8000, 1]):
        c.lens = lens
        c.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        before = c.weights.clone()
        c.attend()
        torch.cuda.synchronize()
        c.check_attend(before)
        c.Kp, c.Vp = c.Vp, c.Kp
    assert torch.equal(c.Vp.view(torch.int16), full[0].view(torch.int16)) and torch.equal(c.Kp.view(torch.int16), full[1].view(torch.int16))


def test_offsets_past_32_bits():
    """A pool of 5 GiB (2.7e9 elements) whose last pages are the cache's, and pages 1 MiB apart."""
    P, H_kv, d, n_pages = 16, 8, 128, 5200
    stride = 512 * 1024
    pool = torch.empty(n_pages * stride, dtype=torch.bfloat16, device=DEV)
    Kp = pool.as_strided((n_pages, P, H_kv, d), (stride, H_kv * d, d, 1))
    Vp = pool[P * H_kv * d:].as_strided((n_pages, P, H_kv, d), (stride, H_kv * d, d, 1))
    small = Cache([200, 97], H=16, H_kv=H_kv, P=P)
    table = torch.arange(2 * small.mp, dtype=torch.int32, device=DEV).view(2, small.mp) + (n_pages - 2 * small.mp)
    Kp[table.view(-1).long()] = small.Kp[small.table.view(-1).long()]
    Vp[table.view(-1).long()] = small.Vp[small.table.view(-1).long()]
    ctx = binding.Paged(binding.make_paged_desc(2, 16, H_kv, d, P, small.mp, n_pages, "bf16", page_stride=stride), DEV)
    out = torch.empty_like(small.out)
    ctx.attend(small.q, small.q_pos, table, Kp, Vp, small.seq_len, out)
    small.attend()
    torch.cuda.synchronize()
    small.check_attend()
    assert torch.equal(out.view(torch.int16), small.out.view(torch.int16))


# ---- append ---------------------------------------------------------------------------------------------------------------------

def _check_append(c, k_new, v_new, n_tok, n_new, K0, V0, w0, p0):
    K, V = K0.clone(), V0.clone()
    boundK = torch.zeros_like(K0, dtype=torch.float64)
    for b, have in enumerate(c.lens):
        have = max(0, min(have, c.cap))
        n = min(max(0, min(n_new[b], n_tok)), c.cap - have)
        assert int(c.seq_len[b]) == (have + n if n else c.lens[b]), b
        for t in range(n):
            page, row, there = (x[-1] for x in po.slots(c.table_h[b], c.P, have + t + 1, c.n_pages))
            at = int(c.q_pos[b]) + t
            if there:
                x = _np(k_new[b, t])
                K[page, row] = torch.from_numpy(po.rope(x, at, c.theta, c.style))
                pair = np.roll(np.abs(x), c.d // 2, axis=-1) if not c.style else np.abs(x).reshape(c.H_kv, -1, 2)[..., ::-1].reshape(c.H_kv, -1)
                boundK[page, row] = torch.from_numpy(2.0 ** -21 * (np.abs(x) + pair))
                V[page, row] = v_new[b, t].cpu().double()
            if c.lists:
                p0[b, :, have + t], w0[b, :, have + t] = at, 0.0
    got = c.Kp.cpu().double()
    bound = boundK + torch.where(boundK > 0, HALF[c.dtype] * K.abs() * (1 + 2.0 ** -6), 0.0)
    same = torch.isnan(got) & torch.isnan(K)
    assert bool((same | ((got - K).abs() <= bound)).all())
    gv = c.Vp.cpu().double()
    assert bool(((torch.isnan(gv) & torch.isnan(V)) | (gv == V)).all())
    if c.lists:
        assert torch.equal(c.pos.cpu(), p0) and torch.equal(c.weights.cpu(), w0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_tok,H_kv,d,P,style", [(1, 8, 128, 16, 0), (1, 32, 128, 16, 1), (1, 1, 64, 1, 0), (3, 3, 64, 7, 1), (8, 2, 128, 8, 0), (9, 2, 64, 16, 1),
                                                  (150, 4, 128, 24, 0), (333, 1, 128, 64, 0)])
def test_append(dtype, n_tok, H_kv, d, P, style):
    lens = [0, 1, 37, 95, 130]
    c = Cache(lens, H=H_kv, H_kv=H_kv, d=d, P=P, dtype=dtype, lists=H_kv, mp=-(-(130 + n_tok // 2 + 1) // P), style=style, joined=n_tok == 8,
              holes=[(2, 38 // P, -1)] if P > 1 else ())
    c.q_pos.copy_(torch.tensor([0, 5, 1000, 131072, 77], dtype=torch.int32))
    g = torch.Generator().manual_seed(7)
    k_new, v_new = (torch.randn(5, n_tok, H_kv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    K0, V0 = c.Kp.cpu().double(), c.Vp.cpu().double()
    w0, p0 = c.weights.cpu().clone(), c.pos.cpu().clone()
    c.ctx.append(k_new, v_new, c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, n_tok=n_tok, pos=c.pos, weights=c.weights)
    torch.cuda.synchronize()
    _check_append(c, k_new, v_new, n_tok, [n_tok] * 5, K0, V0, w0, p0)


@pytest.mark.parametrize("n_tok", [5, 70])
def test_append_of_different_counts(n_tok):
    """n_new: none, some, all, more than there are, fewer than none; a full cache; lengths outside it."""
    lens = [10, 20, 30, 40, 50, 160, 157, -4]
    c = Cache([max(0, n) for n in lens], H=2, H_kv=2, P=16, lists=1, mp=10)
    c.lens = lens
    c.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
    n_new = [0, 3, n_tok, n_tok + 9, -2, 4, n_tok, 2]
    g = torch.Generator().manual_seed(8)
    k_new, v_new = (torch.randn(8, n_tok, 2, 128, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    K0, V0 = c.Kp.cpu().double(), c.Vp.cpu().double()
    w0, p0 = c.weights.cpu().clone(), c.pos.cpu().clone()
    c.ctx.append(k_new, v_new, c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, n_tok=n_tok, n_new=torch.tensor(n_new, dtype=torch.int32, device=DEV), pos=c.pos,
                 weights=c.weights)
    torch.cuda.synchronize()
    _check_append(c, k_new, v_new, n_tok, n_new, K0, V0, w0, p0)


# ---- eviction -------------------------------------------------------------------------------------------------------------------

def _check_evict(c, n_keep, sink, recent, src=True):
    K0, V0, w0, p0, l0 = c.Kp.clone(), c.Vp.clone(), c.weights.clone(), c.pos.clone(), c.seq_len.clone()
    got_src = torch.full((c.B, c.lists, n_keep), -9, dtype=torch.int32, device=DEV) if src else None
    c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, n_keep, n_sink=sink, n_recent=recent, src=got_src)
    torch.cuda.synchronize()
    K, V, w, p, s = K0.clone(), V0.clone(), w0.clone(), p0.clone(), torch.full((c.B, c.lists, n_keep), -1, dtype=torch.int32)
    w_h, p_h = w0.cpu().numpy(), p0.cpu().numpy()
    for b in range(c.B):
        n = max(0, min(int(l0[b]), c.cap))
        assert int(c.seq_len[b]) == (n_keep if n > n_keep else int(l0[b])), b
        for a in range(c.lists):
            line = po.evict(w_h[b, a, :n], p_h[b, a, :n], int(c.q_pos[b]), n_keep, sink, recent)
            s[b, a, : len(line)] = torch.tensor(line, dtype=torch.int32)
            to = [j for j, x in enumerate(line) if x != j]
            if not to:
                continue
            frm = [line[j] for j in to]
            w[b, a, to], p[b, a, to] = w0[b, a, frm], p0[b, a, frm]
            heads = slice(None) if c.lists == 1 else slice(a, a + 1)
            pt, rt, _ = po.slots(c.table_h[b], c.P, n, c.n_pages)
            for new, old in ((K, K0), (V, V0)):
                new[torch.from_numpy(pt[to]).long().to(DEV), torch.from_numpy(rt[to]).long().to(DEV), heads] = \
                    old[torch.from_numpy(pt[frm]).long().to(DEV), torch.from_numpy(rt[frm]).long().to(DEV), heads]
    bits = (lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32))
    if src:
        assert torch.equal(got_src.cpu(), s)
    assert torch.equal(bits(c.weights), bits(w)) and torch.equal(c.pos, p)
    assert torch.equal(bits(c.Kp), bits(K)) and torch.equal(bits(c.Vp), bits(V))


def _positions(c, seed=5):
    """Positions in any order, with gaps, different in every list; the newest token's is q_pos."""
    rng = np.random.default_rng(seed)
    for b in range(c.B):
        for a in range(c.lists):
            p = np.cumsum(rng.integers(1, 3, c.cap)) - 1
            p = p - p[max(0, min(c.lens[b], c.cap) - 1)] + int(c.q_pos[b])
            n = max(0, min(c.lens[b], c.cap))
            p[:n] = p[:n][rng.permutation(n)] if n else p[:n]
            c.pos[b, a] = torch.from_numpy(p.astype(np.int32)).to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H_kv,d,P,per_head", [(1, 128, 16, False), (4, 128, 16, False), (4, 64, 7, True), (2, 128, 1, True), (3, 64, 64, True), (8, 128, 24, False)])
def test_evict(dtype, H_kv, d, P, per_head):
    lens = [0, 1, 63, 64, 65, 100, 257]
    for n_keep, sink, recent in ((64, 4, 16), (1, 0, 0), (63, 16, 0), (200, 0, 50)):
        c = Cache(lens, H=H_kv, H_kv=H_kv, d=d, P=P, dtype=dtype, lists=H_kv if per_head else 1, joined=True)
        _positions(c)
        _check_evict(c, n_keep, sink, recent)


@pytest.mark.parametrize("n,n_keep", [(4096, 4095), (4097, 1), (5000, 4096), (8192, 4097), (9001, 1003), (9001, 9000), (20000, 15000), (40000, 700), (40000, 39990),
                                      (70000, 35000), (200000, 16384), (1048576, 500000)])
def test_evict_long_lists(n, n_keep):
    c = Cache([n, n - 1, n // 2] if n < 1 << 20 else [n], H=1, H_kv=1, d=64, P=64, lists=1)
    _positions(c)
    _check_evict(c, n_keep, 4, min(64, n_keep // 2), src=n != 20000)


@pytest.mark.parametrize("kind", ["equal", "zero", "ends", "nan", "two", "close", "negative"])
@pytest.mark.parametrize("n,n_keep", [(300, 100), (5000, 4999), (6000, 2500), (9000, 8995), (20000, 9000), (140000, 70000)])
def test_evict_weights_that_are_hard_to_rank(kind, n, n_keep):
    c = Cache([n, n - 7], H=2, H_kv=2, d=64, P=16, lists=2)
    _positions(c)
    w = c.weights
    g = torch.Generator(device=DEV).manual_seed(1)
    r = torch.rand(w.shape, generator=g, device=DEV)
    if kind == "equal":
        w.fill_(1.25)
    elif kind == "zero":
        w.copy_(torch.where(r < 0.5, torch.zeros_like(w), -torch.zeros_like(w)))
    elif kind == "ends":
        vals = torch.tensor([float("inf"), -float("inf"), 3.4028235e38, 1e-45, 0.0, -0.0, 1.1754944e-38], device=DEV)
        w.copy_(vals[(r * 7).long().clamp(max=6)])
    elif kind == "nan":
        w.copy_(torch.where(r < 0.7, torch.full_like(w, float("nan")), r))
        w.view(torch.int32)[0, 0, ::3] = -4194303   # a NaN with its sign bit set
    elif kind == "two":
        w.copy_((r < 0.3).float())
    elif kind == "close":
        w.copy_(1.0 + (r * 50).floor() * 2.0 ** -23)
    else:
        w.copy_(r - 0.5)
    _check_evict(c, n_keep, 2, 10)


def test_evict_the_same_context_again_and_shorter():
    """Nothing of an eviction stays in the workspace: long lists, then short ones, then long ones again on one context."""
    c = Cache([30000, 9000, 2000], H=2, H_kv=2, d=64, P=16, lists=2)
    for lens, n_keep in (([30000, 9000, 2000], 1000), ([900, 1001, 5], 999), ([30000, 29999, 1001], 1000), ([30000, 30000, 30000], 29990), ([0, 1, 1], 1)):
        c.lens = lens
        c.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        _positions(c, seed=n_keep)
        c.weights.copy_(torch.rand(c.weights.shape, generator=torch.Generator().manual_seed(n_keep)))
        _check_evict(c, n_keep, 3, 20)


def test_evict_more_protected_than_stay_and_extreme_positions():
    c = Cache([500, 500], H=2, H_kv=2, d=64, P=16, lists=2)
    c.q_pos.copy_(torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
    c.pos[0, 0].fill_(2 ** 31 - 1)
    c.pos[0, 1].fill_(-2 ** 31)
    _check_evict(c, 100, 3, 2 ** 31 - 1)
    c.seq_len.fill_(500)
    _check_evict(c, 100, 0, 0)


def test_evict_leaves_rows_of_missing_pages_alone():
    """Slots on pages outside the pool: neither read nor written; the lists and the length as always."""
    c = Cache([100], H=1, H_kv=1, d=64, P=10, lists=1, holes=[(0, 1, -1), (0, 8, 2 ** 31 - 1)])
    _positions(c)
    K0 = c.Kp.clone()
    src = torch.empty((1, 1, 40), dtype=torch.int32, device=DEV)
    w = c.weights.cpu().numpy()[0, 0]
    line = po.evict(w[:100], c.pos.cpu().numpy()[0, 0, :100], int(c.q_pos[0]), 40, 0, 0)
    c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, 40, src=src)
    torch.cuda.synchronize()
    assert src.cpu().view(-1).tolist() == line and int(c.seq_len[0]) == 40
    page, row, there = po.slots(c.table_h[0], 10, 100, c.n_pages)
    K = K0.clone()
    for j, x in enumerate(line):
        if x != j and there[j] and there[x]:
            K[int(page[j]), int(row[j])] = K0[int(page[x]), int(row[x])]
    assert torch.equal(c.Kp.view(torch.int16), K.view(torch.int16))


# ---- together -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,H,H_kv,d,P,per_head,style", [("bf16", 8, 2, 128, 16, True, 0), ("f32", 4, 4, 64, 7, True, 1), ("bf16", 8, 2, 64, 5, False, 1)])
def test_a_run_of_steps_with_eviction(dtype, H, H_kv, d, P, per_head, style):
    """Prompts enter, then steps of append, attention with weights and eviction to a bound, each held to the oracle on the cache as it is
    on the device; the state behind it is what the steps have to leave."""
    B, bound = 3, 40
    lists = H_kv if per_head else 1
    c = Cache([0, 0, 0], H=H, H_kv=H_kv, d=d, P=P, dtype=dtype, lists=lists, mp=-(-(bound + 12) // P), style=style)
    g = torch.Generator().manual_seed(11)
    c.q_pos.zero_()
    n_new = torch.tensor([12, 3, 0], dtype=torch.int32, device=DEV)
    k, v = (torch.randn(B, 12, H_kv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    c.ctx.append(k, v, c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, n_tok=12, n_new=n_new, pos=c.pos, weights=c.weights)
    c.q_pos += n_new
    total = [12, 3, 0]
    for step in range(60):
        k, v = (torch.randn(B, 1, H_kv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
        c.q.copy_(1.5 * torch.randn(B, H, d, generator=g))
        c.ctx.append(k, v, c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, pos=c.pos, weights=c.weights)
        torch.cuda.synchronize()
        total = [t + 1 for t in total]
        c.lens = [min(t, bound + 1) for t in total]
        assert c.seq_len.tolist() == c.lens
        before = c.weights.clone()
        c.attend()
        torch.cuda.synchronize()
        if step % 7 == 0 or step > 55:
            c.check_attend(before)
        _check_evict(c, bound, 2, 8, src=step % 2 == 0)
        c.q_pos += 1
    pos = c.pos.cpu().numpy()
    for b in range(B):
        n = min(total[b], bound)
        for a in range(lists):
            have = set(pos[b, a, :n].tolist())
            assert len(have) == n and {0, 1} <= have and set(range(total[b] - 8, total[b])) <= have


def test_another_stream_and_a_captured_step():
    """A step on a side stream, then captured into a graph and replayed with eager work between the replays: every replay leaves what
    the eager calls leave on the same state."""
    def make():
        c = Cache([600, 90], H=8, H_kv=2, P=16, lists=2, mp=45)
        _positions(c)
        c.k = torch.randn(2, 1, 2, 128, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
        return c

    def step(c):
        c.ctx.append(c.k, c.k, c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, pos=c.pos, weights=c.weights)
        c.attend()
        c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, 550, n_sink=4, n_recent=32)
        c.q_pos += 1

    def state(c):
        return [t.clone() for t in (c.out, c.Kp, c.Vp, c.weights, c.pos, c.seq_len)]

    a, b = make(), make()
    want = []
    for _ in range(6):
        step(a)
        torch.cuda.synchronize()
        want.append(state(a))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b)
    side.synchronize()
    got = [state(b)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    scratch = torch.zeros(1 << 20, device=DEV)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        got.append(state(b))
        scratch.add_(1.0).sum().item()
    for k, (x, y) in enumerate(zip(want, got)):
        for t, (p, q) in enumerate(zip(x, y)):
            bits = torch.int16 if p.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(p.contiguous().view(bits), q.contiguous().view(bits)), (k, t)


def test_binding_refuses_what_does_not_fit():
    c = Cache([20, 30], lists=2)
    bad = [dict(q=c.q.float()), dict(q=c.q[:1]), dict(q_pos=c.q_pos.long()), dict(table=c.table.cpu()), dict(Kp=c.Kp[:-1]), dict(Vp=c.Vp.transpose(1, 2)),
           dict(seq_len=c.seq_len[:1]), dict(weights=c.weights[:, :1]), dict(out=c.out.transpose(0, 1))]
    for kw in bad:
        a = dict(q=c.q, q_pos=c.q_pos, table=c.table, Kp=c.Kp, Vp=c.Vp, seq_len=c.seq_len, out=c.out, weights=c.weights)
        a.update(kw)
        with pytest.raises(binding.SalsError):
            c.ctx.attend(**a)
    with pytest.raises(binding.SalsError):
        c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, 8, src=torch.zeros((2, 2, 9), dtype=torch.int32, device=DEV))
    with pytest.raises(binding.SalsError):
        c.ctx.append(c.q[:, :2], c.q[:, :2], c.q_pos, c.table, c.Kp, c.Vp, c.seq_len)   # (lists wanted)
    c.ctx.close()
    with pytest.raises(binding.SalsError):
        c.attend()


def test_binding_refuses_counts_of_more_than_32_bits():
    c = Cache([20, 30], lists=2)
    state = lambda: [t.clone().contiguous().view(torch.uint8) for t in (c.seq_len, c.pos, c.weights, c.Kp)]   # (as bits: the pools hold NaN)
    before = state()
    for counts in ((2 ** 32 + 5, 0, 0), (8, 2 ** 32, 0), (8, 0, 2 ** 31), (-1, 0, 0), (8, -2 ** 32, 0)):
        with pytest.raises(binding.SalsError):
            c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, *counts)
    for n_tok in (0, -1, 2 ** 32 + 1):
        with pytest.raises(binding.SalsError):
            c.ctx.append(c.q[:, :2], c.q[:, :2], c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, n_tok=n_tok, pos=c.pos, weights=c.weights)
    assert all(torch.equal(x, y) for x, y in zip(before, state()))
