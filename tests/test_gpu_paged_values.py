"""GPU tests of what the paged cache's attention makes of single values: weights in full fp32, infinite and undefined keys and values.

eps = 2^-24 is half a step of fp32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from oracle import paged_oracle as po  # noqa: E402
from test_gpu_paged import DEV, EPS, HALF, Cache, _np  # noqa: E402


def _small(keys, values, d, dtype, H=1, H_kv=1, P=16):
    """Slots whose keys are `keys` in channel 0 and zero elsewhere, values `values` in all channels; a query of ones in channel 0 at position
    0: logit j is keys[j] / sqrt(d)."""
    n = len(keys)
    c = Cache([n], H=H, H_kv=H_kv, d=d, P=P, dtype=dtype)
    K = torch.zeros(n, H_kv, d)
    K[:, :, 0] = torch.tensor(keys)[:, None]
    V = torch.as_tensor(values, dtype=torch.float32)[:, None, None].expand(n, H_kv, d)
    page, row, _ = po.slots(c.table_h[0], P, n, c.n_pages)
    at = torch.from_numpy(page).long().to(DEV), torch.from_numpy(row).long().to(DEV)
    c.Kp[at] = K.to(c.Kp.dtype).to(DEV)
    c.Vp[at] = V.to(c.Vp.dtype).to(DEV)
    c.q.zero_()
    c.q[:, :, 0] = 1.0
    c.q_pos.zero_()
    return c


# exp(k / 8) of these needs more than 16 bits: a head of 8 and a rounded remainder of 8 are off by 0.57 to 0.95 2^-16 of it, too much ...
TOO_MUCH = [-1.6796875, -4.03125, -3.109375, -2.03125, -3.375, -3.734375, -2.875, -5.25, -3.875, -5.5, -5.375]
# ... and too little
TOO_LITTLE = [-3.78125, -4.40625, -4.90625, -4.28125, -3.421875, -2.96875, -2.6875, -4.625, -3.09375, -2.359375, -3.25]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("copies", [1, 20])
def test_weights_enter_the_sum_in_full(dtype, copies):
    """Values +1 where 16 bits of a weight are too much and -1 where they are too little, and two values that cancel the sum to 2^-17 of
    it, so that the output's own rounding hides nothing.

    Bound, relative to sum p |v|: a logit takes a rounding of the scale, one of the scaled query and two of its three products with the key, of
    at most 5.5 / 8 log2(e) = 1: 4 eps ln 2 of the weight; exp2 2 eps; the sum, of three products a slot, one rounding each, 3 n eps at
    most for the n slots of a wave (and n = 23 in a block of 32) and 10 for joining the waves."""
    keys = (TOO_MUCH + TOO_LITTLE) * copies + [0.0, 0.0]
    sign = np.array(([1.0] * len(TOO_MUCH) + [-1.0] * len(TOO_LITTLE)) * copies)
    p = np.exp(np.array(keys) / 8.0)
    first = -float(torch.tensor(np.sum(p[:-2] * sign)).to(torch.bfloat16))
    second = -float(torch.tensor(np.sum(p[:-2] * sign) + first).to(torch.bfloat16))
    v = np.concatenate([sign, [first, second]])
    c = _small(keys, v, 64, dtype)
    c.attend()
    torch.cuda.synchronize()
    want, size = np.sum(p * v) / p.sum(), np.sum(p * np.abs(v)) / p.sum()
    assert abs(want) < 2.0 ** -16 * size     # (the premise)
    bound = (4 * np.log(2) + 2 + 3 * min(len(keys), 32) + -(-len(keys) // 16) + 10) * EPS * size + HALF[dtype] * abs(want)
    err = np.abs(_np(c.out)[0, 0] - want)
    print(f"    error {err.max() / size * 2 ** 16:.4f} 2^-16 of the sum, bound {bound / size * 2 ** 16:.4f}", flush=True)
    assert (err <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [44, 300, 4096, 30000])
def test_values_of_weight_zero_that_are_not_finite_show(dtype, n):
    """A value row far below the largest logit has weight zero in fp32; zero times NaN or infinity is a NaN, however the sequence is spread
    over waves and workgroups."""
    keys, values = [-2400.0] * 40 + [0.0] * (n - 40), [1.0] * n      # (logits -300 and 0)
    c = _small(keys, values, 64, dtype)
    page, row, _ = po.slots(c.table_h[0], c.P, n, c.n_pages)
    c.Vp[int(page[5]), int(row[5]), 0, 3] = float("nan")
    c.Vp[int(page[39]), int(row[39]), 0, 7] = float("inf")
    c.attend()
    torch.cuda.synchronize()
    out = _np(c.out)[0, 0]
    assert np.isnan(out[[3, 7]]).all()
    # (a mean of ones: the rounding of n terms and that of the result)
    assert (np.abs(np.delete(out, [3, 7]) - 1.0) <= HALF[dtype] + (64 + n / 32) * EPS).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [3, 700])
def test_an_infinite_key_is_a_logit_like_others(dtype, d, n):
    """A key with an infinity against a query of the other sign in that channel: logit -infinity, weight zero; of the same sign: NaN."""
    c = Cache([n, 90], H=6, H_kv=2, d=d, dtype=dtype, lists=2)
    c.q_pos.zero_()
    c.q[0, :, 9] = torch.tensor([0.71875, 1.0, -0.34375, 0.001, 2.0, 3.0], dtype=c.q.dtype, device=DEV)
    page, row, _ = po.slots(c.table_h[0], c.P, n, c.n_pages)
    at = int(page[1]), int(row[1])
    c.Kp[at[0], at[1], :, 9] = -float("inf")
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    out, added = _np(c.out), _np(c.weights - before)[0]
    assert np.isnan(out[0, 2]).all()                       # (its logit is +infinity)
    assert np.isfinite(np.delete(out[0], 2, axis=0)).all() and np.isfinite(out[1]).all()
    assert added[1, 1] == 0.0 and np.isfinite(added[1]).all() and np.isnan(added[0, :n]).all()
    # the others' rows as if that slot were not there
    K, there = c.rows(c.Kp, 0, n)
    V, _ = c.rows(c.Vp, 0, n)
    K[1], there[1] = 0.0, False
    want, p = po.attend(_np(c.q[0]), 0, K, V, there, c.theta)
    size = np.einsum("hn,nhc->hc", p, np.repeat(np.abs(V), 3, axis=1))
    logit = np.einsum("hc,nhc->hn", np.abs(_np(c.q[0])), np.repeat(np.abs(K), 3, axis=1)).max(axis=1) / np.sqrt(d)
    # (a logit: d + 16 roundings of at most the sum of its products; weights twice that; the sum of n terms; the output's rounding)
    bound = HALF[dtype] * np.abs(want) * (1 + 2.0 ** -6) + ((2 * (d + 16) * logit + 2 * (64 + n / 32)) * EPS + 2.0 ** -19)[:, None] * size
    for h in (0, 1, 3, 4, 5):
        assert (np.abs(out[0, h] - want[h]) <= bound[h]).all(), h


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_whose_logits_are_all_minus_infinity_is_zero(dtype):
    c = _small([-float("inf")] * 40, [1.0] * 40, 64, dtype)
    c.attend()
    torch.cuda.synchronize()
    assert not _np(c.out).any()


@pytest.mark.parametrize("lists", [1, 3])
def test_an_eviction_of_a_sequence_with_missing_pages_and_attention_behind_it(lists):
    """What the header says of it: entries move by rank alone; rows only between slots with pages.  Attention behind it gives the slots
    without pages no weight and takes the others' rows as they lie there."""
    c = Cache([120], H=6, H_kv=3, d=64, P=10, lists=lists, holes=[(0, 1, -1), (0, 8, -1)])   # slots 10 .. 19 and 80 .. 89
    keep = 50
    c.q_pos.fill_(119)
    c.pos.copy_(torch.arange(120, dtype=torch.int32, device=DEV).expand(1, lists, 120))
    w = torch.rand(1, lists, 120, generator=torch.Generator().manual_seed(9)) + 0.5
    w[..., 0:30] = 0.001         # free slots, 10 .. 19 without pages; kept ones behind move into them, 80 .. 89 among these
    w[..., 60:90] = 5.0
    c.weights.copy_(w)
    K0, V0, page, row, there = c.Kp.clone(), c.Vp.clone(), *po.slots(c.table_h[0], 10, 120, c.n_pages)
    src = torch.empty((1, lists, keep), dtype=torch.int32, device=DEV)
    c.ctx.evict(c.q_pos, c.table, c.Kp, c.Vp, c.seq_len, c.pos, c.weights, keep, src=src)
    torch.cuda.synchronize()
    assert c.seq_len.tolist() == [keep]
    lost = stale = 0
    for a in range(lists):
        line = po.evict(w[0, a].numpy(), np.arange(120), 119, keep, 0, 0)
        assert src[0, a].tolist() == line == c.pos[0, a, :keep].tolist()
        assert torch.equal(c.weights[0, a, :keep].cpu(), w[0, a, line])
        heads = slice(None) if lists == 1 else slice(a, a + 1)
        for j, x in enumerate(line):
            if there[j]:
                frm = x if there[x] else j
                for new, old in ((c.Kp, K0), (c.Vp, V0)):
                    assert torch.equal(new[int(page[j]), int(row[j]), heads], old[int(page[frm]), int(row[frm]), heads])
            lost += bool(not there[j] and there[x])
            stale += bool(there[j] and not there[x])
    assert lost and stale        # (the premise)
    c.lens = [keep]
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    c.check_attend(before)
    assert torch.equal(c.weights[..., 10:20], before[..., 10:20])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lists", [1, 2])
def test_slots_without_a_page_get_no_weight_beside_a_nan(dtype, lists):
    c = Cache([200, 90], dtype=dtype, lists=lists, holes=[(0, 1, -1), (0, 12, 2 ** 31 - 1)])   # slots 16 .. 31 and 192 .. 199
    c.Kp[int(c.table_h[0, 0]), 3, 1, 5] = float("nan")
    before = c.weights.clone()
    c.attend()
    torch.cuda.synchronize()
    w, was = _np(c.weights), _np(before)
    for gone in (slice(16, 32), slice(192, None)):
        assert np.array_equal(w[0, :, gone], was[0, :, gone])
    assert np.isnan(w[0, -1, :16]).all() and np.isnan(w[0, -1, 32:192]).all() and np.isfinite(w[1]).all()
