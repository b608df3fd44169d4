"""GPU tests of the eviction where there are many lists, and of all three calls on pools past 2^32 elements."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from oracle import paged_oracle as po  # noqa: E402
from paper_2510_24273_amd import binding  # noqa: E402
from test_gpu_paged import DEV, Cache, _positions  # noqa: E402


def _line(w, pos, position, keep, sink, recent):
    """po.evict for weights without NaN, by one sort."""
    n = len(w)
    if n <= keep:
        return np.arange(n)
    protected = (pos < sink) | (pos.astype(np.int64) > position - recent)
    order = np.lexsort((np.arange(n), np.where(protected, 0.0, -(w.astype(np.float64) + 0.0)), ~protected))
    kept = np.zeros(n, bool)
    kept[order[:keep]] = True
    line = np.arange(keep)
    line[~kept[:keep]] = keep + np.flatnonzero(kept[keep:])
    return line


@pytest.mark.parametrize("B,H_kv,lists", [(64, 1, 1), (8, 8, 8), (65, 2, 1)])
@pytest.mark.parametrize("cap,P,gone,kind", [(16387, 7, 1, "random"), (16387, 7, 9, "ties"), (20000, 25, 8, "random"), (20000, 25, 9999, "ties"),
                                             (32768, 64, 1, "ties"), (32768, 64, 8, "random"), (32768, 64, 16000, "random"), (33000, 8, 9, "random"),
                                             (33000, 8, 22000, "ties")])
def test_many_long_lists(B, H_kv, lists, cap, P, gone, kind):
    """Tables of 16385 to 32768 slots with 64 lists and more are a workgroup's each, longer ones are in chunks; the sequences are as long
    as the table, a little and far shorter, and no longer than what is kept."""
    print(f"[case] B={B} H_kv={H_kv} lists={lists} cap={cap} P={P} gone={gone} {kind}", flush=True)
    d, mp, keep = 64, cap // P, cap - gone
    g = torch.Generator(device=DEV).manual_seed(cap + gone)
    n_pages = B * mp + 2
    Kp, Vp = (torch.randint(-2 ** 15, 2 ** 15, (n_pages, P, H_kv, d), generator=g, device=DEV, dtype=torch.int16) for _ in range(2))
    table = torch.randperm(n_pages, generator=g, device=DEV)[: B * mp].to(torch.int32).view(B, mp).contiguous()
    lens = [cap - (0, 0, 1, 5, gone // 2, 3 * gone, cap - keep)[b % 7] for b in range(B)]
    lens = [max(0, n) for n in lens]
    weights = torch.rand(B, lists, cap, generator=g, device=DEV)
    if kind == "ties":
        weights = torch.floor(weights * 3)
    pos = torch.stack([torch.randperm(2 * cap, generator=g, device=DEV)[:cap] for _ in range(B * lists)]).view(B, lists, cap).to(torch.int32)
    q_pos = torch.full((B,), 2 * cap - 1, dtype=torch.int32, device=DEV)
    seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ctx = binding.Paged(binding.make_paged_desc(B, H_kv, H_kv, d, P, mp, n_pages, "bf16", weight_heads=lists), DEV)
    src = torch.full((B, lists, keep), -9, dtype=torch.int32, device=DEV)
    K, V, w, p = Kp.clone(), Vp.clone(), weights.clone(), pos.clone()
    ctx.evict(q_pos, table, Kp.view(torch.bfloat16), Vp.view(torch.bfloat16), seq_len, pos, weights, keep, n_sink=16, n_recent=100, src=src)
    torch.cuda.synchronize()
    w_h, p_h, want = w.cpu().numpy(), p.cpu().numpy(), np.full((B, lists, keep), -1, np.int32)
    at = torch.arange(cap, device=DEV)
    K0, V0, w0, p0 = K.clone(), V.clone(), w.clone(), p.clone()
    for b, n in enumerate(lens):
        page, row = table[b].long()[at // P], at % P
        for a in range(lists):
            line = _line(w_h[b, a, :n], p_h[b, a, :n], 2 * cap - 1, keep, 16, 100)
            want[b, a, : len(line)] = line
            to = np.flatnonzero(line != np.arange(len(line)))
            frm, to = torch.from_numpy(line[to]).to(DEV), torch.from_numpy(to).to(DEV)
            heads = slice(None) if lists == 1 else a
            K[page[to], row[to], heads], V[page[to], row[to], heads] = K0[page[frm], row[frm], heads], V0[page[frm], row[frm], heads]
            w[b, a, to], p[b, a, to] = w0[b, a, frm], p0[b, a, frm]
    assert seq_len.tolist() == [min(n, keep) for n in lens]
    assert np.array_equal(src.cpu().numpy(), want)
    assert torch.equal(weights, w) and torch.equal(pos, p) and torch.equal(Kp, K) and torch.equal(Vp, V)
    if B == 8:   # (the sort against the oracle)
        n = lens[1]
        assert want[1, 3].tolist() == po.evict(w_h[1, 3, :n], p_h[1, 3, :n], 2 * cap - 1, keep, 16, 100)


@pytest.mark.parametrize("lists", [1, 8])
def test_offsets_past_32_bits_of_elements(lists):
    """Pages 2 MiB apart in a pool of 4.4e9 elements, of which the cache has the last: append, attend and evict leave what they leave in a
    small pool."""
    P, H_kv, d, n_pages, stride = 16, 8, 128, 4300, 1 << 20
    pool = torch.empty(n_pages * stride, dtype=torch.bfloat16, device=DEV)
    Kp = pool.as_strided((n_pages, P, H_kv, d), (stride, H_kv * d, d, 1))
    Vp = pool[P * H_kv * d:].as_strided((n_pages, P, H_kv, d), (stride, H_kv * d, d, 1))
    small = Cache([200, 97], H=16, H_kv=H_kv, P=P, lists=lists, mp=14)
    _positions(small)
    first = n_pages - 2 * small.mp
    assert first * stride > 2 ** 32
    table = torch.arange(2 * small.mp, dtype=torch.int32, device=DEV).view(2, small.mp) + first
    used, at = small.table.view(-1).long(), table.view(-1).long()
    Kp[at], Vp[at] = small.Kp[used], small.Vp[used]
    ctx = binding.Paged(binding.make_paged_desc(2, 16, H_kv, d, P, small.mp, n_pages, "bf16", weight_heads=lists, page_stride=stride), DEV)
    pos, weights, seq_len, out = small.pos.clone(), small.weights.clone(), small.seq_len.clone(), torch.empty_like(small.out)
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(2, 5, H_kv, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    bits = lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)

    def same():
        torch.cuda.synchronize()
        for x, y in ((Kp[at], small.Kp[used]), (Vp[at], small.Vp[used]), (pos, small.pos), (weights, small.weights), (seq_len, small.seq_len)):
            assert torch.equal(bits(x), bits(y))

    q_pos = small.q_pos
    same()
    ctx.append(k, v, q_pos, table, Kp, Vp, seq_len, n_tok=5, pos=pos, weights=weights)
    small.ctx.append(k, v, q_pos, small.table, small.Kp, small.Vp, small.seq_len, n_tok=5, pos=small.pos, weights=small.weights)
    same()
    assert seq_len.tolist() == [205, 102]
    small.lens = [205, 102]
    ctx.attend(small.q, q_pos, table, Kp, Vp, seq_len, out, weights=weights)
    small.attend()
    same()
    small.check_attend()
    assert torch.equal(bits(out), bits(small.out))
    ctx.evict(q_pos, table, Kp, Vp, seq_len, pos, weights, 90, n_sink=4, n_recent=10)
    small.ctx.evict(q_pos, small.table, small.Kp, small.Vp, small.seq_len, small.pos, small.weights, 90, n_sink=4, n_recent=10)
    same()
    assert seq_len.tolist() == [90, 90]
