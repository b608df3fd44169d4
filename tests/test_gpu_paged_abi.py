"""GPU tests of the paged cache's C entry points on a context that is ready: every argument that is refused comes back as the error that
the header names, with nothing enqueued, beside the same call with the argument in order."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2510_24273_amd import binding  # noqa: E402
from test_gpu_paged import DEV, Cache  # noqa: E402

OK, BAD = binding.SALS_OK, binding.SALS_ERR_INVALID_ARG


def _calls(c):
    """name -> (entry point, arguments behind the context, their names)."""
    lib, h = binding._lib, c.ctx._h
    p = lambda t: None if t is None else t.data_ptr()
    st = torch.cuda.current_stream().cuda_stream
    c.k_new, c.n_new = torch.zeros(c.B, 3, c.H_kv, c.d, dtype=c.q.dtype, device=DEV), torch.zeros(c.B, dtype=torch.int32, device=DEV)
    c.src = torch.zeros(c.B, max(1, c.lists), 8, dtype=torch.int32, device=DEV)
    cache = [p(c.q_pos), p(c.table), p(c.Kp), p(c.Vp), p(c.seq_len)]
    return {
        "append": (lib.sals_paged_append, h, [p(c.k_new), p(c.k_new)] + cache + [p(c.n_new), 3, p(c.pos), p(c.weights), st],
                   "k_new v_new q_pos table Kp Vp seq_len n_new n_tok pos weights stream".split()),
        "attend": (lib.sals_paged_attend, h, [p(c.q)] + cache + [p(c.weights), p(c.out), st], "q q_pos table Kp Vp seq_len weights out stream".split()),
        "evict": (lib.sals_paged_evict, h, cache + [p(c.pos), p(c.weights), 8, 1, 2, p(c.src), st],
                  "q_pos table Kp Vp seq_len pos weights n_keep n_sink n_recent src stream".split()),
    }


# what each refuses, beside null for every pointer but those named as optional, and misaligned rows
BAD_COUNTS = {"append": [("n_tok", 0), ("n_tok", -1), ("n_tok", (1 << 20) + 1), ("n_tok", -2 ** 31)],
              "attend": [],
              "evict": [("n_keep", 0), ("n_keep", -5), ("n_keep", 65), ("n_keep", 2 ** 31 - 1), ("n_sink", -1), ("n_recent", -1)]}
ALIGNED = {"append": ["k_new", "v_new", "Kp", "Vp", "pos", "weights"], "attend": ["q", "Kp", "Vp", "weights", "out"], "evict": ["Kp", "Vp", "pos", "weights"]}
OPTIONAL = {"append": ["n_new"], "attend": ["weights"], "evict": ["src"]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["append", "attend", "evict"])
@pytest.mark.parametrize("lists", [0, 1, 2])
def test_refusals_of_a_context_that_is_ready(name, lists, dtype):
    c = Cache([8, 5], H=4, H_kv=2, d=64, P=16, mp=4, dtype=dtype, lists=lists)
    fn, h, args, names = _calls(c)[name]
    held = [t for t in (c.Kp, c.Vp, c.seq_len, c.pos, c.weights, c.out, c.src) if t is not None]
    bits = lambda: [t.clone().contiguous().view(torch.uint8) for t in held]
    before = bits()
    given = dict(zip(names, args))
    spare = c.k_new.data_ptr()   # (never read or written: the calls below are refused)
    call = lambda **kw: fn(h, *[{**given, **kw}[n] for n in names])
    refused = [dict([(n, v)]) for n, v in BAD_COUNTS[name]]
    for n in names:
        if n in OPTIONAL[name] or n.startswith("n_") or n == "stream" or given[n] is None:
            continue
        refused.append({n: None})
    refused += [{n: given[n] + 8} for n in ALIGNED[name] if given[n] is not None]
    if lists == 0:
        refused += [{n: spare} for n in ("pos", "weights") if n in names]
        if name == "evict":
            refused += [dict(pos=spare, weights=spare)]
    for kw in refused:
        assert call(**kw) == BAD, (name, kw)
        assert fn(None, *[{**given, **kw}[n] for n in names]) == BAD
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, bits()))
    # in order: taken (an eviction needs lists)
    assert call() == (BAD if name == "evict" and lists == 0 else OK)
    for n in OPTIONAL[name]:
        if not (name == "evict" and lists == 0):
            assert call(**{n: None}) == OK, n
    if name == "evict" and lists:
        assert call(n_keep=64, src=None) == OK and call(n_sink=2 ** 31 - 1, n_recent=2 ** 31 - 1) == OK
    torch.cuda.synchronize()


def test_a_context_is_not_ready_before_it_is_prepared():
    """The same call on a context of the same descriptor and workspace size: refused until sals_paged_prepare has returned."""
    c = Cache([8, 5], H=4, H_kv=2, d=64, P=16, mp=4)
    lib, h = binding._lib, ctypes.c_void_p()
    ws = torch.empty(binding.paged_workspace_bytes(c.ctx.desc), dtype=torch.uint8, device=DEV)
    assert lib.sals_paged_create(ctypes.byref(c.ctx.desc), ws.data_ptr(), ws.numel(), ctypes.byref(h)) == OK
    fn, _, args, _ = _calls(c)["attend"]
    assert fn(h, *args) == BAD
    assert lib.sals_paged_prepare(h, args[-1]) == OK
    assert fn(h, *args) == OK
    torch.cuda.synchronize()
    lib.sals_paged_destroy(h)
    c.check_attend()
