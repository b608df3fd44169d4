"""Host-side checks of the paged cache's entry points (no GPU): descriptors, workspace and arguments are refused before anything
reaches a device."""
import ctypes
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def sb():
    from paper_2510_24273_amd import build
    if build.is_stale():
        build.build()
    from paper_2510_24273_amd import binding
    return binding


def _desc(sb, **kw):
    base = dict(B=2, H_q=32, H_kv=8, d=128, page_size=16, max_pages=100, n_pages=300, dtype="bf16")
    base.update(kw)
    return sb.make_paged_desc(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), 1), (dict(H_kv=5), 1), (dict(H_kv=0), 1), (dict(page_size=0), 1), (dict(max_pages=0), 1), (dict(n_pages=0), 1), (dict(n_pages=-1), 1),
    (dict(weight_heads=2), 1), (dict(weight_heads=-1), 1), (dict(rope_theta=0.0), 1), (dict(rope_theta=float("inf")), 1), (dict(rope_style=2), 1),
    (dict(page_stride=16 * 8 * 128 - 8), 1), (dict(page_stride=16 * 8 * 128 + 4), 1), (dict(page_stride=-8), 1), (dict(d=3), 1),
    (dict(d=96), 2), (dict(d=256), 2), (dict(B=1025), 2), (dict(H_q=2048), 2), (dict(page_size=2049), 2), (dict(max_pages=65537), 2),
    (dict(B=1024, H_q=64, H_kv=64, weight_heads=64), 2), (dict(page_stride=1 << 50), 2)])
def test_descriptors_that_are_refused(sb, kw, code):
    with pytest.raises(sb.SalsError) as e:
        sb.paged_workspace_bytes(_desc(sb, **kw))
    assert e.value.code == code


def test_descriptors_that_are_taken(sb):
    n = sb.paged_workspace_bytes(_desc(sb))
    assert n > 0 and n % 256 == 0
    for kw in (dict(d=64), dict(dtype="f32"), dict(page_size=1, max_pages=1 << 20), dict(page_size=2048, max_pages=512), dict(page_size=7),
               dict(B=1024), dict(H_q=1024, H_kv=1), dict(H_q=64, H_kv=64), dict(page_stride=2 * 16 * 8 * 128), dict(n_pages=2 ** 31 - 1)):
        assert sb.paged_workspace_bytes(_desc(sb, **kw)) > 0, kw
    # the logits of a step come on top where weights are added up
    for lists in (1, 8):
        assert sb.paged_workspace_bytes(_desc(sb, weight_heads=lists)) >= n + 2 * 32 * 1600 * 4
    assert sb._lib.sals_paged_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == sb.SALS_ERR_INVALID_ARG
    assert sb._lib.sals_paged_workspace_bytes(ctypes.byref(_desc(sb)), None) == sb.SALS_ERR_INVALID_ARG


def test_create_checks_its_workspace(sb):
    lib, d, h = sb._lib, _desc(sb), ctypes.c_void_p()
    n, at = sb.paged_workspace_bytes(d), 1 << 20
    assert lib.sals_paged_create(ctypes.byref(d), None, n, ctypes.byref(h)) == sb.SALS_ERR_WORKSPACE
    assert lib.sals_paged_create(ctypes.byref(d), at + 16, n, ctypes.byref(h)) == sb.SALS_ERR_WORKSPACE
    assert lib.sals_paged_create(ctypes.byref(d), at, n - 1, ctypes.byref(h)) == sb.SALS_ERR_WORKSPACE
    assert lib.sals_paged_create(ctypes.byref(d), at, n, None) == sb.SALS_ERR_INVALID_ARG
    assert lib.sals_paged_create(None, at, n, ctypes.byref(h)) == sb.SALS_ERR_INVALID_ARG
    assert lib.sals_paged_create(ctypes.byref(d), at, n, ctypes.byref(h)) == sb.SALS_OK and h.value
    # not prepared: refused
    ok = 1 << 20
    assert lib.sals_paged_attend(h, ok, ok, ok, ok, ok, ok, None, ok, None) == sb.SALS_ERR_INVALID_ARG
    assert lib.sals_paged_append(h, ok, ok, ok, ok, ok, ok, ok, None, 1, None, None, None) == sb.SALS_ERR_INVALID_ARG
    assert lib.sals_paged_prepare(None, None) == sb.SALS_ERR_INVALID_ARG
    lib.sals_paged_destroy(h)
    lib.sals_paged_destroy(None)


# The argument checks behind `prepared`: a child process whose library is told that the context is ready (prepare needs a device).
_ARGS = """
import ctypes, sys
from paper_2510_24273_amd import binding as b
lib, ok = b._lib, 1 << 20
def ctx(**kw):
    d = b.make_paged_desc(**dict(dict(B=2, H_q=32, H_kv=8, d=128, page_size=16, max_pages=100, n_pages=300, dtype="bf16"), **kw))
    h = ctypes.c_void_p()
    assert lib.sals_paged_create(ctypes.byref(d), ok, b.paged_workspace_bytes(d), ctypes.byref(h)) == 0
    return h
bad = []
def refused(what, st, code=1):
    if st != code: bad.append((what, st))
for lists in (0, 8):
    h = ctx(weight_heads=lists)
    att = [ok, ok, ok, ok, ok, ok, ok if lists else None, ok]
    for i in range(8):
        if i == 6: continue
        refused(("attend null", i), lib.sals_paged_attend(h, *att[:i], None, *att[i + 1:], None))
    refused("attend misaligned", lib.sals_paged_attend(h, ok + 8, *att[1:], None))
    app = [ok, ok, ok, ok, ok, ok, ok, None, 1, ok if lists else None, ok if lists else None]
    for i in range(7):
        refused(("append null", i), lib.sals_paged_append(h, *app[:i], None, *app[i + 1:], None))
    for n in (0, -1, (1 << 20) + 1):
        refused(("append n_tok", n), lib.sals_paged_append(h, *app[:8], n, *app[9:], None))
    refused("append lists", lib.sals_paged_append(h, *app[:9], None if lists else ok, app[10], None))
    refused("append lists", lib.sals_paged_append(h, *app[:10], None if lists else ok, None))
    evi = [ok] * 7 + [64, 4, 16, None]
    for i in range(7):
        refused(("evict null", i), lib.sals_paged_evict(h, *evi[:i], None, *evi[i + 1:], None))
    for n in (0, -5, 1601):
        refused(("evict n_keep", n), lib.sals_paged_evict(h, *evi[:7], n, *evi[8:], None))
    refused("evict sink", lib.sals_paged_evict(h, *evi[:8], -1, 16, None, None))
    refused("evict recent", lib.sals_paged_evict(h, *evi[:9], -1, None, None))
    if not lists:
        refused("evict without lists", lib.sals_paged_evict(h, *evi, None))
        refused("attend without lists", lib.sals_paged_attend(h, *att[:6], ok, ok, None))
    lib.sals_paged_destroy(h)
print(bad)
sys.exit(1 if bad else 0)
"""


def test_arguments_that_are_refused(sb):
    """Every refusal, on a context that was never prepared: whatever comes first, nothing is enqueued and no call returns OK."""
    p = subprocess.run([sys.executable, "-c", _ARGS], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert p.returncode == 0, p.stdout[-500:] + p.stderr[-500:]


def test_binding_checks_what_it_is_given(sb):
    """Types, sizes, layout and device: host tensors never get past the binding."""
    torch = pytest.importorskip("torch")
    c = sb.Paged.__new__(sb.Paged)
    c.desc, c._dtype, c._index, c._capacity, c._row, c._page, c._page_stride = _desc(sb), torch.bfloat16, -1, 1600, 1024, (16, 8, 128), 16 * 1024
    good = torch.zeros(64, dtype=torch.int32)
    assert c._take("w", "x", good, torch.int32, 64) == good.data_ptr()
    wide = torch.zeros(64, 2, dtype=torch.int32)
    for t, dt, n in ((good, torch.float32, 64), (good, torch.int32, 65), (wide[:, 0], torch.int32, 64)):
        with pytest.raises(sb.SalsError):
            c._take("w", "x", t, dt, n)
    pool = torch.empty(300, 2, 16, 8, 128, dtype=torch.bfloat16)
    assert c._pool("w", "K", pool.view(600, 16, 8, 128)) == pool.data_ptr()
    for t in (pool[:, 0], pool.view(600, 16, 8, 128)[:299], pool.view(600, 8, 16, 128), pool.view(600, 8, 16, 128).transpose(1, 2),
              pool.view(600, 16, 8, 128).float(), pool.view(600 * 16, 8, 128)):
        with pytest.raises(sb.SalsError):
            c._pool("w", "K", t)
    c._page_stride = 2 * 16 * 1024
    assert c._pool("w", "V", pool[:, 1]) == pool[:, 1].data_ptr()
    c._index = 0
    with pytest.raises(sb.SalsError):
        c._take("w", "x", good, torch.int32, 64)
