"""Host checks of the paged cache's calls: refusals, sizes, and the page division, without a GPU (every
call here is refused before it could launch anything)."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests._build_once import ensure_built

ensure_built()

import paper_2605_30351_amd as vm  # noqa: E402
from paper_2605_30351_amd import _lib as L  # noqa: E402
from workloads import TINY, WAN, WAN_DC, WAN_SINK  # noqa: E402

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)  # never dereferenced
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def dims(d=WAN, **kw):
    s = L.make_dims(d)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def paged(**kw):
    p = L.VideomlaPaged(4, 16, 64, 100, 500, 4, 1, 0, 0x1000, 0x1000, 0x1000, 0x1000, None)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def write(d=None, p=None, x=FAKE, w=FAKE, c=FAKE, k=FAKE, gamma=None):
    d, p = d or dims(), p if p is not None else paged()
    return L.raw().videomla_paged_cache_write(ctypes.byref(d), ctypes.byref(p) if p else None, x, w, gamma,
                                              c, k, None)


def attend(d=None, p=None, q=FAKE, out=FAKE, ws=FAKE, nbytes=1 << 44):
    d, p = d or dims(), p if p is not None else paged()
    return L.raw().videomla_paged_attend(ctypes.byref(d), ctypes.byref(p) if p else None, q, FAKE, FAKE,
                                         FAKE, FAKE, FAKE, out, ws, nbytes, None)


def copy(src, dst, d=None, page=64, pages=32, layers=3, c=FAKE, n=None):
    n = len(src) if n is None else n
    arr = lambda v: (ctypes.c_int32 * max(1, len(v)))(*v)  # noqa: E731
    return L.raw().videomla_pages_copy(ctypes.byref(d or dims()), page, pages, layers, c, FAKE,
                                       ctypes.cast(arr(src), ctypes.c_void_p) if src is not None else None,
                                       ctypes.cast(arr(dst), ctypes.c_void_p), n, None)


@pytest.mark.parametrize("call", [write, attend])
@pytest.mark.parametrize("field,value,code", [
    ("n_seqs", 0, L.EINVAL), ("n_seqs", 4097, L.EUNSUPPORTED), ("n_tokens", 0, L.EINVAL),
    ("n_tokens", -1, L.EINVAL), ("page_tokens", 0, L.EINVAL), ("max_pages", 0, L.EINVAL),
    ("n_pages", 0, L.EINVAL), ("max_new", -1, L.EINVAL), ("mask_block", -1, L.EINVAL),
    ("window_tokens", -1, L.EINVAL), ("max_pages", 1 << 25, L.EUNSUPPORTED),
    ("n_pages", 1 << 25, L.EUNSUPPORTED), ("cu_tokens", None, L.EINVAL), ("kv_len", None, L.EINVAL),
    ("block_table", None, L.EINVAL), ("cu_tokens", 0x1002, L.EALIGN), ("kv_len", 0x1002, L.EALIGN),
    ("block_table", 0x1001, L.EALIGN), ("first_pos", 0x1004, L.EALIGN)])
def test_refuses_bad_descriptions(call, field, value, code):
    assert call(p=paged(**{field: value})) == code
    assert L.raw().videomla_last_error()


@pytest.mark.parametrize("call", [write, attend])
def test_refuses_null_descriptions_and_bad_dims(call):
    assert call(p=False) == L.EINVAL
    assert call(d=dims(d_rope=7)) == L.EINVAL
    assert call(d=dims(WAN_SINK)) == L.EUNSUPPORTED


def test_write_refuses_what_the_ring_write_refuses():
    assert write(d=dims(d_model=1504)) == L.EUNSUPPORTED
    assert write(d=dims(d_model=2112)) == L.EUNSUPPORTED
    for k in ("x", "w", "c", "k"):
        assert write(**{k: None}) == L.EINVAL
        assert write(**{k: ODD}) == L.EALIGN
    assert write(gamma=ODD) == L.EALIGN


def test_attend_refuses_shapes_pointers_and_workspaces():
    assert attend(d=dims(d_c=176)) == L.EUNSUPPORTED
    assert attend(d=dims(d_nope=144)) == L.EUNSUPPORTED
    assert attend(d=dims(d_v=48)) == L.EUNSUPPORTED
    assert attend(p=paged(n_tokens=1 << 28)) == L.EUNSUPPORTED
    assert attend(q=None) == L.EINVAL and attend(out=None) == L.EINVAL
    assert attend(q=ODD) == L.EALIGN and attend(out=ODD) == L.EALIGN
    p, d = paged(), dims()
    need = L.raw().videomla_paged_attend_workspace_bytes(ctypes.byref(d), ctypes.byref(p))
    assert need > 0
    assert attend(nbytes=need - 1) == L.EWORKSPACE and attend(ws=None) == L.EWORKSPACE
    assert attend(ws=ODD) == L.EALIGN


@pytest.mark.parametrize("d", [TINY, *WAN_DC.values()], ids=lambda d: f"dc{d.d_c}")
def test_workspace_size_needs_no_arrays_and_grows_with_the_rows(d):
    size = lambda **kw: L.raw().videomla_paged_attend_workspace_bytes(  # noqa: E731
        ctypes.byref(dims(d)), ctypes.byref(paged(cu_tokens=None, kv_len=None, block_table=None, **kw)))
    assert 0 < size(n_tokens=1, max_new=1) < size(n_tokens=4000, max_new=1) <= size(n_tokens=4000, max_new=0)
    assert size(n_seqs=0) == 0


@pytest.mark.parametrize("src,dst,kw,code", [
    ([0], [32], {}, L.EINVAL), ([32], [0], {}, L.EINVAL), ([-1], [0], {}, L.EINVAL),
    ([0], [-1], {}, L.EINVAL), ([0, 1], [5, 5], {}, L.EINVAL), ([0, 5], [5, 6], {}, L.EINVAL),
    ([3], [3], {}, L.EINVAL), ([0], [1], {"page": 0}, L.EINVAL), ([0], [1], {"pages": 0}, L.EINVAL),
    ([0], [1], {"layers": 0}, L.EINVAL), ([0], [1], {"layers": 65536}, L.EUNSUPPORTED),
    ([0], [1], {"n": -1}, L.EINVAL), ([0], [1], {"c": None}, L.EINVAL), ([0], [1], {"c": ODD}, L.EALIGN),
    ([0], [1], {"pages": 1 << 25}, L.EUNSUPPORTED),
    ([0], [1], {"d": dims(d_c=20), "page": 1}, L.EUNSUPPORTED)])
def test_copy_refuses(src, dst, kw, code):
    assert copy(src, dst, **kw) == code


def test_copy_of_nothing_is_done():
    assert copy([], []) == L.OK


def test_binding_checks_devices_and_shapes():
    import torch
    i32 = torch.zeros(2, dtype=torch.int32)
    p = vm.Paged(cu_tokens=i32, kv_len=i32[:1], block_table=i32.view(1, 2), n_tokens=1, page_tokens=4,
                 n_pages=3)
    with pytest.raises(ValueError, match="device"):
        vm.paged_attend_workspace_bytes(TINY, p)
    with pytest.raises(ValueError, match="block_table"):
        vm.Paged(cu_tokens=i32, kv_len=i32[:1], block_table=i32, n_tokens=1, page_tokens=4,
                 n_pages=3).struct()
    c = torch.zeros(1, 3, 4, 16, dtype=torch.bfloat16)
    k = torch.zeros(1, 3, 4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        vm.pages_copy(TINY, 4, c, k, [0], [1])
    with pytest.raises(ValueError, match="pools"):
        vm.pages_copy(TINY, 2, c, k, [0], [1])
    with pytest.raises(ValueError, match="elements"):
        vm.pages_copy(TINY, 4, c, k, [0], [1, 2])


def test_struct_layout_matches_the_header():
    # 6 int32, 2 int64, 5 pointers
    assert ctypes.sizeof(L.VideomlaPaged) == 24 + 16 + 40


def test_page_division_is_exact(tmp_path):
    """page_of() of csrc/vmla_paged.h against the division, for every page size up to 70,000 at indices
    around its multiples up to 2^30."""
    src = tmp_path / "div.cpp"
    src.write_text('''
#include "vmla_paged.h"
#include <cstdio>
int main() {
  for (int64_t d = 1; d <= (1 << 30); d = d < 70000 ? d + 1 : d * 3) {
    vmla::PagedGeo g{};
    g.page_tokens = (int32_t)d;
    vmla::set_page_division(g);
    for (int64_t k = 0; k < 64; ++k) {
      const int64_t q = k < 32 ? k : ((int64_t(1) << 30) / d) * (k - 31) / 33;
      for (int64_t j = q * d - 1; j <= q * d + 1; ++j)
        if (j >= 0 && j < (int64_t(1) << 31) && vmla::page_of(g, (int32_t)j) != j / d) {
          std::printf("%ld / %ld\\n", (long)j, (long)d);
          return 1;
        }
    }
  }
  return 0;
}
''')
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    exe = tmp_path / "div"
    r = subprocess.run([hipcc, "-O1", "-std=c++17", "-x", "hip", "--cuda-host-only", "-w", f"-I{ROOT}/include",
                        f"-I{ROOT}/paper_2605_30351_amd/csrc", str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("mask,window", [(0, 0), (1, 5), (7, 0)])
def test_the_two_forms_of_the_definition_agree(mask, window):
    from tests.paged_common import Batch, attention_by_sequence
    b = Batch(TINY, [(3, 3, 0), (0, 4, 1), (2, 1, 0), (40, 50, 1000), (1, 0, 0)], page=4, pad=2, mask=mask, window=window,
              seed=3, holes=[(3, 2, -1)])
    for one, two in zip(b.attention(), attention_by_sequence(b, "cpu")):
        assert np.allclose(one, two, rtol=1e-9, atol=1e-12, equal_nan=True)


@pytest.mark.parametrize("d", [TINY, *WAN_DC.values()], ids=lambda d: f"dc{d.d_c}")
@pytest.mark.parametrize("tokens", [1, 3, 40, 5000, 3000000])
def test_a_workspace_serves_every_smaller_bound_on_the_new_tokens(d, tokens):
    size = lambda m: L.raw().videomla_paged_attend_workspace_bytes(  # noqa: E731
        ctypes.byref(dims(d)), ctypes.byref(paged(n_tokens=tokens, n_seqs=1, max_new=m)))
    sizes = [size(m) for m in (1, 2, 3, 8, 40, 5000, 0)]
    assert 0 < sizes[0] and sizes == sorted(sizes)
