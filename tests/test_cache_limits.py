"""Limits of the paged cache's calls that only the largest sizes reach, on the host."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2606_13872_amd as sra
from paper_2606_13872_amd import build
from paper_2606_13872_amd import cache as binding


def _runs(tmp_path):
    """tree_run of csrc/sra_tree.h, compiled for the host."""
    src = tmp_path / "runs.cpp"
    src.write_text('#include "sra_tree.h"\n'
                   'extern "C" int32_t groups() { return sra::kTreeGroups; }\n'
                   'extern "C" int32_t run(int32_t total, int32_t least) { return sra::tree_run(total, least); }\n')
    out = tmp_path / "libruns.so"
    r = subprocess.run([build.hipcc(), *build.COMMON, "-shared", str(src), "-o", str(out)], capture_output=True, text=True,
                       timeout=build.COMPILE_TIMEOUT_S)
    assert r.returncode == 0, r.stderr[-3000:]
    return ctypes.CDLL(os.fspath(out))


def test_runs_cover_the_largest_launch_that_is_accepted(tmp_path):
    """A launch whose contexts fill their table rows costs 2^31 - 128 here; the workgroups' runs have to cover all of it."""
    batch, kv, page, max_pages = 8, 8, 8, 134217684
    fake = 1 << 20
    c = binding._PagedCache(batch, batch, kv, 64, 6, page, max_pages, fake, fake, 0, 0, 0, 0, fake, 0, fake, fake)
    size = ctypes.c_size_t()
    assert binding._lib().sra_tree_workspace_size(ctypes.byref(c), kv, ctypes.byref(size)) == 0
    total = batch * kv * (8 + (max_pages * page + 1 + 31) // 32)  # 8 for beginning a group of rows, its chunks of 32 keys
    assert 2**31 - 256 < total < 2**31
    L = _runs(tmp_path)
    n = L.groups()
    for t in (total, 2**31 - 1, 2**31 - n, 2**31 - n - 1, 0, 1, n - 1, n, n + 1, 16 * n, 16 * n + 1):
        for least in (16, 36):
            run = L.run(t, least)
            assert run >= least and run * n >= t and (run == least or (run - 1) * n < t), (t, least, run)


@pytest.mark.parametrize("tokens,width,batch", [(2**32 + 5, 3, 1), (5, 2**32 + 1, 1), (5, 3, 2**32 + 1), (2**31, 3, 1)])
def test_sizes_past_32_bits_are_refused(tokens, width, batch):
    """They would reach the library cut to their lower 32 bits."""
    def ints(*shape):
        return torch.empty(shape, dtype=torch.int32, device="meta")

    cache = torch.empty(6, 8, 2, 64, dtype=torch.bfloat16, device="meta")
    with pytest.raises(sra.SRAError) as e:
        binding._cache(cache, cache, ints(batch, width), ints(batch), ints(batch + 1), tokens, 2, 64)
    assert e.value.status == 1
