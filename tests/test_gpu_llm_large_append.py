"""An append of more tokens than one launch holds."""
import os
import re

import pytest
import torch

import paper_2505_20932_amd as P

DEV = "cuda:0"
_RULES = os.path.join(os.path.dirname(P.__file__), "csrc", "llm_rules.h")


def test_a_launch_counts_fewer_than_2_to_the_32_threads():
    at = re.search(r"kAppendBlocksPerLaunch = \(\(int64_t\)1 << (\d+)\) / (\d+);", open(_RULES).read())
    assert 2 ** int(at.group(1)) // int(at.group(2)) * 256 < 2 ** 32


@pytest.mark.gpu
def test_2_to_the_26_tokens():
    """Eight heads of 128, keys and values in the same 137 GB: 2^32 threads of four tokens each and some more.  A few tokens around the borders
    of the launches, the first and the last have slots."""
    heads, d, page = 8, 128, 16
    n = 2 ** 26 + 9
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 * 2 ** 30:
        pytest.skip("needs 160 GiB of free device memory")
    print(f"append of {n} tokens", flush=True)
    x = torch.empty(n, heads, d, dtype=torch.float16, device=DEV)
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    live = torch.cat([torch.arange(a, min(a + 40, n), device=DEV) for a in (0, 2 ** 25 - 20, 2 ** 26 - 20, n - 12)]).unique()
    x[live] = torch.randn(len(live), heads, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).half()
    slots[live] = torch.arange(len(live), device=DEV)
    pages = len(live) // page + 1
    kc, vc = (torch.full((pages, heads, page, d), 3.0, dtype=torch.float16, device=DEV) for _ in range(2))
    P.llm_kv_append(x, x, slots, kc, vc)
    torch.cuda.synchronize()
    for c in (kc, vc):
        rows = c.transpose(1, 2).reshape(-1, heads, d)
        assert torch.equal(rows[:len(live)], x[live]) and (rows[len(live):] == 3.0).all()
    del x
    torch.cuda.empty_cache()
