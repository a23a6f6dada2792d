"""The compiled gfx950 code of kernels whose results the next launch of a layer reads (no GPU)."""
import re

import pytest

from test_device_code_cpu import device_code      # noqa: F401 (a fixture)


@pytest.mark.parametrize("kernel,kinds", [("paged_load_kernel", 36), ("rope_kernel", 20)])
def test_results_stay_in_the_caches_for_their_reader(device_code, kernel, kinds):      # noqa: F811
    """No store with the non-temporal hint: it ends the launch earlier, and whoever reads the rows next waits for memory instead."""
    functions, stores = set(), 0
    for lines in device_code:
        inside = None
        for line in lines:
            label = re.match(r"[0-9a-f]+ <(\w+)>:", line)
            if label:
                inside = label.group(1) if kernel in label.group(1) else None
                if inside:
                    functions.add(inside)
            elif inside and re.search(r"\b(global|flat|buffer)_store_", line):
                stores += 1
                assert not re.search(r"\bnt\b", line), (inside, line.strip())
    assert len(functions) == kinds and stores >= kinds
