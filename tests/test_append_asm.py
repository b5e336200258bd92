"""Static checks of the append kernels' assembly (no GPU needed)."""

import re

import pytest

from test_kernel_asm import _asm, _have_hipcc, _kernels

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not installed")


def test_arguments_come_in_few_groups():
    """Every argument is loaded by scalar loads, in groups: the kernel of one token is a chain of loads already (starts, lengths,
    page, words), and a wait for arguments before each use adds as many steps to it. A choice between fields of the argument
    struct once became a vector load from the chosen one's address."""
    kernels = {name: [t for kind, t, _ in code if kind == "ins"] for name, code in _kernels(_asm("fa_paged_kernel.hip")).items()
               if "fa_append_kernel" in name}
    assert len(kernels) == 4
    for name, code in kernels.items():
        waits = [t for t in code if re.match(r"s_waitcnt\b.*lgkmcnt", t)]
        pairs = [t for t in code if re.match(r"global_load_dwordx2\b", t)]
        assert any(re.match(r"s_load", t) for t in code)
        assert len(waits) <= 8 and not pairs, (name, waits, pairs)
