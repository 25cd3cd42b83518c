"""More sequences than the kernels count are refused (addresses are never followed)."""
import pytest

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import build as B
from tests.test_paged_refusals import UNSUPPORTED, cache, heads, ref, sequences


@pytest.mark.parametrize("seqs", [2**30 + 1, 2**31 - 1])
def test_refused(seqs):
    B.build()
    s = sequences(seqs=seqs, table_stride=0)
    assert P.lib().ttf_attend(ref(heads(8)), ref(s), ref(cache()), 0.1, 1, 0, ref(heads(8)), None) == UNSUPPORTED
    assert P.lib().ttf_cache_append(ref(heads()), ref(heads()), None, None, None, ref(s), ref(cache()), None, None) == UNSUPPORTED
