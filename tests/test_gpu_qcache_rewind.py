"""Rewinding to rows that are held as codes alone."""
import pytest

import paper_2605_12471_amd as kv
from test_gpu_qcache import Fold

pytestmark = pytest.mark.gpu


def test_rows_left_as_codes_cannot_be_gone_back_into():
    """300 rows, rewound to 128, of which no bf16 rows are left: not even 64 rows back from what is appended then, up to where two blocks are new."""
    f = Fold(8, 2, 64, 600)

    def to(n):
        f.cache.truncate(0, n)
        f.k, f.v = f.k[:n], f.v[:n]

    def refused(*places):
        for n in places:
            with pytest.raises(kv.KvFoldError) as e:
                f.cache.truncate(0, n)
            assert e.value.status == -3 and f.cache.length(0) == len(f.k)
    f.append(300)
    refused(191, 129, 65, 301)
    to(128)
    f.append(10)
    refused(74, 127, 1)
    to(129)
    f.step(30)
    to(128)
    f.check_rows()
    f.append(72)
    refused(74, 127)
    to(136)            # 64 rows back
    f.step(100)        # 236
    refused(127)
    to(172)
    f.check_rows()
    to(64)
    f.append(3)
    refused(63)
    f.check_rows()
