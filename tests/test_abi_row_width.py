"""The widest rows of the routing calls: a lane goes on by up to 64 elements at a
time, so a width within 64 of the largest int would wrap in the kernels' loops.
Such a call is refused on the host."""
import pytest

import paper_2107_02103_amd as P
from paper_2107_02103_amd import binding as B

FAKE = 4096          # never dereferenced: validation fails first


@pytest.mark.parametrize("width", [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 127])
@pytest.mark.parametrize("elem", ["F64", "F32", "F16", "BF16"])
def test_rows_whose_ends_wrap_are_refused(width, elem):
    a = dict(stream=0, elem=getattr(P, "DPC_ELEM_" + elem), ntok=1, topk=1, width=width, x=FAKE, ldx=width, weight=None,
             pos=FAKE)
    for call in (lambda: P.dpc_route_gather(**a, rows=FAKE, y=FAKE, ldy=width),
                 lambda: P.dpc_route_combine(**a, y=FAKE, ldy=width),
                 lambda: P.dpc_route_combine_bwd(**a, rows=FAKE, dy=FAKE, lddy=width, dx=FAKE, lddx=width, dweight=FAKE)):
        with pytest.raises(P.DpcError) as e:
            call()
        assert e.value.status == B.DPC_ENOTSUP
