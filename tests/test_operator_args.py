"""CPU checks of the feed-forward and update entry points' refusals at their limits (no pointer here is ever
dereferenced: every call is stopped by its last check, the workspace's)."""
import os

import pytest

FAKE = 0x10000  # non-null, aligned


@pytest.fixture(scope="module")
def gs():
    import paper_1710_09854_amd as m

    if not (os.path.exists(m.LIB_PATH) and os.path.exists(m.INSTR_LIB_PATH)):
        from paper_1710_09854_amd import build

        build.build()
    return m


def test_workspace_of_long_pitches(gs):
    """Leading dimensions over 4,000,000 take the workspace of operands that are copied; that one is enough for any."""
    L = gs.lib()
    T, d, f, far = 40, 64, 96, 4_000_008
    for back in (0, 1):
        near, copied = (L.gspar_gated_ff_workspace_bytes(T, d, f, a, back) for a in (1, 0))
        assert 0 < near < copied

        def call(ldx, ldg, ldu, nbytes):
            if back:
                return L.gspar_gated_ff_backward(FAKE, f, FAKE, ldx, FAKE, ldg, FAKE, ldu, FAKE, 1, T, d, f, 0, FAKE, d, FAKE, d,
                                                 FAKE, d, FAKE, nbytes, None)
            return L.gspar_gated_ff_forward(FAKE, ldx, FAKE, ldg, FAKE, ldu, 1, T, d, f, 0, FAKE, f, None, FAKE, nbytes, None)

        for ld in ((far, d, d), (d, far, d), (d, d, far)):
            assert call(*ld, near) == gs.ERR_WORKSPACE and call(*ld, copied - 1) == gs.ERR_WORKSPACE
