"""The sequence layers' GPU tests again, with a comparison that an infinity or NaN among the results does not pass.

Workspaces are filled with NaN before calls and operands are surrounded by NaN and infinities there, so this is what shows
that neither reaches a result."""
import pytest

from tests import parity as PT
from tests import test_gpu_sequence as sequence

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    PT.torch_dev()
    from tests import sequence_case, sequence_strict
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(sequence_case, "close", sequence_strict.close)
        yield sequence_case


globals().update({name: test for name, test in vars(sequence).items() if name.startswith("test_")})
