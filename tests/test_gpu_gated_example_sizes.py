"""The example that trains a gated block, where rows do not fill the buffers that were asked for."""
import pytest

from test_gpu_gated_example import _example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,buffers,said", [(90, 16, 1), (91, 16, 1), (7, 5, 2), (3, 8, 1)])
def test_fewer_buffers_than_asked_for(rows, buffers, said):
    """90 rows in 16 buffers: 15 of six rows and none left for the last one."""
    lines = []
    losses, linear = _example().train(rows=rows, p=8, hidden=16, classes=3, buffers=buffers, batch=1, passes=1, iterations=said, say=lines.append)
    assert len(losses) == said and len(lines) == said + 1 and all(x > 0 for x in losses) and linear > 0
