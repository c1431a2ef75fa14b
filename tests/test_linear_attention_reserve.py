"""What rnn_linear_attention_reserve takes and how much it holds."""
import pytest

from paper_2307_11339_amd import rnn
from test_linear_attention import gpu  # noqa: F401  (the fixture)


def test_plans_of_more_steps_than_are_taken():
    for T, B in ((2 ** 31 - 1, 1), (2 ** 31 - 60, 1), (2 ** 30 + 1, 1), (2 ** 29 + 1, 2)):
        assert rnn.rnn_linear_attention_plan_query(1, 1, 64, 64, rnn.RNN_F32, T, B)[0] == rnn.RNN_EUNSUPPORTED
    rc, plan = rnn.rnn_linear_attention_plan_query(1, 1, 64, 64, rnn.RNN_F32, 2 ** 30, 1)
    assert rc == rnn.RNN_OK and (plan["pieces"] - 1) * plan["piece_steps"] < 2 ** 30 <= plan["pieces"] * plan["piece_steps"]


@pytest.mark.gpu
@pytest.mark.parametrize("key_size,mib", [(8, 8), (32, 8), (64, 16), (96, 24), (128, 32), (136, 48), (192, 48), (200, 64), (256, 64)])
def test_what_is_held(gpu, key_size, mib):
    layer = rnn.rnn_linear_attention_create(1, 1, key_size, 64, rnn.RNN_F32, [0.9], 1.0)
    tables = rnn.rnn_linear_attention_device_bytes(layer)
    for T, B in ((2 ** 31 - 1, 1), (2 ** 31 - 60, 1), (2 ** 30, 2)):
        assert rnn.rnn_linear_attention_reserve(layer, T, B) == rnn.RNN_EUNSUPPORTED
        assert rnn.rnn_linear_attention_device_bytes(layer) == tables
    for _ in range(2):
        assert rnn.rnn_linear_attention_reserve(layer, 10000, 1) == rnn.RNN_OK
        assert rnn.rnn_linear_attention_device_bytes(layer) == tables + (mib << 20)
    rnn.rnn_linear_attention_destroy(layer)
