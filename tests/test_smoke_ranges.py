"""The smoke run's check of the examples' first losses is as narrow as it was when it was made for the first of them."""
import inspect


def test_first_losses():
    import __graft_entry__ as entry

    assert set(entry.FIRST_LOSS) == {"tiny_layer", "gated_layer"}
    assert all(low >= 0.8 and high <= 1.3 for low, high in entry.FIRST_LOSS.values())
    assert "low * guess < first < high * guess" in inspect.getsource(entry.smoke)
