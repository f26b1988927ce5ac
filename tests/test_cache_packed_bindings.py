"""The bindings of the cache and the packed calls, on the host: what they hold on to."""
import pytest

import paper_2503_02130_amd as fox

ATTRIBUTES = ("k", "v", "c", "page_table", "k_exp", "v_exp", "dtype", "device", "n_pages", "page",
              "max_pages", "B", "H", "H_kv", "d")


@pytest.mark.parametrize("name", ATTRIBUTES)
def test_a_cache_is_set_once(name):
    """Its addresses and sizes are taken when it is made: another tensor behind the same name
    would leave the calls with memory that nobody holds."""
    cache = object.__new__(fox.PagedCache)
    with pytest.raises(AttributeError):
        setattr(cache, name, None)
    cache.__dict__[name] = 1
    with pytest.raises(AttributeError):
        setattr(cache, name, 2)
    with pytest.raises(AttributeError):
        delattr(cache, name)
    assert getattr(cache, name) == 1
