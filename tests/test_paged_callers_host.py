"""What callers may hand the paged calls, without a GPU: pages of a class of their own, numbers that 32-bit
fields do not hold."""
import pytest

import fake_cuda
import paper_2606_27550_gb300 as tv
from test_paged_host import Setup as Setup16
from test_paged_host import fake_path, lib  # noqa: F401
from test_paged_q4_host import Setup, s  # noqa: F401


class OwnPages(tv.Pages):
    """A subclass, with something of its own."""

    __slots__ = ("name",)


class OwnPagesQ4(tv.PagesQ4):
    __slots__ = ("name",)


class Holder:
    """An object that is no subclass: what the calls read of pages, no more."""

    def __init__(self, pages):
        self._c, self.dtype = pages.as_c(), pages.dtype


def test_pages_of_a_callers_own_class(lib, s):  # noqa: F811
    """Subclasses, and objects with the same C struct and type, are served by every call of their kind and refused by
    the others."""
    p16, q4 = s.pages16, s.pages
    calls16 = ((lambda **kw: Setup16.store(s, **kw), 1), (lambda **kw: Setup16.attend(s, **kw), 2),
               (lambda **kw: Setup16.accept(s, **kw), 1), (s.store_norm, 1))
    calls4 = ((s.store_q4, 1), (s.load, 1), (s.attend, 2), (s.accept, 1))
    own16 = (OwnPages(p16.k, p16.v), Holder(p16))
    own4 = (OwnPagesQ4(q4.k, q4.v, 16, 64, q4.dtype), Holder(q4))
    for calls, own, others in ((calls16, own16, own4), (calls4, own4, own16)):
        for fn, launches in calls:
            for pages in own:
                fn(pages=pages)
                assert len(fake_cuda.launches(lib)) == launches
            for pages in (*others, object()):
                with pytest.raises(TypeError):
                    fn(pages=pages)
    assert fake_cuda.launches(lib) == []


BIG = 2 ** 40 * 1e30  # past 32 bits


@pytest.mark.parametrize("name", ["store", "store_norm", "store_q4"])
def test_numbers_past_32_bits_are_refused_by_the_library(lib, s, name):  # noqa: F811
    """A theta, eps or offset whose 32-bit value is infinite, a section past 32 bits: refused as other bad values are."""
    fn = (lambda **kw: Setup16.store(s, pages=s.pages16, **kw)) if name == "store" else getattr(s, name)
    bad = [dict(rope_theta=BIG), dict(rope_theta=-BIG), dict(sections=(2 ** 31,)), dict(sections=(-2 ** 31 - 1,))]
    if name != "store":
        bad += [dict(eps=BIG), dict(weight_offset=-BIG)]
    for kw in bad:
        with pytest.raises(tv.TreeVerifyError) as e:
            fn(**kw)
        assert e.value.status == tv.TB_EINVAL
    assert fake_cuda.launches(lib) == []
