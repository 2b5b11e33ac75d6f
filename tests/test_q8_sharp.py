"""The sharp inputs over the 8-bit cache are what they are said to be (host only; that a lost plane breaks their
bounds is shown for the same numbers in test_window_sharp.py)."""
import pytest

import q8_sharp as S8


@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("Ek,Ev", [(127, 127), (71, 71), (191, 191), (96, 159)])
@pytest.mark.parametrize("kind", S8.KINDS)
def test_the_exact_answers_are_the_definition(kind, Ek, Ev, dense):
    c, given, q = S8.case(kind, 2, 2, 4, 2, 64, 6, Ek, Ev, dense)
    S8.definition_agrees(kind, c, given, q, Ev, range(2))
