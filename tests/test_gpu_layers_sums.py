"""How exact the float32 linear layer's sums are (GPU): chains of the tensor cores' additions, every term product of the gradients of W, sums over
many rows."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_35099_b200 as e3j

pytestmark = pytest.mark.gpu
U = 2.0 ** -24   # half a step of float32
