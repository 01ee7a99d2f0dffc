"""Exact attention over packed prompts where numbers come near the ends of their types: scores far apart, values that nobody may see, rows beside others."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
from test_gpu_prompt import DT, check, inputs, offsets

pytestmark = pytest.mark.gpu
