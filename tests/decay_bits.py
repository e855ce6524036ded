"""How many bits the states of decay attention hold that bf16 tokens leave, by the root mean square of their errors.

f = 2^-24. A state sums exp(g n) k v over the tokens that it remembers. What is off by independent parts of each term, relative to the term, is off by as
much relative to the sum:
  - a weight is a power whose exponent is off by 2 f |g n| and its function by f at most, and its product with the value rounds: 1.5 f;
  - the weighted value is taken as three bf16 terms: nothing is left out but what is below 2^-24. As two, the rest after 16 bits is: a rest of half a
    step of 8 bits is uniform and of 2^-8 / sqrt(12) of a value of mantissas between 1 and 2, 0.7 of that on average; twice: (0.7 2^-8 /
    sqrt(12))^2 = 10.5 f;
  - a state is rounded with every chunk that it remembers (by its weight, and by two times three products added), 0.3 to 0.5 f each, less for the
    chunks that decays of at least 0.05 a token have left behind: four chunks' 28 roundings, 2.2 f, and as much in a scan over segments.
Together 3.5 f with three terms; STATE leaves twice that, and two terms are off by more than 10.
"""
import torch

F = 2.0 ** -24
STATE = 7.0
DECAYS = (-0.05, -0.1, -0.3, -1.0)


def rms(got, want, heads=1):
    """The root mean square error relative to the values', in f, of each head (an axis of both)."""
    other = [i for i in range(want.dim()) if i != heads]
    return ((got - want).square().mean(other).sqrt() / want.square().mean(other).sqrt() / F).tolist()


def split(x, terms):
    """Float32 values as the sum of so many bf16 terms."""
    total, left = torch.zeros_like(x, dtype=torch.float64), x
    for _ in range(terms):
        t = left.bfloat16().float()
        total += t
        left = left - t
    return total
