"""Operands whose products are exact in fp32, of numbers with so many bits that every part counts of a product that is taken as bf16 parts."""
import torch

# Bits of two factors: 24 are what fp32 holds and three bf16 parts of 8, hi, mid and lo, all count; of 12 bits the first two; of one bit the first alone.
# Together (lo and mid and hi times hi, hi times mid and lo, mid times mid) they have all six products of parts that are taken.
BITS = {"f32": [(24, 1), (1, 24), (12, 12)], "bf16": [(8, 1), (1, 8), (4, 4)]}


def numbers(rows, cols, bits, g):
    """Whole numbers of exactly so many bits, of both signs, on the generator's device; of one bit: powers of two from 1 to 8."""
    shape, device = (rows, cols), g.device
    if bits == 1:
        n = 2 ** torch.randint(0, 4, shape, generator=g, device=device)
    else:
        n = torch.randint(2 ** (bits - 1), 2 ** bits, shape, generator=g, device=device) | 1
    return (n * (2 * torch.randint(0, 2, shape, generator=g, device=device) - 1)).float()


def parts(x):
    """hi, mid, lo: each the nearest bf16 number to what the ones before leave."""
    out = []
    for _ in range(3):
        p = x.bfloat16().float()
        out.append(p)
        x = x - p
    return out


SIX = [(2, 0), (1, 0), (1, 1), (0, 1), (0, 2), (0, 0)]


def one_place(rows, cols, bits, g):
    """(places, matrix): a row has one number, in column 7 i + 3 of row i, modulo their number."""
    places = (7 * torch.arange(rows, device=g.device) + 3) % cols
    m = torch.zeros(rows, cols, device=g.device)
    m.scatter_(1, places[:, None], numbers(rows, 1, bits, g))
    return places, m
