"""The page tables of a cache on the host as the header describes them, one sequence and one entry after another: a shared page
that a sequence is about to write into is replaced, wherever in its table it lies."""
import plain


class Pages(plain.Pages):
    def resize(self, want):
        before = list(self.refs)
        free = [i for i, r in enumerate(before) if r == 0]
        src, dst, missing, used = [-1] * self.B, [-1] * self.B, [0] * self.B, 0
        for b, w in enumerate(want):
            if w < 0:
                continue
            n, row, held, kv = -(-w // self.ps), self.table[b], self.count[b], self.kv[b]
            # entries that positions kv .. w-1 lie in: those held whose page somebody else names too, and those not held
            mine = [e for e in range(kv // self.ps, min(n, held)) if before[row[e]] > 1] if w > kv else []
            mine += range(held, n)
            missing[b] = len(mine)
            if n > self.cap[b]:
                continue
            pages, used = free[used:used + len(mine)], used + len(mine)  # (a sequence that finds too few takes its place all the same)
            if len(pages) < len(mine):
                continue
            missing[b] = 0
            for e in range(n, held):
                self.refs[row[e]] -= 1
                row[e] = -1
            for e, page in zip(mine, pages):
                if e < held:
                    self.refs[row[e]] -= 1
                    if e * self.ps < kv:           # tokens before kv lie in it
                        src[b], dst[b] = row[e], page
                row[e] = page
                self.refs[page] = 1
            self.count[b], self.kv[b] = n, min(kv, w)
        return src, dst, missing

    def written_twice(self, before_kv, want):
        """Pages that positions before_kv[b] .. want[b]-1 of two sequences lie in."""
        seen, twice = {}, []
        for b, (kv, w) in enumerate(zip(before_kv, want)):
            for e in range(kv // self.ps, min(-(-w // self.ps), self.count[b])) if w > kv else ():
                if self.table[b][e] in seen:
                    twice.append((self.table[b][e], seen[self.table[b][e]], b))
                seen[self.table[b][e]] = b
        return twice
