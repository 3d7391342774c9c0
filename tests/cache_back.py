"""The page tables' step that takes tokens back, in front of ``cache_reference.assign_pages``."""
import cache_reference as ref


def take_back(table, lengths, free, count, page_size, back):
    """table, lengths, free and count after step 0, sequence by sequence."""
    table, lengths, free = table.clone(), lengths.clone(), free.clone()
    pages, cap = len(free), table.shape[1] * page_size
    count = min(max(int(count), 0), pages)
    for b in range(len(lengths)):
        had = min(max(int(lengths[b]), 0), cap)
        left = had - min(max(int(back[b]), 0), had)
        for i in range(-(-left // page_size), -(-had // page_size)):
            if 0 <= int(table[b, i]) < pages:
                if count < pages:
                    free[count] = table[b, i]
                    count += 1
                table[b, i] = -1
        if back[b] > 0:
            lengths[b] = left
    return table, lengths, free, count


def assign_pages(table, lengths, new, free, count, page_size, tokens, window, sinks, back):
    table, lengths, free, count = take_back(table, lengths, free, count, page_size, back)
    return ref.assign_pages(table, lengths, new, free, count, page_size, tokens, window, sinks)
